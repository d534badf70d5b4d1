"""The linear layers on the GPU against plain 64-bit forms (tests/layer_cases.py;
the oracle is held to the same in test_layers_oracle.py), every output equal:
sizes around the tiles' and the steps' edges, every activation with and without
a residual, extremes, unaligned bases, bytes around the output left alone."""
import numpy as np
import pytest

import layer_cases as R
from test_layers_oracle import options

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fq():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2111_13824_amd as fq
    return fq


def dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def host(t):
    import torch
    torch.cuda.synchronize()
    return t.cpu().numpy()


def say(*a):
    print("CASE", *a, flush=True)


def guarded(shape, dtype, offset=0):
    """An output inside a larger buffer of 0x55 bytes, `offset` bytes off its
    alignment, and a check that the bytes around it are as they were."""
    import torch
    n = int(np.prod(shape)) * dtype.itemsize
    buf = torch.full((n + 512,), 0x55, dtype=torch.uint8, device="cuda:0")
    lo = 256 + offset
    out = buf[lo:lo + n].view(dtype).view(shape)

    def intact():
        b = host(buf)
        return (b[:lo] == 0x55).all() and (b[lo + n:] == 0x55).all()
    return out, intact


def unaligned(a, offset):
    """The same int8 matrix on a base `offset` bytes off a 256-byte boundary."""
    import torch
    buf = torch.zeros(a.size + 256, dtype=torch.int8, device="cuda:0")
    view = buf[offset:offset + a.size].view(a.shape)
    view.copy_(dev(a))
    return view


def run(fq, p, act="none", residual=False, zp_y=0, bits=8, offset=0, seed=0):
    T, N = p["x"].shape[0], p["w"].shape[0]
    s_y = p["s_y"] * 255 / ((1 << bits) - 1) * (8 if act == "table" else 1)
    x, w = (unaligned(a, offset) if offset else dev(a) for a in (p["x"], p["w"]))
    f, m = fq.linear_fold_int8(w, dev(p["s_w"]), p["s_x"], s_y, p["zp_x"], dev(p["bias"]))
    rf, rm = R.fold(p["w"], p["s_w"], p["s_x"], s_y, p["zp_x"], p["bias"])
    assert np.array_equal(host(f), rf) and np.array_equal(host(m), rm)
    more = options(act, residual, T, N, seed)
    more_d = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in more.items()}
    y, intact = guarded((T, N), x.dtype, offset)
    fq.linear_int8(x, w, f, m, zp_y, bits, y=y, **more_d)
    ref = R.linear(p["x"], p["w"], rf, rm, zp_y, bits, **more)
    assert np.array_equal(host(y), ref)
    assert intact()


# rows around the widths of the tiles (16, 32, 64, 128, 256) and their multiples
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 197, 255, 256, 257,
                               511, 520, 1030])
@pytest.mark.parametrize("K,N", [(64, 64), (192, 96), (100, 70)])
def test_rows(fq, T, K, N):
    say("rows", T, K, N)
    run(fq, R.layer(T, K, N, seed=T, zp_x=5), zp_y=-3)


# inputs around the units of 16, the steps of 64 and 128, and the ends of the range
@pytest.mark.parametrize("K", [1, 2, 3, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 80, 96, 112, 127, 128,
                               129, 144, 160, 191, 192, 193, 240, 256, 257, 272, 320, 384, 448, 512, 516,
                               1008, 1024, 4096, 4111, 32767, 32768])
@pytest.mark.parametrize("T,N", [(1, 33), (20, 40), (200, 150)])
def test_inputs(fq, K, T, N):
    if K > 10000 and T > 20:
        T = 70
    say("inputs", K, T, N)
    run(fq, R.layer(T, K, N, seed=K, zp_x=-7), zp_y=2)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 7, 8, 9, 12, 15, 16, 17, 20, 31, 32, 33, 36, 63, 64, 65, 68,
                               127, 128, 129, 132, 192, 255, 256, 257, 260, 300, 1000, 1001])
@pytest.mark.parametrize("T,K", [(1, 256), (5, 100), (70, 128), (270, 64)])
def test_channels(fq, N, T, K):
    say("channels", N, T, K)
    run(fq, R.layer(T, K, N, seed=N))


@pytest.mark.parametrize("T,K,N", [(T, 64, 1000) for T in (1025, 1026, 1055, 1057, 1087, 1088)]
                         + [(T, 67, 1000) for T in (1023, 1024, 1025, 1056, 1087)]
                         + [(1000, K, 1000) for K in (1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 65, 96, 112, 127,
                                                      128, 129, 144, 240, 255, 256, 257, 272, 400, 528)]
                         + [(1000, K, N) for K in (64, 70)
                            for N in (1001, 1002, 1003, 1007, 1009, 1023, 1025, 1039, 1057, 1087, 1088)])
def test_edges_of_small_tiles(fq, T, K, N):
    """Rows, inputs and channels that end inside tiles of 64 x 64."""
    say("small tiles", T, K, N)
    run(fq, R.layer(T, K, N, seed=T + K + N, zp_x=6), residual=True, zp_y=-4, seed=K)


@pytest.mark.parametrize("act", ["none", "relu", "table"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,K,N", [(1, 128, 256), (40, 96, 100), (130, 192, 260), (600, 64, 512),
                                   (33, 50, 27), (300, 77, 131), (2100, 256, 1024)])
def test_epilogues(fq, act, residual, T, K, N):
    for bits, zp in ((8, 0), (8, -128), (4, 7), (2, -1), (6, 31)):
        say("epilogue", act, residual, T, K, N, bits, zp)
        run(fq, R.layer(T, K, N, seed=bits, zp_x=zp), act, residual, zp, bits, seed=T)


@pytest.mark.parametrize("name,T,K,N", [(n, *p) for n in R.KERNELS for p in R.PRODUCTS[n]])
def test_every_kernel(fq, name, T, K, N):
    """Each kernel on each of its products (that they are its, the CPU test of the
    same list holds), with a residual on every second."""
    say("kernel", name, T, K, N)
    run(fq, R.layer(T, K, N, seed=K, zp_x=-3), "none", K % 32 == 0, 5, seed=N)


@pytest.mark.parametrize("name", R.KERNELS)
@pytest.mark.parametrize("act,residual", [("none", True), ("relu", False), ("relu", True),
                                          ("table", False), ("table", True), ("int32", False)])
def test_every_kernel_and_epilogue(fq, name, act, residual):
    T, K, N = R.PRODUCTS[name][0]
    say("kernel", name, act, residual)
    p = R.layer(T, K, N, seed=T)
    if act == "int32":
        f = np.random.default_rng(K).integers(-2 ** 30, 2 ** 30, N).astype(np.int32)
        out, intact = guarded((T, N), dev(f).dtype, 4)
        fq.linear_int32(dev(p["x"]), dev(p["w"]), dev(f), out=out)
        assert np.array_equal(host(out), R.sums(p["x"], p["w"], f)) and intact()
    else:
        run(fq, p, act, residual, -20, 7, seed=K)


@pytest.mark.parametrize("offset", [1, 2, 4, 8, 12, 15])
@pytest.mark.parametrize("T,K,N", [(1, 64, 64), (9, 48, 20), (150, 128, 132), (260, 100, 64),
                                   (1000, 128, 1001), (1100, 100, 700)])
def test_unaligned_bases(fq, offset, T, K, N):
    say("offset", offset, T, K, N)
    run(fq, R.layer(T, K, N, seed=offset), "relu", True, 1, 8, offset, seed=T)


@pytest.mark.parametrize("T,K,N", [(1, 64, 64), (13, 100, 37), (70, 701, 1001), (300, 256, 256),
                                   (129, 16, 4), (1, 32768, 3), (65, 32768, 65), (2100, 128, 1024),
                                   (1000, 272, 1001), (1100, 101, 700)])
def test_accumulators(fq, T, K, N):
    say("int32", T, K, N)
    p = R.layer(T, K, N, seed=K)
    f = np.random.default_rng(K).integers(-2 ** 30, 2 ** 30, N).astype(np.int32)
    for fold in (None, f):
        for offset in (0, 4):
            out, intact = guarded((T, N), dev(f).dtype, offset)
            fq.linear_int32(dev(p["x"]), dev(p["w"]), dev(fold), out=out)
            assert np.array_equal(host(out), R.sums(p["x"], p["w"], fold)), (fold is None, offset)
            assert intact()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_extremes(fq, T):
    """Sums of the largest magnitude: +-(2^29 + 2^30 - 1), and multipliers that
    saturate, vanish or hit ties exactly."""
    K, N = 32768, 70
    say("extremes", T)
    x = np.full((T, K), -128, np.int8)
    w = np.where(np.arange(N)[:, None] % 2, -128, 127).astype(np.int8) * np.ones((1, K), np.int8)
    f = np.where(np.arange(N) % 2, 2 ** 30, -2 ** 30).astype(np.int32)
    assert np.array_equal(host(fq.linear_int32(dev(x), dev(w), dev(f))), R.sums(x, w, f))
    big = np.finfo(np.float32).max
    for m in (big, 0.0, 2.0 ** -24, 2.0 ** -40):
        mul = np.full(N, m, np.float32)
        for more in ({}, dict(relu=True), dict(table=np.linspace(-200, 200, 4096).astype(np.float32),
                                               zp_t=4095)):
            for res in ({}, dict(residual=np.full((T, N), 127, np.int8), zp_r=-128, mul_r=2.0 ** 20)):
                kw = dict(more, **res)
                kd = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
                got = host(fq.linear_int8(dev(x), dev(w), dev(f), dev(mul), 3, **kd))
                with np.errstate(over="ignore"):
                    assert np.array_equal(got, R.linear(x, w, f, mul, 3, **kw)), (m, list(kw))


@pytest.mark.parametrize("T,N", [(1, 70), (4200, 130), (2600, 2050), (5500, 2050)])
def test_largest_sums(fq, T, N):
    """Every row the same, so one row of the plain form is the reference."""
    import torch
    K = 32768
    say("largest sums", T, N)
    x = torch.full((T, K), -128, dtype=torch.int8, device="cuda:0")
    w = np.where(np.arange(N)[:, None] % 2, -128, 127).astype(np.int8) * np.ones((1, K), np.int8)
    f = np.where(np.arange(N) % 2, 2 ** 30, -2 ** 30).astype(np.int32)
    got = host(fq.linear_int32(x, dev(w), dev(f)))
    assert (got == R.sums(np.full((1, K), -128, np.int8), w, f)).all()


@pytest.mark.parametrize("T", [3, 40, 300])
def test_ties_go_to_the_even_neighbour(fq, T):
    """mul = 1/2 and 1/4 put every second or fourth sum on a tie, the zero point
    inside the rounding."""
    g = np.random.default_rng(T)
    x, w = (g.integers(-3, 4, (n, 32)).astype(np.int8) for n in (T, 48))
    f = g.integers(-20, 20, 48).astype(np.int32)
    say("ties", T)
    for m in (0.5, 0.25):
        mul = np.full(48, m, np.float32)
        for zp in (0, 1, -7):
            for kw in ({}, dict(relu=True), dict(residual=g.integers(-9, 9, (T, 48)).astype(np.int8),
                                                 zp_r=1, mul_r=0.5)):
                kd = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in kw.items()}
                got = host(fq.linear_int8(dev(x), dev(w), dev(f), dev(mul), zp, **kd))
                assert np.array_equal(got, R.linear(x, w, f, mul, zp, **kw)), (m, zp, list(kw))


def test_matches_the_oracle(fq, orc):
    p = R.layer(50, 130, 90, seed=4, zp_x=9)
    f, m = orc.linear_fold_int8(p["w"], p["s_w"], p["s_x"], p["s_y"], 9, p["bias"])
    say("oracle")
    gf, gm = fq.linear_fold_int8(dev(p["w"]), dev(p["s_w"]), p["s_x"], p["s_y"], 9, dev(p["bias"]))
    assert np.array_equal(host(gf), f) and np.array_equal(host(gm), m)
    for act in ("none", "relu", "table"):
        more = options(act, True, 50, 90, 1)
        kd = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in more.items()}
        y = fq.linear_int8(dev(p["x"]), dev(p["w"]), gf, gm, 4, **kd)
        assert np.array_equal(host(y), orc.linear_int8(p["x"], p["w"], f, m, 4, **more))


@pytest.mark.parametrize("K", [1, 5, 63, 64, 65, 100, 1000, 4099, 32768])
def test_fold(fq, orc, K):
    """Channels without a usable scale, biases without a value or beyond the
    clip; the sums of rows of any length."""
    g = np.random.default_rng(K)
    N = 37
    w = g.integers(-128, 128, (N, K)).astype(np.int8)
    w[0] = -128
    s_w = np.exp(g.normal(0, 3, N)).astype(np.float32)
    bias = g.normal(0, 5, N).astype(np.float32)
    s_w[1:5] = 0.0, -1.0, np.inf, np.nan
    bias[5:9] = np.nan, np.inf, -np.inf, 1e30
    s_w[9], s_w[10] = 1e-38, 3e38
    say("fold", K)
    for zp in (0, -128, 127):
        f, m = fq.linear_fold_int8(dev(w), dev(s_w), 0.013, 0.02, zp, dev(bias))
        rf, rm = orc.linear_fold_int8(w, s_w, 0.013, 0.02, zp, bias)
        assert np.array_equal(host(f), rf) and np.array_equal(host(m), rm)


@pytest.mark.parametrize("T,K,N", [(5, 64, 48), (200, 64, 192), (600, 128, 512), (90, 50, 27), (1100, 64, 700),
                                   (1000, 50, 1001)])
def test_output_over_the_residual(fq, T, K, N):
    say("in place", T, K, N)
    p = R.layer(T, K, N, seed=1)
    f, m = R.fold(p["w"], p["s_w"], p["s_x"], p["s_y"], 0, p["bias"])
    r = np.random.default_rng(2).integers(-128, 128, (T, N)).astype(np.int8)
    buf = dev(r)
    fq.linear_int8(dev(p["x"]), dev(p["w"]), dev(f), dev(m), residual=buf, mul_r=0.7, y=buf)
    assert np.array_equal(host(buf), R.linear(p["x"], p["w"], f, m, residual=r, mul_r=0.7))


def test_empty_and_prepared_calls_and_streams(fq):
    import torch
    p = R.layer(300, 128, 256, seed=3)
    x, w = dev(p["x"]), dev(p["w"])
    f, m = fq.linear_fold_int8(w, dev(p["s_w"]), p["s_x"], p["s_y"], 0, dev(p["bias"]))
    assert fq.linear_int8(x[:0], w, f, m).shape == (0, 256)
    assert fq.linear_int32(x[:0], w).shape == (0, 256)
    ref = R.linear(p["x"], p["w"], host(f), host(m))
    say("streams")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty((300, 256), dtype=torch.int8, device="cuda:0") for _ in streams]
    calls = [fq.linear_int8(x, w, f, m, y=o, stream=s, prepare=True) for o, s in zip(outs, streams)]
    for _ in range(3):
        for c in calls:
            c()
    for o in outs:
        assert np.array_equal(host(o), ref)


def test_offsets_beyond_32_bits(fq):
    """Outputs and inputs whose byte offsets pass 2^31 and 2^32: the rows at the
    ends and around the borders against the plain form."""
    import torch
    say("far rows")
    K, N = 16, 1040
    T = (1 << 32) // N + 300
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    x = torch.randint(-128, 128, (T, K), generator=g, device="cuda:0", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda:0", dtype=torch.int8)
    mul = torch.full((N,), 2.0 ** -9, device="cuda:0")
    y = fq.linear_int8(x, w, None, mul)
    picks = torch.cat([torch.arange(max(0, c - 150), min(T, c + 150)) for c in
                       (0, (1 << 31) // N, (1 << 32) // N, T)]).to("cuda:0")
    ref = R.linear(host(x[picks]), host(w), None, host(mul))
    assert np.array_equal(host(y[picks]), ref)
    del y
    # a long input: T K beyond 2^32
    K, N = 32768, 20
    T = (1 << 32) // K + 70
    x = torch.randint(-128, 128, (T, K), generator=g, device="cuda:0", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g, device="cuda:0", dtype=torch.int8)
    out = fq.linear_int32(x, w)
    picks = torch.cat([torch.arange(max(0, c - 20), min(T, c + 20)) for c in
                       (0, (1 << 31) // K, (1 << 32) // K, T)]).to("cuda:0")
    assert np.array_equal(host(out[picks]), R.sums(host(x[picks]), host(w)))
