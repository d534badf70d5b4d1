"""Rotary positions and the heads' way back to rows on the GPU against plain
64-bit forms (tests/layer_cases.py) and the oracle, every output equal."""
import numpy as np
import pytest

import layer_cases as R
from test_linear_gpu import dev, fq, guarded, host, say, unaligned  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 3, 64, 197, 1000])
@pytest.mark.parametrize("P", [1, 3, 16, 30, 32, 64, 128])
@pytest.mark.parametrize("axes", [1, 2, 3, 8])
def test_table(fq, T, P, axes):  # noqa: F811
    """An entry differs from the correctly rounded one only where 2^14 cos t lies
    within 2^-36 of the middle of two integers (two units in the last place of a
    cosine, 2 * 2^-53, times 2^14, and as much for the host's own): none of
    these inputs does."""
    say("table", T, P, axes)
    g = np.random.default_rng(T + P)
    pos = g.integers(-2 ** 31, 2 ** 31, (axes, T)).astype(np.int32)
    pos[0, 0] = 0
    pos[:, T // 2] = -2 ** 31
    freq = 10000.0 ** (-np.arange(P) / P)
    axis = (np.arange(P) % (axes + 1)).astype(np.uint8)      # one beyond the last
    table, intact = guarded((T, P, 2), dev(np.zeros(1, np.int16)).dtype, 4)
    fq.rope_table_int16(dev(pos), dev(freq), dev(axis), table=table)
    t = pos[np.minimum(axis, axes - 1)].T.astype(np.float64) * freq
    exact = 16384.0 * np.stack((np.cos(t), np.sin(t)), -1)
    assert (np.abs(exact - np.floor(exact) - 0.5) > 2.0 ** -36).all()
    assert np.array_equal(host(table), np.rint(exact).astype(np.int16))
    assert intact()


def rope(fq, B, L, Hq, Hkv, d, P, il, own_rows=False, offset=0, bits=8, zps=(0, 0, 0), out_off=0):  # noqa: F811
    g = np.random.default_rng(B * L + d + P)
    qkv = g.integers(-128, 128, (B, L, (Hq + 2 * Hkv) * d)).astype(np.int8)
    table = None
    if P:
        pos = g.integers(0, 100_000, (2, B * L if own_rows else L)).astype(np.int32)
        table = R.rope_table(pos, 10000.0 ** (-np.arange(P) / P), (np.arange(P) & 1).astype(np.uint8))
    kw = dict(zp_x=zps[0], zp_q=zps[1], zp_k=zps[2], bits=bits, interleaved=il)
    s = (0.05, 0.07 * 255 / (2 ** bits - 1), 0.06 * 255 / (2 ** bits - 1))
    x = unaligned(qkv, offset) if offset else dev(qkv)
    outs = [guarded((B, h, L, d), x.dtype, out_off) for h in (Hq, Hkv, Hkv)]
    fq.rope_qkv_int8(x, dev(table), Hq, Hkv, *s, **kw, **{n: o for n, (o, _) in zip("qkv", outs)})
    for n, (o, intact), ref in zip("qkv", outs, R.rope(qkv, table, Hq, Hkv, *s, **kw)):
        assert np.array_equal(host(o), ref), n
        assert intact(), n


# head sizes of whole units of 16 bytes, of 8, of 4, odd ones; all, some and one
# of their pairs turned
@pytest.mark.parametrize("d,P", [(64, 32), (32, 16), (128, 64), (64, 16), (64, 30), (64, 1), (80, 40),
                                 (72, 36), (48, 24), (96, 32), (256, 128), (40, 20), (8, 4), (2, 1), (1, 0),
                                 (37, 18), (37, 5), (64, 0), (16, 8), (66, 33), (36, 18), (20, 8)])
@pytest.mark.parametrize("il", [False, True])
def test_heads(fq, d, P, il):  # noqa: F811
    for B, L, Hq, Hkv in ((1, 1, 1, 1), (2, 7, 3, 3), (3, 33, 4, 2)):
        say("rope", d, P, il, B, L, Hq, Hkv)
        rope(fq, B, L, Hq, Hkv, d, P, il, own_rows=L == 7, zps=(3, -2, 1))


@pytest.mark.parametrize("B,L,Hq,Hkv", [(1, 197, 3, 3), (5, 64, 12, 1), (300, 1, 8, 2), (1, 2000, 1, 1),
                                        (2, 50, 48, 12), (1, 3, 1024, 1024), (7, 65, 5, 5)])
@pytest.mark.parametrize("il", [False, True])
def test_shapes(fq, B, L, Hq, Hkv, il):  # noqa: F811
    for own_rows in (False, True):
        say("shape", B, L, Hq, Hkv, il, own_rows)
        rope(fq, B, L, Hq, Hkv, 64, 32, il, own_rows, zps=(-128, 5, 127))


@pytest.mark.parametrize("bits,zps", [(8, (127, -128, 127)), (4, (0, -8, 7)), (2, (1, 1, -2)),
                                      (6, (-5, 31, -32))])
@pytest.mark.parametrize("d,P", [(64, 32), (37, 10)])
def test_grids(fq, bits, zps, d, P):  # noqa: F811
    for il in (False, True):
        say("grid", bits, zps, d, P, il)
        rope(fq, 2, 40, 3, 3, d, P, il, bits=bits, zps=zps)


@pytest.mark.parametrize("offset,out_off", [(1, 0), (4, 0), (8, 4), (0, 1), (0, 8), (3, 5)])
def test_unaligned(fq, offset, out_off):  # noqa: F811
    for d, P in ((64, 32), (64, 20), (80, 40)):
        say("unaligned", offset, out_off, d, P)
        rope(fq, 2, 30, 4, 2, d, P, True, offset=offset, out_off=out_off)
        rope(fq, 2, 30, 4, 2, d, P, False, offset=offset, out_off=out_off)


def test_saturation_and_ties(fq):  # noqa: F811
    """m = 2^-15: every odd value of the unturned part is a tie; m = 2^4 and the
    largest multiplier saturate."""
    g = np.random.default_rng(0)
    qkv = g.integers(-128, 128, (2, 9, 3 * 32)).astype(np.int8)
    table = R.rope_table(np.arange(9, dtype=np.int32)[None], 0.5 ** np.arange(8), np.zeros(8, np.uint8))
    say("saturation")
    for s_x, s_q, s_k in ((0.5, 1.0, 0.25), (2.0 ** 18, 1.0, 2.0), (1e30, 1e-30, 1.0)):
        got = fq.rope_qkv_int8(dev(qkv), dev(table), 1, 1, s_x, s_q, s_k, zp_q=3)
        with np.errstate(over="ignore"):
            table_q = R.rope(qkv, table, 1, 1, s_x, max(s_q, s_x * 2.0 ** -100), s_k, zp_q=3)
        for a, b in zip(got, table_q):
            assert np.array_equal(host(a), b)


def test_empty(fq):  # noqa: F811
    import torch
    z = torch.zeros((0, 5, 96), dtype=torch.int8, device="cuda:0")
    t = torch.zeros((5, 16, 2), dtype=torch.int16, device="cuda:0")
    say("empty")
    assert [o.numel() for o in fq.rope_qkv_int8(z, t, 1, 1, 1.0, 1.0, 1.0)] == [0, 0, 0]
    assert fq.requant_heads_int8(torch.zeros((2, 3, 0, 8), dtype=torch.int32, device="cuda:0"), 1.0, 1.0,
                                 0).shape == (2, 0, 24)


@pytest.mark.parametrize("B,H,L,d", [(1, 1, 1, 1), (2, 3, 5, 7), (1, 12, 197, 64), (3, 5, 145, 37),
                                     (2, 4, 33, 32), (4, 2, 64, 48), (1, 2, 9, 256), (1, 1024, 2, 3),
                                     (2, 3, 50, 36), (1, 3, 7, 66)])
@pytest.mark.parametrize("bits,zp", [(8, 0), (4, -8), (6, 20)])
def test_heads_to_rows(fq, orc, B, H, L, d, bits, zp):  # noqa: F811
    g = np.random.default_rng(d)
    q = (g.normal(0, 1, (B, H, L, d)) * 2.0 ** 22).astype(np.int32)
    q.flat[0], q.flat[-1] = -2 ** 31, 2 ** 31 - 1
    for s_in, s_out, off in ((2.0 ** -22, 0.02, 0), (0.75, 2.0 ** 17, 0), (1e-12, 1e3, 0), (3.0, 0.1, 0),
                             (2.0 ** -22, 0.02, 1), (2.0 ** -22, 0.02, 4)):
        say("merge", B, H, L, d, bits, s_in, s_out, off)
        y, intact = guarded((B, L, H * d), dev(np.zeros(1, np.int8)).dtype, off)
        x = dev(q)
        if off == 4:                           # int32 on a base of 4 bytes
            import torch
            buf = torch.zeros(q.size + 1, dtype=torch.int32, device="cuda:0")
            x = buf[1:].view(q.shape)
            x.copy_(dev(q))
        fq.requant_heads_int8(x, s_in, s_out, zp, bits, y=y)
        assert np.array_equal(host(y), orc.requant_heads_int8(q, s_in, s_out, zp, bits))
        assert intact()


def test_offsets_beyond_32_bits(fq):  # noqa: F811
    """The last image of a batch of more than 2^32 bytes is that image alone."""
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(2)
    B, L, Hq, Hkv, d = 2500, 577, 16, 16, 64
    table = dev(R.rope_table(np.arange(L, dtype=np.int32)[None], 0.9 ** np.arange(32),
                             np.zeros(32, np.uint8)))
    say("far images", B)
    qkv = torch.randint(-128, 128, (B, L, (Hq + 2 * Hkv) * d), generator=g, device="cuda:0",
                        dtype=torch.int8)
    for head in (64, 37):                      # 37 of the same bytes: the kernel of single values
        x = qkv if head == 64 else qkv.view(-1)[:B * L * 48 * 37].view(B, L, 48 * 37)
        t = table[:, :16] if head == 37 else table
        kw = dict(interleaved=head == 37)
        far = fq.rope_qkv_int8(x, t.contiguous(), Hq, Hkv, 0.05, 0.07, 0.06, **kw)
        for b in (0, B // 2, B - 1):
            one = fq.rope_qkv_int8(x[b:b + 1].clone(), t.contiguous(), Hq, Hkv, 0.05, 0.07, 0.06, **kw)
            for a, c in zip(far, one):
                assert torch.equal(a[b:b + 1], c)
        del far
    q = qkv.view(-1)[:4 * (B // 2 * 16 * L * 64) // 4 * 4].view(torch.int32).view(-1)
    n = q.numel() // (16 * L * 64)
    q = q[:n * 16 * L * 64].view(n, 16, L, 64)
    y = fq.requant_heads_int8(q, 2.0 ** -30, 0.02, 1)
    for b in (0, n - 1):
        assert torch.equal(y[b:b + 1], fq.requant_heads_int8(q[b:b + 1].clone(), 2.0 ** -30, 0.02, 1))


def test_matches_the_oracle(fq, orc):  # noqa: F811
    g = np.random.default_rng(5)
    pos = g.integers(0, 5000, (3, 40)).astype(np.int32)
    freq, axis = 10000.0 ** (-np.arange(15) / 15), (np.arange(15) // 5).astype(np.uint8)
    qkv = g.integers(-128, 128, (2, 20, 8 * 32)).astype(np.int8)
    say("oracle")
    table = fq.rope_table_int16(dev(pos), dev(freq), dev(axis))
    ref = orc.rope_table_int16(pos, freq, axis)
    assert np.array_equal(host(table), ref)
    for il in (False, True):
        got = fq.rope_qkv_int8(dev(qkv), table, 4, 2, 0.05, 0.06, 0.07, 1, 2, 3, interleaved=il)
        for a, b in zip(got, orc.rope_qkv_int8(qkv, ref, 4, 2, 0.05, 0.06, 0.07, 1, 2, 3, interleaved=il)):
            assert np.array_equal(host(a), b)
