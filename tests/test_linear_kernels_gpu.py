"""Every kernel of the linear layers by itself: rows, channels and inputs around
the edges of its tiles, every epilogue on ties, on the largest sums and with
tables of every size, and operands on bases of the least alignment.  Which
product takes which kernel is held on the CPU (test_layers_abi.py).

Rows come again every 331 rows, a prime above every tile, so that one small
plain form is the reference of a large product and no two rows of a tile, nor
the same rows of two tiles next to each other, are alike."""
import numpy as np
import pytest

import layer_cases as R
from test_linear_gpu import dev, fq, guarded, host, say, unaligned  # noqa: F401

pytestmark = pytest.mark.gpu

PERIOD = 331


def repeated(a, T):
    return a[np.arange(T) % len(a)]


def check(fq, T, x, w, f, mul, **kw):  # noqa: F811
    """linear_int8 of T rows, x's and the residual's over and over, against the plain
    form of x alone."""
    more = dict(kw)
    for n in ("table", "residual"):
        if n in more:
            more[n] = dev(repeated(more[n], T) if n == "residual" else more[n])
    y, intact = guarded((T, len(w)), dev(x[:1]).dtype)
    fq.linear_int8(dev(repeated(x, T)), dev(w), dev(f), dev(mul), y=y, **more)
    with np.errstate(over="ignore"):
        ref = R.linear(x, w, f, mul, **kw)
    got = host(y)
    assert np.array_equal(got, repeated(ref, T)), [(n, v if np.isscalar(v) else "") for n, v in kw.items()]
    assert intact()


@pytest.mark.parametrize("name,T,K,N", [(n, *p) for n in R.EDGES for p in R.EDGES[n]])
def test_edges_of_every_tile(fq, name, T, K, N):  # noqa: F811
    """The requantized result, with a residual, and the int32 sums."""
    say("edges", name, T, K, N)
    p = R.layer(min(T, PERIOD), K, N, seed=K + N, zp_x=-3)
    f, m = R.fold(p["w"], p["s_w"], p["s_x"], p["s_y"], -3, p["bias"])
    r = np.random.default_rng(N).integers(-128, 128, p["x"].shape[:1] + (N,)).astype(np.int8)
    check(fq, T, p["x"], p["w"], f, m, zp_y=5, residual=r, zp_r=7, mul_r=0.6)
    out, intact = guarded((T, N), dev(f).dtype)
    fq.linear_int32(dev(repeated(p["x"], T)), dev(p["w"]), dev(f), out=out)
    assert np.array_equal(host(out), repeated(R.sums(p["x"], p["w"], f), T))
    assert intact()


@pytest.mark.parametrize("T,K,N", R.WIDE)
def test_wide_products_of_few_rows(fq, T, K, N):  # noqa: F811
    """One line of tiles, most of whose rows are not there: every epilogue."""
    say("wide", T, K, N)
    p = R.layer(T, K, N, seed=T, zp_x=4)
    f, m = R.fold(p["w"], p["s_w"], p["s_x"], p["s_y"], 4, p["bias"])
    r = np.random.default_rng(N).integers(-128, 128, (T, N)).astype(np.int8)
    table = np.random.default_rng(T).normal(0, 60, 256).astype(np.float32)
    for kw in ({}, dict(relu=True), dict(table=table, zp_t=128)):
        check(fq, T, p["x"], p["w"], f, m, zp_y=-9, **kw)
        check(fq, T, p["x"], p["w"], f, m, zp_y=-9, residual=r, zp_r=3, mul_r=0.7, **kw)
    out, intact = guarded((T, N), dev(f).dtype, 4)
    fq.linear_int32(dev(p["x"]), dev(p["w"]), dev(f), out=out)
    assert np.array_equal(host(out), R.sums(p["x"], p["w"], f)) and intact()


@pytest.mark.parametrize("name", R.KERNELS)
@pytest.mark.parametrize("mul,zp", [(0.5, 1), (0.25, -7)])
def test_ties_go_to_the_even_neighbour_in_every_kernel(fq, name, mul, zp):  # noqa: F811
    T, K, N = R.PRODUCTS[name][0]
    say("ties", name, mul, zp)
    g = np.random.default_rng(T)
    x = g.integers(-3, 4, (min(T, PERIOD), K)).astype(np.int8)
    w = g.integers(-3, 4, (N, K)).astype(np.int8)
    f = g.integers(-20, 20, N).astype(np.int32)
    m = np.full(N, mul, np.float32)
    r = g.integers(-9, 9, (len(x), N)).astype(np.int8)
    table = (np.arange(64) * 0.5 - 16).astype(np.float32)      # every second value between two steps
    for kw in ({}, dict(relu=True), dict(table=table, zp_t=32)):
        check(fq, T, x, w, f, m, zp_y=zp, **kw)
        check(fq, T, x, w, f, m, zp_y=zp, residual=r, zp_r=1, mul_r=0.5, **kw)


@pytest.mark.parametrize("name", R.KERNELS)
def test_extremes_in_every_kernel(fq, name):  # noqa: F811
    """The largest sums of a product of this length, multipliers that saturate or
    vanish, and the ends of the residual's range."""
    T, K, N = R.PRODUCTS[name][0]
    say("extremes", name)
    x = np.full((1, K), -128, np.int8)
    w = np.where(np.arange(N)[:, None] % 2, -128, 127).astype(np.int8) * np.ones((1, K), np.int8)
    f = np.where(np.arange(N) % 2, 2 ** 30, -2 ** 30).astype(np.int32)
    table = np.linspace(-200, 200, 4096).astype(np.float32)
    for m in (np.finfo(np.float32).max, 0.0, 2.0 ** -24, 2.0 ** -40):
        mul = np.full(N, m, np.float32)
        for kw in ({}, dict(relu=True), dict(table=table, zp_t=4095)):
            check(fq, T, x, w, f, mul, zp_y=3, **kw)
            for r, zp_r, mul_r in ((127, -128, 2.0 ** 20), (-128, 127, 2.0 ** 20), (127, 0, 2.0 ** -20)):
                check(fq, T, x, w, f, mul, zp_y=3, residual=np.full((1, N), r, np.int8), zp_r=zp_r,
                      mul_r=mul_r, **kw)


@pytest.mark.parametrize("name", R.KERNELS)
@pytest.mark.parametrize("table_bits", [4, 8, 9, 10, 12])
def test_tables_in_every_kernel(fq, name, table_bits):  # noqa: F811
    """Tables that no two entries of are alike, their indices spread over the whole
    and past both ends."""
    T, K, N = R.PRODUCTS[name][0]
    say("table", name, table_bits)
    size = 1 << table_bits
    p = R.layer(min(T, PERIOD), K, N, seed=table_bits)
    # the sums' spread is 1.5 (R.layer), the table reaches over 3 of it
    f, m = R.fold(p["w"], p["s_w"], p["s_x"], 9.0 / size, 0, p["bias"])
    table = np.random.default_rng(size).permutation(np.linspace(-127, 127, size)).astype(np.float32)
    at = np.rint(R.f32(R.sums(p["x"], p["w"], f)) * m + size // 2)
    assert (at < 0).any() and (at >= size).any()
    assert at.size < 40 * size or len(np.unique(np.clip(at, 0, size - 1))) > size * 0.99 - 1
    check(fq, T, p["x"], p["w"], f, m, zp_y=-2, table=table, zp_t=size // 2)
    r = np.random.default_rng(N).integers(-128, 128, (len(p["x"]), N)).astype(np.int8)
    check(fq, T, p["x"], p["w"], f, m, zp_y=-2, table=table, zp_t=size // 2, residual=r, mul_r=0.3)


def shifted(a, n):
    """A copy of `a` on a base n elements off a 256-byte boundary."""
    import torch
    t = dev(a)
    buf = torch.zeros(t.numel() + 64, dtype=t.dtype, device=t.device)
    view = buf[n:n + t.numel()].view(t.shape)
    view.copy_(t)
    return view


@pytest.mark.parametrize("name", R.KERNELS)
@pytest.mark.parametrize("n,byte", [(1, 1), (2, 6), (3, 15)])
def test_vectors_and_residuals_of_the_least_alignment(fq, name, n, byte):  # noqa: F811
    """fold, mul and the table on 4-byte boundaries, the residual on any; x and w stay
    on their own, so that the kernel does."""
    T, K, N = R.PRODUCTS[name][0]
    say("alignment", name, n, byte)
    p = R.layer(min(T, PERIOD), K, N, seed=n)
    f, m = R.fold(p["w"], p["s_w"], p["s_x"], 9.0 / 256, 0, p["bias"])
    table = np.random.default_rng(n).normal(0, 60, 256).astype(np.float32)
    r = np.random.default_rng(N).integers(-128, 128, (len(p["x"]), N)).astype(np.int8)
    x, w, res = dev(repeated(p["x"], T)), dev(p["w"]), unaligned(repeated(r, T), byte)
    fd, md, td = shifted(f, n), shifted(m, n), shifted(table, n)
    assert fd.data_ptr() % 16 == md.data_ptr() % 16 == td.data_ptr() % 16 == 4 * n
    for kw in ({}, dict(table=table, zp_t=128)):
        got = fq.linear_int8(x, w, fd, md, table=td if kw else None, zp_t=128, residual=res, mul_r=0.4)
        assert np.array_equal(host(got), repeated(R.linear(p["x"], p["w"], f, m, residual=r, mul_r=0.4, **kw), T))
    assert np.array_equal(host(fq.linear_int32(x, w, fd)), repeated(R.sums(p["x"], p["w"], f), T))
