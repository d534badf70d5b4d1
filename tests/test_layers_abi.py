"""Refusals of the linear layers, the rotary positions and the heads' way back
to rows, in the C ABI and in the binding, and the constants that the host
derives.  Every call here fails its checks, is empty, or runs against a host
build whose launchers only keep their arguments (built with AddressSanitizer
and UndefinedBehaviorSanitizer where the environment variable names one)."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2111_13824_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SAN_LIB = os.environ.get("FQVIT_LAYER_TEST_LIB")


def host_library(out, flags=()):
    csrc = os.path.join(ROOT, "paper_2111_13824_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", *flags, "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "fqvit_abi.cpp"), os.path.join(HERE, "abi_launch_stubs.cpp"),
                    os.path.join(HERE, "layer_launch_stubs.cpp"), "-o", out], check=True)
    return out


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return B.load(SAN_LIB or host_library(str(tmp_path_factory.mktemp("host") / "libhost.so")))


def caller(lib, name, **defaults):
    """call(**changes): the entry point with its arguments, some changed, and
    whether it reached its launcher."""
    def call(**kw):
        assert set(kw) <= set(defaults), kw
        n = lib.fq_test_layer_calls()
        rc = getattr(lib, name)(*dict(defaults, **kw).values(), None)
        return rc, lib.fq_test_layer_calls() - n
    return call


RAN, EMPTY = (B.FQ_OK, 1), (B.FQ_OK, 0)
NULL, SHAPE, PARAM = (B.FQ_ERR_NULL, 0), (B.FQ_ERR_SHAPE, 0), (B.FQ_ERR_PARAM, 0)


def test_fold_refusals(lib):
    call = caller(lib, "linear_fold_int8", w=1, N=8, K=16, s_w=1, bias=None, zp=0, s_x=0.5, s_y=0.5,
                  fold=1, mul=1)
    assert call() == RAN and call(bias=1) == RAN and call(K=32768, N=1 << 20) == RAN
    assert call(mul=None, s_y=0.0) == RAN           # without multipliers the step is unused
    for k, v in (("N", 0), ("N", (1 << 20) + 1), ("K", 0), ("K", 32769), ("N", -1)):
        assert call(**{k: v}) == SHAPE
    for k, v in (("zp", 128), ("zp", -129), ("s_x", 0.0), ("s_x", float("inf")), ("s_y", -1.0),
                 ("s_y", float("nan"))):
        assert call(**{k: v}) == PARAM
    for k in ("w", "s_w", "fold"):
        assert call(**{k: None}) == NULL


def test_linear_refusals(lib):
    call = caller(lib, "linear_int8", x=1, T=4, w=1, N=8, K=16, fold=1, mul=1, act=0, table=None,
                  tbits=0, zp_t=0, res=None, zp_r=0, mul_r=1.0, zp=0, bits=8, y=1)
    assert call() == RAN and call(fold=None) == RAN and call(act=1) == RAN
    assert call(act=2, table=1, tbits=4, zp_t=15) == RAN and call(res=1, zp_r=-128) == RAN
    assert call(T=0, x=None, y=None) == EMPTY
    # what is not used is not looked at
    assert call(tbits=99, zp_t=-5, zp_r=1000, mul_r=0.0) == RAN
    for k, v in (("T", -1), ("N", 0), ("K", 0), ("K", 32769), ("N", (1 << 20) + 1), ("T", 1 << 41)):
        assert call(**{k: v}) == SHAPE
    # fewer than 2^24 tiles of 64 x 64
    assert call(T=(1 << 30) - 64, N=64) == RAN and call(T=(1 << 30) - 63, N=64) == SHAPE
    assert call(T=1 << 24, N=1 << 20) == SHAPE
    for k, v in (("act", 3), ("act", -1), ("bits", 1), ("bits", 9), ("zp", 128), ("zp", -129)):
        assert call(**{k: v}) == PARAM
    assert call(bits=4, zp=8) == PARAM
    for k, v in (("tbits", 3), ("tbits", 13), ("zp_t", -1), ("zp_t", 16)):
        assert call(**dict(dict(act=2, table=1, tbits=4), **{k: v})) == PARAM
    for k, v in (("zp_r", 128), ("zp_r", -129), ("mul_r", 0.0), ("mul_r", float("nan")),
                 ("mul_r", 2.0 ** 21), ("mul_r", -1.0)):
        assert call(res=1, **{k: v}) == PARAM
    for k in ("x", "w", "mul", "y"):
        assert call(**{k: None}) == NULL
    assert call(act=2, tbits=4) == NULL


def test_linear_int32_refusals(lib):
    call = caller(lib, "linear_int32", x=1, T=4, w=1, N=8, K=16, fold=1, out=1)
    assert call() == RAN and call(fold=None) == RAN and call(T=0, x=None) == EMPTY
    for k, v in (("T", -1), ("N", 0), ("K", 0), ("K", 32769)):
        assert call(**{k: v}) == SHAPE
    for k in ("x", "w", "out"):
        assert call(**{k: None}) == NULL


def test_products_of_the_gpu_tests_reach_every_kernel(lib):
    import layer_cases as R
    assert set(R.PRODUCTS) == set(R.KERNELS)
    call = caller(lib, "linear_int32", x=16, T=1, w=16, N=1, K=1, fold=None, out=1)
    for name, products in R.PRODUCTS.items():
        for T, K, N in products:
            assert call(T=T, K=K, N=N) == RAN
            assert R.KERNELS[lib.fq_test_linear_kernel()] == name, (name, T, K, N)
    # rows of whole units on other bases take the register path
    for x, w in ((20, 16), (16, 24)):
        call(T=1000, K=64, N=1000, x=x, w=w)
        assert R.KERNELS[lib.fq_test_linear_kernel()] == "tile64r"


def test_wide_products_of_few_rows_take_tiles(lib):
    """9 to 32 rows of products whose channels come to several workgroups of few rows a CU
    take one line of tiles (32 x 1024 x 32768: 9.5 us, 16.5 in the kernel of 32 rows); narrow
    ones, and up to 8 rows all, do not."""
    import layer_cases as R
    call = caller(lib, "linear_int8", x=16, T=1, w=16, N=1, K=1, fold=None, mul=16, act=0, table=None,
                  tbits=0, zp_t=0, res=None, zp_r=0, mul_r=1.0, zp=0, bits=8, y=1)

    def kernel(T, K, N):
        assert call(T=T, K=K, N=N) == RAN
        return R.KERNELS[lib.fq_test_linear_kernel()]

    for T, K, N in R.WIDE:
        assert kernel(T, K, N) == ("tile64" if K % 16 == 0 else "tile64r"), (T, K, N)
    for T in (17, 24, 32):
        for K in (768, 1024, 2048, 4096):
            for N in (1024, 4096, 8192):
                assert kernel(T, K, N) in ("rows16", "rows32"), (T, K, N)
            for N in (16384, 32768, 65536):
                assert kernel(T, K, N) == "tile64", (T, K, N)
            assert kernel(T, K + 1, 32769) == "tile64r"
    for T in (1, 2, 8):
        for N in (1, 4096, 65536, 1 << 20):
            assert kernel(T, 1024, N) == kernel(T, 1001, N) == "rows16"


def test_edges_of_the_gpu_tests_are_those_of_the_tiles(lib):
    """Each product of EDGES takes its kernel, and each kernel's reach the edges of its
    tiles: rows and channels of whole tiles, one less and one more."""
    import layer_cases as R
    assert set(R.EDGES) == set(R.KERNELS) - {"rows16", "rows32"}
    call = caller(lib, "linear_int32", x=16, T=1, w=16, N=1, K=1, fold=None, out=1)
    for name, products in R.EDGES.items():
        bn, bt, _ = WORKGROUPS[name]
        for T, K, N in products:
            assert call(T=T, K=K, N=N) == RAN
            assert R.KERNELS[lib.fq_test_linear_kernel()] == name, (name, T, K, N)
        assert {T % bt for T, _, _ in products} >= {0, 1, bt - 1}, name
        assert {N % bn for _, _, N in products} >= {0, 1, bn - 1}, name
        # ends inside a unit of 16, and on one
        assert {N % 16 for _, _, N in products} >= {0, 1, 15}, name


# channels, rows and threads of a workgroup
WORKGROUPS = dict(rows16=(16, 16, 512), rows32=(16, 32, 512), tile64=(64, 64, 256), tile128=(128, 128, 256),
                  tile256x128=(256, 128, 512), tile256x192=(256, 192, 512), tile256x256=(256, 256, 512),
                  tile256x320=(256, 320, 512), tile64r=(64, 64, 256), tile128r=(128, 128, 256),
                  tile256r=(256, 256, 512))


@pytest.mark.parametrize("x", [16, 17])
def test_no_launch_has_more_threads_than_the_hardware_takes(lib, x):
    """The sizes that the entry points allow, up to their limits: fewer than 2^32
    threads a launch, in whichever kernel the product takes."""
    import layer_cases as R
    call = caller(lib, "linear_int32", x=x, T=1, w=16, N=1, K=16, fold=None, out=1)
    for N in (1, 64, 65, 128, 192, 256, 257, 1000, 4096, 1 << 16, 1 << 20):
        most = ((1 << 24) - 1) // (-(-N // 64)) * 64
        for T in (most, most - 63, most - 64, most // 2, most // 2 + 1, most // 64, 17, 16):
            for K in (16, 128, 4096, 32768):
                assert call(T=T, N=N, K=K) == RAN
                bn, bt, threads = WORKGROUPS[R.KERNELS[lib.fq_test_linear_kernel()]]
                assert -(-N // bn) * -(-T // bt) * threads < 1 << 32, (T, K, N)


def test_rope_refusals(lib):
    call = caller(lib, "rope_table_int16", pos=1, axes=3, T=5, freq=1, axis=1, P=4, table=4)
    assert call() == RAN and call(T=0, pos=None) == EMPTY and call(T=1 << 25, P=128) == RAN
    for k, v in (("axes", 0), ("axes", 9), ("T", -1), ("T", (1 << 25) + 1), ("P", 0), ("P", 129)):
        assert call(**{k: v}) == SHAPE
    assert call(table=2) == PARAM
    for k in ("pos", "freq", "axis", "table"):
        assert call(**{k: None}) == NULL

    call = caller(lib, "rope_qkv_int8", qkv=1, B=2, L=5, Hq=4, Hkv=2, d=64, s_x=0.5, zp_x=0, table=4,
                  rows=5, P=32, il=0, s_q=0.5, zp_q=0, s_k=0.5, zp_k=0, bits=8, q=1, k=1, v=1)
    assert call() == RAN and call(rows=10, il=1) == RAN and call(P=0, table=None, rows=0) == RAN
    assert call(B=0, qkv=None) == EMPTY and call(L=0, rows=0, q=None) == EMPTY
    assert call(B=1 << 20, L=32, rows=32) == RAN and call(B=(1 << 20) + 1, L=32, rows=32) == SHAPE
    for k, v in (("B", -1), ("L", -1), ("Hq", 0), ("Hkv", 0), ("Hq", 1025), ("d", 0), ("d", 257),
                 ("P", -1), ("P", 33), ("rows", 4), ("rows", 6), ("rows", 20), ("B", 1 << 40)):
        assert call(**{k: v}) == SHAPE, (k, v)
    for k, v in (("il", 2), ("bits", 1), ("bits", 9), ("zp_x", 128), ("zp_q", 128), ("zp_k", -129),
                 ("s_x", 0.0), ("s_q", float("nan")), ("s_k", float("inf")), ("table", 6)):
        assert call(**{k: v}) == PARAM, (k, v)
    assert call(bits=4, zp_q=8) == PARAM and call(bits=4, zp_k=-9) == PARAM
    for k in ("qkv", "q", "k", "v", "table"):
        assert call(**{k: None}) == NULL


def test_requant_heads_refusals(lib):
    call = caller(lib, "requant_heads_int8", q=1, B=2, H=3, L=5, d=64, si=0.5, so=0.25, zp=0, bits=8,
                  y=1)
    assert call() == RAN and call(B=0, q=None) == EMPTY and call(L=0, y=None) == EMPTY
    for k, v in (("B", -1), ("H", 0), ("H", 1025), ("L", -1), ("d", 0), ("d", 257), ("B", 1 << 40)):
        assert call(**{k: v}) == SHAPE
    for k, v in (("si", 0.0), ("so", float("inf")), ("bits", 1), ("bits", 9), ("zp", 128)):
        assert call(**{k: v}) == PARAM
    assert call(q=None) == NULL and call(y=None) == NULL


def test_derived_constants(lib):
    """add_r and the rotation's multipliers, rounded once; the dyadic form."""
    f, i = np.zeros(3, np.float32), np.zeros(3, np.int64)
    for zp_r, mul_r, zp in ((0, 0.3, 0), (-128, 7.0, 5), (127, 2.0 ** -20 * 1.3, -128)):
        assert caller(lib, "linear_int8", x=1, T=4, w=1, N=8, K=16, fold=1, mul=1, act=0, table=None,
                      tbits=0, zp_t=0, res=1, zp_r=zp_r, mul_r=mul_r, zp=zp, bits=8, y=1)() == RAN
        lib.fq_test_multipliers(f.ctypes.data_as(ctypes.c_void_p))
        assert f[0] == np.float32(zp - (128 + zp_r) * float(np.float32(mul_r)))
    rope = caller(lib, "rope_qkv_int8", qkv=1, B=2, L=5, Hq=4, Hkv=2, d=64, s_x=0.05, zp_x=0, table=4,
                  rows=5, P=32, il=0, s_q=0.07, zp_q=0, s_k=1e-38, zp_k=0, bits=8, q=1, k=1, v=1)
    assert rope(s_x=3e38) == RAN                    # the ratio leaves binary32
    lib.fq_test_multipliers(f.ctypes.data_as(ctypes.c_void_p))
    assert f[2] == np.finfo(np.float32).max
    assert rope(rows=10) == RAN
    lib.fq_test_multipliers(f.ctypes.data_as(ctypes.c_void_p))
    lib.fq_test_integers(i.ctypes.data_as(ctypes.c_void_p))
    assert f[1] == np.float32(float(np.float32(0.05)) / (16384 * float(np.float32(0.07))))
    assert i[2] == 1
    assert caller(lib, "requant_heads_int8", q=1, B=2, H=3, L=5, d=64, si=0.75, so=1.0, zp=0, bits=8,
                  y=1)() == RAN
    lib.fq_test_integers(i.ctypes.data_as(ctypes.c_void_p))
    assert (i[0], i[1]) == (3 << 29, 31)


def test_a_build_without_the_kernels_says_so(tmp_path):
    """The host code alone loads; a call that needs a missing kernel returns a
    status instead of ending the process."""
    csrc = os.path.join(ROOT, "paper_2111_13824_amd", "csrc")
    out = str(tmp_path / "libalone.so")
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "fqvit_abi.cpp"), os.path.join(HERE, "abi_launch_stubs.cpp"),
                    "-o", out], check=True)
    alone = B.load(out)
    assert alone.linear_int32(1, 4, 1, 8, 16, None, 1, None) == B.FQ_ERR_HIP
    assert alone.rope_table_int16(1, 1, 5, 1, 1, 4, 4, None) == B.FQ_ERR_HIP


def test_activation_tables(lib):
    from math import erf, exp, tanh, pi, sqrt
    f = {0: lambda t: t * (1 + erf(t / sqrt(2))) / 2,
         1: lambda t: t * (1 + tanh(sqrt(2 / pi) * (t + 0.044715 * t ** 3))) / 2,
         2: lambda t: t / (1 + exp(-t))}
    for kind in f:
        for bits, zp, s_t, s_y in ((4, 0, 0.5, 0.25), (10, 512, 1 / 64, 0.05), (12, 4095, 0.004, 1e-3)):
            table = np.zeros((1 << bits) + 1, np.float32)
            assert lib.fq_activation_table(kind, s_t, zp, bits, s_y, table.ctypes.data) == B.FQ_OK
            t = float(np.float32(s_t)) * (np.arange(1 << bits) - zp)
            ref = np.array([f[kind](v) for v in t]) / float(np.float32(s_y))
            # rounding to binary32 (half a step) and a few roundings in binary64;
            # 1 + erf and 1 + tanh cancel below 0, to within t 2^-53 / s_y
            assert np.all(np.abs(table[:-1] - ref) <= np.abs(ref) * 2.0 ** -24 * 1.01 +
                          np.abs(t) * 2.0 ** -50 / s_y + 2.0 ** -149)
            assert table[-1] == 0
    table = np.zeros(16, np.float32)
    assert lib.fq_activation_table(2, 1e4, 8, 4, 1.0, table.ctypes.data) == B.FQ_OK
    assert np.all(table[:9] == 0) and table[9] == 1e4   # far below 0 SiLU is 0
    for args in ((3, 1.0, 0, 4, 1.0), (-1, 1.0, 0, 4, 1.0), (0, 0.0, 0, 4, 1.0), (0, 1.0, 16, 4, 1.0),
                 (0, 1.0, -1, 4, 1.0), (0, 1.0, 0, 3, 1.0), (0, 1.0, 0, 13, 1.0),
                 (0, 1.0, 0, 4, float("nan")), (0, 3e38, 0, 4, 1e-3)):
        assert lib.fq_activation_table(*args, table.ctypes.data) == B.FQ_ERR_PARAM
    assert lib.fq_activation_table(0, 1.0, 0, 4, 1.0, None) == B.FQ_ERR_NULL


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_activation_tables_beyond_binary32(lib, kind):
    """A table whose ends are small and whose middle, near the function's
    extremum below 0, is beyond binary32 in steps of the output; one whose end
    is; and the largest that fit.  A refused table is left as it was."""
    table = np.full(4096, 7, np.float32)
    for s_t, zp, s_y in ((0.01, 4095, 1e-42), (0.01, 0, 1e-42), (0.01, 4095, 2.0 ** -131)):
        assert lib.fq_activation_table(kind, s_t, zp, 12, s_y, table.ctypes.data) == B.FQ_ERR_PARAM
        assert (table == 7).all()
    # the extrema are -0.17 and -0.28: in steps of 2^-129 below 2^128
    assert lib.fq_activation_table(kind, 0.01, 4095, 12, 2.0 ** -129, table.ctypes.data) == B.FQ_OK
    assert np.isfinite(table).all() and table.min() < -2.0 ** 126
    # exactly the largest finite value: f(t) = t far above 0
    big = float(np.finfo(np.float32).max)
    assert lib.fq_activation_table(kind, big / 4, 11, 4, 1.0, table.ctypes.data) == B.FQ_OK
    assert np.isfinite(table).all() and table[15] == np.float32(big)


@pytest.mark.skipif(bool(SAN_LIB), reason="needs torch, which the sanitizer run leaves out")
def test_binding_refusals(lib, monkeypatch):
    """Dtypes, shapes and layouts, then the device."""
    torch = pytest.importorskip("torch")
    import paper_2111_13824_amd as fq
    monkeypatch.setattr(B, "_lib", lib)
    i8, f32, i32 = torch.int8, torch.float32, torch.int32
    z = lambda *shape, dtype=i8: torch.zeros(*shape, dtype=dtype)
    x, w, fold, mul = z(4, 8), z(3, 8), z(3, dtype=i32), z(3, dtype=f32)
    for call in (lambda: fq.linear_int8(x, w, fold, mul), lambda: fq.linear_int32(x, w),
                 lambda: fq.linear_fold_int8(w, mul, 1.0),
                 lambda: fq.rope_table_int16(z(3, 5, dtype=i32), z(4, dtype=torch.float64),
                                             z(4, dtype=torch.uint8)),
                 lambda: fq.rope_qkv_int8(z(2, 5, 32), None, 2, 1, 1.0, 1.0, 1.0),
                 lambda: fq.requant_heads_int8(z(2, 3, 5, 8, dtype=i32), 1.0, 1.0, 0)):
        with pytest.raises(ValueError, match="device tensor"):
            call()
    with pytest.raises(TypeError, match="x must be torch.int8"):
        fq.linear_int8(x.float(), w, fold, mul)
    with pytest.raises(TypeError, match="mul must be a torch.Tensor"):
        fq.linear_int8(x, w, fold, [1.0, 2.0, 3.0])
    with pytest.raises(ValueError, match="x must have 2 dimensions"):
        fq.linear_int8(x[0], w, fold, mul)
    with pytest.raises(ValueError, match=r"w must be \[3, 8\], got \[3, 7\]"):
        fq.linear_int8(x, w[:, :7].contiguous(), fold, mul)
    with pytest.raises(ValueError, match="x must be contiguous"):
        fq.linear_int8(z(8, 4).t(), w, fold, mul)
    with pytest.raises(ValueError, match=r"fold must be \[3\]"):
        fq.linear_int8(x, w, fold[:2], mul)
    with pytest.raises(ValueError, match=r"residual must be \[4, 3\]"):
        fq.linear_int8(x, w, fold, mul, residual=x)
    with pytest.raises(ValueError, match=r"y must be \[4, 3\]"):
        fq.linear_int8(x, w, fold, mul, y=x)
    with pytest.raises(ValueError, match="not both"):
        fq.linear_int8(x, w, fold, mul, relu=True, table=z(16, dtype=f32))
    with pytest.raises(ValueError, match="power of two"):
        fq.linear_int8(x, w, fold, mul, table=z(17, dtype=f32))
    with pytest.raises(ValueError, match=r"table must be \[16\]"):
        fq.linear_int8(x, w, fold, mul, table=z(4, 4, dtype=f32))
    with pytest.raises(ValueError, match=r"out must be \[4, 3\]"):
        fq.linear_int32(x, w, fold, out=z(4, 4, dtype=i32))
    with pytest.raises(ValueError, match=r"s_w must be \[3\]"):
        fq.linear_fold_int8(w, z(4, dtype=f32), 1.0)
    with pytest.raises(ValueError, match="kind"):
        fq.activation_table("tan", 1.0, 1.0, device="cpu")
    with pytest.raises(ValueError, match="table_bits"):
        fq.activation_table("gelu", 1.0, 1.0, table_bits=20, device="cpu")
    with pytest.raises(B.FqError):
        fq.activation_table("gelu", 0.0, 1.0, device="cpu")
    assert fq.activation_table("silu", 0.5, 1.0, device="cpu")[512] == 0
    with pytest.raises(ValueError, match=r"axis must be \[4\]"):
        fq.rope_table_int16(z(3, 5, dtype=i32), z(4, dtype=torch.float64), z(3, dtype=torch.uint8))
    qkv, table = z(2, 5, 32), z(5, 4, 2, dtype=torch.int16)
    with pytest.raises(ValueError, match="qkv must be"):
        fq.rope_qkv_int8(qkv, table, 3, 1, 1.0, 1.0, 1.0)
    with pytest.raises(ValueError, match=r"table must be \[5, 4, 2\]"):
        fq.rope_qkv_int8(qkv, table[..., :1], 2, 1, 1.0, 1.0, 1.0)
    with pytest.raises(ValueError, match=r"q must be \[2, 2, 5, 8\]"):
        fq.rope_qkv_int8(qkv, table, 2, 1, 1.0, 1.0, 1.0, q=z(2, 2, 5, 9))
    with pytest.raises(ValueError, match=r"y must be \[2, 5, 24\]"):
        fq.requant_heads_int8(z(2, 3, 5, 8, dtype=i32), 1.0, 1.0, 0, y=z(2, 5, 25))


def test_the_binding_cuts_no_integer(lib, monkeypatch):
    """ctypes keeps the low 32 bits of an integer: a row of 2^32 + 16 inputs would
    be a row of 16.  Sizes and scalars beyond 32 bits are refused, in every entry
    point, and reach no launcher; the ends of the range go through."""
    monkeypatch.setattr(B, "_lib", lib)
    good = (16, 1, 16, 3, 16, None, 16, 0)             # x, T, w, N, K, fold, out, stream
    n = lib.fq_test_layer_calls()
    for prepare in (False, True):
        for at in (3, 4):
            for bad in (2 ** 32 + 16, -2 ** 32 + 16, 2 ** 31, -2 ** 31 - 1, 2 ** 70):
                args = (*good[:at], bad, *good[at + 1:])
                with pytest.raises(ValueError, match="32-bit"):
                    B._invoke("linear_int32", args, (), prepare, None)
        for end in (2 ** 31 - 1, -2 ** 31):
            with pytest.raises(B.FqError):
                call = B._invoke("linear_int32", (*good[:3], end, *good[4:]), (), prepare, None)
                call()
    assert lib.fq_test_layer_calls() == n
    B._invoke("linear_int32", good, (), False, None)
    assert lib.fq_test_layer_calls() == n + 1
    for name, types in B.SIGNATURES.items():
        narrow = [i for i, t in enumerate(types) if t is ctypes.c_int32]
        assert len(narrow) > 1
        for at in narrow:
            args = [2 ** 32 + 1 if i == at else 1 for i in range(len(types))]
            with pytest.raises(ValueError, match="32-bit"):
                B._narrow(name, args)
    # what is no integer is left to ctypes
    with pytest.raises(ctypes.ArgumentError):
        B._invoke("linear_int32", (*good[:3], 3.0, *good[4:]), (), False, None)
    if SAN_LIB:                                        # that run leaves torch out
        return
    pytest.importorskip("torch")
    import paper_2111_13824_amd as fq
    with pytest.raises(ValueError, match="32-bit"):
        fq.activation_table("gelu", 1.0, 1.0, zp_t=2 ** 32 + 8, table_bits=4, device="cpu")


@pytest.mark.skipif(bool(SAN_LIB), reason="this is the run that starts it")
def test_host_code_under_sanitizers(tmp_path):
    from test_sanitizers import SAN, _env
    env = _env({"FQVIT_LAYER_TEST_LIB": host_library(str(tmp_path / "libsan.so"), SAN)})
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-s", "-p",
                        "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert r.returncode == 0 and " passed" in out, out[-4000:]
