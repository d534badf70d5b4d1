"""Refusals of the step over a stream of tokens (norm, cache, attention, eviction), in
the C ABI and in the binding.  Every call here fails its checks, is empty, or runs
against a host build whose launchers only keep their arguments (built with
AddressSanitizer and UndefinedBehaviorSanitizer where the environment variable names
one).  The plain forms of the other tests are held to the oracle here."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from paper_2111_13824_amd import binding as B
from test_layers_abi import EMPTY, NULL, PARAM, RAN, SHAPE, caller

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
SAN_LIB = os.environ.get("FQVIT_DECODE_TEST_LIB")
BIG = 2 ** 31 - 1
HEADROOM = (B.FQ_ERR_HEADROOM, 0)


def host_library(out, flags=()):
    csrc = os.path.join(ROOT, "paper_2111_13824_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", *flags, "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "fqvit_abi.cpp"), os.path.join(HERE, "abi_launch_stubs.cpp"),
                    os.path.join(HERE, "decode_launch_stubs.cpp"), "-o", out], check=True)
    return out


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return B.load(SAN_LIB or host_library(str(tmp_path_factory.mktemp("host") / "libhost.so")))


NORM = dict(x=1, zp_x=0, alpha=1, K=3, m_x=1.0, r=1, T=4, C=8, gamma=1, eps=1.0)


def test_norm_refusals(lib):
    one = caller(lib, "rmsnorm_int8", **NORM, s_out=0.5, zp=0, bits=8, h=1, y=1)
    rows = caller(lib, "rmsnorm_rows_int8", **NORM, bits=8, h=1, y=1, scales=1)
    for call in (one, rows):
        assert call() == RAN and call(T=(1 << 24) - 1, C=8192) == RAN and call(alpha=None, K=99) == RAN
        # without a branch nothing of it is looked at
        assert call(x=None, zp_x=999, K=-1, m_x=0.0) == RAN
        assert call(T=0, r=None, y=None) == EMPTY
        for k, v in (("T", -1), ("T", 1 << 24), ("C", 0), ("C", 8193)):
            assert call(**{k: v}) == SHAPE
        for k, v in (("bits", 1), ("bits", 9), ("eps", -1.0), ("eps", float("nan")), ("eps", float("inf")),
                     ("zp_x", 128), ("zp_x", -129), ("m_x", 0.0), ("m_x", 64.5), ("m_x", float("nan")),
                     ("K", -1), ("K", 8)):
            assert call(**{k: v}) == PARAM
        for k in ("r", "gamma", "h", "y"):
            assert call(**{k: None}) == NULL
    for k, v in (("s_out", 0.0), ("s_out", float("inf")), ("zp", 128), ("zp", -129)):
        assert one(**{k: v}) == PARAM
    assert one(bits=4, zp=8) == PARAM and rows(scales=None) == NULL
    ints = (ctypes.c_longlong * 3)()
    one(x=None)
    lib.fq_test_integers(ints)
    assert ints[2] == 0


def cache_refusals(call):
    for k, v in (("pages", 0), ("pages", (1 << 30) + 1), ("page", 8), ("page", 48), ("page", 2048),
                 ("max_pages", 0), ("max_pages", (1 << 16) + 1), ("B", -1), ("Hkv", 0), ("Hkv", 1025),
                 ("B", 32769), ("d", 8), ("d", 72), ("d", 144), ("d", 0), ("d", -16), ("page", -16)):
        assert call(**{k: v}) == SHAPE, (k, v)
    for k in ("k_pages", "v_pages"):
        assert call(**{k: 8}) == PARAM and call(**{k: None}) == NULL
    assert call(weight=4) == PARAM
    for k in ("table", "length"):
        assert call(**{k: None}) == NULL


def test_append_refusals(lib):
    call = caller(lib, "kv_cache_append_int8", k=16, v=16, B=3, Hkv=2, L=5, d=64, n_new=None, k_pages=16,
                  v_pages=16, weight=None, pages=9, page=16, table=4, max_pages=4, length=4)
    assert call() == RAN and call(weight=8, n_new=4, d=128, page=1024) == RAN
    assert call(B=0, k=None) == EMPTY and call(L=0, v=None) == EMPTY
    cache_refusals(call)
    assert call(L=-1) == SHAPE and call(L=(1 << 20) + 1) == SHAPE
    assert call(B=1024, Hkv=64, L=64 * 254 - 1) == RAN and call(B=1024, Hkv=64, L=64 * 254) == SHAPE
    for k in ("k", "v"):
        assert call(**{k: 8}) == PARAM and call(**{k: None}) == NULL


ATTEND = dict(q=16, B=3, Hq=4, Hkv=2, L=5, d=64, n_new=None, k_pages=16, v_pages=16, weight=None, pages=9,
              page=16, table=4, max_pages=4, length=4, zp_q=0, zp_k=0, zp_v=0, causal=1, s=2.0 ** -10,
              bits=4, n=20, out=16, ws=None, size=0)


def test_attention_refusals(lib):
    call = caller(lib, "lis_attention_paged", **ATTEND)
    assert call() == RAN and call(weight=8, n_new=4, causal=0, bits=1) == RAN
    assert call(B=0, q=None) == EMPTY and call(L=0, out=None) == EMPTY
    cache_refusals(call)
    for k, v in (("L", -1), ("L", (1 << 20) + 1), ("Hq", 5), ("Hq", 0), ("Hq", 1026)):
        assert call(**{k: v}) == SHAPE
    # fewer than 2^24 workgroups of 16 rows; a tile more than the rows fill is counted
    assert call(B=1, Hq=1024, Hkv=1, L=1 << 20) == SHAPE and call(B=3, Hq=2, L=1 << 20) == RAN
    for k, v in (("zp_q", 128), ("zp_k", -129), ("zp_v", 300), ("causal", 2), ("bits", 0), ("bits", 5),
                 ("n", 0), ("n", 31), ("s", 0.0), ("s", 0.6), ("s", float("nan")), ("q", 8), ("out", 8)):
        assert call(**{k: v}) == PARAM, (k, v)
    for k in ("q", "out"):
        assert call(**{k: None}) == NULL
    # the sum of 2^20 keys at this depth leaves 64 bits
    assert call(n=30, max_pages=1 << 16) == HEADROOM and call(n=20, max_pages=1 << 16) == RAN
    # the workspace: there, large enough, aligned
    assert call(L=7) == NULL and call(L=7, ws=16, size=95) == PARAM and call(L=7, ws=8, size=96) == PARAM
    assert call(L=7, ws=16, size=96) == RAN
    need = lib.fq_lis_attention_paged_workspace_bytes
    assert need(3, 4, 2, 7, 64, 64) == 96 and need(3, 4, 2, 5, 64, 64) == 0
    assert need(0, 4, 2, 7, 64, 64) == need(3, 5, 2, 7, 64, 64) == need(3, 4, 2, 7, 64, 1 << 21) == 0
    ints = (ctypes.c_longlong * 3)()
    call(Hq=6, page=64)
    lib.fq_test_integers(ints)
    assert (ints[0], ints[1]) == (3, 6)


def test_evict_refusals(lib):
    call = caller(lib, "kv_cache_evict", k_pages=16, v_pages=16, weight=8, pages=9, Hkv=2, page=16, d=64,
                  table=4, max_pages=4, length=4, B=3, keep=20, recent=4, table_out=8, max_out=2,
                  length_out=4, kept=4)
    assert call() == RAN and call(recent=0) == RAN and call(recent=20) == RAN
    assert call(table_out=4, max_out=4) == RAN and call(table_out=4, max_out=3) == SHAPE
    assert call(B=0, kept=None) == EMPTY
    cache_refusals(call)
    for k, v in (("keep", 0), ("keep", -1), ("keep", 33), ("keep", (1 << 20) + 1), ("max_out", 0),
                 ("max_out", 1), ("max_out", 1 << 17)):
        assert call(**{k: v}) == SHAPE, (k, v)
    assert call(recent=21) == PARAM and call(recent=-1) == PARAM
    for k in ("weight", "table_out", "length_out", "kept"):
        assert call(**{k: None}) == NULL


def test_a_build_without_the_kernels_says_so(tmp_path):
    csrc = os.path.join(ROOT, "paper_2111_13824_amd", "csrc")
    out = str(tmp_path / "libalone.so")
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "fqvit_abi.cpp"), os.path.join(HERE, "abi_launch_stubs.cpp"),
                    "-o", out], check=True)
    alone = B.load(out)
    assert alone.lis_attention_paged(*ATTEND.values(), None) == B.FQ_ERR_HIP
    assert alone.fq_lis_attention_paged_workspace_bytes(3, 4, 2, 7, 64, 64) == 0


def test_the_binding_cuts_no_integer(lib):
    for name, types in B.DECODE_SIGNATURES.items():
        narrow = [i for i, t in enumerate(types) if t is ctypes.c_int32]
        for at in narrow:
            with pytest.raises(ValueError, match="32-bit"):
                B._narrow(name, [2 ** 32 + 1 if i == at else 1 for i in range(len(types))])


def test_the_binding_refuses():
    if SAN_LIB:
        return
    torch = pytest.importorskip("torch")
    import paper_2111_13824_amd as fq
    i8, i16, i32, i64 = torch.int8, torch.int16, torch.int32, torch.int64
    z = lambda *shape, dtype=i8: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    r, gamma = z(4, 8, dtype=i16), torch.ones(8)
    with pytest.raises(ValueError, match="device tensor"):
        fq.rmsnorm_int8(r, gamma, 1.0, 1.0)
    with pytest.raises(TypeError, match="r must be torch.int16"):
        fq.rmsnorm_int8(z(4, 8), gamma, 1.0, 1.0)
    with pytest.raises(ValueError, match=r"gamma must be \[8\]"):
        fq.rmsnorm_rows_int8(r, torch.ones(7), 1.0)
    with pytest.raises(ValueError, match="give x"):
        fq.rmsnorm_int8(r, gamma, 1.0, 1.0, alpha=z(8, dtype=torch.uint8))
    with pytest.raises(ValueError, match=r"scales must be \[4\]"):
        fq.rmsnorm_rows_int8(r, gamma, 1.0, scales=torch.ones(5))
    kp, vp, w = z(5, 2, 16, 32), z(5, 2, 32, 16), z(5, 2, 16, dtype=i64)
    table, length = z(3, 4, dtype=i32), z(3, dtype=i32)
    k, q = z(3, 2, 1, 32), z(3, 4, 1, 32)
    calls = {
        "append": lambda **kw: fq.kv_cache_append_int8(**dict(dict(k=k, v=k, k_pages=kp, v_pages=vp, table=table,
                                                                   length=length), **kw)),
        "attend": lambda **kw: fq.lis_attention_paged(**dict(dict(q=q, k_pages=kp, v_pages=vp, table=table,
                                                                  length=length, s_logit=0.01,
                                                                  workspace=z(0, dtype=torch.uint8)), **kw)),
        "evict": lambda **kw: fq.kv_cache_evict(**dict(dict(k_pages=kp, v_pages=vp, weight=w, table=table,
                                                            length=length, keep=20), **kw))}
    for call in calls.values():
        with pytest.raises(ValueError, match="device tensor"):
            call()
        with pytest.raises(ValueError, match=r"v_pages must be \[5, 2, 32, 16\]"):
            call(v_pages=z(5, 2, 16, 32))
        with pytest.raises(TypeError, match="table must be torch.int32"):
            call(table=z(3, 4, dtype=i64))
        with pytest.raises(ValueError, match=r"length must be \[3\]"):
            call(length=z(2, dtype=i32))
        with pytest.raises(ValueError, match="4 dimensions"):
            call(k_pages=z(5, 2, 16))
        with pytest.raises(ValueError, match="contiguous"):
            call(v_pages=z(5, 2, 16, 32).transpose(2, 3))
        with pytest.raises(ValueError, match=r"weight must be \[5, 2, 16\]"):
            call(weight=z(5, 2, 17, dtype=i64))
    with pytest.raises(ValueError, match="hold 2 heads of 48"):
        calls["append"](k=z(3, 2, 1, 48))
    with pytest.raises(ValueError, match="heads of 48"):
        calls["attend"](q=z(3, 4, 1, 48))
    with pytest.raises(TypeError, match="weight must be"):
        calls["evict"](weight=None)
    with pytest.raises(ValueError, match=r"kept must be \[3, 2, 20\]"):
        calls["evict"](kept=z(3, 2, 21, dtype=i32))


def test_the_plain_attention_is_the_oracle_s(orc):
    """tests/decode_cases.py against lis_attention_qk of the oracle, on the keys that a
    token sees."""
    import decode_cases as R
    for case in R.ATTEND:
        c, q, length, n_new, s, more = R.attend_case(case)
        out, grown = R.attend(c, q, length, n_new, s, **more)
        n = dict(n="exp_n")
        args = {n.get(k, k): v for k, v in more.items() if k != "causal"}
        page, Hkv = case[5], case[2]
        weight = np.zeros_like(grown)
        for b in range(len(length)):
            for h in range(q.shape[1]):
                for i in range(0, n_new[b], 1 if len(length) < 3 else 3):
                    seen = length[b] - n_new[b] + i + 1 if more.get("causal", True) else length[b]
                    if not 0 < seen <= 4096:
                        assert seen > 0 or not out[b, h, i].any()
                        continue
                    p, g = np.arange(seen), h // (q.shape[1] // Hkv)
                    at, slot = c["table"][b, p // page], p % page
                    k, v = c["k"][at, g, slot][None], c["v"][at, g, :, slot][None]
                    ref = orc.lis_attention_qk(q[b, h, i][None, None], k, v, s, **args)
                    assert np.array_equal(ref[0, 0], out[b, h, i])
                    # the weight is the product with values of 1
                    one = orc.lis_attention_qk(q[b, h, i][None, None], k, np.ones_like(v), s,
                                               **dict(args, zp_v=0))
                    weight[at[0], g, slot[0]] += one[0, 0, 0]
        if len(length) < 3 and max(length) <= 4096:
            assert weight.sum() == grown.sum()


@pytest.mark.skipif(bool(SAN_LIB), reason="this is the run that starts it")
def test_host_code_under_sanitizers(tmp_path):
    from test_sanitizers import SAN, _env
    env = _env({"FQVIT_DECODE_TEST_LIB": host_library(str(tmp_path / "libsan.so"), SAN)})
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-q", "-s", "-p",
                        "no:cacheprovider", "-k", "refusals or integer"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert r.returncode == 0 and " passed" in out, out[-4000:]
