"""The step over a stream of tokens on the GPU against plain 64-bit forms
(tests/decode_cases.py), every output equal: whole numbers, and scales that are
correctly rounded on both sides."""
import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, guarded, host, say  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- Root-mean-square norm ----------------------------------------------------

WIDTHS = (1, 7, 8, 31, 32, 33, 96, 128, 129, 300, 512, 513, 768, 1001, 1024, 1025, 2048, 2304, 4096, 4097, 8192)


@pytest.mark.parametrize("C", WIDTHS)
def test_norm_widths(fq, C):  # noqa: F811
    for T in (1, 2, 67):
        say("norm", T, C)
        a = R.norm_inputs(T, C, seed=C)
        branch = dict(x=a["x"], zp_x=3, alpha=a["alpha"], K=3, m_x=1.75)
        on = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in branch.items()}
        r, gamma = dev(a["r"]), dev(a["gamma"])
        ref = R.norm(a["r"], a["gamma"], 1.5, 0.05, -7, **branch)
        for got, want in zip(fq.rmsnorm_int8(r, gamma, 1.5, 0.05, -7, **on), ref):
            assert np.array_equal(host(got), want)
        for got, want in zip(fq.rmsnorm_rows_int8(r, gamma, 1.5, bits=6, **on),
                             R.norm(a["r"], a["gamma"], 1.5, bits=6, **branch)):
            assert np.array_equal(host(got), want)
        for got, want in zip(fq.rmsnorm_int8(r, gamma, 0.0, 0.03), R.norm(a["r"], a["gamma"], 0.0, 0.03)):
            assert np.array_equal(host(got), want)


def test_norm_extremes(fq):  # noqa: F811
    """Rows of zeros, of one value, at both ends of 16 bits; sums that leave them; a
    branch at its ends; steps at theirs."""
    C = 640
    g = np.random.default_rng(0)
    r = g.integers(-32768, 32768, (9, C)).astype(np.int16)
    r[0], r[1], r[2] = 0, -32768, 32767
    r[3] = 0
    r[3, 5] = 1
    x = g.integers(-128, 128, (9, C)).astype(np.int8)
    x[0] = 0
    x[4], x[5] = 127, -128
    gamma = g.normal(0, 2, C).astype(np.float32)
    gamma[:3] = 0, -0.0, 1e-30
    for eps in (0.0, 1e-3, 3e38):
        for m_x, zp_x, K in ((64.0, -128, 7), (2.0 ** -20, 127, 0), (0.5, 0, 3), (1 / 3, 0, 7)):
            alpha = g.integers(0, 256, C).astype(np.uint8)
            branch = dict(x=x, zp_x=zp_x, alpha=alpha, K=K, m_x=m_x)
            on = {k: dev(v) if isinstance(v, np.ndarray) else v for k, v in branch.items()}
            say("norm extremes", eps, m_x)
            for bits, s_out, zp in ((8, 0.01, 0), (2, 1e-6, 1), (4, 100.0, -8)):
                ref = R.norm(r, gamma, eps, s_out, zp, bits, **branch)
                for got, want in zip(fq.rmsnorm_int8(dev(r), dev(gamma), eps, s_out, zp, bits, **on), ref):
                    assert np.array_equal(host(got), want)
                for got, want in zip(fq.rmsnorm_rows_int8(dev(r), dev(gamma), eps, bits, **on),
                                     R.norm(r, gamma, eps, bits=bits, **branch)):
                    assert np.array_equal(host(got), want)


def test_norm_in_place_and_unaligned(fq):  # noqa: F811
    import torch
    for T, C, off in ((5, 1024, 0), (3, 1024, 2), (64, 40, 2), (7, 701, 0)):
        say("norm in place", T, C, off)
        a = R.norm_inputs(T, C, seed=T)
        r, r_ok = guarded((T, C), torch.int16, off)
        y, y_ok = guarded((T, C), torch.int8, off + 1)
        s, s_ok = guarded((T,), torch.float32, 4)
        r.copy_(dev(a["r"]))
        h, y1 = fq.rmsnorm_int8(r, dev(a["gamma"]), 1.0, 0.05, x=dev(a["x"]), h=r, y=y)
        ref = R.norm(a["r"], a["gamma"], 1.0, 0.05, x=a["x"])
        assert h is r and y1 is y
        assert np.array_equal(host(r), ref[0]) and np.array_equal(host(y), ref[1])
        r.copy_(dev(a["r"]))
        fq.rmsnorm_rows_int8(r, dev(a["gamma"]), 1.0, h=r, y=y, scales=s)
        for got, want in zip((r, y, s), R.norm(a["r"], a["gamma"], 1.0)):
            assert np.array_equal(host(got), want)
        assert r_ok() and y_ok() and s_ok()
    h, y = fq.rmsnorm_int8(torch.empty((0, 64), dtype=torch.int16, device="cuda:0"),
                           torch.ones(64, device="cuda:0"), 1.0, 1.0)
    assert h.shape == y.shape == (0, 64)


# ---- Append ----------------------------------------------------------------------

APPEND = [(1, 1, 1, 16, 16, [1], [1]), (3, 2, 1, 64, 32, [5, 100, 1], [1, 1, 0]),
          (2, 3, 15, 80, 16, [15, 47], [15, 9]), (2, 2, 16, 128, 64, [16, 80], [16, 16]),
          (3, 1, 77, 48, 16, [77, 140, 63], [77, 13, 0]), (2, 4, 130, 64, 64, [130, 257], [130, 129]),
          (1, 2, 300, 112, 1024, [333], [300]), (4, 1, 64, 32, 128, [64, 65, 128, 127], [64] * 4),
          (1, 1, 640, 96, 32, [640], [640]),
          # more new tokens than keys: the first ones have no place
          (2, 2, 20, 64, 16, [5, 0], [20, 20]), (2, 2, 3, 64, 16, [1, 2], [3, 3])]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "x".join(map(str, c[:5])))
def test_append(fq, case):  # noqa: F811
    B, Hkv, L, d, page, length, n_new = case
    for weights in (True, False):
        say("append", case, weights)
        c = R.cache(B, Hkv, d, page, max(max(length), 1), seed=L)
        g = np.random.default_rng(L)
        k, v = (g.integers(-128, 128, (B, Hkv, L, d)).astype(np.int8) for _ in range(2))
        kp, vp, w = dev(c["k"]), dev(c["v"]), dev(c["weight"])
        length_, new_ = np.array(length, np.int32), np.array(n_new, np.int32)
        fq.kv_cache_append_int8(dev(k), dev(v), kp, vp, dev(c["table"]), dev(length_),
                                n_new=None if n_new == [L] * B else dev(new_),
                                weight=w if weights else None)
        ref = R.append(c, k, v, length_, new_)
        assert np.array_equal(host(kp), ref[0]) and np.array_equal(host(vp), ref[1])
        assert np.array_equal(host(w), ref[2] if weights else c["weight"])


# ---- Attention -------------------------------------------------------------------

@pytest.mark.parametrize("case", R.ATTEND, ids=lambda c: "x".join(map(str, c[:6])) + str(c[6][-1]))
def test_attention(fq, case):  # noqa: F811
    import torch
    c, q, length, n_new, s, more = R.attend_case(case)
    say("attend", case[:8], s, more)
    names = dict(n="exp_n")
    on = {names.get(k, k): v for k, v in more.items()}
    out, intact = guarded(q.shape, torch.int32)
    before = host(out).copy()
    ref, grown = R.attend(c, q, length, n_new, s, out=before, **more)
    args = (dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]), dev(length), s)
    w = dev(c["weight"])
    fq.lis_attention_paged(*args, n_new=dev(n_new), out=out, **on)
    assert np.array_equal(host(out), ref)
    out.copy_(dev(before))
    fq.lis_attention_paged(*args, n_new=dev(n_new), out=out, weight=w, **on)
    assert np.array_equal(host(out), ref) and intact()
    assert np.array_equal(host(w), c["weight"] + grown)
    if (n_new == q.shape[2]).all():
        assert np.array_equal(host(fq.lis_attention_paged(*args, **on)), ref)


def test_attention_of_a_long_cache(fq):  # noqa: F811
    """70001 keys: sums beyond 2^53, weights of 1 of almost every key."""
    c = R.cache(1, 1, 64, 64, 70001, seed=4)
    q = np.random.default_rng(5).integers(-40, 41, (1, 3, 2, 64)).astype(np.int8)
    length = np.array([70001], np.int32)
    ref, grown = R.attend(c, q, length, [2], 2.0 ** -10, zp_v=7)
    w = dev(c["weight"])
    say("attend long")
    out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]), dev(length), 2.0 ** -10,
                                 zp_v=7, weight=w)
    assert np.array_equal(host(out), ref) and np.array_equal(host(w), c["weight"] + grown)


def test_places_beyond_two_gibibytes(fq):  # noqa: F811
    """A cache of 2.3 GiB of keys and as much of values whose last pages are used:
    append, attention, eviction."""
    import torch
    Hkv, d, page, pages = 2, 128, 256, 37000
    say("big cache")
    kp = torch.zeros((pages, Hkv, page, d), dtype=torch.int8, device="cuda:0")
    vp = torch.zeros((pages, Hkv, d, page), dtype=torch.int8, device="cuda:0")
    w = torch.zeros((pages, Hkv, page), dtype=torch.int64, device="cuda:0")
    assert kp.numel() > 1 << 31
    small = R.cache(1, Hkv, d, page, 1000, seed=2, spare=0)
    where = np.array([[pages - 1, 3, pages - 2, pages - 5]], np.int32)
    order = small["table"][0]
    g = np.random.default_rng(1)
    length, n = np.array([900], np.int32), 700
    k, v = (g.integers(-60, 61, (1, Hkv, n, d)).astype(np.int8) for _ in range(2))
    for to, frm in ((kp, "k"), (vp, "v"), (w, "weight")):
        for j in range(4):
            to[int(where[0, j])].copy_(dev(small[frm][order[j]]))
    fq.kv_cache_append_int8(dev(k), dev(v), kp, vp, dev(where), dev(length), weight=w)
    small["k"], small["v"], small["weight"] = R.append(small, k, v, length, [n])
    q = g.integers(-60, 61, (1, 2, 3, d)).astype(np.int8)
    out = fq.lis_attention_paged(dev(q), kp, vp, dev(where), dev(length), 2.0 ** -12, weight=w, exp_n=14)
    ref, grown = R.attend(small, q, length, [3], 2.0 ** -12, n=14)
    assert np.array_equal(host(out), ref)
    small["weight"] += grown
    n_out, kept = fq.kv_cache_evict(kp, vp, w, dev(where), dev(length), 300, 20)
    ref = R.evict(small, length, 300, 20)
    assert np.array_equal(host(n_out), ref[3]) and np.array_equal(host(kept), ref[4])
    for j in range(4):
        for got, want in zip((kp, vp, w), ref[:3]):
            assert np.array_equal(host(got[int(where[0, j])]), want[order[j]])


# ---- Eviction --------------------------------------------------------------------

@pytest.mark.parametrize("case", R.EVICT, ids=lambda c: "x".join(map(str, c[:4])) + c[7])
def test_evict(fq, case):  # noqa: F811
    c, length, keep, recent, to = R.evict_case(case)
    for elsewhere in (False, True):
        say("evict", case, elsewhere)
        on = [dev(c[n]) for n in ("k", "v", "weight")]
        table, n = dev(c["table"]), dev(length)
        n_out, kept = fq.kv_cache_evict(*on, table, n, keep, recent, length_out=None if elsewhere else n,
                                        table_out=dev(to) if elsewhere else None)
        ref = R.evict(c, length, keep, recent, to if elsewhere else None)
        for got, want in zip((*on, n_out, kept), ref):
            assert np.array_equal(host(got), want)
        assert np.array_equal(host(n), length if elsewhere else ref[3])


def test_evict_in_place_through_another_table(fq):  # noqa: F811
    """table_out with the first entries of table, in memory of its own, for one sequence,
    and other pages for the other: many tiles of places, of which those in place have
    to follow one another."""
    c, length, keep, recent, to = R.evict_case((2, 2, 64, 32, [2800, 2500], 1900, 60, "any"))
    to[0] = c["table"][0]
    pages = -(-keep // 32)
    to = np.ascontiguousarray(to[:, :pages])
    on = [dev(c[n]) for n in ("k", "v", "weight")]
    n_out, kept = fq.kv_cache_evict(*on, dev(c["table"]), dev(length), keep, recent, table_out=dev(to))
    ref = R.evict(c, length, keep, recent, to)
    for got, want in zip((*on, n_out, kept), ref):
        assert np.array_equal(host(got), want)
