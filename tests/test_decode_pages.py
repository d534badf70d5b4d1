"""Table entries that name no page read as page 0 and are never written through, by the
attention's weights, the append or the eviction; entries behind a sequence's last key
are not read."""
import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, host, say  # noqa: F401

pytestmark = pytest.mark.gpu


def spoiled(table, pages, at):
    bad = table.copy()
    for n, (b, j) in enumerate(at):
        bad[b, j] = (-1, pages, 1 << 30, -2 ** 31)[n % 4]
    return bad


def aside(c, bad):
    """The cache with one page more, a copy of page 0, in the place of the entries that are none."""
    spare = c["k"].shape[0]
    more = {n: np.concatenate([c[n], c[n][:1]]) for n in ("k", "v", "weight")}
    more["table"] = np.where((bad < 0) | (bad >= spare), spare, bad).astype(np.int32)
    return more, spare


# every way of the attention: few rows with their logits in LDS and in parts, chunks whole and
# in parts, pages that hold a tile and smaller ones, the thresholds and the 64-bit form
CASES = [((2, 4, 2, 3, 64, 16, [100, 77], [3, 3], {}), [(0, 1), (0, 3), (1, 4)]),
         ((1, 2, 2, 40, 64, 64, [300], [40], {}), [(0, 1), (0, 3)]),
         ((1, 4, 1, 1, 128, 32, [6000], [1], {}), [(0, 1), (0, 3), (0, 100), (0, 187)]),
         ((2, 4, 2, 24, 32, 16, [2500, 1100], [24, 20], {}), [(0, 0), (0, 70), (1, 3)]),
         ((1, 16, 1, 1, 64, 128, [3000], [1], dict(s=2e-4, n=14)), [(0, 2), (0, 23)]),
         ((2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=0.1, n=30, causal=False)), [(0, 2), (1, 0), (1, 12)]),
         ((1, 2, 1, 5, 48, 1024, [1500], [5], {}), [(0, 1)])]


@pytest.mark.parametrize("case,at", CASES, ids=lambda x: "x".join(map(str, x[:6])) if len(x) > 5 else "")
def test_weights_are_not_added_through_them(fq, case, at):  # noqa: F811
    c, q, length, n_new, s, more = R.attend_case(case)
    page = case[5]
    bad = spoiled(c["table"], c["k"].shape[0], at)
    other, spare = aside(c, bad)
    for b, n in enumerate(length):              # what lies behind the last key
        bad[b, -(-n // page):] = 2 ** 31 - 1
    ref, grown = R.attend(other, q, length, n_new, s, **more)
    assert grown[spare].any()
    on = {dict(n="exp_n").get(k, k): v for k, v in more.items()}
    w = dev(c["weight"])
    say("no pages", case)
    out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(bad), dev(length), s, n_new=dev(n_new),
                                 weight=w, **on)
    rows = np.arange(q.shape[2])[None] < n_new[:, None]
    assert np.array_equal(host(out).swapaxes(1, 2)[rows], ref.swapaxes(1, 2)[rows])
    assert np.array_equal(host(w), c["weight"] + grown[:spare])


def test_lengths_beyond_the_table(fq):  # noqa: F811
    c, q, length, n_new, s, _ = R.attend_case((2, 2, 2, 1, 64, 16, [48, 48], [1, 1], {}))
    most = c["table"].shape[1] * 16
    ref, _ = R.attend(c, q, np.array([most, 0]), n_new, s)
    say("lengths beyond the table")
    out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]),
                                 dev(np.array([most + 77, -5], np.int32)), s)
    assert np.array_equal(host(out), ref)


@pytest.mark.parametrize("L", (3, 40))
def test_an_append_leaves_them_out(fq, L):  # noqa: F811
    g = np.random.default_rng(2)
    c = R.cache(1, 2, 64, 16, 64, seed=9)
    bad = c["table"].copy()
    bad[0, 1], bad[0, 2] = -7, 1 << 30
    k, v = (g.integers(-128, 128, (1, 2, L, 64)).astype(np.int8) for _ in range(2))
    kp, vp, w = dev(c["k"]), dev(c["v"]), dev(c["weight"])
    n = np.array([33], np.int32)
    say("append no pages", L)
    fq.kv_cache_append_int8(dev(k), dev(v), kp, vp, dev(bad), dev(n), weight=w)
    more, spare = aside(c, bad)
    for got, want in zip((kp, vp, w), R.append(more, k, v, n, [L])):
        assert np.array_equal(host(got), want[:spare])


def test_an_eviction_leaves_them_out(fq):  # noqa: F811
    c, length, keep, recent, to = R.evict_case((1, 2, 64, 16, [100], 40, 4, "any"))
    bad = to.copy()
    bad[0, 1] = -1
    kp, vp, w = dev(c["k"]), dev(c["v"]), dev(c["weight"])
    say("evict no pages")
    _, kept = fq.kv_cache_evict(kp, vp, w, dev(c["table"]), dev(length), keep, recent, table_out=dev(bad))
    more, spare = aside(c, bad)
    to, more["table"] = more["table"], c["table"]
    ref = R.evict(more, length, keep, recent, to)
    for got, want in zip((kp, vp, w), ref):
        assert np.array_equal(host(got), want[:spare])
    assert np.array_equal(host(kept), ref[4])
