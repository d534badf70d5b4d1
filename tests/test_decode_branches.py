"""Ways of the attention over a cache that sizes alone reach: one launch of few rows for
many key heads, with as many logits in LDS as it holds and more pages than are looked up
at once; chunks of more sequences than are put in order of length; and as many sequences
as a call takes, through append, attention and eviction."""
import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, host, say  # noqa: F401

pytestmark = pytest.mark.gpu


def ragged(B, Hkv, d, page, most, length, seed):
    """A cache that holds the pages of these lengths alone; other entries of the tables name none."""
    g = np.random.default_rng(seed)
    held = [-(-int(n) // page) for n in length]
    order = g.permutation(sum(held))
    table = np.full((B, most // page), 2 ** 31 - 1, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n

    def ints(shape, dev):
        return np.clip(np.rint(g.normal(0, dev, shape)), -128, 127).astype(np.int8)

    return dict(k=ints((at, Hkv, page, d), 19.6), v=ints((at, Hkv, d, page), 40.0),
                weight=g.integers(0, 1 << 40, (at, Hkv, page)), table=table)


def short(B, *long):
    return [*long, *(7 * i % 150 for i in range(B - len(long)))]


# (B, Hq, Hkv, L, d, page, keys that a table names, lengths, more)
CASES = [(128, 1, 1, 1, 64, 16, 16384, short(128, 16384, 8193, 9000), {}),
         (128, 1, 1, 1, 128, 64, 16384, short(128, 4097, 16384, 0, 12345), dict(zp_q=4, zp_v=-3)),
         (130, 1, 1, 1, 16, 1024, 16384, short(130, 16383, 8192), dict(s=2e-4, n=14)),
         (64, 16, 4, 1, 64, 32, 4096, short(64, 4096, 4095, 3000), {}),
         (64, 8, 2, 2, 96, 16, 2048, short(64, 2048, 1025), dict(causal=False)),
         (32, 64, 4, 1, 32, 16, 1024, short(32, 1024, 1000), dict(bits=3)),
         # 17 rows and more of more than 64 sequences: whole, in parts, the 64-bit form
         (65, 2, 2, 17, 32, 16, 512, short(65, 500, 512), {}),
         (70, 2, 1, 9, 64, 64, 2048, short(70, 2000, 1, 1500, 1024), dict(zp_q=-128)),
         (66, 1, 1, 40, 80, 32, 1024, short(66, 1024, 0, 41), {}),
         (65, 3, 1, 6, 48, 16, 1040, short(65, 1040), dict(s=0.1, n=26))]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:7])))
def test_attention(fq, case):  # noqa: F811
    B, Hq, Hkv, L, d, page, most, length, more = case
    more = dict(more)
    s = more.pop("s", 2.0 ** -10)
    c = ragged(B, Hkv, d, page, most, length, seed=B)
    g = np.random.default_rng(B + 1)
    q = np.clip(np.rint(g.normal(more.get("zp_q", 0), 19.6, (B, Hq, L, d))), -128, 127).astype(np.int8)
    length = np.array(length, np.int32)
    n_new = np.minimum(length, L - g.integers(0, 2, B) * (L > 1)).astype(np.int32)
    ref, grown = R.attend(c, q, length, n_new, s, **more)
    on = {dict(n="exp_n").get(k, k): v for k, v in more.items()}
    w = dev(c["weight"])
    rows = np.arange(L)[None] < n_new[:, None]
    say("branches", case[:7])
    for weight in (None, w):
        out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]), dev(length), s,
                                     n_new=dev(n_new), weight=weight, **on)
        assert np.array_equal(host(out).swapaxes(1, 2)[rows], ref.swapaxes(1, 2)[rows])
    assert np.array_equal(host(w), c["weight"] + grown)


@pytest.mark.parametrize("L", (1, 16, 17))
def test_as_many_sequences_as_a_call_takes(fq, L):  # noqa: F811
    """61 sequences, over and over: every copy gives what the plain forms give for the first."""
    B, N, d, page = 65536, 61, 16, 32
    g = np.random.default_rng(L)
    length = np.array([L + i % (33 - L) for i in range(N)], np.int32)
    one = ragged(N, 1, d, page, page, length, seed=3)
    k, v, q = (np.clip(np.rint(g.normal(0, 30, (N, 1, L, d))), -128, 127).astype(np.int8) for _ in range(3))
    n_new = np.full(N, L)
    first = one["table"][:, 0]
    which = np.arange(B) % N
    on = [dev(one[m][first][which]) for m in ("k", "v", "weight")]
    table = dev(np.random.default_rng(5).permutation(B).astype(np.int32)[:, None])
    place = np.argsort(host(table)[:, 0])           # the sequence of each page
    for t in on:
        t.copy_(t[dev(place)])
    n = dev(length[which])
    args = [dev(a[which]) for a in (k, v, q)]
    say("many sequences", L)
    fq.kv_cache_append_int8(*args[:2], *on[:2], table, n, weight=on[2])
    one["k"], one["v"], one["weight"] = R.append(one, k, v, length, n_new)
    for got, m in zip(on, ("k", "v", "weight")):
        assert np.array_equal(host(got), one[m][first][which][place])
    out = fq.lis_attention_paged(args[2], *on[:2], table, n, 2.0 ** -10, weight=on[2])
    ref, grown = R.attend(one, q, length, n_new, 2.0 ** -10)
    one["weight"] = one["weight"] + grown
    assert np.array_equal(host(out), ref[which])
    assert np.array_equal(host(on[2]), one["weight"][first][which][place])
    n_out, kept = fq.kv_cache_evict(*on, table, n, 12, 3)
    one["k"], one["v"], one["weight"], ref_n, ref_kept = R.evict(one, length, 12, 3)
    assert np.array_equal(host(n_out), ref_n[which]) and np.array_equal(host(kept), ref_kept[which])
    for got, m in zip(on, ("k", "v", "weight")):
        assert np.array_equal(host(got), one[m][first][which][place])
