"""Lengths beyond what the table can name: the append and the attention count a new
token's place from the length as it is.  The append leaves out what has no slot, the
attention's tokens see the keys up to their places, of those that the table names."""
import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, host, say  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(c, q, length, n_new, s, causal):
    """Token by token, with the keys that each one sees."""
    most = c["table"].shape[1] * c["k"].shape[2]
    out, grown = np.zeros(q.shape, np.int32), np.zeros(c["weight"].shape, np.int64)
    for i in range(q.shape[2]):
        seen = length - n_new + i + 1 if causal else length
        ref, more = R.attend(c, q[:, :, i:i + 1], np.clip(seen, 0, most), (i < n_new).astype(int), s, causal=False)
        out[:, :, i:i + 1] = ref
        grown += more
    return out, grown


# (sequences' keys in the table, B, Hq, Hkv, L, d, page, lengths less what the table names, new tokens)
CASES = [(96, 3, 4, 2, 3, 64, 16, [1, 2, 5], [3, 3, 3]), (192, 2, 2, 2, 40, 32, 64, [3, 39], [40, 40]),
         (192, 3, 2, 2, 20, 128, 64, [25, -3, 1000], [20, 17, 9]), (6016, 1, 4, 1, 2, 64, 32, [1], [2]),
         (4096, 2, 4, 2, 33, 64, 64, [30, 2 ** 31 - 1 - 4096], [33, 33]), (1024, 1, 2, 1, 9, 16, 1024, [4], [9]),
         (64, 2, 2, 1, 17, 48, 16, [-2 ** 31, -70], [17, 17])]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[:7])))
def test_new_tokens_at_the_table_s_end(fq, case):  # noqa: F811
    most, B, Hq, Hkv, L, d, page, beyond, n_new = case
    g = np.random.default_rng(most)
    c = R.cache(B, Hkv, d, page, most, seed=L)
    assert c["table"].shape[1] * page == most
    length = np.clip(np.array(beyond, np.int64) + most, -2 ** 31, 2 ** 31 - 1)
    n_new = np.array(n_new, np.int64)
    q = np.clip(np.rint(g.normal(0, 20, (B, Hq, L, d))), -128, 127).astype(np.int8)
    k, v = (np.clip(np.rint(g.normal(0, 20, (B, Hkv, L, d))), -128, 127).astype(np.int8) for _ in range(2))
    c["k"], c["v"], c["weight"] = old = R.append(c, k, v, length, n_new)
    say("lengths", case)
    n, new = dev(length.astype(np.int32)), dev(n_new.astype(np.int32))
    for causal in (True, False):
        fresh = R.cache(B, Hkv, d, page, most, seed=L)
        on = [dev(fresh[m]) for m in ("k", "v", "weight")]
        table = dev(c["table"])
        fq.kv_cache_append_int8(dev(k), dev(v), *on[:2], table, n, n_new=new, weight=on[2])
        for got, want in zip(on, old):
            assert np.array_equal(host(got), want)
        out = fq.lis_attention_paged(dev(q), *on[:2], table, n, 2.0 ** -10, n_new=new, causal=causal, weight=on[2])
        ref, grown = attend(c, q, length, n_new, 2.0 ** -10, causal)
        rows = np.arange(L)[None] < n_new[:, None]
        assert np.array_equal(host(out).swapaxes(1, 2)[rows], ref.swapaxes(1, 2)[rows])
        assert np.array_equal(host(on[2]), old[2] + grown)
