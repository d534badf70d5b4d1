"""The step over a stream of tokens as it is run: a decoder layer of the framework's
integer operators, chunk by chunk and token by token over a paged cache that is cut to a
budget, against the oracle and the plain forms, eagerly and replayed from graphs; other
streams than the current one; calls that overlap; pages that the table names wrongly."""
import numpy as np
import pytest

import decode_cases as R
from test_linear_gpu import dev, fq, host, say  # noqa: F401

pytestmark = pytest.mark.gpu

PAGE, D = 16, 64


class Stream:
    """A layer of width C with Hq and Hkv heads of 64 for B streams, its cache, and the
    same calls through the library (device tensors) and the plain forms (numpy)."""

    def __init__(self, B, Hq, Hkv, C, most, seed):
        self.B, self.Hq, self.Hkv, self.C, self.most = B, Hq, Hkv, C, most
        g = np.random.default_rng(seed)
        self.g = g
        self.gamma = (1 + 0.3 * g.normal(size=C)).astype(np.float32)
        self.alpha = g.integers(0, 3, C).astype(np.uint8)
        widths = dict(qkv=(C, (Hq + 2 * Hkv) * D), proj=(Hq * D, C))
        self.w = {n: np.clip(np.rint(g.normal(0, 40, (o, i))), -128, 127).astype(np.int8)
                  for n, (i, o) in widths.items()}
        self.s_w = {n: (np.exp(g.uniform(-0.5, 0.5, o)) * 0.6 / (40 * np.sqrt(i))).astype(np.float32)
                    for n, (i, o) in widths.items()}
        self.freq = 100.0 ** (-np.arange(D // 2) / (D // 2))
        self.axis = np.zeros(D // 2, np.uint8)
        self.cache = R.cache(B, Hkv, D, PAGE, most, seed)
        self.length = np.zeros(B, np.int32)
        self.seen = np.zeros(B, np.int32)           # tokens of each stream so far (positions)

    def tokens(self, L, n_new):
        """A chunk's stream and branch, the lengths after it, its positions."""
        g = self.g
        r = np.clip(np.rint(g.normal(0, 400, (self.B * L, self.C))), -32768, 32767).astype(np.int16)
        x = np.clip(np.rint(g.normal(0, 36, (self.B * L, self.C))), -128, 127).astype(np.int8)
        at = self.seen[:, None] + np.arange(L)[None]
        return dict(r=r, x=x, positions=at.reshape(1, -1).astype(np.int32), n_new=n_new,
                    length=(self.length + n_new).astype(np.int32))


def layer_on(fq, m, t, cache, put, **more):  # noqa: F811
    """The library's pass: every intermediate tensor."""
    B, L = m.B, t["r"].shape[0] // m.B
    keep = {}
    keep["h"], keep["norm"] = fq.rmsnorm_int8(t["r"], put(m.gamma), 1.0, 0.02, x=t["x"],
                                              alpha=put(m.alpha), m_x=3.0)
    fold = {n: fq.linear_fold_int8(put(m.w[n]), put(m.s_w[n]), 0.02, 0.03) for n in m.w}
    keep["qkv"] = rows = fq.linear_int8(keep["norm"], put(m.w["qkv"]), *fold["qkv"])
    table = fq.rope_table_int16(t["positions"], put(m.freq), put(m.axis))
    q, k, v = fq.rope_qkv_int8(rows.view(B, L, -1), table, m.Hq, m.Hkv, 0.03, 0.04, 0.04)
    keep.update(q=q, k=k, v=v)
    fq.kv_cache_append_int8(k, v, *cache[:2], t["table"], t["length"], n_new=t["n_new"], weight=cache[2])
    out = fq.lis_attention_paged(q, *cache[:2], t["table"], t["length"], 0.04 * 0.04 / 8,
                                 n_new=t["n_new"], weight=cache[2], **more)
    keep["attention"] = out
    rows = fq.requant_heads_int8(out, 0.03 / 2 ** 15, 0.01, 0)
    keep["proj"] = fq.linear_int8(rows.view(B * L, -1), put(m.w["proj"]), *fold["proj"])
    return keep


def layer_plain(orc, m, t):
    """The same on the host, the norm and the cache by the plain forms."""
    B, L = m.B, t["r"].shape[0] // m.B
    keep = {}
    keep["h"], keep["norm"] = R.norm(t["r"], m.gamma, 1.0, 0.02, x=t["x"], alpha=m.alpha, m_x=3.0)
    fold = {n: orc.linear_fold_int8(m.w[n], m.s_w[n], 0.02, 0.03) for n in m.w}
    keep["qkv"] = rows = orc.linear_int8(keep["norm"], m.w["qkv"], *fold["qkv"])
    table = orc.rope_table_int16(t["positions"], m.freq, m.axis)
    q, k, v = orc.rope_qkv_int8(rows.reshape(B, L, -1), table, m.Hq, m.Hkv, 0.03, 0.04, 0.04)
    keep.update(q=q, k=k, v=v)
    c = m.cache
    c["k"], c["v"], c["weight"] = R.append(c, k, v, t["length"], t["n_new"])
    out, grown = R.attend(c, q, t["length"], t["n_new"], 0.04 * 0.04 / 8)
    c["weight"] = c["weight"] + grown
    keep["attention"] = out
    rows = orc.requant_heads_int8(out, 0.03 / 2 ** 15, 0.01, 0)
    keep["proj"] = orc.linear_int8(rows.reshape(B * L, -1), m.w["proj"], *fold["proj"])
    return keep


def test_streams_over_a_cache_with_a_budget(fq, orc):  # noqa: F811
    """Chunks, single tokens and evictions in turn: 3 streams, 40 tokens and more kept at
    24 keys of each head."""
    import torch
    m = Stream(3, 4, 2, 192, 96, seed=1)
    on = [dev(m.cache[n]) for n in ("k", "v", "weight")]
    table = dev(m.cache["table"])
    for step, (L, n_new) in enumerate([(20, [20, 7, 1]), (1, [1, 1, 1]), (33, [33, 0, 21]), (1, [1, 1, 0]),
                                       (2, [2, 1, 2])]):
        say("stream", step, L, n_new)
        t = m.tokens(L, np.array(n_new, np.int32))
        ref = layer_plain(orc, m, t)
        d = {k: dev(v) for k, v in t.items()}
        d["table"] = table
        out = torch.zeros((m.B, m.Hq, L, D), dtype=torch.int32, device="cuda:0")    # rows that stay
        got = layer_on(fq, m, d, on, dev, out=out)
        for n in ref:
            assert np.array_equal(host(got[n]), ref[n]), (step, n)
        m.seen += t["n_new"]
        c = m.cache
        for a, n in zip(on, ("k", "v", "weight")):
            assert np.array_equal(host(a), c[n]), (step, n)
        length = d["length"]
        _, kept = fq.kv_cache_evict(*on, table, length, 24, 5, length_out=length)
        c["k"], c["v"], c["weight"], m.length, ref_kept = R.evict(c, t["length"], 24, 5)
        assert np.array_equal(host(kept), ref_kept) and np.array_equal(host(length), m.length)
        for a, n in zip(on, ("k", "v", "weight")):
            assert np.array_equal(host(a), c[n]), (step, n)
        assert len(np.unique(ref["attention"])) > 8


def test_a_step_replayed_from_a_graph(fq):  # noqa: F811
    """Token steps from one graph, eager work between the replays: every result as from eager
    calls.  Two graphs share nothing but the cache."""
    import torch
    m = Stream(2, 4, 2, 128, 96, seed=5)
    kept = {}

    def put(a):
        if id(a) not in kept:
            kept[id(a)] = (a, dev(a))
        return kept[id(a)][1]

    start = [dev(m.cache[n]) for n in ("k", "v", "weight")]
    cache = [t.clone() for t in start]
    tokens = [m.tokens(1, np.array([1, 1], np.int32)) for _ in range(5)]
    for i, t in enumerate(tokens):
        t["length"] = np.array([40 + i, 9 + i], np.int32)
    t = {k: dev(v) for k, v in tokens[0].items()}
    t["table"] = dev(m.cache["table"])
    evicted = dev(np.array([60, 61], np.int32))

    def step():
        keep = layer_on(fq, m, t, cache, put)
        keep["length"], keep["kept"] = fq.kv_cache_evict(*cache, t["table"], evicted, 50, 4)
        return keep

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = step()
        graphs.append((g, out))
    torch.cuda.synchronize()
    for i, new in enumerate(tokens):
        say("graph", i)
        for n, a in new.items():
            t[n].copy_(dev(a))
        for c, s in zip(cache, start):
            c.copy_(s)
        g, out = graphs[i % 2]
        for a in out.values():
            a.fill_(1)
        g.replay()
        torch.cuda.synchronize()
        after = [c.clone() for c in cache]
        got = {n: a.clone() for n, a in out.items()}
        for c, s in zip(cache, start):
            c.copy_(s)
        eager = step()
        torch.cuda.synchronize()
        for n in eager:
            assert torch.equal(got[n], eager[n]), (i, n)
        for a, b in zip(after, cache):
            assert torch.equal(a, b), i


def attend_args(case):
    c, q, length, n_new, s, more = R.attend_case(case)
    return (c, q, length, n_new, s, more), (dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]), dev(length), s)


def test_two_streams_at_once(fq):  # noqa: F811
    """Calls of every way on two streams that overlap, each with the workspace that the binding
    makes for it; a long cache keeps both busy."""
    import torch
    cases = [(1, 4, 2, 1, 64, 64, [9000], [1], {}), (2, 4, 2, 9, 64, 16, [1300, 700], [9, 9], {}),
             (1, 4, 2, 20, 64, 64, [5000], [20], {}), (2, 2, 2, 1, 128, 32, [90, 400], [1, 1], {})]
    made = [attend_args(c) for c in cases]
    want = [R.attend(c, q, length, n_new, s)[0] for (c, q, length, n_new, s, _), _ in made]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    say("two streams")
    got = []
    for rep in range(6):
        for i, (_, args) in enumerate(made):
            got.append((i, fq.lis_attention_paged(*args, stream=streams[(rep + i) % 2])))
    torch.cuda.synchronize()
    for i, out in got:
        assert np.array_equal(host(out), want[i]), i


def test_outputs_come_from_the_memory_of_their_stream(fq):  # noqa: F811
    import torch
    side = torch.cuda.Stream()
    c, length, keep, recent, _ = R.evict_case(R.EVICT[1])
    _, args = attend_args((1, 4, 2, 1, 64, 64, [9000], [1], {}))
    r = torch.zeros((4, 64), dtype=torch.int16, device="cuda:0")
    ones = torch.ones(64, device="cuda:0")
    on = [dev(c[n]) for n in ("k", "v", "weight", "table")]
    n = dev(length)
    torch.cuda.synchronize()
    for name, call in (("norm", lambda: fq.rmsnorm_int8(r, ones, 1.0, 1.0, stream=side)),
                       ("rows", lambda: fq.rmsnorm_rows_int8(r, ones, 1.0, stream=side)),
                       ("attend", lambda: (fq.lis_attention_paged(*args, stream=side),)),
                       ("evict", lambda: fq.kv_cache_evict(*on, n, keep, recent, stream=side))):
        say("stream memory", name)
        out = call()
        torch.cuda.synchronize()
        for t in out:
            pool, = [s["stream"] for s in torch.cuda.memory_snapshot()
                     if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]]
            assert pool == side.cuda_stream, name


def test_pages_that_are_none(fq):  # noqa: F811
    """Table entries that name no page read as page 0 and are never written through; entries
    behind a sequence's last key are not read; lengths beyond the table are its end."""
    say("bad pages")
    for case in ((2, 4, 2, 3, 64, 16, [100, 77], [3, 3], {}), (1, 2, 2, 40, 64, 64, [300], [40], {}),
                 (1, 4, 1, 1, 128, 32, [6000], [1], {})):
        c, q, length, n_new, s, _ = R.attend_case(case)
        page = case[5]
        bad = c["table"].copy()
        bad[0, 1], bad[0, 3] = -1, c["k"].shape[0]
        zero = dict(c, table=np.where((bad < 0) | (bad >= c["k"].shape[0]), 0, bad))
        for b, n in enumerate(length):          # what lies behind the last key
            bad[b, -(-n // page):] = 2 ** 31 - 1
        ref, grown = R.attend(zero, q, length, n_new, s)
        w = dev(c["weight"])
        out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(bad), dev(length), s, weight=w)
        assert np.array_equal(host(out), ref) and np.array_equal(host(w), c["weight"] + grown)
    # lengths beyond the table
    c, q, length, n_new, s, _ = R.attend_case((2, 2, 2, 1, 64, 16, [48, 48], [1, 1], {}))
    most = c["table"].shape[1] * 16
    ref, _ = R.attend(c, q, np.array([most, 0]), n_new, s)
    out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]),
                                 dev(np.array([most + 77, -5], np.int32)), s)
    assert np.array_equal(host(out), ref)
    # writes: an append's and an eviction's
    g = np.random.default_rng(2)
    for L in (3, 40):
        c = R.cache(1, 2, 64, 16, 64, seed=9)
        bad = c["table"].copy()
        bad[0, 1], bad[0, 2] = -7, 1 << 30
        k, v = (g.integers(-128, 128, (1, 2, L, 64)).astype(np.int8) for _ in range(2))
        kp, vp, w = dev(c["k"]), dev(c["v"]), dev(c["weight"])
        n = np.array([33], np.int32)
        fq.kv_cache_append_int8(dev(k), dev(v), kp, vp, dev(bad), dev(n), weight=w)
        spare = c["k"].shape[0]
        more = {m: np.concatenate([c[m], c[m][:1]]) for m in ("k", "v", "weight")}
        more["table"] = np.where((bad < 0) | (bad >= spare), spare, bad)      # a page that is thrown away
        ref = R.append(more, k, v, n, [L])
        for got, want in zip((kp, vp, w), ref):
            assert np.array_equal(host(got), want[:spare])
    c, length, keep, recent, to = R.evict_case((1, 2, 64, 16, [100], 40, 4, "any"))
    bad = to.copy()
    bad[0, 1] = -1
    kp, vp, w = dev(c["k"]), dev(c["v"]), dev(c["weight"])
    n_out, kept = fq.kv_cache_evict(kp, vp, w, dev(c["table"]), dev(length), keep, recent, table_out=dev(bad))
    spare = c["k"].shape[0]
    more = {m: np.concatenate([c[m], c[m][:1]]) for m in ("k", "v", "weight")}
    more["table"] = c["table"]
    ref = R.evict(more, length, keep, recent, np.where(bad < 0, spare, bad))
    for got, want in zip((kp, vp, w), ref):
        assert np.array_equal(host(got), want[:spare])
    assert np.array_equal(host(kept), ref[4])


def test_sequences_that_share_pages(fq):  # noqa: F811
    """A common beginning kept once: read by both, its weight collected from both."""
    say("shared pages")
    c, q, length, n_new, s, _ = R.attend_case((2, 4, 2, 2, 64, 16, [100, 100], [2, 2], {}))
    c["table"][1, :4] = c["table"][0, :4]
    ref, grown = R.attend(c, q, length, n_new, s)
    w = dev(c["weight"])
    out = fq.lis_attention_paged(dev(q), dev(c["k"]), dev(c["v"]), dev(c["table"]), dev(length), s, weight=w)
    assert np.array_equal(host(out), ref) and np.array_equal(host(w), c["weight"] + grown)


def test_a_prepared_call_and_its_workspace(fq):  # noqa: F811
    """A prepared call runs again and again on changed contents, in a workspace of the
    caller's; one that is too small is refused."""
    import torch
    say("prepared")
    (c, q, length, n_new, s, _), args = attend_args((1, 4, 2, 1, 64, 64, [9000], [1], {}))
    need = fq.lis_attention_paged_workspace_bytes(1, 4, 2, 1, 64, c["table"].shape[1] * 64)
    assert need > 0
    ws = torch.full((need,), 0x55, dtype=torch.uint8, device="cuda:0")
    out = torch.zeros(q.shape, dtype=torch.int32, device="cuda:0")
    call = fq.lis_attention_paged(*args, out=out, workspace=ws, prepare=True)
    for shift in range(3):
        q1 = np.roll(q, shift, axis=-1)
        args[0].copy_(dev(q1))
        call()
        assert np.array_equal(host(out), R.attend(c, q1, length, n_new, s)[0])
    with pytest.raises(fq.FqError) as e:
        fq.lis_attention_paged(*args, workspace=ws[:need - 1])
    assert e.value.status == fq.binding.FQ_ERR_PARAM
