"""The operators together, as a quantized transformer layer runs them: LayerNorm,
the query-key-value layer, rotary positions, attention from Q and K, heads back
to rows, the projection with its residual, LayerNorm, the two layers of the
perceptron with GELU and the second residual.  Every intermediate tensor against
the oracle, eagerly and replayed from a graph."""
import numpy as np
import pytest

import layer_cases as R
import workloads as W
from test_linear_gpu import dev, fq, host, say  # noqa: F401

pytestmark = pytest.mark.gpu


class Layer:
    """Parameters of a layer of width C with H heads of 64; the same calls on the
    oracle's functions (numpy) and on the library's (device tensors)."""

    def __init__(self, B, L, C, H, Hkv, seed):
        self.B, self.L, self.C, self.H, self.Hkv, self.d = B, L, C, H, Hkv, 64
        g = np.random.default_rng(seed)
        ln = W.ln_inputs(B * L, C, seed=seed)
        self.x, self.ln = ln["x_q"], ln
        # the fixed residual scale of the row's tensor, for the test's purposes
        self.widths = dict(qkv=(C, (H + 2 * Hkv) * 64), proj=(H * 64, C), fc1=(C, 4 * C), fc2=(4 * C, C))
        self.w = {n: np.clip(np.rint(g.normal(0, 40, (o, i))), -128, 127).astype(np.int8)
                  for n, (i, o) in self.widths.items()}
        self.s_w = {n: (np.exp(g.uniform(-0.5, 0.5, o)) * 0.6 / (40 * np.sqrt(i))).astype(np.float32)
                    for n, (i, o) in self.widths.items()}
        self.bias = {n: g.normal(0, 0.2, o).astype(np.float32) for n, (_, o) in self.widths.items()}
        side = max(1, int(np.sqrt(L)))
        i = np.arange(L)
        self.pos = np.stack((i // side, i % side)).astype(np.int32)
        self.freq = 100.0 ** (-np.arange(32) / 32.0)
        self.axis = (np.arange(32) // 16).astype(np.uint8)

    def step(self, lib, put, x, attention):
        B, L, H, Hkv, ln = self.B, self.L, self.H, self.Hkv, self.ln
        keep = {}
        w = {n: put(v) for n, v in self.w.items()}
        s_in = dict(qkv=ln["s_out"], proj=0.01, fc1=ln["s_out"], fc2=0.02)
        zp_in = dict(qkv=ln["zp_out"], proj=0, fc1=ln["zp_out"], fc2=-100)
        s_out = dict(qkv=0.03, proj=0.04, fc1=16.0 / 1024, fc2=0.05)
        par = {n: lib.linear_fold_int8(w[n], put(self.s_w[n]), s_in[n], s_out[n], zp_in[n],
                                       bias=put(self.bias[n])) for n in w}

        def norm(v):
            return lib.ptf_layernorm_int8(v, ln["zp_in"], put(ln["alpha"]), ln["K"], put(ln["gamma"]),
                                          put(ln["beta"]), ln["s_out"], ln["zp_out"], ln["bits"])

        keep["norm1"] = h = norm(x)
        keep["qkv"] = h = lib.linear_int8(h, w["qkv"], *par["qkv"])
        table = lib.rope_table_int16(put(self.pos), put(self.freq), put(self.axis))
        q, k, v = lib.rope_qkv_int8(h.reshape(B, L, -1), table, H, Hkv, 0.03, 0.04, 0.04, zp_k=2)
        keep.update(q=q, k=k, v=v)
        # the queries of a shared key head are one longer unit
        out = attention(q.reshape(B * Hkv, H // Hkv * L, 64), k.reshape(B * Hkv, L, 64),
                        v.reshape(B * Hkv, L, 64), 0.04 * 0.04 / 8, 0, 2)
        keep["attention"] = out
        rows = lib.requant_heads_int8(out.reshape(B, H, L, 64), 0.03 / 2 ** 15, 0.01, 0)
        keep["rows"] = rows = rows.reshape(B * L, -1)
        keep["proj"] = x1 = lib.linear_int8(rows, w["proj"], *par["proj"], residual=x, zp_r=ln["zp_in"],
                                            mul_r=0.8, zp_y=ln["zp_in"])
        h = norm(x1)
        gelu = put(self.gelu)
        keep["fc1"] = h = lib.linear_int8(h, w["fc1"], *par["fc1"], table=gelu, zp_t=512, zp_y=-100)
        keep["fc2"] = lib.linear_int8(h, w["fc2"], *par["fc2"], residual=x1, zp_r=ln["zp_in"], mul_r=0.9)
        return keep

    @property
    def gelu(self):
        import paper_2111_13824_amd as fq  # noqa: F811
        return fq.activation_table("gelu", 16.0 / 1024, 0.02, 512, 10, device="cpu").numpy()


@pytest.mark.parametrize("B,L,C,H,Hkv", [(2, 49, 192, 3, 3), (1, 197, 256, 4, 2), (3, 1, 128, 2, 1)])
def test_a_layer(fq, orc, B, L, C, H, Hkv):  # noqa: F811
    say("layer", B, L, C, H, Hkv)
    layer = Layer(B, L, C, H, Hkv, seed=L)

    def attend(q, k, v, s, zq, zk):
        return fq.lis_attention_qk(q, k, v, s, zp_q=zq, zp_k=zk)

    def attend_ref(q, k, v, s, zq, zk):
        return orc.lis_attention_qk(q, k, v, s, zp_q=zq, zp_k=zk)

    got = layer.step(fq, dev, dev(layer.x), attend)
    ref = layer.step(orc, lambda a: a, layer.x, attend_ref)
    for name in ref:
        assert np.array_equal(host(got[name]), ref[name]), name
        assert len(np.unique(ref[name])) > 8, name       # the scales leave something to compare


def test_a_layer_replayed_from_a_graph(fq):  # noqa: F811
    import torch
    say("graph")
    layer = Layer(2, 65, 192, 3, 3, seed=9)
    x0 = dev(layer.x)
    x = x0.clone()
    kept = {}

    def put(a):       # uploaded once, outside the capture
        if id(a) not in kept:
            kept[id(a)] = (a, dev(a))
        return kept[id(a)][1]

    table = layer.gelu

    class Fixed(Layer):
        gelu = table

    layer.__class__ = Fixed

    def attend(q, k, v, s, zq, zk):
        return fq.lis_attention_qk(q, k, v, s, zp_q=zq, zp_k=zk)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(fq, put, x, attend)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer.step(fq, put, x, attend)
    torch.cuda.synchronize()
    for rep in range(4):
        x.copy_(torch.roll(x0, shifts=31 * rep, dims=0))
        for t in out.values():
            t.fill_(1)
        g.replay()
        torch.cuda.synchronize()
        eager = layer.step(fq, put, x, attend)
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], eager[n]), (rep, n)
