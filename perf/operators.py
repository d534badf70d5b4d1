"""Operators of the integer layers around the attention: the linear layer with
its epilogue, rotary positions on queries and keys, and the way back from heads
to rows.  Each case is one pass through one of them.

Every case has a "kind":

  linear  int8 activations [T, K] times int8 weights [N, K], plus the folded bias;
          out "int8": requantized per channel, through an activation ("none",
          "relu", or "gelu": a table of 2^table_bits entries) and, with
          "residual", added to an int8 residual of its own scale; out "int32":
          the accumulators themselves;
  rope    the int8 result [B, L, (Hq + 2 Hkv) d] of the query-key-value layer
          split into heads, queries and keys rotated by positions of 1 to 3 axes
          (time, height, width) and requantized; "fresh": the rotation table is
          made from the positions in the pass, as for images of differing sizes
          or the next token, else it is kept, as for a batch of equal images;
  merge   the int32 attention result [B, H, L, d] requantized to int8 [B, L, H d].

The definitions, written with RN = rounding to the nearest binary32 and rint =
rounding to the nearest integer (ties to even), both of the exact real value:

  acc = sum_k x w + fold,  a = RN(acc)
  int8 without residual:  y = clip(rint(v + zp_y)), v = a mul_n, max(a mul_n, 0) or
      table[u] with u = clip(rint(a mul_n + zp_t), 0, 2^table_bits - 1)
  int8 with residual:  z = RN((r + 128) mul_r + RN(zp_y - (128 + zp_r) mul_r)),
      y = clip(rint(RN(v + z))), where v is RN(max(a mul_n, 0)) for "relu"
  rope table:  c = rint(2^14 cos t), s = rint(2^14 sin t), t = position x frequency
  rope:  (p, q) -> (p c - q s, p s + q c) of values less their zero point, then
      clip(rint(. m + zp)), m = RN(s_x / (2^14 s_out)); values are kept as they are
  merge:  clip(floor((N2 q + 2^(N1 - 1)) / 2^N1) + zp), N2 / 2^N1 the 31-bit
      dyadic form of the ratio of the scales

All results are whole numbers (points of the b-bit grid and int32 sums, as the
next integer layer takes them), so both forms give the same ones.

Inputs follow quantized vision transformers: activations and weights are rounded
normals that use most of int8, weight scales are log-uniform per channel, the
output scale lets a few values reach the ends of the grid.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"


def listed():
    return [
        # One token or one pooled row through a widening layer with GELU: the
        # weights are read once, latency is all that counts.
        dict(name="linear_one_row", kind="linear", T=1, K=1024, N=4096, out="int8", act="gelu",
             table_bits=10, residual=False, bits=8, zp_x=3, zp_y=-5),
        # The narrowing layer of DeiT-T for one image, with its residual.
        dict(name="linear_deit_tiny_fc2", kind="linear", T=197, K=768, N=192, out="int8",
             act="none", table_bits=0, residual=True, bits=8, zp_x=0, zp_y=0),
        # Class scores of a pruned width: odd in every size, int32 out.
        dict(name="linear_odd_head", kind="linear", T=333, K=701, N=1001, out="int32", act="none",
             table_bits=0, residual=False, bits=8, zp_x=-7, zp_y=0),
        # Swin-S's first patch merging at batch 32: many short rows.
        dict(name="linear_swin_merge_b32", kind="linear", T=25088, K=384, N=192, out="int8",
             act="none", table_bits=0, residual=False, bits=8, zp_x=0, zp_y=0),
        # Query, key and value of ViT-B/16 at a throughput batch.
        dict(name="linear_vit_base_qkv_b64", kind="linear", T=12608, K=768, N=2304, out="int8",
             act="none", table_bits=0, residual=False, bits=8, zp_x=0, zp_y=0),
        # The two layers of ViT-L/16's perceptron at 384 px, the largest products.
        dict(name="linear_vit_large_fc1_b16", kind="linear", T=9232, K=1024, N=4096, out="int8",
             act="gelu", table_bits=10, residual=False, bits=8, zp_x=0, zp_y=-96),
        dict(name="linear_vit_large_fc2_b16", kind="linear", T=9232, K=4096, N=1024, out="int8",
             act="none", table_bits=0, residual=True, bits=8, zp_x=-96, zp_y=0),
        # One image of DeiT-T with positions of its own: two short launches.
        dict(name="rope_deit_tiny_b1", kind="rope", B=1, L=197, Hq=3, Hkv=3, d=64, P=32, axes=2,
             interleaved=False, fresh=True, bits=8, zp=0),
        # A batch of ViT-L images on one grid: the table is shared.
        dict(name="rope_vit_large_b16", kind="rope", B=16, L=577, Hq=16, Hkv=16, d=64, P=32,
             axes=2, interleaved=False, fresh=False, bits=8, zp=0),
        # Two clips of 16 frames of 196 patches, three axes, shared key heads.
        dict(name="rope_video_b2", kind="rope", B=2, L=3136, Hq=12, Hkv=4, d=64, P=30, axes=3,
             interleaved=True, fresh=True, bits=8, zp=2),
        # Attention of ViT-B/16 back to rows for the projection.
        dict(name="merge_vit_base_b64", kind="merge", B=64, H=12, L=197, d=64, bits=8, zp=0),
        # A small batch with a ragged head.
        dict(name="merge_ragged", kind="merge", B=3, H=5, L=145, d=37, bits=6, zp=3),
    ]


# ---------------------------------------------------------------------------
# Drawn cases
# ---------------------------------------------------------------------------

WIDTHS = (96, 192, 384, 512, 768, 1024, 1536, 2304, 4096)
MOST_PRODUCTS = 9232 * 1024 * 4096
MOST_QKV = 16 * 577 * 3 * 16 * 64
MOST_HEADS = 64 * 12 * 197 * 64


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng):
    return rng.choice(WIDTHS) if rng.random() < 0.5 else _log(rng, 16, 4096)


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear", "rope", "rope", "merge"))
    if kind == "linear":
        K, N = _width(rng), _width(rng)
        T = _log(rng, 1, max(1, min(25088, MOST_PRODUCTS // (K * N))))
        out = rng.choice(("int8", "int8", "int8", "int32"))
        act = rng.choice(("none", "none", "relu", "gelu")) if out == "int8" else "none"
        bits = rng.choice((8, 8, 6, 4))
        half = 1 << (bits - 1)
        return dict(kind=kind, T=T, K=K, N=N, out=out, act=act,
                    table_bits=rng.choice((8, 10, 12)) if act == "gelu" else 0,
                    residual=out == "int8" and rng.random() < 0.4, bits=bits,
                    zp_x=rng.randint(-128, 127), zp_y=rng.randint(-half, half - 1))
    if kind == "rope":
        d = rng.choice((32, 64, 64, 64, 72, 80, 128))
        P = d // 2 if rng.random() < 0.6 else rng.randint(1, d // 2)
        Hkv = rng.choice((1, 2, 3, 4, 6, 12, 16))
        Hq = Hkv * rng.choice((1, 1, 1, 2, 4))
        L = _log(rng, 1, 3136)
        B = _log(rng, 1, max(1, MOST_QKV // (L * (Hq + 2 * Hkv) * d)))
        return dict(kind=kind, B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, P=P, axes=rng.randint(1, 3),
                    interleaved=rng.random() < 0.5, fresh=rng.random() < 0.5,
                    bits=rng.choice((8, 8, 6, 4)), zp=rng.randint(-8, 7))
    H, L, d = rng.choice((3, 5, 6, 12, 16)), _log(rng, 1, 577), rng.choice((32, 64, 64, 48, 37))
    B = _log(rng, 1, max(1, MOST_HEADS // (H * L * d)))
    bits = rng.choice((8, 8, 6, 4))
    half = 1 << (bits - 1)
    return dict(kind=kind, B=B, H=H, L=L, d=d, bits=bits, zp=rng.randint(-half, half - 1))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _int8(gen, shape, dev, zp=0):
    x = torch.randn(shape, generator=gen, device=DEV) * dev + zp
    return x.round_().clamp_(-128, 127).to(torch.int8)


def _prepare_linear(case, gen):
    T, K, N, bits = case["T"], case["K"], case["N"], case["bits"]
    st = dict(case=case, x=_int8(gen, (T, K), 36.0, case["zp_x"]), w=_int8(gen, (N, K), 40.0))
    # scales that the products' spread asks for: a layer's result has a deviation
    # of about 1.5, GELU's input lies on a grid of [-8, 8), the output grid
    # reaches about three deviations
    s_x = 0.02
    spread = torch.exp(torch.rand(N, generator=gen, device=DEV) * 1.4 - 0.7)
    s_w = (1.5 * spread / (s_x * 36.0 * 40.0 * math.sqrt(K))).float()
    s_y = 9.0 / ((1 << bits) - 1)
    s_pre = 16.0 / (1 << case["table_bits"]) if case["act"] == "gelu" else s_y
    bias = torch.randn(N, generator=gen, device=DEV) * 0.3
    s_acc = s_x * s_w.double()
    rows = st["w"].sum(1, dtype=torch.int64)
    st["fold"] = (torch.round(bias.double() / s_acc) - case["zp_x"] * rows).to(torch.int32)
    st["mul"] = (s_acc / s_pre).float()
    if case["act"] == "gelu":
        st["zp_t"] = 1 << (case["table_bits"] - 1)
        u = torch.arange(1 << case["table_bits"], device=DEV, dtype=torch.float64)
        t = (u - st["zp_t"]) * s_pre
        st["table"] = (0.5 * t * (1 + torch.erf(t / math.sqrt(2.0))) / s_y).float()
    if case["residual"]:
        st["r"] = _int8(gen, (T, N), 40.0)
        st["zp_r"] = 4
        st["mul_r"] = float(np.float32(0.03 / s_y))
    return st


def _prepare_rope(case, gen):
    B, L, P, axes = case["B"], case["L"], case["P"], case["axes"]
    heads = case["Hq"] + 2 * case["Hkv"]
    levels = (1 << case["bits"]) - 1
    st = dict(case=case, qkv=_int8(gen, (B, L, heads * case["d"]), 36.0, case["zp"]), s_x=0.05,
              zp_x=case["zp"], s_q=0.07 * 255 / levels, s_k=0.06 * 255 / levels)
    # positions of each batch entry from an origin of its own when the table is
    # made in the pass (a long stream's next frames), one grid for all otherwise
    rows = B * L if case["fresh"] else L
    i = torch.arange(rows, device=DEV) % L
    side = max(1, math.isqrt(min(L, 196)))
    grid = torch.stack((i // (side * side), i // side % side, i % side))[3 - axes:]
    start = torch.randint(0, 100_000 if case["fresh"] else 8, (axes, B if case["fresh"] else 1),
                          generator=gen, device=DEV)
    st["positions"] = (grid + start.repeat_interleave(L, 1)).to(torch.int32).contiguous()
    p = torch.arange(P, device=DEV, dtype=torch.float64)
    st["freq"] = torch.pow(torch.tensor(10000.0, device=DEV, dtype=torch.float64), -p / P)
    st["axis"] = (torch.arange(P, device=DEV) * axes // P).to(torch.uint8)
    if not case["fresh"]:
        st["table"] = _plain_table(st)
    return st


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["kind"] == "linear":
        return _prepare_linear(case, gen)
    if case["kind"] == "rope":
        return _prepare_rope(case, gen)
    # Sums of codes times values: a few reach beyond the output grid.
    q = torch.randn((case["B"], case["H"], case["L"], case["d"]), generator=gen, device=DEV)
    s_out = 1.0 / (1 << case["bits"])
    return dict(case=case, q=(q * 600_000.0).round_().to(torch.int32), s_in=2.0 ** -22, s_out=s_out)


# ---------------------------------------------------------------------------
# Plain forms.  Sums of int8 products reach 2^31 and requantization decides at
# the middle between two steps, so they are computed in 64 bits.
# ---------------------------------------------------------------------------

def _grid(case):
    half = 1 << (case["bits"] - 1)
    return -half, half - 1


def _rn(v):
    return v.float().double()


def _plain_linear(st):
    case = st["case"]
    acc = st["x"].double() @ st["w"].double().t() + st["fold"].double()
    if case["out"] == "int32":
        return acc.to(torch.int32)
    v = _rn(acc) * st["mul"].double()
    if case["act"] == "gelu":
        u = torch.clamp(torch.round(v + st["zp_t"]), 0, (1 << case["table_bits"]) - 1)
        v = st["table"][u.long()].double()
    elif case["act"] == "relu":
        v = torch.clamp_min(_rn(v) if case["residual"] else v, 0.0)
    if case["residual"]:
        m = st["mul_r"]
        c = float(np.float32(case["zp_y"] - (128 + st["zp_r"]) * m))
        v = _rn(v + _rn((st["r"].double() + 128) * m + c))
    else:
        v = v + case["zp_y"]
    return torch.clamp(torch.round(v), *_grid(case)).to(torch.int8)


def _plain_table(st):
    t = st["positions"][st["axis"].long()].t().double() * st["freq"]
    both = torch.stack((torch.cos(t), torch.sin(t)), -1)
    return torch.round(both * 16384.0).to(torch.int16)


def _plain_rope(st):
    case = st["case"]
    B, L, Hq, Hkv, d, P = (case[n] for n in ("B", "L", "Hq", "Hkv", "d", "P"))
    table = _plain_table(st) if case["fresh"] else st["table"]
    heads = st["qkv"].view(B, L, Hq + 2 * Hkv, d).transpose(1, 2)
    x = heads[:, :Hq + Hkv].double() - st["zp_x"]
    cos, sin = table.view(-1, 1, L, P, 2).double().unbind(-1)
    y = x * 16384.0
    first, second = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if case["interleaved"] else \
        (slice(0, P), slice(P, 2 * P))
    p, q = x[..., first], x[..., second]
    y[..., first] = p * cos - q * sin
    y[..., second] = p * sin + q * cos
    out = []
    for part, s in ((y[:, :Hq], st["s_q"]), (y[:, Hq:], st["s_k"])):
        m = float(np.float32(float(np.float32(st["s_x"])) / (16384.0 * float(np.float32(s)))))
        out.append(torch.clamp(torch.round(part * m + case["zp"]), *_grid(case)).to(torch.int8))
    return (*out, heads[:, Hq + Hkv:].contiguous())


def _dyadic(s_in, s_out):
    ratio = float(np.float32(s_in)) / float(np.float32(s_out))
    shift = min(max(31 - math.frexp(ratio)[1], 0), 62)
    return min(math.floor(math.ldexp(ratio, shift)), 2 ** 31 - 1), shift


def _plain_merge(st):
    case = st["case"]
    mult, shift = _dyadic(st["s_in"], st["s_out"])
    half = (1 << shift) >> 1
    v = ((st["q"].to(torch.int64) * mult + half) >> shift) + case["zp"]
    v = torch.clamp(v, *_grid(case)).to(torch.int8)
    return v.transpose(1, 2).reshape(case["B"], case["L"], case["H"] * case["d"])


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def _own_linear(st):
    import paper_2111_13824_amd as fq

    case = st["case"]
    if case["out"] == "int32":
        return fq.linear_int32(st["x"], st["w"], st["fold"])
    more = {}
    if case["act"] == "gelu":
        more.update(table=st["table"], zp_t=st["zp_t"])
    elif case["act"] == "relu":
        more.update(relu=True)
    if case["residual"]:
        more.update(residual=st["r"], zp_r=st["zp_r"], mul_r=st["mul_r"])
    return fq.linear_int8(st["x"], st["w"], st["fold"], st["mul"], zp_y=case["zp_y"],
                          bits=case["bits"], **more)


def _own_rope(st):
    import paper_2111_13824_amd as fq

    case = st["case"]
    table = fq.rope_table_int16(st["positions"], st["freq"], st["axis"]) if case["fresh"] else \
        st["table"]
    return fq.rope_qkv_int8(st["qkv"], table, case["Hq"], case["Hkv"], st["s_x"], st["s_q"],
                            st["s_k"], zp_x=st["zp_x"], zp_q=case["zp"], zp_k=case["zp"],
                            bits=case["bits"], interleaved=case["interleaved"])


def _own_merge(st):
    import paper_2111_13824_amd as fq

    return fq.requant_heads_int8(st["q"], st["s_in"], st["s_out"], st["case"]["zp"],
                                 bits=st["case"]["bits"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"linear": _own_linear, "rope": _own_rope, "merge": _own_merge}[kind](state)
    return {"linear": _plain_linear, "rope": _plain_rope, "merge": _plain_merge}[kind](state)


def work(case):
    if case["kind"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        size = T * N * (4 if case["out"] == "int32" else 1) * (2 if case["residual"] else 1)
        size += T * K + N * K + 4 * N + (4 * N if case["out"] == "int8" else 0)
        size += 4 << case["table_bits"] if case["act"] == "gelu" else 0
        return {"bytes": size, "flops": 2 * T * K * N}
    if case["kind"] == "rope":
        values = case["B"] * case["L"] * (case["Hq"] + 2 * case["Hkv"]) * case["d"]
        rows = case["B"] * case["L"] if case["fresh"] else case["L"]
        read = 4 * case["axes"] * rows + 9 * case["P"] if case["fresh"] else 4 * rows * case["P"]
        turned = case["B"] * case["L"] * (case["Hq"] + case["Hkv"]) * case["P"]
        return {"bytes": 2 * values + read, "flops": 6 * turned}
    values = case["B"] * case["H"] * case["L"] * case["d"]
    return {"bytes": 5 * values, "flops": 2 * values}


# ---------------------------------------------------------------------------
# The definitions once more, on the host
# ---------------------------------------------------------------------------

def _host(st, *names):
    return [st[n].cpu().numpy() for n in names]


def _f32(v):
    return np.asarray(v).astype(np.float32).astype(np.float64)


def _exact_linear(case, st):
    x, w, fold, mul = _host(st, "x", "w", "fold", "mul")
    weights = np.ascontiguousarray(w.T).astype(np.float64)
    parts, step = [], max(1, (1 << 22) // case["N"])
    lo, hi = _grid(case)
    for i in range(0, case["T"], step):
        acc = np.matmul(x[i:i + step].astype(np.float64), weights)
        acc += fold
        if case["out"] == "int32":
            parts.append(acc.astype(np.int32))
            continue
        v = _f32(acc) * mul
        if case["act"] == "gelu":
            table, = _host(st, "table")
            at = np.minimum(np.maximum(np.rint(v + st["zp_t"]), 0), len(table) - 1).astype(np.int64)
            v = np.take(table, at).astype(np.float64)
        if case["residual"]:
            m = st["mul_r"]
            z = _f32((st["r"][i:i + step].cpu().numpy() + 128.0) * m +
                     _f32(case["zp_y"] - (128 + st["zp_r"]) * m))
            v = _f32(z + (np.maximum(_f32(v), 0) if case["act"] == "relu" else v))
        else:
            v = (np.maximum(v, 0) if case["act"] == "relu" else v) + case["zp_y"]
        parts.append(np.minimum(np.maximum(np.rint(v), lo), hi).astype(np.int8))
    return np.concatenate(parts)


def _exact_rope(case, st):
    B, L, Hq, Hkv, d, P = (case[n] for n in ("B", "L", "Hq", "Hkv", "d", "P"))
    pos, freq, axis, qkv = _host(st, "positions", "freq", "axis", "qkv")
    # as complex numbers: (p + q i) e^(i t) on the table's grid
    t = pos.T[:, axis].astype(np.float64) * freq
    turn = np.rint(16384.0 * np.cos(t)) + 1j * np.rint(16384.0 * np.sin(t))
    turn = turn.reshape(-1, L, 1, P)
    x = qkv.reshape(B, L, Hq + 2 * Hkv, d)
    lo, hi = _grid(case)
    at = np.arange(P)
    one, two = (2 * at, 2 * at + 1) if case["interleaved"] else (at, at + P)
    out = []
    for part, s in ((x[:, :, :Hq], st["s_q"]), (x[:, :, Hq:Hq + Hkv], st["s_k"])):
        v = part.astype(np.float64) - st["zp_x"]
        turned = (v[..., one] + 1j * v[..., two]) * turn
        v *= 16384.0
        v[..., one], v[..., two] = turned.real, turned.imag
        v = np.rint(v * _f32(_f32(st["s_x"]) / (16384.0 * _f32(s))) + case["zp"])
        out.append(np.ascontiguousarray(np.clip(v, lo, hi).astype(np.int8).swapaxes(1, 2)))
    return (*out, np.ascontiguousarray(x[:, :, Hq + Hkv:].swapaxes(1, 2)))


def _exact_merge(case, st):
    mult, shift = _dyadic(st["s_in"], st["s_out"])
    q, = _host(st, "q")
    # floor((N2 q + 2^(N1-1)) / 2^N1), head by head into the rows
    lo, hi = _grid(case)
    out = np.empty((case["B"], case["L"], case["H"], case["d"]), np.int8)
    for h in range(case["H"]):
        v = (q[:, h].astype(np.int64) * mult + (2 ** shift // 2)) // 2 ** shift
        out[:, :, h] = np.minimum(np.maximum(v + case["zp"], lo), hi)
    return out.reshape(case["B"], case["L"], -1)


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _exact_linear, "rope": _exact_rope, "merge": _exact_merge}[case["kind"]](case, st)
