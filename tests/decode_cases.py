"""Inputs and plain 64-bit forms for the tests of the step over a stream of tokens:
numpy, written from the definitions in include/fqvit.h, token by token."""
import numpy as np


def f32(v):
    """Rounded to the nearest binary32, as binary64."""
    return np.asarray(v, np.float64).astype(np.float32).astype(np.float64)


# ---- Root-mean-square norm ----------------------------------------------------

def stream_sum(r, x=None, zp_x=0, alpha=None, K=3, m_x=1.0):
    h = r.astype(np.int64)
    if x is not None:
        lift = np.minimum(np.zeros(r.shape[1], int) if alpha is None else alpha.astype(int), K)
        h = h + np.rint((x.astype(np.int64) - zp_x) * 2 ** lift * f32(m_x)).astype(np.int64)
    return np.clip(h, -32768, 32767)


def norm(r, gamma, eps, s_out=None, zp_out=0, bits=8, **branch):
    """(h, y) with a scale, else (h, y, scales)."""
    h = stream_sum(r, **branch)
    mean = (h * h).sum(1) / np.float64(r.shape[1]) + f32(eps)
    with np.errstate(divide="ignore"):
        rho = np.where(mean > 0, 1.0 / np.sqrt(mean), 0.0)
    g = gamma.astype(np.float64)
    half = 1 << (bits - 1)
    if s_out is not None:
        f = f32(g * f32(rho / f32(s_out))[:, None])
        y = np.clip(np.rint(h * f + zp_out), -half, half - 1)
        return h.astype(np.int16), y.astype(np.int8)
    t = half - 1.0
    a = f32(g * h)
    top = np.abs(a).max(1)
    with np.errstate(divide="ignore"):
        q = np.where(top > 0, f32(t / top), 0.0)
    return (h.astype(np.int16), np.rint(a * q[:, None]).astype(np.int8),
            (f32(top * f32(rho)) / t).astype(np.float32))


def norm_inputs(T, C, seed, wide=300.0):
    g = np.random.default_rng(seed)
    r = np.clip(np.rint(g.normal(0, wide, (T, C)) * np.exp(g.normal(0, 1, C))), -32768, 32767)
    return dict(r=r.astype(np.int16), gamma=(1 + 0.5 * g.normal(size=C)).astype(np.float32),
                x=np.clip(np.rint(g.normal(3, 36, (T, C))), -128, 127).astype(np.int8),
                alpha=g.integers(0, 6, C).astype(np.uint8))


# ---- The cache -----------------------------------------------------------------

def cache(B, Hkv, d, page, keys, seed, zp=0, spread=19.6, spare=2):
    """Pages full of values, and tables of sequences of at most `keys` keys on them."""
    g = np.random.default_rng(seed)
    n = max(1, -(-keys // page))
    pages = B * n + spare
    table = g.permutation(pages)[:B * n].reshape(B, n).astype(np.int32)

    def ints(shape, dev, mid=0):
        return np.clip(np.rint(g.normal(mid, dev, shape)), -128, 127).astype(np.int8)

    return dict(k=ints((pages, Hkv, page, d), spread, zp), v=ints((pages, Hkv, d, page), 40.0),
                weight=g.integers(0, 1 << 40, (pages, Hkv, page)), table=table)


def place(table, b, p, page):
    return table[b, p // page], p % page


def append(c, k, v, length, n_new):
    kp, vp, w = c["k"].copy(), c["v"].copy(), c["weight"].copy()
    page = kp.shape[2]
    for b in range(len(length)):
        for i in range(n_new[b]):
            p = length[b] - n_new[b] + i
            if 0 <= p < c["table"].shape[1] * page:
                at, s = place(c["table"], b, p, page)
                kp[at, :, s], vp[at, :, :, s], w[at, :, s] = k[b, :, i], v[b, :, i], 0
    return kp, vp, w


def constants(s):
    s = float(np.float32(s))
    return (-int(np.floor(-0.69314718055994530942 / s)), int(np.floor(1.353 / s)),
            int(np.floor(0.344 / ((0.3585 * s) * s))))


def codes(logits, s, bits, n):
    """Log-Int-Softmax codes of a row of integers (at least one), exactly."""
    step, q_b, q_c = constants(s)
    u = np.minimum(int(logits.max()) - logits.astype(np.int64), n * step)
    z = u // step
    e = ((q_b - u + z * step) ** 2 + q_c) * (np.int64(1) << (n - z))
    S = sum(int(x) for x in np.add.reduceat(e, np.arange(0, len(e), 64)))
    assert 2 * S + int(e.max()) < 1 << 63
    ratio = (2 * np.int64(S) + e) // (2 * e)
    # I-Log2: the first set bit's place, and one more where the bit below it is set
    code = np.zeros(len(e), np.int64)
    for i, r in enumerate(ratio.tolist()):
        m = r.bit_length() - 1
        code[i] = m + (r >> (m - 1) & 1 if m else 0)
    return np.minimum(code, (1 << bits) - 1)


def attend(c, q, length, n_new, s, zp_q=0, zp_v=0, bits=4, n=20, causal=True, out=None):
    """(out, what each slot's weight grows by)."""
    B, Hq, L, d = q.shape
    page, Hkv = c["k"].shape[2], c["k"].shape[1]
    out = np.zeros(q.shape, np.int32) if out is None else out.copy()
    grown = np.zeros(c["weight"].shape, np.int64)
    top = (1 << bits) - 1
    for b in range(B):
        for hq in range(Hq):
            h = hq // (Hq // Hkv)
            for i in range(n_new[b]):
                seen = length[b] - n_new[b] + i + 1 if causal else length[b]
                out[b, hq, i] = 0
                if seen <= 0:
                    continue
                p = np.arange(seen)
                at, slot = c["table"][b, p // page], p % page
                k, v = c["k"][at, h, slot].astype(np.int64), c["v"][at, h, :, slot].astype(np.int64)
                w = np.int64(1) << (top - codes(k @ (q[b, hq, i].astype(np.int64) - zp_q), s, bits, n))
                out[b, hq, i] = w @ (v - zp_v)
                np.add.at(grown, (at, h, slot), w)
    return out, grown


def evict(c, length, keep, recent, table_out=None):
    """(k, v, weight, length, kept)"""
    kp, vp, w = c["k"].copy(), c["v"].copy(), c["weight"].copy()
    B, Hkv, page = len(length), kp.shape[1], kp.shape[2]
    to = c["table"] if table_out is None else table_out
    kept = np.full((B, Hkv, keep), -1, np.int32)
    for b in range(B):
        n = int(length[b])
        for h in range(Hkv):
            mine = [int(c["weight"][place(c["table"], b, p, page)[0], h, p % page]) for p in range(n)]
            old = sorted(range(max(n - recent, 0)), key=lambda p: (-mine[p], p)) if n > keep else range(n)
            stay = sorted([*old[:keep - recent], *range(n - recent, n)]) if n > keep else list(old)
            kept[b, h, :len(stay)] = stay
            for j, p in enumerate(stay):
                (a0, s0), (a1, s1) = place(c["table"], b, p, page), place(to, b, j, page)
                kp[a1, h, s1], vp[a1, h, :, s1] = c["k"][a0, h, s0], c["v"][a0, h, :, s0]
                w[a1, h, s1] = c["weight"][a0, h, s0]
    return kp, vp, w, np.minimum(length, keep).astype(np.int32), kept


# Attention over the cache: (B, Hq, Hkv, L, d, page, lengths, new tokens, more).  One
# token and chunks, rows that see nothing, lengths around the edges of blocks, tiles and
# pages, every width of head, shared and single key heads, scales from fine to coarse.
ATTEND = [
    (1, 1, 1, 1, 16, 16, [1], [1], {}),
    (2, 3, 3, 1, 64, 16, [0, 197], [1, 1], {}),
    (4, 2, 2, 1, 32, 16, [15, 16, 17, 1], [1, 1, 1, 0], {}),
    (3, 6, 2, 5, 64, 32, [63, 64, 65], [5, 0, 3], dict(zp_q=5, zp_v=3)),
    (3, 4, 4, 7, 48, 16, [3, 127, 129], [7, 7, 7], dict(zp_q=-128, zp_v=-128)),
    (2, 8, 1, 3, 128, 64, [300, 255], [3, 2], dict(zp_q=127, zp_v=127)),
    (1, 12, 4, 33, 80, 128, [257], [33], dict(bits=3)),
    (2, 2, 1, 70, 112, 32, [70, 200], [70, 61], dict(bits=2, zp_q=-3)),
    (2, 5, 5, 4, 96, 256, [400, 513], [4, 4], dict(causal=False, zp_v=9)),
    (2, 4, 2, 9, 64, 1024, [1, 1300], [9, 9], dict(causal=False, bits=1)),
    (1, 3, 3, 130, 64, 64, [130], [130], {}),
    (1, 16, 2, 17, 64, 16, [700], [17], dict(s=2.0 ** -8)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=0.5)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=0.1, n=30)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=0.03, n=3)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=0.01, n=1)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=1e-4, n=12)),
    (2, 2, 2, 20, 64, 32, [90, 400], [20, 20], dict(s=2.5e-4, n=16, zp_q=1)),
    (1, 4, 2, 1, 64, 64, [5000], [1], {}),
    (1, 2, 2, 2, 64, 64, [3000], [2], dict(flat=True)),
    (1, 2, 2, 2, 64, 64, [900], [2], dict(spread=127.0, s=2e-4, n=14)),
    (33, 2, 1, 1, 64, 16, list(range(33)), [1] * 33, {}),
    # keys in parts: many rows and few, wide heads, parts that hold nothing, general scales
    (1, 4, 2, 20, 64, 64, [5000], [20], {}),
    (2, 2, 1, 40, 128, 32, [4100, 70], [40, 33], dict(zp_q=-2, zp_v=1)),
    (1, 2, 1, 9, 32, 16, [3001], [9], dict(s=2e-4, n=14)),
    (2, 16, 2, 2, 96, 16, [2100, 1], [2, 1], dict(bits=3)),
    (1, 16, 1, 1, 64, 128, [3000], [1], dict(s=2e-4, n=14, zp_q=-128, zp_v=5)),
    (3, 8, 1, 2, 128, 64, [2049, 0, 1500], [2, 2, 0], dict(causal=False)),
    (65, 2, 1, 2, 16, 16, [3 * i % 50 for i in range(65)], [2] * 65, {}),
    # narrow heads in parts, the 64-bit form in parts, parts that only some sequences fill
    (2, 4, 2, 24, 32, 16, [2500, 1100], [24, 20], dict(zp_q=3, zp_v=-4)),
    (1, 6, 2, 30, 16, 32, [1700], [30], dict(causal=False, bits=2)),
    (1, 4, 1, 17, 80, 64, [1800], [17], dict(s=0.1, n=30)),
    (3, 4, 2, 50, 48, 256, [3000, 200, 60], [50, 50, 40], {}),
    # chunks of so many heads that their keys stay whole: more than 16 tiles of 64 keys, in
    # pages that hold a tile and in smaller ones
    (16, 32, 32, 17, 16, 64, [2300 - 120 * i for i in range(16)], [17 - i % 3 for i in range(16)], {}),
    (8, 64, 64, 17, 16, 16, [1090, 1025, 1024, 1500, 2049, 17, 0, 1], [17] * 8, dict(zp_q=2)),
]


def attend_case(case, seed=1):
    B, Hq, Hkv, L, d, page, length, n_new, more = case
    more = dict(more)
    s, spread, flat = more.pop("s", 2.0 ** -10), more.pop("spread", 19.6), more.pop("flat", False)
    zp_q = more.get("zp_q", 0)
    c = cache(B, Hkv, d, page, max(length), seed, spread=spread)
    g = np.random.default_rng(seed + 100)
    q = np.clip(np.rint(g.normal(zp_q, spread, (B, Hq, L, d))), -128, 127).astype(np.int8)
    if flat:                    # equal logits: every code the same, exact ties
        q[:] = zp_q
    return c, q, np.array(length, np.int32), np.array(n_new, np.int32), s, more


# Eviction: (B, Hkv, d, page, lengths, keep, recent, kind of weights)
EVICT = [
    (1, 1, 16, 16, [1], 1, 0, "any"),
    (2, 3, 64, 16, [577, 100], 197, 49, "any"),
    (3, 2, 32, 32, [0, 64, 65], 64, 64, "any"),
    (2, 2, 128, 16, [300, 299], 40, 0, "equal"),
    (2, 1, 80, 64, [1500, 1025], 1024, 1, "few"),
    (1, 2, 48, 256, [3000], 1, 0, "any"),
    (1, 2, 64, 64, [2500], 1700, 300, "wide"),
    (2, 2, 112, 1024, [2048, 7], 2048, 5, "any"),
    (1, 2, 64, 32, [2049], 2048, 2047, "few"),
    (2, 2, 96, 16, [700, 650], 350, 10, "signs"),
    # more keys than a workgroup holds at once in eight and in 32 registers a thread
    (1, 2, 16, 16, [9000], 5000, 700, "any"),
    (1, 1, 16, 64, [20000], 300, 0, "few"),
    (1, 1, 16, 1024, [40000], 33000, 2, "signs"),
    (1, 1, 16, 64, [35001], 100, 99, "equal"),
]


def evict_case(case, seed=3):
    B, Hkv, d, page, length, keep, recent, kind = case
    n = -(-max(max(length), keep) // page) * page
    c = cache(B, Hkv, d, page, 2 * n, seed)
    g = np.random.default_rng(seed + 7)
    shape = c["weight"].shape
    c["weight"] = {"any": c["weight"], "equal": np.full(shape, 12345, np.int64),
                   "few": g.integers(0, 3, shape) << 33, "wide": g.integers(0, 1 << 62, shape),
                   "signs": g.integers(-(1 << 62), 1 << 62, shape)}[kind]
    half = c["table"].shape[1] // 2
    both = c["table"]
    c["table"] = np.ascontiguousarray(both[:, :half])
    return c, np.array(length, np.int32), keep, recent, np.ascontiguousarray(both[:, half:])
