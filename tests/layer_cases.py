"""Inputs and plain 64-bit forms for the tests of the linear layers, the rotary
positions and the heads' way back to rows.  The plain forms are numpy, written
from the definitions in include/fqvit.h; integer products go through binary64,
where sums of int8 products are exact."""
import numpy as np


def f32(v):
    """Rounded to the nearest binary32, as binary64."""
    return np.asarray(v, np.float64).astype(np.float32).astype(np.float64)


def fold(w, s_w, s_x, s_y=1.0, zp_x=0, bias=None):
    s_n = float(np.float32(s_x)) * s_w.astype(np.float64)
    b = np.zeros(len(w)) if bias is None else np.rint(bias.astype(np.float64) / s_n)
    b = np.clip(b, -2.0 ** 30, 2.0 ** 30)
    rows = w.astype(np.int64).sum(1)
    return ((b.astype(np.int64) - zp_x * rows).astype(np.int32),
            (s_n / float(np.float32(s_y))).astype(np.float32))


def sums(x, w, fold_=None):
    s = x.astype(np.float64) @ w.astype(np.float64).T
    return s if fold_ is None else s + fold_


def linear(x, w, fold_, mul, zp_y=0, bits=8, relu=False, table=None, zp_t=0, residual=None, zp_r=0,
           mul_r=1.0):
    a, m = f32(sums(x, w, fold_)), mul.astype(np.float64)
    v = a * m
    if table is not None:
        v = table.astype(np.float64)[np.clip(np.rint(v + zp_t), 0, len(table) - 1).astype(np.int64)]
    elif relu:
        v = np.maximum(f32(v) if residual is not None else v, 0)
    if residual is None:
        v = v + zp_y
    else:
        mr = float(np.float32(mul_r))
        v = f32(v + f32((residual.astype(np.float64) + 128) * mr + f32(zp_y - (128 + zp_r) * mr)))
    half = 1 << (bits - 1)
    return np.clip(np.rint(v), -half, half - 1).astype(np.int8)


def rope_table(positions, freq, axis):
    t = positions[np.minimum(axis, len(positions) - 1)].T.astype(np.float64) * freq
    return np.rint(16384.0 * np.stack((np.cos(t), np.sin(t)), -1)).astype(np.int16)


def rope(qkv, table, Hq, Hkv, s_x, s_q, s_k, zp_x=0, zp_q=0, zp_k=0, bits=8, interleaved=False):
    B, L, row = qkv.shape
    heads = Hq + 2 * Hkv
    x = qkv.reshape(B, L, heads, row // heads)
    f = (x.astype(np.int64) - zp_x)
    out = f * 16384
    if table is not None:
        P = table.shape[1]
        at = np.arange(P)
        one, two = (2 * at, 2 * at + 1) if interleaved else (at, at + P)
        c, s = table.astype(np.int64).reshape(-1, L, 1, P, 2).transpose(4, 0, 1, 2, 3)
        out[..., one] = f[..., one] * c - f[..., two] * s
        out[..., two] = f[..., one] * s + f[..., two] * c
    half = 1 << (bits - 1)

    def grid(part, scale, zp):
        m = f32(float(np.float32(s_x)) / (16384.0 * float(np.float32(scale))))
        return np.clip(np.rint(part * m + zp), -half, half - 1).astype(np.int8).transpose(0, 2, 1, 3)

    return (grid(out[:, :, :Hq], s_q, zp_q), grid(out[:, :, Hq:Hq + Hkv], s_k, zp_k),
            x[:, :, Hq + Hkv:].transpose(0, 2, 1, 3))


def layer(T, K, N, seed, zp_x=0, spread=36.0):
    """A quantized layer's inputs: x, w, weight scales, bias and scales that fill
    the output grid."""
    g = np.random.default_rng(seed)
    x = np.clip(np.rint(g.normal(zp_x, spread, (T, K))), -128, 127).astype(np.int8)
    w = np.clip(np.rint(g.normal(0, 40, (N, K))), -128, 127).astype(np.int8)
    s_x = np.float32(0.02)
    s_w = (np.exp(g.uniform(-0.7, 0.7, N)) * 1.5 / (s_x * spread * 40 * np.sqrt(K))).astype(np.float32)
    bias = g.normal(0, 0.3, N).astype(np.float32)
    return dict(x=x, w=w, s_w=s_w, bias=bias, s_x=float(s_x), s_y=9.0 / 255, zp_x=zp_x)


# Products (T, K, N) for every kernel of the linear layers, by the name of their
# tile (linear_plan.h): rows and channels that end inside a tile and a unit, one
# stage of inputs and many, whole and ragged ones.  The first is the smallest.
KERNELS = ("rows16", "rows32", "tile64", "tile128", "tile256x128", "tile256x192", "tile256x256",
           "tile256x320", "tile64r", "tile128r", "tile256r")
PRODUCTS = {
    "rows16": [(5, 80, 300), (16, 1001, 77), (17, 80, 300), (32, 1001, 77), (31, 64, 16), (100, 80, 300),
               (33, 16, 70), (500, 384, 64), (100, 49, 70), (230, 301, 70), (33, 7, 5), (70, 129, 66)],
    "rows32": [(97, 48, 1900), (24, 64, 4100), (32, 1001, 4097), (20, 7, 4099), (128, 1024, 1001),
               (394, 4096, 200), (250, 1001, 300)],
    "tile64": [(640, 80, 1000), (1000, 400, 1001), (1030, 16, 1000), (1130, 80, 1001), (1260, 48, 1001),
               (900, 384, 700), (300, 1024, 520), (1300, 16, 1290)],
    "tile128": [(1000, 80, 2050), (1000, 48, 2050), (2170, 272, 1001), (1000, 400, 2050)],
    "tile256x128": [(4120, 80, 1001), (1000, 48, 4100), (4120, 272, 1001), (2170, 128, 3000),
                    (5420, 80, 2050), (5550, 48, 2050), (5420, 208, 2050)],
    "tile256x192": [(3860, 80, 2050), (2690, 48, 3000), (3860, 272, 2050), (3860, 192, 2050)],
    "tile256x256": [(5420, 256, 2050), (5420, 272, 2050), (5550, 400, 2050), (5420, 336, 2050)],
    "tile256x320": [(7760, 80, 2050), (7370, 208, 2050), (7370, 400, 2050), (7760, 320, 2050)],
    "tile64r": [(1000, 49, 700), (1500, 301, 500), (1300, 129, 666), (1400, 7, 1290), (900, 65, 1001)],
    "tile128r": [(2960, 131, 2050), (2050, 301, 2050), (4130, 301, 1001)],
    "tile256r": [(4000, 49, 2050), (3870, 131, 2050), (4130, 65, 2050)],
}

# Products (T, K, N) of every tile kernel whose rows and channels end on, one before,
# one after and a unit away from the edges of its tiles, with one stage of inputs
# to seven, whole and ragged ones.
EDGES = {
    "tile64": [(319, 128, 832), (448, 112, 896), (577, 144, 448), (4160, 256, 63), (3328, 384, 65),
        (2753, 416, 81), (2367, 512, 111), (161, 592, 784), (161, 768, 752), (4160, 896, 31), (1935, 48,
        193)],
    "tile128": [(5503, 128, 384), (5504, 112, 384), (2689, 144, 768), (5504, 256, 383), (6656, 384,
        257), (6529, 416, 273), (8319, 512, 239), (6625, 592, 272), (8225, 768, 240), (8256, 896, 223),
        (6543, 48, 257)],
    "tile256x128": [(5503, 64, 768), (5504, 48, 768), (1153, 80, 3328), (5504, 128, 767), (6656, 192,
        513), (6529, 224, 529), (8319, 256, 495), (6625, 272, 528), (1185, 384, 3312), (8256, 448, 479),
        (8207, 48, 385)],
    "tile256x192": [(2495, 128, 3328), (2496, 112, 3328), (5377, 144, 1536), (2496, 256, 3327), (13248,
        384, 513), (13057, 416, 529), (10943, 512, 751), (13217, 592, 528), (5409, 768, 1520), (11072,
        896, 735), (10959, 48, 641)],
    "tile256x256": [(4863, 256, 2560), (4864, 256, 2560), (6913, 256, 1792), (4864, 256, 2559), (16384,
        384, 513), (16385, 416, 529), (16383, 512, 751), (16353, 592, 528), (6945, 768, 1776), (16576,
        896, 735), (16399, 256, 641)],
    "tile256x320": [(13119, 128, 1280), (13120, 112, 1280), (21761, 144, 768), (7680, 256, 2303),
        (22080, 384, 513), (21761, 416, 529), (9279, 512, 1775), (22049, 592, 528), (6433, 768, 2544),
        (22016, 896, 735), (21775, 48, 641)],
    "tile64r": [(319, 129, 832), (320, 127, 832), (385, 259, 640), (3136, 17, 127), (3328, 379, 65),
        (1409, 520, 81), (2751, 641, 47), (417, 15, 912), (161, 767, 752), (4160, 903, 31), (1935, 33,
        193)],
    "tile128r": [(4479, 129, 1408), (4480, 127, 1408), (2689, 259, 1920), (7040, 129, 895), (7296, 379,
        513), (7041, 520, 401), (8319, 641, 367), (7649, 129, 784), (8225, 767, 368), (8256, 903, 223),
        (7567, 129, 769)],
    "tile256r": [(11007, 65, 768), (11008, 63, 768), (5377, 131, 1536), (7424, 17, 1279), (13312, 187,
        513), (13057, 264, 529), (16639, 321, 495), (16609, 15, 528), (16417, 383, 496), (16576, 455,
        479), (13583, 33, 641)],
}

# Products (T, K, N) of 9 to 32 rows whose channels are many: one line of tiles.
WIDE = [(9, 1024, 40000), (16, 272, 45001), (17, 768, 16384), (31, 272, 33017), (32, 1024, 32768),
        (10, 301, 50001), (16, 500, 50001), (17, 1001, 16385), (32, 129, 33000)]
