"""The oracle's linear layers, rotary positions and heads-to-rows against plain
64-bit forms in numpy (tests/layer_cases.py), and against values worked out by
hand: ties, saturation, the turn by a quarter.  No GPU."""
import numpy as np
import pytest

import layer_cases as R

ACTS = ("none", "relu", "table")


def options(act, residual, T, N, seed):
    """Arguments of the activation and the residual for linear_int8."""
    g = np.random.default_rng(seed + 99)
    more = {}
    if act == "relu":
        more["relu"] = True
    elif act == "table":
        more["table"] = g.normal(0, 60, 64).astype(np.float32)
        more["zp_t"] = 21
    if residual:
        more["residual"] = g.integers(-128, 128, (T, N)).astype(np.int8)
        more["zp_r"], more["mul_r"] = -9, 0.37
    return more


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("T,K,N,bits,zp_x,zp_y", [(1, 1, 1, 8, 0, 0), (7, 33, 5, 8, -11, 4),
                                                  (20, 100, 31, 4, 90, -8), (3, 640, 17, 2, -128, 1)])
def test_linear_matches_plain_form(orc, act, residual, T, K, N, bits, zp_x, zp_y):
    p = R.layer(T, K, N, seed=T + K, zp_x=zp_x)
    s_y = p["s_y"] * 255 / ((1 << bits) - 1) * (8 if act == "table" else 1)
    f, m = orc.linear_fold_int8(p["w"], p["s_w"], p["s_x"], s_y, zp_x, p["bias"])
    rf, rm = R.fold(p["w"], p["s_w"], p["s_x"], s_y, zp_x, p["bias"])
    assert np.array_equal(f, rf) and np.array_equal(m, rm)
    assert np.array_equal(orc.linear_int32(p["x"], p["w"], f), R.sums(p["x"], p["w"], f))
    more = options(act, residual, T, N, seed=K)
    y = orc.linear_int8(p["x"], p["w"], f, m, zp_y, bits, **more)
    assert np.array_equal(y, R.linear(p["x"], p["w"], f, m, zp_y, bits, **more))


def test_linear_by_hand(orc):
    # acc = 2 * 3 + 4 * (-5) + 1 = -13; -13 / 2 = -6.5 goes to the even -6
    x, w = np.array([[2, 4]], np.int8), np.array([[3, -5]], np.int8)
    one = np.array([1], np.int32)
    for mul, zp, expect in ((0.5, 0, -6), (0.5, 1, -6), (0.5, 3, -4), (0.25, 0, -3), (1e30, 7, -128),
                            (0.0, 7, 7)):
        assert orc.linear_int8(x, w, one, [mul], zp)[0, 0] == expect, (mul, zp)
    assert orc.linear_int8(x, w, one, [0.5], 5, relu=True)[0, 0] == 5
    # residual: (10 - 2) * 0.5 + (-13 * 0.5) = -2.5 -> -2
    assert orc.linear_int8(x, w, one, [0.5], 0, residual=[[10]], zp_r=2, mul_r=0.5)[0, 0] == -2
    # table: rint(-6.5 + 8) = 2
    assert orc.linear_int8(x, w, one, [0.5], 1, table=np.arange(16) * 3.0, zp_t=8)[0, 0] == 7


def test_fold_of_channels_without_a_scale(orc):
    w = np.full((5, 4), 3, np.int8)
    s_w = np.array([0.0, -1.0, np.inf, np.nan, 0.5], np.float32)
    f, m = orc.linear_fold_int8(w, s_w, 0.5, 0.25, 2, np.array([1, 1, 1, 1, np.nan], np.float32))
    assert f.tolist() == [-24] * 5 and m.tolist() == [0, 0, 0, 0, 1]
    f, _ = orc.linear_fold_int8(w[:2], np.float32([1e-9, 1e-9]), 1.0, 1.0, 0, np.float32([9, -9]))
    assert f.tolist() == [2 ** 30, -2 ** 30]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,L,Hq,Hkv,d,P,own_rows", [(1, 1, 1, 1, 2, 1, False), (2, 5, 4, 2, 9, 3, True),
                                                     (3, 4, 3, 3, 16, 8, False)])
def test_rope_matches_plain_form(orc, interleaved, B, L, Hq, Hkv, d, P, own_rows):
    g = np.random.default_rng(L)
    pos = g.integers(-1000, 100_000, (3, B * L if own_rows else L)).astype(np.int32)
    freq, axis = 10000.0 ** (-np.arange(P) / P), (np.arange(P) % 4).astype(np.uint8)
    table = orc.rope_table_int16(pos, freq, axis)
    assert np.array_equal(table, R.rope_table(pos, freq, axis))
    qkv = g.integers(-128, 128, (B, L, (Hq + 2 * Hkv) * d)).astype(np.int8)
    kw = dict(zp_x=-3, zp_q=5, zp_k=-2, bits=6, interleaved=interleaved)
    got = orc.rope_qkv_int8(qkv, table, Hq, Hkv, 0.05, 0.2, 0.3, **kw)
    for a, b in zip(got, R.rope(qkv, table, Hq, Hkv, 0.05, 0.2, 0.3, **kw)):
        assert np.array_equal(a, b)


def test_rope_by_hand(orc):
    # no turn, a quarter, a half: (a, b) -> (a, b), (-b, a), (-a, -b)
    table = orc.rope_table_int16([[0, 1, 2]], [np.pi / 2], [0])
    assert table.reshape(3, 2).tolist() == [[16384, 0], [0, 16384], [-16384, 0]]
    qkv = np.tile(np.array([10, 20, 10, 20, 1, 2], np.int8), (1, 3, 1))
    q, k, v = orc.rope_qkv_int8(qkv, table, 1, 1, 0.5, 0.5, 1.0)
    assert q[0, 0].tolist() == [[10, 20], [-20, 10], [-10, -20]]
    assert k[0, 0].tolist() == [[5, 10], [-10, 5], [-5, -10]]
    assert v[0, 0].tolist() == [[1, 2]] * 3


def test_turned_attention_depends_on_the_distance_alone():
    """What rotary positions are for: the product of a query at position i and a
    key at j is that at i + 1000 and j + 1000, within the table's rounding: each
    of the four entries of a pair is off by half a step of 2^-14, so a product
    of two pairs of values up to 128 by less than 2 * 128^2 * 4 * 2^-15 * 2."""
    g = np.random.default_rng(0)
    P = 16
    q, k = g.integers(-90, 91, (2, 2 * P)).astype(np.float64)
    freq, axis = 10000.0 ** (-np.arange(P) / P), np.zeros(P, np.uint8)

    def turned(x, at):
        c, s = R.rope_table(np.array([[at]]), freq, axis)[0].T / 16384.0
        return np.concatenate((x[:P] * c - x[P:] * s, x[:P] * s + x[P:] * c))

    for i, j in ((0, 0), (5, 3), (700, 20)):
        near, far = (turned(q, i + o) @ turned(k, j + o) for o in (0, 1000))
        assert abs(near - far) < P * 2 * 128 ** 2 * 4 * 2.0 ** -15 * 2


def test_heads_to_rows(orc):
    g = np.random.default_rng(1)
    q = g.integers(-2 ** 31, 2 ** 31, (2, 3, 4, 5)).astype(np.int32)
    flat = orc.requant_dyadic_int8(np.ascontiguousarray(q.transpose(0, 2, 1, 3)), 1e-9, 0.02, 3)
    assert np.array_equal(orc.requant_heads_int8(q, 1e-9, 0.02, 3), flat.reshape(2, 4, 15))
