"""The serving part of the oracle against hand-made examples and closed forms (CPU)."""
from fractions import Fraction

import numpy as np

from oracle import serving


def test_unpack_and_linear_by_hand():
    packed = np.array([[0x1F, 0x0A]], np.uint8)                       # codes 15, 1, 10 and an odd tail
    assert serving.unpack4(packed, 3, False).tolist() == [[15, 1, 10]]
    assert serving.unpack4(packed, 3, True).tolist() == [[-1, 1, -6]]
    x = np.array([[2.0, 3.0, 5.0]])
    y = serving.linear(x, packed, np.array([[0.5, 2.0]]), np.array([[8, 200]], np.uint8), np.array([1.0]), 3, 2, False)
    # group 0: (15-8)*0.5*2 + (1-8)*0.5*3 ; group 1: a zero point above 15 counts as 15: (10-15)*2*5 ; bias 1
    assert y.tolist() == [[7.0 - 10.5 - 50.0 + 1.0]]


def test_linear_equals_exact_rationals():
    g = np.random.default_rng(5)
    n, k, group = 3, 71, 32
    codes = g.integers(0, 256, (n, 36), dtype=np.uint8)
    scales = g.uniform(0.01, 1, (n, 3)).astype(np.float16)
    x = g.normal(size=(2, k)).astype(np.float16)
    y = serving.linear(x, codes, scales, None, None, k, group, True)
    for r in range(2):
        for o in range(n):
            want = Fraction(0)
            for c in range(k):
                q = int(codes[o, c // 2]) >> (4 * (c % 2)) & 15
                want += Fraction(q - 16 if q > 7 else q) * Fraction(float(scales[o, c // group])) * Fraction(float(x[r, c]))
            assert abs(Fraction(float(y[r, o])) - want) <= abs(want) / 10**12 + Fraction(1, 10**12)


def test_schedule_by_hand():
    table = np.full((3, 3), -1, np.int32)
    table[0, 0], table[2, :2] = 7, (5, 6)
    # block of 4: request 0 goes 3 -> 6 (one block), request 1 stays empty, request 2 goes 8 -> 9 (one block)
    got = serving.schedule([3, 0, 8], [3, 0, 1], table, [10, 11, 12], 4, 6)
    assert got[0].tolist() == [[7, 12, -1], [-1, -1, -1], [5, 6, 11]]
    assert got[1].tolist() == [0, 3, 3, 4] and got[2].tolist() == [6, 0, 9]
    assert got[3].tolist() == [7 * 4 + 3, 12 * 4, 12 * 4 + 1, 11 * 4, -1, -1]
    assert got[4].tolist() == [1, 4, 2, 0]
    refused = serving.schedule([3, 0, 8], [3, 0, 1], table, [10], 4, 6)
    assert np.array_equal(refused[0], table) and refused[1].tolist() == [0] * 4 and refused[2].tolist() == [3, 0, 8]
    assert set(refused[3].tolist()) == {-1} and refused[4].tolist() == [1, 0, 0, 1]


def test_append_keeps_and_rescales():
    codes = np.zeros((2, 1, 16, 64), np.int8)
    scale = np.full((2, 1), 0.5, np.float32)
    codes[1, 0, 0] = 100                                              # stands for 50.0
    x = np.zeros((1, 1, 64), np.float32)
    x[0, 0, 3] = 127.0
    c, s = serving.append(codes, scale, x, [16 + 1])
    assert s[1, 0] == 1.0 and s[0, 0] == 0.5                          # grown to 127 / 127; the other block is as it was
    assert (c[1, 0, 0] == 50).all() and c[1, 0, 1, 3] == 127 and c[1, 0, 1].sum() == 127
    c2, s2 = serving.append(c, s, x / 1000, [16 + 2])                 # a smaller token leaves the scale alone
    assert s2[1, 0] == 1.0 and np.array_equal(c2[1, 0, :2], c[1, 0, :2]) and not c2[1, 0, 2].any()
    c3, s3 = serving.append(c2, s2, x * 0, [16])                      # offset 0 starts the block anew
    assert s3[1, 0] == np.float32(2.0 ** -100) and not c3[1, 0, 0].any()
    odd = x.copy()
    odd[0, 0, :3] = (np.inf, -np.inf, np.nan)
    c4, s4 = serving.append(c3, s3, odd, [0])
    assert s4[0, 0] == 1.0 and c4[0, 0, 0, :4].tolist() == [127, -127, -127, 127]
    assert np.array_equal(serving.read(c4, s4, [0, -1])[0, 0, 3:5], [127.0, 0.0]) and not serving.read(c4, s4, [-1]).any()


def test_append_is_within_half_a_step():
    g = np.random.default_rng(9)
    x = g.normal(size=(16, 2, 64)).astype(np.float32)
    c, s = serving.append(np.zeros((1, 2, 16, 64), np.int8), np.ones((1, 2), np.float32), x, np.arange(16))
    back = serving.read(c, s, np.arange(16))
    assert (np.abs(back - x) <= 0.5001 * s[0][None, :, None]).all()
    assert np.abs(c).max(axis=(0, 2, 3)).tolist() == [127, 127]


def test_attention_closed_forms():
    g = np.random.default_rng(3)
    ck, cv = np.zeros((4, 2, 16, 64), np.int8), g.integers(-127, 128, (4, 2, 16, 64)).astype(np.int8)
    ones = np.ones((4, 2), np.float32)
    table = np.array([[2, 0], [1, 3]])
    q = g.normal(size=(3, 4, 64))
    y, lse = serving.attention(q, ck, ones, cv, ones * 0.5, [0, 2, 3], [20, 1], table, 0.125)
    first = cv[[2, 0]].transpose(1, 0, 2, 3).reshape(2, 32, 64) * 0.5
    assert np.allclose(y[1, 1], first[0, :20].mean(0)) and np.allclose(y[0, 3], first[1, :19].mean(0))   # equal keys: the mean
    assert np.allclose(lse[1], np.log(20)) and np.allclose(y[2, 0], cv[1, 0, 0] * 0.5) and np.allclose(lse[2], 0)
    y, lse = serving.attention(q, ck, ones, cv, ones, [0, 2, 3], [1, 0], table, 0.125)
    assert not y[0].any() and not y[2].any() and np.isneginf(lse[0]).all() and np.allclose(lse[1], 0)    # rows that see nothing
    y, lse = serving.attention(q, ck, ones, cv, ones, [0, 2, 3], [20, 9], table, 0.125, window=1)
    assert np.allclose(y[1, 2], cv[0, 1, 3])                                                             # only itself
