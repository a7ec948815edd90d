"""Pins of oracle/cache_oracle.py: rows in 4 bits by hand, rotations as complex numbers, selections written out."""

import math

import numpy as np

from oracle import cache_oracle as co


def test_codes_by_hand():
    x = np.zeros(64, np.float16)
    # group 0: largest 6 -> e = 0; ties between codes go to the even one
    x[:14] = [6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.0, 0.26, 5.004, 4.996]
    # group 1: largest 6.004 -> e = 1: halved
    x[32:36] = [6.004, 3.0, -1.0, 0.5]
    codes, exps = co.quantise_row(x)
    assert list(codes[:14]) == [7, 15, 0, 2, 2, 4, 4, 6, 6, 8, 8, 1, 7, 6]
    assert list(exps) == [127, 128] and list(codes[32:36]) == [5, 3, 9, 0]
    y = co.values(co.pack(codes), exps)
    assert list(y[:9]) == [6, -6, 0, 1, 1, 2, 2, 4, 4] and list(y[32:36]) == [6, 3, -1, 0]
    assert co.pack(codes)[0] == 7 | 15 << 4 and co.pack(codes)[1] == 0 | 2 << 4


def test_codes_at_the_ends_of_the_range():
    x = np.zeros(32, np.float16)
    assert co.quantise_row(x)[1][0] == 127 - 23
    x[0], x[1] = 2.0 ** -24, -3 * 2.0 ** -24       # the smallest fp16 numbers
    codes, exps = co.quantise_row(x)
    assert exps[0] == 127 - 23 and codes[0] == 1 and codes[1] == 8 + 3
    x[0], x[1] = 65504, 40960                      # over 6 * 2^13: the largest code
    codes, exps = co.quantise_row(x)
    assert exps[0] == 127 + 13 and codes[0] == 7 and codes[1] == 6 and co.values(co.pack(codes), exps)[0] == 49152
    for bad in (np.inf, -np.inf, np.nan):
        x[5] = bad
        codes, exps = co.quantise_row(x)
        assert exps[0] == 255 and (codes == 0).all() and np.isnan(co.values(co.pack(codes), exps)).all()


def test_values_are_within_a_quarter_and_fp16_numbers():
    rng = np.random.default_rng(3)
    x = np.clip(rng.standard_normal(32 * 400) * np.exp2(rng.uniform(-25, 15, 400)).repeat(32), -65504, 65504).astype(np.float16)
    codes, exps = co.quantise_row(x)
    y = co.values(co.pack(codes), exps)
    unit = np.exp2(exps.astype(np.float64) - 127).repeat(32)
    assert (np.abs(y - x) <= 0.25 * np.maximum(np.abs(x.astype(np.float64)), unit)).all()
    assert (y.astype(np.float16) == y).all() and (np.signbit(y) == np.signbit(x)).all()
    assert (co.quantise_row(y.astype(np.float16))[0] == codes)[np.abs(codes.reshape(-1, 32) & 7).max(1).repeat(32) > 6].all()


def test_rotation_is_a_product_of_complex_numbers():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 64)).astype(np.float16)
    angle = rng.uniform(0, 50, 24)
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    w = cos.astype(np.float64) + 1j * sin.astype(np.float64)
    for interleaved in (False, True):
        y = co.rotate(x, cos, sin, interleaved)
        a, b = ((slice(0, 48, 2), slice(1, 48, 2)) if interleaved else (slice(0, 24), slice(24, 48)))
        z = (x[:, a].astype(np.float64) + 1j * x[:, b].astype(np.float64)) * w
        assert np.abs(y[:, a] - z.real).max() < 2.0 ** -9 and np.abs(y[:, b] - z.imag).max() < 2.0 ** -9
        assert (y[:, 48:] == x[:, 48:]).all()
    quarter = co.rotate(x, np.zeros(32, np.float32), np.ones(32, np.float32), False)
    assert (quarter[:, :32] == -x[:, 32:]).all() and (quarter[:, 32:] == x[:, :32]).all()


def test_scores_bound_every_logit():
    rng = np.random.default_rng(7)
    k, q = rng.standard_normal((16, 64)).astype(np.float16), rng.standard_normal((3, 64)).astype(np.float16)
    lo, hi = co.bounds(k)
    assert co.score(q, lo, hi) >= (q.astype(np.float64) @ k.T.astype(np.float64)).max()
    one = k[:1]
    assert math.isclose(co.score(q, *co.bounds(one)), (q.astype(np.float64) @ one[0].astype(np.float64)).max())
    k[3, 5] = np.nan
    assert math.isnan(co.score(q, *co.bounds(k)))


def test_selection_by_hand():
    nan, inf = math.nan, math.inf
    assert co.select([3.0, 1.0, 2.0, -inf], 4) == [0, 1, 2, 3]
    assert co.select([3.0, 1.0, 2.0, 9.0, 0.0], 3) == [0, 3, 4]
    assert co.select([1.0, 1.0, 1.0, 1.0, -5.0], 3) == [0, 1, 4]           # ties: the lower ones
    assert co.select([0.0, -0.0, 0.0, 7.0], 3) == [0, 1, 3]                # zeros are one value
    assert co.select([inf, nan, 5.0, nan, 0.0], 3) == [1, 3, 4]
    assert co.select([-inf, -1.0, -inf, 0.0], 2) == [1, 3]
    assert co.select([5.0, 4.0, 3.0], 1) == [2]                            # the token's own block
