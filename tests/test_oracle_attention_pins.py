"""Pins of oracle/attention_oracle.py: closed forms, a sum over pairs written out, e4m3 by hand."""

import numpy as np

from oracle import attention_oracle as ao


def test_attention_closed_forms():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((7, 4)), rng.standard_normal((7, 4))
    out, lse, spread = ao.attention(np.zeros((3, 4)), k, v, 2)      # equal logits: means of what is seen
    for i in range(3):
        assert np.allclose(out[i], v[:3 + i].mean(0)) and np.isclose(lse[i], np.log(3 + i))
        assert np.allclose(spread[i], np.abs(v[:3 + i]).mean(0))
    out, lse, _ = ao.attention(rng.standard_normal((2, 4)), k, v, -1)    # row 0 sees nothing, row 1 one key
    assert (out[0] == 0).all() and lse[0] == -np.inf and np.allclose(out[1], v[0])


def test_attention_against_a_sum_over_pairs():
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal((n, 8)) for n in (3, 6, 6))
    out, lse, _ = ao.attention(q, k, v, 3, scale=0.4)
    for i in range(3):
        z, acc = 0.0, np.zeros(8)
        for j in range(4 + i):
            w = np.exp(0.4 * sum(q[i, c] * k[j, c] for c in range(8)))
            z += w
            acc += w * v[j]
        assert np.allclose(out[i], acc / z) and np.isclose(lse[i], np.log(z))


def test_e4m3_by_hand():
    assert ao.E4M3[126] == 448 and ao.E4M3[119] == 240 and ao.E4M3[8] == 2.0 ** -6 and ao.E4M3[1] == 2.0 ** -9
    # 448 keeps e = 0; just above needs e = 1; a tie goes to the even code
    c, e = ao.quantise_row([448.0, 1.0, -1.0, 1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10])
    assert e == 127 and c.tolist() == [126, 0x38, 0xb8, 0x38, 0x3a, 0, 2]
    c, e = ao.quantise_row([448.25, 0.0])
    assert e == 128 and ao.values(c, e)[0] == 448.0
    c, e = ao.quantise_row([65504.0, -57344.0])
    assert e == 135 and ao.values(c, e).tolist() == [61440.0, -57344.0]
    c, e = ao.quantise_row([0.0, -0.0])
    assert e == 112 and c.tolist() == [0, 128]
    c, e = ao.quantise_row([np.inf, 2.0, np.nan])
    assert c[0] == 127 and c[2] == 127 and ao.values(c, e)[1] == 2.0 and np.isnan(ao.values(c, e)[0])


def test_every_value_of_a_row_is_a_half():
    rng = np.random.default_rng(3)
    for scale in (2.0 ** -24, 2.0 ** -20, 1e-4, 1.0, 300.0, 60000.0):
        x = (rng.uniform(-1, 1, 64) * scale).astype(np.float16)
        y = ao.values(*ao.quantise_row(x))
        assert (y == y.astype(np.float16)).all()
        e = ao.quantise_row(x)[1] - 127
        assert (np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x.astype(np.float64)), 2.0 ** (e - 10))).all()
