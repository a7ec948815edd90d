"""The sum by which blocks are selected (csrc/fc_select_blocks.h, score_exactly): products' multiples of 2^-10 and what is
left of them, added up apart in 64 bits in any order and rounded once, give the correctly rounded sum.  No GPU."""

import math

import numpy as np


def _split_sum(x, rng):
    cut = (x + 1.5 * 2.0 ** 42) - 1.5 * 2.0 ** 42
    parts = []
    for terms in (cut, x - cut):
        terms = list(terms[rng.permutation(len(terms))])
        while len(terms) > 1:                        # any tree
            i, j = sorted(rng.choice(len(terms), 2, replace=False))
            b, a = terms.pop(j), terms.pop(i)
            terms.append(a + b)
        parts.append(terms[0])
    return parts[0] + parts[1]


def test_any_order_gives_the_sum_rounded_once():
    rng = np.random.default_rng(8)
    plain = 0
    for n in range(300):
        # fp16 numbers of the whole range, largest and smallest ones among them, and products that cancel
        a = (rng.choice([-1, 1], 128) * rng.integers(0, 0x7c00, 128).astype(np.uint16).view(np.float16).astype(np.float64))
        b = (rng.choice([-1, 1], 128) * rng.integers(0, 0x7c00, 128).astype(np.uint16).view(np.float16).astype(np.float64))
        if n % 3 == 1:
            a[64:], b[64:] = a[:64], -b[:64]
            b[3] = 2.0 ** -24
        elif n % 3 == 2:
            a[:], b[:] = 65504, 65504 * (1 if n % 2 else -1)
            a[5] = b[5] = 2.0 ** -24
        x = a * b
        assert (x.astype(np.float32) == x).all()      # (what the kernel makes of a product is exact)
        assert _split_sum(x, rng) == math.fsum(x)
        plain += x.sum() != math.fsum(x)
    assert plain > 50                                 # sums of the products themselves are not
