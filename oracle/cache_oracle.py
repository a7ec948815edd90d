"""CPU oracle of rows in 4 bits, of rows rotated by their positions and of attention over selected
blocks (test infrastructure; shares no code with the library).

  * 4-bit rows: 32 channels are a group of e2m1 codes (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6) times
    2^e, e the smallest integer in [-23, 13] with max |x| <= 6 * 2^e (13 where none is); nearest code,
    ties to the even one, found by comparison with every number that a code stands for; a group with a
    channel that is no finite number is not a number: exponent byte 255, codes 0;
  * rotation: (a, b) -> (a cos - b sin, b cos + a sin) in fp64, rounded to fp32 and then to fp16;
  * bounds: smallest and largest of each channel over a block's tokens, not a number where one is;
  * selection: the blocks with the best sums of max(q lo, q hi), the sums rounded correctly
    (math.fsum), ties to the lower one, the last block always.
"""

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def quantise_row(x):
    """One row of fp16 numbers -> (codes uint8 [d], exponents + 127 uint8 [d / 32])."""
    x = np.asarray(x, np.float64)
    codes = np.zeros(x.shape, np.uint8)
    exps = np.zeros(len(x) // GROUP, np.uint8)
    for g in range(len(exps)):
        part = x[g * GROUP:(g + 1) * GROUP]
        if not np.isfinite(part).all():
            exps[g] = 255
            continue
        e = -23
        while np.abs(part).max() > 6.0 * 2.0 ** e and e < 13:
            e += 1
        exps[g] = e + 127
        d = np.abs(E2M1 - np.abs(part)[:, None] / 2.0 ** e)
        nearest = d == d.min(1, keepdims=True)
        # (two are as near: the even one)
        c = np.where(nearest.sum(1) == 1, nearest.argmax(1), (nearest & (np.arange(8) % 2 == 0)).argmax(1))
        codes[g * GROUP:(g + 1) * GROUP] = c | np.where(np.signbit(part), 8, 0)
    return codes, exps


def pack(codes):
    """Codes [..., d] -> bytes [..., d / 2], the even channel's code in the low half."""
    return codes[..., ::2] | (codes[..., 1::2] << 4)


def values(packed, exponents):
    """What packed codes [..., d / 2] and exponents + 127 [..., d / 32] stand for, fp64."""
    codes = np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (-1,))
    x = np.where(codes & 8, -E2M1[codes & 7], E2M1[codes & 7])
    scale = np.where(exponents == 255, np.nan, np.exp2(np.asarray(exponents, np.float64) - 127))
    return (x.reshape(x.shape[:-1] + (-1, GROUP)) * scale[..., None]).reshape(x.shape)


def rotate(x, cos, sin, interleaved):
    """Rows [..., d] of fp16 numbers, angles of their position [rotary / 2] fp32 -> fp16 rows."""
    x = np.asarray(x, np.float16)
    n = 2 * len(cos)
    out = x.copy()
    cos, sin = np.asarray(cos, np.float64), np.asarray(sin, np.float64)
    a_at, b_at = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    a, b = x[..., a_at].astype(np.float64), x[..., b_at].astype(np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        out[..., a_at] = (a * cos - b * sin).astype(np.float32).astype(np.float16)
        out[..., b_at] = (b * cos + a * sin).astype(np.float32).astype(np.float16)
    return out


def bounds(k):
    """k [tokens][d] of one block -> (smallest [d], largest [d])."""
    return np.min(k, 0), np.max(k, 0)     # (numpy's propagate what is not a number)


def score(q, lo, hi):
    """q [heads][d], lo and hi [d], fp16 numbers: the largest over the heads of the sum of max(q lo, q hi)."""
    best = -math.inf
    for row in np.asarray(q, np.float64):
        terms = np.fmax(row * np.asarray(lo, np.float64), row * np.asarray(hi, np.float64))
        s = math.nan if np.isnan(terms).any() else math.fsum(terms) if np.isfinite(terms).all() else terms.sum()
        if math.isnan(s):
            return math.nan
        best = max(best, s)
    return best


def select(scores, n_select):
    """scores of a request's blocks (the last entry is not looked at) -> ascending entries of those read."""
    n = len(scores)
    if n <= n_select:
        return list(range(n))
    order = sorted(range(n - 1), key=lambda b: (not math.isnan(scores[b]), -scores[b] if not math.isnan(scores[b]) else 0.0, b))
    return sorted(order[:n_select - 1]) + [n - 1]
