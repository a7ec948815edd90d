"""CPU oracle of the attention over whole prompts and chunks of new tokens, and of the 8-bit
rows (test infrastructure; shares no code with the library).

  * attention: query row i of a request (all of one head) sees keys 0 .. first + i;
    out = softmax(scale * q K^T) V, lse = log sum exp(scale * q k), both over the keys that
    the row sees, in fp64;
  * 8-bit rows: codes of the OCP e4m3 numbers times 2^e, e the smallest integer in [-15, 8]
    with max |x| <= 448 * 2^e; nearest code, ties to the even one, found by comparison with
    every number that a code stands for; codes stop at 240 where e = 8.
"""

import numpy as np


def attention(q, k, v, first, scale=None):
    """q [rows][d], k and v [keys][d] -> (out [rows][d], lse [rows], spread [rows][d]);
    spread = softmax . |V|, what an error bound of a result is made of."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    if scale is None or scale <= 0:
        scale = 1.0 / np.sqrt(q.shape[1])
    out = np.zeros_like(q)
    spread = np.zeros_like(q)
    lse = np.full(q.shape[0], -np.inf)
    for i in range(q.shape[0]):
        n = min(k.shape[0], first + i + 1)
        if n <= 0:
            continue
        t = scale * (k[:n] @ q[i])
        top = t.max()
        w = np.exp(t - top)
        lse[i] = top + np.log(w.sum())
        w /= w.sum()
        out[i] = w @ v[:n]
        spread[i] = w @ np.abs(v[:n])
    return out, lse, spread


def _e4m3_values():
    """The magnitude of every code without a sign, 0..126 (127 is not a number)."""
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append(np.ldexp(1 + m / 8, e - 7) if e else np.ldexp(m / 8, -6))
    return np.array(out)


E4M3 = _e4m3_values()


def quantise_row(x):
    """One row of fp16 numbers -> (codes uint8, exponent + 127)."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x)
    top = np.abs(x[finite]).max() if finite.any() else 0.0
    e = -15
    while top > 448.0 * 2.0 ** e:
        e += 1
    assert e <= 8, "not an fp16 number"
    codes = np.zeros(x.shape, np.uint8)
    last = 119 if e == 8 else 126      # 240, 448
    for i, v in enumerate(x):
        if not np.isfinite(v):
            codes[i] = 127
            continue
        d = np.abs(E4M3[:last + 1] - abs(v) / 2.0 ** e)
        best = np.flatnonzero(d == d.min())
        c = best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]
        codes[i] = c | (128 if np.signbit(v) else 0)
    return codes, e + 127


def values(codes, exponent):
    """What codes (any shape) and their rows' exponents + 127 (without the last axis) stand for."""
    mag = np.append(E4M3, np.nan)[codes & 127]
    return np.where(codes & 128, -mag, mag) * np.exp2(np.asarray(exponent, np.float64) - 127)[..., None]
