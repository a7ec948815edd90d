"""A decode step over an 8-bit pool whose heads are cut into segments, or taken by 16 wavefronts, or by
four in a call of more heads than CUs, against 64 bits."""

import numpy as np
import pytest

from attention_util import Chunk
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


class LongChunk(Chunk):
    """An 8-bit pool whose rows are made all at once (what it holds is read back, not compared)."""

    def image8(self):
        import torch
        x = self.kv.astype(np.float32)
        e = np.clip(np.ceil(np.log2(np.abs(x).max(-1) / 448.0)), -15, 8)
        codes = torch.from_numpy(x / np.exp2(e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        flat = x.shape[:2] + (-1,)
        return np.concatenate([codes.reshape(flat), (e + 127).astype(np.uint8).reshape(flat)], 2)


def tolerance(q, k, v, out, spread):
    """Per channel, one query.  A logit: the scaled query rounded, d products and sums in fp32, the row's
    power of two exact: (d + 4) 2^-24 of the magnitudes summed, in log2 units 1.45 times that, absolutely.
    A weight: exp2 of the hardware, 2^-22, once for itself and once for each time that the maximum moved
    behind it (a key at most each, and the joins, fewer than 2^7).  Sums of n terms: n 2^-24.  Numerator
    and denominator both; then the division and the result, 2^-23."""
    n, d = k.shape
    mag = (np.abs(k) @ np.abs(q)).max() / np.sqrt(d)
    delta = (d + 4) * 2.0 ** -24 * mag * 1.45 + (n + 128) * (2.0 ** -22 + 2.0 ** -24)
    return 2 * delta * spread + 2.0 ** -23 * np.abs(out) + 1e-30


def _check(lens, heads, dim, layers, seed=0):
    import torch
    c = LongChunk(lens, [0] * len(lens), heads, 1, dim, dtype="e4m3", seed=seed, layers=layers)
    try:
        q = np.random.default_rng(seed + 1).standard_normal((len(lens), layers, heads, dim)).astype(np.float16)
        got = c.fc.fc_decode_attention(c.pool, c.table_dev, c.lens, torch.from_numpy(q).to(c.dev)).cpu().numpy()
        for layer in range(layers):
            rows = c.pool_rows(layer)
            for r, n in enumerate(lens):
                k, v = c.cached(rows, r)
                for h in range(heads):
                    x = q[r, layer, h].astype(np.float64)
                    if n == 0:
                        assert (got[r, layer, h] == 0).all()
                        continue
                    want, _, spread = (y[0] for y in ao.attention(x[None], k[h], v[h], n - 1))
                    err = np.abs(got[r, layer, h] - want)
                    assert (err <= tolerance(x, k[h], v[h], want, spread)).all(), (layer, r, h, err.max())
    finally:
        c.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[2100, 0, 40, 700], [8000], [2049, 2049, 1], [3000, 1024, 1023, 512, 511]], ids=str)
def test_heads_cut_into_segments(lens, dim):
    _check(lens, 2, dim, 1, seed=dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,heads,layers", [([2048, 241, 16, 0], 2, 2), ([1024] + [48] * 7, 17, 2), ([1000] + [30] * 7, 17, 2)], ids=str)
def test_heads_whole_and_more_heads_than_compute_units(lens, heads, layers, dim):
    """16 wavefronts a head; more heads than CUs, the longest cut in two; the same with four wavefronts a whole head."""
    _check(lens, heads, dim, layers, seed=dim + 1)
