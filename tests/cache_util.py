"""Batches for the tests of rows in 4 bits, of rotated rows and of attention over selected blocks: a pool of
any of the three formats filled by the oracles, its rows read back, and bounds of a result in fp32."""

import numpy as np

from attention_util import Chunk, blocks_for
from oracle import attention_oracle as ao
from oracle import cache_oracle as co


def encode(x, fmt):
    """Rows [..., d] of fp16 numbers -> (codes as the pool's bytes [..., n], exponents [..., m])."""
    lead = x.shape[:-1]
    rows = [co.quantise_row(r) if fmt == "e2m1" else ao.quantise_row(r) for r in x.reshape(-1, x.shape[-1])]
    codes = np.stack([co.pack(c) if fmt == "e2m1" else c for c, _ in rows])
    exps = np.stack([np.atleast_1d(e) for _, e in rows]).astype(np.uint8)
    return codes.reshape(lead + (-1,)), exps.reshape(lead + (-1,))


def image(kv, fmt):
    """[layer][block][2][head][16][d] fp16 -> the pool's bytes [layer][block][...], or kv itself."""
    if fmt == "f16":
        return kv
    codes, exps = encode(kv, fmt)
    n = kv.shape[:2]
    return np.concatenate([codes.reshape(n + (-1,)), exps.reshape(n + (-1,))], -1)


def rows_of(image_, fmt, heads, dim):
    """The pool's bytes (or fp16 rows) [...][block] -> values [...][block][2][head][16][d], fp64."""
    if fmt == "f16":
        return image_.astype(np.float64)
    per = 32 * heads * dim // (2 if fmt == "e2m1" else 1)
    codes, exps = image_[..., :per], image_[..., per:]
    lead = image_.shape[:-1]
    codes = codes.reshape(lead + (2, heads, 16, -1))
    if fmt == "e2m1":
        return co.values(codes, exps.reshape(lead + (2, heads, 16, -1)))
    return ao.values(codes, exps.reshape(lead + (2, heads, 16)))


def dtype_of(fmt):
    from paper_2503_08461_amd import fastcache as fc
    return {"f16": fc.FC_DTYPE_F16, "e4m3": fc.FC_DTYPE_E4M3, "e2m1": fc.FC_DTYPE_E2M1}[fmt]


class Cache(Chunk):
    """Chunk (attention_util) over a pool of fmt "f16", "e4m3" or "e2m1"."""

    def __init__(self, lens, news, heads, group, dim, fmt="e2m1", kv=None, **kw):
        import torch
        super().__init__(lens, news, heads, group, dim, **kw)
        self.fmt = fmt
        if kv is not None:
            self.kv = kv(self)
        self.fc.fc_pool_destroy(self.pool)
        self.kv_dev = torch.from_numpy(image(self.kv, fmt)).to(self.dev)
        self.pool = self.fc.fc_pool_create(self.kv_dev, self.n_blocks, self.layers, heads, dim, dtype=dtype_of(fmt))

    def pool_rows(self, layer):
        return rows_of(self.kv_dev[layer].cpu().numpy(), self.fmt, self.heads, self.dim)

    def upload(self):
        """self.kv into the pool."""
        import torch
        self.kv_dev.copy_(torch.from_numpy(image(self.kv, self.fmt)))

    def new_bounds(self, fill=0.0):
        import torch
        return torch.full((self.layers, self.n_blocks, self.heads, 2, self.dim), fill, dtype=torch.float16, device=self.dev)


def decode_check(c, q, got, scale=None):
    """A decode step's fp32 result [request][layer][head][d] against 64 bits.

    A logit is a sum of d products in fp32, of queries that the scale was multiplied into: d + 4 roundings of
    2^-24 of the magnitudes summed; exp2 in fp32 2^-22, and as much for each of the up to ten factors that
    states are joined with; sums of n numbers n 2^-24: all of it in numerator and denominator, and the
    quotient 2^-22 of itself."""
    d = c.dim
    s = scale or 1.0 / np.sqrt(d)
    for layer in range(c.layers):
        rows = c.pool_rows(layer)
        for r, n in enumerate(c.lens.tolist()):
            k, v = c.cached(rows, r)
            for h in range(c.heads):
                mine = got[r, layer, h].astype(np.float64)
                if n == 0:
                    assert (mine == 0).all()
                    continue
                want, _, spread = ao.attention(q[r, layer, h][None], k[h], v[h], n - 1, s)
                mag = s * (np.abs(k[h]) @ np.abs(q[r, layer, h].astype(np.float64))).max()
                delta = (d + 4) * 2.0 ** -24 * mag + 11 * 2.0 ** -22 + n * 2.0 ** -24
                err, tol = np.abs(mine - want[0]), 2 * delta * spread[0] + 2.0 ** -22 * np.abs(want[0]) + 1e-30
                assert (err <= tol).all(), (r, layer, h, n, (err / tol).max())
