"""Batches for the tests of the attention over prompts and chunks: packed rows, a pool with a
permuted block table, the oracle's results and the error bound of a result."""

import numpy as np

from oracle import attention_oracle as ao


def blocks_for(n):
    return (n + 15) // 16


def bounds(q, k, v, out, spread, n_seen, scale=None):
    """How far a result may be off, per row and channel.  q, k, v: fp64, one head.

    A logit is a sum of d products in fp32, scaled, each step off by 2^-24 of the magnitudes
    summed, d + 2 steps: delta; exp2 in fp32 adds 2^-22 and the sums' own rounding n 2^-24 at
    most; both enter numerator and denominator.  The numerator is rounded to fp16 for the
    product (2^-11, or 2^-25 below 2^-14 where the denominator is at least 1), the result too."""
    d = q.shape[1]
    scale = scale or 1.0 / np.sqrt(d)
    mag = scale * (np.abs(q) @ np.abs(k).T).max(1, initial=0.0)
    delta = (d + 2) * 2.0 ** -24 * mag + 2.0 ** -22 + n_seen * 2.0 ** -24
    vmax = np.abs(v).max(initial=0.0)
    return 2.0 ** -11 * np.abs(out) + (2.0 ** -11 + 2 * delta)[:, None] * spread * (1 + 2.0 ** -10) + \
        (n_seen * 2.0 ** -25 * vmax)[:, None] + 2.0 ** -25


def lse_bound(q, k, lse, n_seen, scale=None):
    """The logits' error, the sum's, a logarithm in fp32 (2^-22 of its value) and its scaling."""
    d = q.shape[1]
    scale = scale or 1.0 / np.sqrt(d)
    mag = scale * (np.abs(q) @ np.abs(k).T).max(1, initial=0.0)
    return (d + 4) * 2.0 ** -24 * mag + 2.0 ** -21 + n_seen * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse)


def check(q, k, v, first, got, lse=None, scale=None):
    """One request's rows of one query head against the oracle; lse: of the last rows, or None."""
    want, want_lse, spread = ao.attention(q, k, v, first, scale)
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n_seen = np.clip(first + 1 + np.arange(len(q)), 0, len(k))
    err = np.abs(got.astype(np.float64) - want)
    tol = bounds(q, k, v, want, spread, n_seen, scale)
    assert (err <= tol).all(), "out: off by %g where %g is allowed (row %d)" % (
        err.flat[(err - tol).argmax()], tol.flat[(err - tol).argmax()], (err - tol).argmax() // q.shape[1])
    if lse is not None and len(lse):
        w = want_lse[len(want_lse) - len(lse):]
        tol = lse_bound(q, k, want_lse, n_seen, scale)[len(want_lse) - len(lse):]
        assert (np.abs(lse - w) <= tol).all(), "lse: off by %g" % np.abs(lse - w).max()


class Chunk:
    """A pool and a batch of requests with `lens` tokens, of which the last `news` are new: the
    older ones' rows lie in the pool, the new ones' are packed.  rng values, four loud key channels."""

    def __init__(self, lens, news, heads, group, dim, seed=0, dtype="f16", layers=2, strided=True, spare=3):
        import torch
        from paper_2503_08461_amd import fastcache as fc
        rng = np.random.default_rng(seed)
        self.fc, self.dev = fc, torch.device("cuda:0")
        self.lens, self.news = np.array(lens, np.int32), np.array(news, np.int32)
        self.heads, self.group, self.dim, self.layers = heads, group, dim, layers
        need = [blocks_for(n) for n in lens]
        self.n_blocks = sum(need) + spare
        loud = np.where(rng.random((heads, dim)).argsort(-1).argsort(-1) < 4, 8.0, 1.0)
        kv = rng.standard_normal((layers, self.n_blocks, 2, heads, 16, dim))
        kv[:, :, 0] *= loud[:, None, :]
        self.kv = kv.astype(np.float16)
        ids = rng.permutation(self.n_blocks)
        self.table = np.full((len(lens), max(need + [1]) + 1), -1, np.int32)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = ids[at:at + n]
            at += n
        total = int(self.news.sum())
        self.q = rng.standard_normal((total, heads * group, dim)).astype(np.float16)
        self.k = (rng.standard_normal((total, heads, dim)) * loud).astype(np.float16)
        self.v = rng.standard_normal((total, heads, dim)).astype(np.float16)
        self.e4m3 = dtype == "e4m3"
        self.table_dev = torch.from_numpy(self.table).to(self.dev)
        if self.e4m3:
            self.kv_dev = torch.from_numpy(self.image8()).to(self.dev)
        else:
            self.kv_dev = torch.from_numpy(self.kv).to(self.dev)
        self.pool = fc.fc_pool_create(self.kv_dev, self.n_blocks, layers, heads, dim,
                                      dtype=fc.FC_DTYPE_E4M3 if self.e4m3 else fc.FC_DTYPE_F16)
        if strided:   # parts of one projection's rows
            x = torch.from_numpy(np.concatenate([self.q, self.k, self.v], 1)).to(self.dev)
            h, hq = heads, heads * group
            self.q_dev, self.k_dev, self.v_dev = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
        else:         # head-major
            self.q_dev, self.k_dev, self.v_dev = (
                torch.from_numpy(np.ascontiguousarray(x.transpose(1, 0, 2))).to(self.dev).transpose(0, 1)
                for x in (self.q, self.k, self.v))

    def image8(self):
        """The pool's rows quantised by the oracle, as the 8-bit pool holds them."""
        n_l, nb, _, h, _, d = self.kv.shape
        out = np.zeros((n_l, nb, 32 * h * (d + 1)), np.uint8)
        for idx in np.ndindex(n_l, nb):
            codes = np.zeros((2, h, 16, d), np.uint8)
            exps = np.zeros((2, h, 16), np.uint8)
            for row in np.ndindex(2, h, 16):
                codes[row], exps[row] = ao.quantise_row(self.kv[idx][row])
            out[idx] = np.concatenate([codes.ravel(), exps.ravel()])
        return out

    def pool_rows(self, layer):
        """[block][2][head][slot][d] of one layer as the device has it now, fp64."""
        x = self.kv_dev[layer].cpu().numpy()
        if not self.e4m3:
            return x.astype(np.float64)
        h, d = self.heads, self.dim
        codes = x[:, :32 * h * d].reshape(-1, 2, h, 16, d)
        return ao.values(codes, x[:, 32 * h * d:].reshape(-1, 2, h, 16))

    def cached(self, rows, r):
        """(K, V) of request r, [head][token][d]."""
        n = int(self.lens[r])
        x = rows[self.table[r, :blocks_for(n)]].transpose(1, 2, 0, 3, 4)
        x = x.reshape(2, self.heads, -1, self.dim)[:, :, :n]
        return x[0], x[1]

    def check(self, layer, out, lse=None, window=0, scale=None):
        rows = self.pool_rows(layer)
        out = out.cpu().numpy()
        lse = None if lse is None else lse.cpu().numpy()
        at = 0
        for r, n in enumerate(self.news.tolist()):
            if n == 0:
                continue
            k, v = self.cached(rows, r)
            for j in range(self.heads * self.group):
                h = j // self.group
                mine = None if lse is None else lse[r, layer, j, max(0, window - n):]
                check(self.q[at:at + n, j], k[h], v[h], int(self.lens[r]) - n, out[at:at + n, j], mine, scale)
            at += n

    def close(self):
        self.fc.fc_pool_destroy(self.pool)
