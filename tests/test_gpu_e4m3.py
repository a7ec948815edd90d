"""The 8-bit pool: quantised copies and appends bit by bit, attention over it in 64 bits."""

import numpy as np
import pytest

from attention_util import Chunk, blocks_for
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu

RTOL, ATOL = 1e-3, 1e-4   # as the fp16 pool's decode attention: fp32 sums and hardware exp2


def _hard_rows(rng, n, dim):
    """Rows over fp16's whole range: subnormal, ordinary, largest numbers, ties, zeros, not finite."""
    x = rng.standard_normal((n, dim)) * np.exp2(rng.uniform(-26, 14, (n, 1)))
    x = np.clip(x, -65504, 65504).astype(np.float16)
    x[0] = 0
    x[1, :4] = [65504, -57344, 57376, 61440]
    x[2] = np.float16(448) * (np.arange(dim) % 2 * 2 - 1)
    x[3, 0] = np.float16(448.25)
    x[4] = (np.arange(dim) % 33) * np.float16(2.0 ** -4) + np.float16(1)   # ties between codes
    x[4, -1] = 448
    x[5] = np.arange(dim).astype(np.float16) * np.float16(2.0 ** -24)
    x[6, 3], x[6, 5], x[6, 6] = np.inf, -np.inf, np.nan
    x[7] = np.inf
    x[8, 1:] = -0.0
    return x


@pytest.mark.parametrize("dim", [64, 128])
def test_quantise_batch_bit_by_bit(dim):
    """Ragged lengths, a request switched off, an empty one; slots behind the last token and other
    blocks keep what they had; the blocks come from fc_extend_batch."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    rng = np.random.default_rng(dim)
    lens = [33, 0, 16, 5, 48]
    enable = np.array([1, 1, 1, 0, 1], np.int32)
    heads, layers = 3, 2
    c = Chunk(lens, [0] * 5, heads, 1, dim, layers=layers)
    nb8 = 12
    kv8 = torch.full((layers, nb8, 32 * heads * (dim + 1)), 0xA5, dtype=torch.uint8, device=c.dev)
    pool8 = fc.fc_pool_create(kv8, nb8, layers, heads, dim, dtype=fc.FC_DTYPE_E4M3)
    try:
        kv = c.kv.reshape(-1, dim)
        kv[:] = np.concatenate([_hard_rows(rng, 64, dim) for _ in range(len(kv) // 64 + 1)])[rng.permutation(len(kv))]
        c.kv_dev.copy_(torch.from_numpy(c.kv))
        table8 = torch.full((5, 4), -1, dtype=torch.int32, device=c.dev)
        lens8 = np.zeros(5, np.int32)
        fc.fc_extend_batch(pool8, table8, lens8, (c.lens * enable).astype(np.int32))
        fc.fc_quantise_batch(pool8, table8, c.pool, c.table_dev, c.lens, enable)
        torch.cuda.synchronize()
        want = np.full(tuple(kv8.shape), 0xA5, np.uint8)
        t8 = table8.cpu().numpy()
        for r, n in enumerate(lens):
            for t in range(n if enable[r] else 0):
                for layer in range(layers):
                    for which in range(2):
                        for h in range(heads):
                            codes, e = ao.quantise_row(c.kv[layer, c.table[r, t // 16], which, h, t % 16])
                            row = (which * heads + h) * 16 + t % 16
                            at = want[layer, t8[r, t // 16]]
                            at[row * dim:(row + 1) * dim] = codes
                            at[32 * heads * dim + row] = e
        got = kv8.cpu().numpy()
        nan = (want & 127 == 127) & (np.arange(want.shape[-1]) < 32 * heads * dim)   # (either sign)
        assert ((got == want) | (nan & (got & 127 == 127))).all()
    finally:
        c.close()
        fc.fc_pool_destroy(pool8)


def _decode_want(c, q):
    out = np.zeros(q.shape)
    for layer in range(c.layers):
        rows = c.pool_rows(layer)
        for r, n in enumerate(c.lens.tolist()):
            if n:
                k, v = c.cached(rows, r)
                for h in range(c.heads):
                    out[r, layer, h] = ao.attention(q[r, layer, h][None], k[h], v[h], n - 1)[0][0]
    return out


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[1, 0, 15, 16, 17, 65, 300], [511, 40], [513, 0, 1, 256, 257]], ids=str)
def test_decode_attention(lens, dim):
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk(lens, [0] * len(lens), 2, 1, dim, dtype="e4m3", seed=dim)
    try:
        q = np.random.default_rng(4).standard_normal((len(lens), c.layers, c.heads, dim)).astype(np.float16)
        got = fc.fc_decode_attention(c.pool, c.table_dev, c.lens, torch.from_numpy(q).to(c.dev)).cpu().numpy()
        want = _decode_want(c, q)
        assert (np.abs(got - want) <= RTOL * np.abs(want) + ATOL).all(), np.abs(got - want).max()
    finally:
        c.close()


@pytest.mark.parametrize("dim", [64, 128])
def test_append_quantises_the_new_rows(dim):
    """Three steps over block boundaries, a request switched off, then attention over all."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    rng = np.random.default_rng(9)
    lens = [15, 16, 0, 30]
    c = Chunk(lens, [0] * 4, 3, 1, dim, dtype="e4m3", spare=8)
    try:
        fc.fc_pool_import_state(c.pool, np.array(sorted(set(range(c.n_blocks)) - set(c.table[c.table >= 0].tolist())) +
                                                 [0] * int((c.table >= 0).sum()), np.int32), 8)
        want = c.kv_dev.cpu().numpy()
        enable = np.array([1, 1, 1, 0], np.int32)
        for step in range(3):
            new = _hard_rows(rng, 4 * c.layers * 2 * 3, dim).reshape(4, c.layers, 2, 3, dim)
            new[~np.isfinite(new)] = 1
            before = c.lens.copy()
            fc.fc_append_batch(c.pool, c.table_dev, c.lens, torch.from_numpy(new).to(c.dev), enable)
            assert (c.lens == before + enable).all()
            c.table = c.table_dev.cpu().numpy()
            for r in range(3):
                blk, slot = c.table[r, before[r] // 16], before[r] % 16
                for layer, which, h in np.ndindex(c.layers, 2, 3):
                    codes, e = ao.quantise_row(new[r, layer, which, h])
                    row = (which * 3 + h) * 16 + slot
                    want[layer, blk, row * dim:(row + 1) * dim] = codes
                    want[layer, blk, 96 * dim + row] = e
        assert (c.kv_dev.cpu().numpy() == want).all()
    finally:
        c.close()


def test_nan_reaches_the_output():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([300, 300], [0, 0], 1, 1, 128, dtype="e4m3", layers=1)
    try:
        c.kv_dev[0, int(c.table[1, 3]), 5 * 128 + 7] = 127       # K, slot 5
        q = torch.ones((2, 1, 1, 128), dtype=torch.float16, device=c.dev)
        got = fc.fc_decode_attention(c.pool, c.table_dev, c.lens, q)
        assert torch.isnan(got[1]).all() and not torch.isnan(got[0]).any()
    finally:
        c.close()
