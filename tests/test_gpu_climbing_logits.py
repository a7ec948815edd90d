"""Attention where the running maximum moves: logits that climb by a little less and a little more than
the kernels let a maximum run ahead (2^8), that fall, and that jump, through short and long caches, few and
many rows, all sources of keys, whole and split."""

import numpy as np
import pytest

from attention_util import check
from oracle import attention_oracle as ao
from test_gpu_split_e4m3 import LongChunk, tolerance

pytestmark = pytest.mark.gpu

LOUD = 8.0   # of the query, in the four channels that carry the climb


def heights(n, pattern, per, rng):
    """A logit for each of n tokens, in log2 units; per: the tokens in which a wavefront goes on by one tile."""
    step = np.arange(n) // 32 * (32.0 / per)
    if pattern == "under":
        return 7.9 * step
    if pattern == "over":
        return 8.1 * step
    if pattern == "down":
        return 8.1 * (step[-1] - step)
    return rng.choice([0.0, 7.9, 8.1, 20.0, 60.0], size=-(-n // 32))[np.arange(n) // 32]


def keys_of(logits, dim, rng):
    """fp16 rows whose product with (LOUD x 4, 0, ...) is near the logits: multiples of 64, 8, 1 and 1/8 in
    the first four channels, which 8-bit rows hold as they are."""
    k = 0.5 * rng.standard_normal((len(logits), dim))
    x = logits * np.log(2.0) * np.sqrt(dim) / LOUD
    assert x.max() < 512
    for c, unit in enumerate((64.0, 8.0, 1.0, 0.125)):
        k[:, c] = np.floor(x / unit) * unit
        x = x - k[:, c]
    return k.astype(np.float16)


def _batch(lens, news, heads, group, dim, dtype, pattern, per, seed):
    """Every token's K and V through fc_store_chunk; the queries of the last `news`."""
    import torch
    rng = np.random.default_rng(seed)
    c = LongChunk(lens, lens, heads, 1, dim, dtype=dtype, seed=seed, layers=1)
    for h in range(heads):
        at = 0
        for n in lens:
            c.k[at:at + n, h] = keys_of(heights(n, pattern, per, rng), dim, rng)
            at += n
    c.k_dev, c.v_dev = torch.from_numpy(c.k).to(c.dev), torch.from_numpy(c.v).to(c.dev)
    c.fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.lens, c.k_dev, c.v_dev)
    c.news = np.array(news, np.int32)
    c.group = group
    q = 0.25 * rng.standard_normal((int(c.news.sum()), heads * group, dim))
    q[:, :, :4] = LOUD
    c.q = q.astype(np.float16)
    c.q_dev = torch.from_numpy(c.q).to(c.dev)
    return c


PATTERNS = ["under", "over", "down", "jumps"]


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
@pytest.mark.parametrize("lens,news,group,dim,per", [
    ([1000, 70], [1, 1], 4, 128, 128),     # few rows, a head whole: a wavefront has every fourth 32 keys
    ([1000, 33], [5, 3], 4, 64, 128),
    ([3000, 513], [1, 2], 2, 128, 128),    # ... and split
    ([900, 300], [130, 40], 1, 128, 64),   # many rows: every 64 keys
    ([640], [200], 3, 64, 64),
    ([2100], [100], 1, 64, 64),            # ... and split
], ids=str)
def test_chunks(lens, news, group, dim, per, dtype, pattern):
    import torch
    c = _batch(lens, news, 2, group, dim, dtype, pattern, per, seed=dim + len(lens))
    try:
        window = 4
        lse = torch.full((len(lens), 1, 2 * group, window), 7.0, device=c.dev)
        out = c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=window)
        c.check(0, out, lse, window)
    finally:
        c.close()


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("n,dim", [(900, 128), (700, 64), (30, 128)])
def test_prompts(n, dim, pattern):
    c = _batch([n], [n], 2, 1, dim, "f16", pattern, 64, seed=n)
    try:
        out = c.fc.fc_prefill_attention(c.pool, 0, c.q_dev, c.k_dev, c.v_dev, c.lens).cpu().numpy()
        for h in range(2):
            check(c.q[:, h], c.k[:, h], c.v[:, h], 0, out[:, h])
    finally:
        c.close()


@pytest.mark.parametrize("pattern", PATTERNS)
@pytest.mark.parametrize("n,dim", [(200, 64), (1500, 128), (3000, 64), (3000, 128)])
def test_decode_step_over_8_bits(n, dim, pattern):
    c = _batch([n], [1], 2, 1, dim, "e4m3", pattern, 64, seed=n)
    try:
        got = c.fc.fc_decode_attention(c.pool, c.table_dev, c.lens, c.q_dev[:, None]).cpu().numpy()
        k, v = c.cached(c.pool_rows(0), 0)
        for h in range(2):
            x = c.q[0, h].astype(np.float64)
            want, _, spread = (y[0] for y in ao.attention(x[None], k[h], v[h], n - 1))
            assert (np.abs(got[0, 0, h] - want) <= tolerance(x, k[h], v[h], want, spread)).all()
    finally:
        c.close()
