"""The longest caches in 8 bits, 32768 tokens: a decode step, single tokens, a chunk, with a scale."""

import numpy as np
import pytest

from oracle import attention_oracle as ao
from test_gpu_split_e4m3 import LongChunk, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 0.21])
def test_the_longest_caches(dim, scale):
    import torch
    c = LongChunk([32768, 32767, 17], [1, 40, 17], 1, 2, dim, dtype="e4m3", layers=1, seed=dim)
    try:
        fc = c.fc
        fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        lse = torch.zeros((3, 1, 2, 17), device=c.dev)
        out = fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=17, scale=scale)
        c.check(0, out, lse, 17, scale or None)
        q = np.random.default_rng(2).standard_normal((3, 1, 1, dim)).astype(np.float16)
        got = fc.fc_decode_attention(c.pool, c.table_dev, c.lens, torch.from_numpy(q).to(c.dev), scale=scale).cpu().numpy()
        rows = c.pool_rows(0)
        for r, n in enumerate(c.lens.tolist()):
            k, v = c.cached(rows, r)
            x = q[r, 0, 0].astype(np.float64)
            want, _, spread = (y[0] for y in ao.attention(x[None], k[0], v[0], n - 1, scale or None))
            # (the tolerance is of logits times 1 / sqrt(dim): a larger scale makes them that much larger)
            most = tolerance(x * max(1.0, scale * np.sqrt(dim)), k[0], v[0], want, spread)
            assert (np.abs(got[r, 0, 0] - want) <= most).all()
    finally:
        c.close()
