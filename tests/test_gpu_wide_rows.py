"""Packed rows whose offsets pass 32 bits: the largest strides that fc_rows takes, by token and by head."""

import numpy as np
import pytest

from attention_util import Chunk, check

pytestmark = pytest.mark.gpu


def _spread(x, token_stride, head_stride, dev):
    """The rows of x [token][head][channel] at these strides, in memory of their own."""
    import torch
    n, h, d = x.shape
    memory = torch.empty((n - 1) * token_stride + (h - 1) * head_stride + d, dtype=torch.float16, device=dev)
    rows = memory.as_strided((n, h, d), (token_stride, head_stride, 1))
    rows.copy_(torch.from_numpy(x))
    return rows


@pytest.mark.parametrize("token_stride,head_stride", [(1 << 24, 128), (128, 0x7ffffff8), (1 << 24, 0x7ffffff8)])
@pytest.mark.parametrize("lens", [[120], [9, 5]], ids=str)   # (128 tokens of 2^24 are a head's stride and 8: rows would overlap)
def test_largest_strides(lens, token_stride, head_stride):
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk(lens, lens, 2, 2, 128, layers=1)
    try:
        # (a token's heads, or a head's tokens, one after the other: results may not overlap)
        out_strides = (token_stride, 128) if token_stride > 128 else (128, head_stride)
        q, k, v = (_spread(x, token_stride, head_stride, c.dev) for x in (c.q, c.k, c.v))
        out = _spread(np.zeros_like(c.q), *out_strides, c.dev)
        fc.fc_prefill_attention(c.pool, 0, q, k, v, c.lens, out=out)
        packed = fc.fc_prefill_attention(c.pool, 0, *(torch.from_numpy(x).to(c.dev) for x in (c.q, c.k, c.v)), c.lens)
        fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.lens, k, v)
        paged = fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.lens, q)
        assert torch.equal(out, packed)
        c.check(0, paged)
        at = 0
        for n in lens:
            for h in range(4):
                check(c.q[at:at + n, h], c.k[at:at + n, h // 2], c.v[at:at + n, h // 2], 0, packed[at:at + n, h].cpu().numpy())
            at += n
    finally:
        c.close()
