"""Results written over their queries: as into memory of their own."""

import pytest

from attention_util import Chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
@pytest.mark.parametrize("strided", [True, False])
@pytest.mark.parametrize("lens,news,heads,group", [([300, 40, 5], [200, 40, 1], 2, 3), ([64, 33], [4, 32], 3, 1),
                                                   ([2100, 1100], [1, 40], 1, 2)], ids=str)
def test_results_over_their_queries(lens, news, heads, group, strided, dtype):
    import torch
    c = Chunk(lens, news, heads, group, 64, dtype=dtype, layers=1, strided=strided)
    try:
        for _ in range(3):
            q = c.q_dev.clone(memory_format=torch.preserve_format)
            c.fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
            want = c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q)
            got = c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q, out=q)
            assert torch.equal(got, want)
        q = c.q_dev.clone()
        want = c.fc.fc_prefill_attention(c.pool, 0, q, c.k_dev, c.v_dev, c.news)
        assert torch.equal(c.fc.fc_prefill_attention(c.pool, 0, q, c.k_dev, c.v_dev, c.news, out=q), want)
    finally:
        c.close()
