"""Selected blocks whose scores, selection and attention are launches of their own, with several heads of K and V that
select each for itself, in parts of the blocks and tiles of the tokens, and with results that are joined from segments;
and the attention over 4 bits of up to 16 rows of several heads, cut into segments.  Which way these calls go is held by
test_sparse_paths.py."""

import numpy as np
import pytest

from cache_util import Cache
from test_gpu_sparse import _step

pytestmark = pytest.mark.gpu

# lens, new tokens, heads of K and V, query heads of each, channels, blocks selected
APART = [
    ([1500, 1300], [5, 2], 3, 4, 128, 70),            # two parts, selections longer than a segment
    ([6200], [1], 2, 1, 128, 30),                     # a single token of a long cache, seven parts
    ([1100, 60, 700], [2, 1, 3], 2, 40, 64, 6),       # more rows than the one launch takes
    ([1300, 1113, 300], [1, 1, 1], 5, 4, 64, 66),     # single tokens, one of which reads all of its blocks
    ([1500], [17], 4, 5, 128, 65),                    # twelve tokens a tile, two tiles
    ([1500], [2], 2, 40, 128, 70),                    # many rows a token, cut into segments
]
# the same over 4 bits without a selection: lens, new tokens, heads, query heads of each, channels
FEW_ROWS = [([1500, 2100], [1, 4], 3, 4, 128), ([2500, 40, 1111], [2, 1, 2], 2, 8, 64)]


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lens,news,heads,group,dim,n_select", APART, ids=str)
def test_heads_that_select_apart(fmt, lens, news, heads, group, dim, n_select):
    c = Cache(lens, news, heads, group, dim, fmt=fmt, seed=3, layers=1)
    try:
        _, selected = _step(c, 0, n_select)
        # (that heads are mixed up would not show if they chose the same)
        assert (selected[0] != selected[0, :1]).any()
    finally:
        c.close()


@pytest.mark.parametrize("lens,news,heads,group,dim", FEW_ROWS, ids=str)
def test_few_rows_of_several_heads_in_segments(lens, news, heads, group, dim):
    import torch
    c = Cache(lens, news, heads, group, dim, seed=5, layers=1)
    try:
        lse = torch.zeros((len(lens), 1, heads * group, 1), device=c.dev)
        out = c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=1)
        c.check(0, out, lse, 1)
    finally:
        c.close()
