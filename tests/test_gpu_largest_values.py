"""Attention over values at the end of fp16's range: a mean of finite values is finite, and infinite
where a value that a row sees is."""

import numpy as np
import pytest

from attention_util import Chunk, check

pytestmark = pytest.mark.gpu

TOP = 65504.0


def _values(c, infinite):
    """V of channels 0 to 3: the largest number, its negative, both in turn, and one infinity."""
    import torch
    at = 0
    for n in c.lens.tolist():
        v = c.v[at:at + n]
        v[:, :, 0], v[:, :, 1] = TOP, -TOP
        v[:, :, 2] = np.where(np.arange(n) % 2, TOP, -TOP)[:, None]
        if infinite:
            v[n // 2, :, 3] = np.inf
        at += n
    c.v_dev = torch.from_numpy(c.v).to(c.dev)


def _check(c, rows_of, out, infinite):
    """rows_of: (queries' rows, first row's last key) of every request."""
    at = start = 0
    for n, new in zip(c.lens.tolist(), rows_of):
        for j in range(c.heads * c.group):
            h = j // c.group
            v = np.where(np.isfinite(c.v[start:start + n, h]), c.v[start:start + n, h], 0)
            got = out[at:at + new, j].copy()
            if infinite:
                sees = n - new + np.arange(new) >= n // 2
                assert (got[sees, 3] == np.inf).all() and np.isfinite(got[~sees, 3]).all()
                got[:, 3] = 0
                v[:, 3] = 0
            assert np.isfinite(got).all()
            check(c.q[at:at + new, j], c.k[start:start + n, h], v, n - new, got)
        at += new
        start += n


@pytest.mark.parametrize("infinite", [False, True])
@pytest.mark.parametrize("group,dim", [(1, 128), (4, 64)])
@pytest.mark.parametrize("lens,news", [([70, 33, 500], [1, 3, 8]), ([300, 140], [300, 130]), ([2100], [2]), ([2100], [70])], ids=str)
def test_chunks(lens, news, group, dim, infinite):
    import torch
    if infinite and lens == [2100]:
        # (a key of no weight times infinity is not a number, as in the definition's own arithmetic)
        lens, news = [40], news[:1] if news[0] < 40 else [40]
    c = Chunk(lens, lens, 2, 1, dim, layers=1, seed=dim + len(lens))
    try:
        _values(c, infinite)
        c.k = (c.k * 0.25).astype(np.float16)
        c.k_dev = torch.from_numpy(c.k).to(c.dev)
        c.fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.lens, c.k_dev, c.v_dev)
        c.group = group
        n = np.array(news, np.int32)
        c.q = np.random.default_rng(5).standard_normal((int(n.sum()), 2 * group, dim)).astype(np.float16)
        out = c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, n, torch.from_numpy(c.q).to(c.dev))
        _check(c, news, out.cpu().numpy(), infinite)
    finally:
        c.close()


@pytest.mark.parametrize("infinite", [False, True])
@pytest.mark.parametrize("lens", [[9], [200, 31, 64]], ids=str)
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts(lens, dim, infinite):
    import torch
    c = Chunk(lens, lens, 2, 2, dim, layers=1, seed=dim)
    try:
        _values(c, infinite)
        c.k = (c.k * 0.25).astype(np.float16)
        c.k_dev = torch.from_numpy(c.k).to(c.dev)
        out = c.fc.fc_prefill_attention(c.pool, 0, c.q_dev, c.k_dev, c.v_dev, c.lens)
        _check(c, lens, out.cpu().numpy(), infinite)
    finally:
        c.close()


@pytest.mark.parametrize("weight", [128.0635, 128.07, 128.1, 64.035])
@pytest.mark.parametrize("n,new,far", [(200, 1, 130), (200, 130, 69), (2100, 1, 130), (2100, 100, 69)])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_mean_of_equal_values(dim, n, new, far, weight):
    """Every value the largest number: so is every result, however the weights are rounded.  Nearly all
    weight is on a later key that the running maximum is left behind for, a weight that fp16 holds only
    to 2^-11 of it: the rounded numerators over the exact sum are past 65520, where fp16 becomes infinite."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([n], [n], 1, 1, dim, layers=1)
    try:
        k = np.zeros((n, 1, dim), np.float16)
        k[:, 0, 0] = -3                 # (weights of 2^-21 and less)
        k[0, 0, 0], k[far, 0, 0] = 0, 1
        v = np.full((n, 1, dim), TOP, np.float16)
        v[:, :, 1::2] = -TOP
        q = np.zeros((n, 1, dim), np.float16)
        q[:, 0, 0] = 1
        q, k, v = (torch.from_numpy(x).to(c.dev) for x in (q, k, v))
        scale = float(np.log(weight))
        fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.lens, k, v)
        outs = [fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, np.array([new], np.int32), q[:new], scale=scale)]
        if n == 200:
            outs.append(fc.fc_prefill_attention(c.pool, 0, q, k, v, c.lens, scale=scale))
        for out in outs:
            out = out.cpu().numpy().astype(np.float64)
            # (half a step of the result, half a step of every numerator, which go the same way at worst)
            assert (np.abs(out - np.where(np.arange(dim) % 2, -TOP, TOP)) <= 2.0 ** -10 * TOP).all(), np.abs(out).max()
    finally:
        c.close()
