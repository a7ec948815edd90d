"""New tokens' rows rotated on their way into the pool: bit by bit, in every format and layout."""

import numpy as np
import pytest

from cache_util import Cache, encode
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu

N_POSITIONS = 700


def _table(rotary, dev, seed=0):
    """Cosines and sines of fp32 that are not those of any angles: the call does not know."""
    import torch
    x = np.random.default_rng(seed).uniform(-1, 1, (N_POSITIONS, 2, rotary // 2)).astype(np.float32)
    return x, torch.from_numpy(x).to(dev)


def _want(c, angles, positions, interleaved, layer):
    """(q rotated, the pool's bytes afterwards)."""
    q = c.q_dev.cpu().numpy().copy()
    k, v = c.k_dev.cpu().numpy(), c.v_dev.cpu().numpy()
    pool = c.kv_dev.cpu().numpy()
    d, h = c.dim, c.heads
    row = 0
    for r, n in enumerate(c.news.tolist()):
        for i in range(n):
            t = int(c.lens[r]) - n + i
            w = angles[int(positions[r]) + i]
            q[row] = co.rotate(q[row], w[0], w[1], interleaved)
            new = np.stack([co.rotate(k[row], w[0], w[1], interleaved), v[row]])
            block, slot = c.table[r, t // 16], t % 16
            if c.fmt == "f16":
                pool[layer, block, :, :, slot] = new
            else:
                codes, exps = encode(new, c.fmt)
                per, e_per = codes.shape[-1], exps.shape[-1]
                for which, j in np.ndindex(2, h):
                    at = (which * h + j) * 16 + slot
                    pool[layer, block, at * per:(at + 1) * per] = codes[which, j]
                    pool[layer, block, 32 * h * per + at * e_per:32 * h * per + (at + 1) * e_per] = exps[which, j]
            row += 1
    return q, pool


def _same(a, b):
    """The same bits, any not-a-number for another one."""
    if a.dtype == np.float16:
        return ((a.view(np.uint16) == b.view(np.uint16)) | (np.isnan(a) & np.isnan(b))).all()
    return (a == b).all()


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("dim,rotary,interleaved", [(64, 64, False), (64, 32, True), (64, 16, False), (128, 128, True),
                                                    (128, 128, False), (128, 48, False), (128, 80, True)])
def test_bit_by_bit(fmt, dim, rotary, interleaved):
    """Ragged chunks, one without new tokens, positions ahead of the caches, queries with heads of their own
    number; strided and head-major rows; the pool's other bytes as they were."""
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([33, 16, 40, 5], [33, 1, 0, 2], 3, 5, dim, fmt=fmt, strided=rotary != 48, seed=rotary)
    try:
        angles, table = _table(rotary, c.dev)
        positions = np.array([0, 400, -7, N_POSITIONS - 2], np.int32)
        q, pool = _want(c, angles, positions, interleaved, 1)
        got = fc.fc_rotate_store_chunk(c.pool, 1, c.table_dev, c.lens, c.news, fc.Rotation(table, interleaved), c.q_dev, c.k_dev,
                                       c.v_dev, positions=positions)
        assert _same(got.cpu().numpy(), q)
        assert _same(c.kv_dev.cpu().numpy(), pool)
    finally:
        c.close()


def test_positions_of_a_whole_cache_by_default_and_q_in_place():
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([100, 33], [3, 33], 2, 2, 128, fmt="f16")
    try:
        angles, table = _table(128, c.dev)
        q, pool = _want(c, angles, [97, 0], False, 0)
        before_k, before_v = c.k_dev.clone(), c.v_dev.clone()
        out = fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, fc.Rotation(table), c.q_dev, c.k_dev, c.v_dev,
                                       q_out=c.q_dev)
        assert out is c.q_dev and _same(c.q_dev.cpu().numpy(), q) and _same(c.kv_dev.cpu().numpy(), pool)
        assert (c.k_dev == before_k).all() and (c.v_dev == before_v).all()    # parts of the same rows
    finally:
        c.close()


def test_without_queries_and_one_token():
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([1], [1], 1, 1, 64, fmt="e2m1", layers=1)
    try:
        angles, table = _table(64, c.dev)
        _, pool = _want(c, angles, [0], True, 0)
        assert fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, fc.Rotation(table, True), None, c.k_dev, c.v_dev) is None
        assert _same(c.kv_dev.cpu().numpy(), pool)
    finally:
        c.close()


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
def test_numbers_at_the_ends(fmt):
    """Overflow to infinity, infinite and no numbers, zeros of both signs, subnormal ones, sums that cancel."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([32], [32], 1, 1, 64, fmt=fmt, layers=1)
    try:
        rng = np.random.default_rng(8)
        x = np.clip(rng.standard_normal((32, 1, 64)) * np.exp2(rng.uniform(-26, 17, (32, 1, 64))), -65504, 65504).astype(np.float16)
        x[0], x[1], x[2, 0, 3], x[3, 0, 40], x[4, 0, 5] = 0, -0.0, np.inf, np.nan, -np.inf
        x[5] = 65504
        x[6, 0, 32:] = x[6, 0, :32]
        for t in (c.q_dev, c.k_dev, c.v_dev):
            t.copy_(torch.from_numpy(x))
        angles, table = _table(64, c.dev)
        angles[6, 1] = angles[6, 0]                     # (a cos - a cos)
        angles[7] = 0
        angles[8, 0], angles[8, 1] = 1, 0
        table.copy_(torch.from_numpy(angles))
        q, pool = _want(c, angles, [0], False, 0)
        got = fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, fc.Rotation(table), c.q_dev, c.k_dev, c.v_dev)
        assert _same(got.cpu().numpy(), q)
        got = c.kv_dev.cpu().numpy()
        if fmt == "e4m3":                               # (codes that are not numbers have either sign)
            nan = (pool & 127 == 127) & (np.arange(pool.shape[-1]) < 32 * 64)
            got[nan & (got & 127 == 127)] = pool[nan & (got & 127 == 127)]
        assert _same(got, pool)
    finally:
        c.close()


def test_more_requests_than_arguments_hold():
    from paper_2503_08461_amd import fastcache as fc
    n = 170
    c = Cache([1 + i % 40 for i in range(n)], [i % 2 for i in range(n)], 1, 2, 64, fmt="e4m3", layers=1)
    try:
        angles, table = _table(64, c.dev)
        positions = np.arange(n, dtype=np.int32) * 3
        q, pool = _want(c, angles, positions, False, 0)
        got = fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, fc.Rotation(table), c.q_dev, c.k_dev, c.v_dev,
                                       positions=positions)
        assert _same(got.cpu().numpy(), q) and _same(c.kv_dev.cpu().numpy(), pool)
    finally:
        c.close()


def test_a_table_behind_32_bits():
    """Positions whose rows of the table begin behind 2^32 bytes."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([20], [3], 2, 1, 128, fmt="f16", layers=1)
    try:
        n = (1 << 32) // 512 + 10
        table = torch.zeros((n, 2, 64), device=c.dev)
        angles, few = _table(128, c.dev)
        table[-3:] = few[:3]
        q, pool = _want(c, angles, [0], False, 0)
        got = fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, fc.Rotation(table), c.q_dev, c.k_dev, c.v_dev,
                                       positions=np.array([n - 3], np.int32))
        assert _same(got.cpu().numpy(), q) and _same(c.kv_dev.cpu().numpy(), pool)
    finally:
        c.close()
