"""Bounds of blocks bit by bit, selections entry by entry, and the attention over what was selected in 64 bits."""

import math

import numpy as np
import pytest

from attention_util import blocks_for, check
from cache_util import Cache
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


def _bounds(c, layer, last=None):
    """The oracle's bounds of every block of the batch, [request][block][head] -> (lo, hi)."""
    rows = c.pool_rows(layer)
    out = []
    for r, n in enumerate(c.lens.tolist()):
        k, _ = c.cached(rows, r)
        out.append([[co.bounds(k[h, b * 16:(b + 1) * 16]) for h in range(c.heads)] for b in range(blocks_for(n))])
    return out


def _same(a, b):
    return ((a == b) | (np.isnan(a) & np.isnan(b))).all()


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("dim", [64, 128])
def test_block_bounds(fmt, dim):
    """Whole caches, then those of a few new tokens: other entries as they were, slots behind the last token
    without influence, what is not a number kept."""
    import torch
    c = Cache([33, 0, 16, 5, 47], [2, 0, 16, 1, 18], 3, 1, dim, fmt=fmt, seed=dim)
    try:
        c.kv[0, c.table[0, 0], 0, 1, 3, 7] = np.nan
        c.kv[0, c.table[2, 0], 0, 2, 15, :3] = [np.inf, -np.inf, np.nan] if fmt == "f16" else np.nan
        c.kv[0, c.table[3, 0], 0, :, 5:] = np.nan                   # behind the last token
        c.kv[0, c.table[4, 2], 0, :, 15:] = np.nan
        c.upload()
        for news, layer in ((c.lens, 0), (c.news, 1)):
            bounds = c.new_bounds(7.0)
            c.fc.fc_block_bounds(c.pool, layer, c.table_dev, c.lens, news, bounds)
            want = np.full(tuple(bounds.shape), 7.0)
            for r, blocks in enumerate(_bounds(c, layer)):
                for b in range((int(c.lens[r]) - int(news[r])) // 16 if news[r] else len(blocks), len(blocks)):
                    for h in range(c.heads):
                        want[layer, c.table[r, b], h] = blocks[b][h]
            assert _same(bounds.cpu().numpy().astype(np.float64), want)
    finally:
        c.close()


def _step(c, layer, n_select, bounds=None, want_selected=None, scale=0.0, **kw):
    """One call, its selection against the oracle's and its result against 64 bits over what was selected."""
    import torch
    if bounds is None:
        bounds = c.new_bounds()
        c.fc.fc_block_bounds(c.pool, layer, c.table_dev, c.lens, c.lens, bounds)
    selected = torch.full((int(c.news.sum()), c.heads, n_select), -9, dtype=torch.int32, device=c.dev)
    out = c.fc.fc_sparse_attention(c.pool, layer, c.table_dev, c.lens, c.news, bounds, n_select, c.q_dev, selected=selected,
                                   scale=scale, **kw)
    got, out_ = selected.cpu().numpy(), out.cpu().numpy()
    q_all, held = c.q_dev.cpu().numpy() if "out" not in kw else c.q, bounds[layer].cpu().numpy()
    rows = c.pool_rows(layer)
    t = 0
    for r, n in enumerate(c.news.tolist()):
        k, v = c.cached(rows, r) if n else (None, None)
        for i in range(n):
            seen = int(c.lens[r]) - n + i + 1
            nb = blocks_for(seen)
            for h in range(c.heads):
                q = q_all[t, h * c.group:(h + 1) * c.group]
                scores = [co.score(q, *held[c.table[r, b], h]) for b in range(nb - 1)] + [0.0] if nb > n_select else [0.0] * nb
                want = co.select(scores, n_select)
                assert got[t, h].tolist() == want + [-1] * (n_select - len(want)), (t, h)
                tok = np.concatenate([np.arange(b * 16, min(b * 16 + 16, seen)) for b in want])
                for j in range(c.group):
                    check(q[j:j + 1], k[h][tok], v[h][tok], len(tok) - 1, out_[t:t + 1, h * c.group + j], scale=scale or None)
            t += 1
    return out, selected


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lens,news,heads,group,dim,n_select", [
    ([1], [1], 1, 1, 64, 1), ([1], [1], 1, 1, 128, 9), ([300, 16, 17, 33, 0], [1, 1, 1, 3, 0], 2, 4, 128, 3),
    ([300, 97], [5, 2], 3, 1, 64, 1), ([500, 700], [1, 18], 2, 5, 64, 7), ([400], [1], 1, 40, 128, 6),
    ([260, 5, 64], [1, 1, 1], 40, 1, 64, 16),
    ([290, 40], [4, 3], 2, 2, 64, 1), ([1200, 90, 333], [1, 1, 2], 1, 64, 64, 5), ([300, 90], [1, 2], 2, 20, 128, 4),
    ([310, 50, 1], [1, 2, 1], 2, 32, 64, 4)], ids=str)
def test_selection_and_attention(fmt, lens, news, heads, group, dim, n_select):
    c = Cache(lens, news, heads, group, dim, fmt=fmt, seed=n_select, layers=2 if fmt == "f16" else 1)
    try:
        _step(c, c.layers - 1, n_select)
    finally:
        c.close()


@pytest.mark.parametrize("lens,news,n_select,fmt", [
    ([4100, 2000], [1, 2], 30, "f16"), ([1041], [1], 64, "f16"), ([1040], [1], 66, "f16"), ([32768], [1], 2047, "f16"),
    ([6300, 2000], [2, 2], 30, "f16"), ([6400, 300, 4600], [34, 3, 1], 7, "e2m1"), ([7000], [2], 100, "e4m3"),
    ([7000, 4113], [1, 1], 100, "e2m1")], ids=str)
def test_long_caches(lens, news, n_select, fmt):
    """Scores made by several workgroups, all of the keys that the selection can hold, segments of the result."""
    c = Cache(lens, news, 1, 2, 64, fmt=fmt, layers=1)
    try:
        _step(c, 0, n_select)
    finally:
        c.close()


def test_many_heads_of_long_caches():
    """One workgroup for scores, selection and attention: many tokens of a few blocks, single ones of many."""
    c = Cache([6400 + 16 * i for i in range(3)] * 7, [1] * 21, 7, 1, 64, fmt="f16", layers=1)
    try:
        _step(c, 0, 20)
    finally:
        c.close()
    c = Cache([1100 + 16 * i for i in range(3)] * 3, [20] * 9, 3, 1, 64, fmt="f16", layers=1)
    try:
        assert int(c.news.sum()) * c.heads >= 512
        _step(c, 0, 20)
    finally:
        c.close()


@pytest.mark.parametrize("n", [600, 4000, 7000])
def test_ties_go_to_the_lower_blocks(n):
    """Queries of zeros, blocks that are the same, scores that differ in the last of 64 bits' places."""
    import torch
    c = Cache([n, n, n], [1, 1, 1], 1, 2, 64, fmt="f16", layers=1)
    try:
        c.q[0] = 0
        c.kv[0, c.table[1, 3::2]] = c.kv[0, c.table[1, 2]]
        # request 2: one channel decides by 2^-24 * 2^-14 beside sums of some 64 * 2^10
        c.q[2] = np.float16(2.0 ** 5)
        c.q[2, :, 9] = np.float16(2.0 ** -14)
        ids = c.table[2][c.table[2] >= 0]
        c.kv[0, ids] = np.float16(2.0 ** 5)
        for i, b in enumerate(ids):
            c.kv[0, b, 0, :, :, 9] = np.float16((i * 7 % 11) * 2.0 ** -24)
        c.upload()
        c.q_dev.copy_(torch.from_numpy(c.q))
        for n_select in (2, 7, 37):
            _, selected = _step(c, 0, n_select)
            assert selected[0, 0].tolist() == list(range(n_select - 1)) + [blocks_for(n) - 1]
    finally:
        c.close()


@pytest.mark.parametrize("n,lens", [(600, 1), (1600, 1), (7000, 1), (7000, 3)])
@pytest.mark.parametrize("dim", [64, 128])
def test_scores_whose_order_of_sums_would_decide(n, lens, dim):
    """Sums that lose what blocks differ by where large products that cancel come first: the score is the sum
    of all of them, rounded once."""
    import torch
    c = Cache([n] * lens, [1] * lens, 1, 2, dim, fmt="f16", layers=1)
    try:
        c.q[:] = 0
        c.q[:, :, [0, 2]] = np.float16(2.0 ** 15)
        c.q[:, :, 1] = 1
        for r in range(lens):
            ids = c.table[r, :blocks_for(n)]
            c.kv[0, ids] = 0
            for i, b in enumerate(ids):
                # 2^30 + 2^-24 (7 i mod 61) - 2^30: 31 and 24 bits, 2 more than there are
                c.kv[0, b, 0, :, :, 0] = np.float16(2.0 ** 15 if i % 2 else 0)
                c.kv[0, b, 0, :, :, 1] = np.float16((i * 7 % 61) * 2.0 ** -24)
                c.kv[0, b, 0, :, :, 2] = np.float16(-2.0 ** 15 if i % 2 else 0)
        c.upload()
        c.q_dev.copy_(torch.from_numpy(c.q))
        for n_select in (2, 7, 25):
            _step(c, 0, n_select, scale=2.0 ** -31)
    finally:
        c.close()


@pytest.mark.parametrize("n", [400, 7000])
def test_scores_that_are_not_finite(n):
    """Blocks with keys that are infinite or not numbers: they are read, and what they hold shows."""
    import torch
    c = Cache([n, n, n], [1, 1, 1], 1, 1, 64, fmt="f16", layers=1)
    try:
        c.q[:] = np.abs(c.q) + np.float16(0.1)
        c.kv[0, c.table[0, 5], 0, 0, 3, 2] = np.nan
        c.kv[0, c.table[1, 6], 0, 0, 3, 2] = np.inf
        c.kv[0, c.table[2, 7], 0, 0, :, 2] = -np.inf            # the worst of all: never selected
        c.upload()
        c.q_dev.copy_(torch.from_numpy(c.q))
        bounds = c.new_bounds()
        c.fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.lens, bounds)
        selected = torch.empty((3, 1, 4), dtype=torch.int32, device=c.dev)
        out = c.fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, 4, c.q_dev, selected=selected)
        assert 5 in selected[0, 0].tolist() and 6 in selected[1, 0].tolist() and 7 not in selected[2, 0].tolist()
        assert torch.isnan(out[0]).all() and torch.isnan(out[1]).all() and torch.isfinite(out[2]).all()
    finally:
        c.close()


def test_a_new_key_shows_at_once():
    """The token's own block is read whatever its bounds say, and earlier tokens of a chunk do not see later ones."""
    import torch
    c = Cache([100], [3], 1, 1, 64, fmt="f16", layers=1)
    try:
        bounds = c.new_bounds()
        c.fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens - 3, c.lens - 3, bounds)   # as before the new tokens
        c.fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        _step(c, 0, 2, bounds=bounds)
    finally:
        c.close()


def test_more_tokens_than_arguments_hold_and_results_in_place():
    import torch
    c = Cache([200] * 80, [2] * 80, 1, 1, 64, fmt="e4m3", layers=1)
    try:
        assert int(c.news.sum()) > 149
        c.q_dev = c.q_dev.contiguous()
        _step(c, 0, 5, out=c.q_dev, scale=0.3)
    finally:
        c.close()


def test_all_blocks_are_the_whole_attention():
    import torch
    for fmt in ("f16", "e4m3", "e2m1"):
        c = Cache([300, 2000, 15], [1, 2, 1], 2, 4, 128, fmt=fmt, layers=1)
        try:
            bounds = c.new_bounds(float("nan"))                 # (not looked at)
            out = c.fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, 125, c.q_dev)
            c.check(0, out)
        finally:
            c.close()


def test_far_bounds():
    """Bounds that lie behind 2^32 bytes."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    heads, dim = 40, 128
    n_blocks = (1 << 32) // (512 * heads) + 40
    dev = torch.device("cuda:0")
    kv = torch.zeros((1, n_blocks, 17 * heads * dim), dtype=torch.uint8, device=dev)
    bounds = torch.zeros((1, n_blocks, heads, 2, dim), dtype=torch.float16, device=dev)
    pool = fc.fc_pool_create(kv, n_blocks, 1, heads, dim, dtype=fc.FC_DTYPE_E2M1)
    try:
        table = torch.arange(n_blocks - 8, n_blocks, dtype=torch.int32, device=dev)[None]
        lens, one = np.array([120], np.int32), np.array([1], np.int32)
        gen = torch.Generator(dev).manual_seed(1)
        x = torch.randn((120, heads, dim), generator=gen, device=dev).half()
        fc.fc_store_chunk(pool, 0, table, lens, lens, x, x)
        fc.fc_block_bounds(pool, 0, table, lens, lens, bounds)
        assert int((bounds[0, :-8] != 0).sum()) == 0 and int((bounds[0, -8:] != 0).sum()) > 0
        q = torch.randn((1, heads, dim), generator=gen, device=dev).half()
        far = torch.empty((1, heads, 3), dtype=torch.int32, device=dev)
        near = torch.empty_like(far)
        out = fc.fc_sparse_attention(pool, 0, table, lens, one, bounds, 3, q, selected=far)
        kv[0, :8], bounds[0, :8] = kv[0, -8:], bounds[0, -8:]
        assert (fc.fc_sparse_attention(pool, 0, table - (n_blocks - 8), lens, one, bounds, 3, q, selected=near) == out).all()
        assert (near == far).all() and int(far[..., 2].unique()) == 7
    finally:
        fc.fc_pool_destroy(pool)
