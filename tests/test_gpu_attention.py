"""Attention over whole prompts and over chunks of new tokens (fc_prefill_attention,
fc_extend_batch, fc_store_chunk, fc_chunk_attention) against a plain definition in 64 bits."""

import numpy as np
import pytest

from attention_util import Chunk, blocks_for, check
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


def _prefill(lens, heads, group, dim, window=0, seed=0, strided=True, scale=0.0):
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk(lens, lens, heads, group, dim, seed=seed, strided=strided)
    try:
        lse = torch.full((len(lens), c.layers, heads * group, window), 7.0, device=c.dev) if window else None
        out = fc.fc_prefill_attention(c.pool, 1, c.q_dev, c.k_dev, c.v_dev, c.lens, lse_out=lse, window=window, scale=scale)
        torch.cuda.synchronize()
        out = out.cpu().numpy()
        at = 0
        for r, n in enumerate(lens):
            for j in range(heads * group):
                h = j // group
                rows = slice(at, at + n)
                mine = lse[r, 1, j, max(0, window - n):].cpu().numpy() if window and n else None
                check(c.q[rows, j], c.k[rows, h], c.v[rows, h], 0, out[rows, j], mine, scale or None)
            at += n
        if window:   # what is no row of this layer stays
            assert (lse[:, 0] == 7.0).all()
            for r, n in enumerate(lens):
                assert (lse[r, 1, :, :max(0, window - n)] == 7.0).all()
    finally:
        c.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[1], [2, 1, 0, 31], [32], [33], [63, 64, 65], [127, 128, 129], [257, 16, 500]], ids=str)
def test_prompts(lens, dim):
    _prefill(lens, 2, 1, dim, window=16)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 8), (2, 4), (3, 5), (1, 33), (1, 64)])
def test_prompts_with_grouped_heads(heads, group, dim):
    _prefill([1, 40, 7, 150], heads, group, dim, window=33, strided=False)


def test_a_long_prompt_and_a_scale():
    _prefill([1500], 1, 2, 128, window=64, scale=0.31)


def _chunk(lens, news, heads, group, dim, dtype="f16", window=0, seed=0, strided=True, scale=0.0):
    """Stores the new rows and attends; the pool before and after, byte by byte."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk(lens, news, heads, group, dim, seed=seed, dtype=dtype, strided=strided)
    try:
        before = c.kv_dev.cpu().numpy()
        fc.fc_store_chunk(c.pool, 1, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        lse = torch.full((len(lens), c.layers, heads * group, window), 7.0, device=c.dev) if window else None
        out = fc.fc_chunk_attention(c.pool, 1, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=window, scale=scale)
        torch.cuda.synchronize()
        want = before.copy()
        at = 0
        for r, n in enumerate(news):
            for i in range(n):
                t = lens[r] - n + i
                blk, slot = c.table[r, t // 16], t % 16
                for which, x in ((0, c.k), (1, c.v)):
                    for h in range(heads):
                        if dtype == "f16":
                            want[1, blk, which, h, slot] = x[at, h]
                        else:
                            codes, e = ao.quantise_row(x[at, h])
                            row = (which * heads + h) * 16 + slot
                            want[1, blk, row * dim:(row + 1) * dim] = codes
                            want[1, blk, 32 * heads * dim + row] = e
                at += 1
        assert (c.kv_dev.cpu().numpy() == want).all()
        c.check(1, out, lse, window, scale or None)
        if window:
            assert (lse[:, 0] == 7.0).all()
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,news", [
    ([1], [1]), ([16, 17, 0, 33], [1, 0, 0, 1]), ([40, 300, 129, 64], [1, 1, 1, 1]), ([100, 7], [5, 7]),
    ([200, 90, 1], [33, 64, 1]), ([513, 48], [100, 48]), ([300], [300])], ids=str)
def test_chunks(lens, news, dim, dtype):
    _chunk(lens, news, 2, 1, dim, dtype, window=3)


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
@pytest.mark.parametrize("heads,group", [(1, 8), (2, 4), (3, 5), (1, 64)])
def test_chunks_with_grouped_heads(heads, group, dtype):
    _chunk([150, 33, 64, 20], [1, 33, 7, 4], heads, group, 128, dtype, window=8, strided=False)


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
@pytest.mark.parametrize("dim", [64, 128])
def test_long_caches_are_split(dim, dtype):
    """Few heads: the keys of a head are split over workgroups and the states joined."""
    _chunk([2100, 513, 5, 1025], [1, 3, 1, 2], 1, 2, dim, dtype, window=2)
    _chunk([1500, 40], [40, 40], 1, 1, dim, dtype, window=64)


def test_a_scale():
    _chunk([140, 60], [2, 50], 2, 2, 64, scale=0.05, window=4)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_what_a_row_does_not_see_has_no_influence(bad, dim):
    """Not a number and infinities in later tokens' K and V, and behind the last token of a block:
    rows before them are what they are without; rows that see them are not numbers, or infinite."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    lens, news = [75, 40, 200], [75, 1, 70]
    c = Chunk(lens, news, 1, 2, dim)
    try:
        at = 40                                       # of request 0
        c.v_dev[at, 0, 3] = bad
        c.k_dev[75 + 1 + 30, 0, 5] = float("nan")     # request 2, its new token 30
        c.v_dev[75 + 1 + 30, 0, 5] = -float(bad)
        for r, n in enumerate(lens):                  # behind the last tokens
            blk = int(c.table[r, n // 16])
            if n % 16:
                c.kv_dev[1, blk, :, :, n % 16:] = bad
        fc.fc_store_chunk(c.pool, 1, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        out = fc.fc_chunk_attention(c.pool, 1, c.table_dev, c.lens, c.news, c.q_dev).cpu().numpy()
        pre = fc.fc_prefill_attention(c.pool, 1, c.q_dev[:75], c.k_dev[:75], c.v_dev[:75], c.lens[:1]).cpu().numpy()
        rows = c.pool_rows(1)
        for j in range(2):
            k, v = c.cached(rows, 0)
            for got in (out, pre):
                check(c.q[:at, j], k[0][:at], v[0][:at], 0, got[:at, j])
                x = got[at:75, j, 3]
                assert (np.isnan(x) if np.isnan(bad) else x == np.inf).all()
                keep = np.arange(dim) != 3
                check(c.q[:75, j], k[0], np.where(np.isfinite(v[0]), v[0], 0.0), 0, np.where(keep, got[:75, j], ao.attention(
                    c.q[:75, j], k[0], np.where(np.isfinite(v[0]), v[0], 0.0), 0)[0]))
            k, v = c.cached(rows, 1)
            check(c.q[75:76, j], k[0], v[0], 39, out[75:76, j])
            k, v = c.cached(rows, 2)
            check(c.q[76:106, j], k[0][:160], v[0][:160], 130, out[76:106, j])
            assert np.isnan(out[106:, j]).all()       # the key is not a number
    finally:
        c.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("fill", [0x00, 0x7e, 0xff])
def test_what_lies_behind_the_last_token_of_an_8_bit_block(fill, dim):
    """Codes and exponents of slots that hold no token: zeros, the largest numbers, not a number."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    lens, news = [5, 40, 200, 81], [5, 1, 70, 17]
    c = Chunk(lens, news, 2, 2, dim, dtype="e4m3")
    try:
        h = c.heads
        for r, n in enumerate(lens):
            if n % 16:
                block = c.kv_dev[1, int(c.table[r, n // 16])]
                block[:32 * h * dim].view(2, h, 16, dim)[:, :, n % 16:] = fill
                block[32 * h * dim:].view(2, h, 16)[:, :, n % 16:] = fill
        # a token that only the last rows see is not a number
        c.v_dev[5 + 1 + 60, 1, 7] = float("nan")
        fc.fc_store_chunk(c.pool, 1, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        out = fc.fc_chunk_attention(c.pool, 1, c.table_dev, c.lens, c.news, c.q_dev).cpu().numpy()
        assert np.isnan(out[5 + 1 + 60:76, 2:, 7]).all()
        out[5 + 1 + 60:76, 2:] = 0
        assert np.isfinite(out).all()
        rows = c.pool_rows(1)
        at = 0
        for r, n in enumerate(news):
            k, v = c.cached(rows, r)
            for j in range(4):
                seen = 60 if r == 2 and j >= 2 else n     # rows before the one that is not a number
                check(c.q[at:at + seen, j], k[j // 2][:lens[r] - n + seen], v[j // 2][:lens[r] - n + seen], lens[r] - n,
                      out[at:at + seen, j])
            at += n
    finally:
        c.close()


def test_extend_pops_in_batch_order():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    kv = torch.zeros((2, 40, 2, 2, 16, 64), dtype=torch.float16, device="cuda:0")
    pool = fc.fc_pool_create(kv, 40, 2, 2, 64)
    try:
        fc.fc_set_debug_checks(pool, True)
        table = torch.full((4, 12), -1, dtype=torch.int32, device="cuda:0")
        lens = np.zeros(4, np.int32)
        fc.fc_extend_batch(pool, table, lens, np.array([17, 0, 16, 1], np.int32))
        assert lens.tolist() == [17, 0, 16, 1] and fc.fc_pool_num_free(pool) == 36
        assert table[:, :2].tolist() == [[0, 1], [-1, -1], [2, -1], [3, -1]]
        fc.fc_extend_batch(pool, table, lens, np.array([15, 160, 1, 15], np.int32))
        assert lens.tolist() == [32, 160, 17, 16]
        assert table[0].tolist() == [0, 1] + [-1] * 10 and table[1].tolist() == list(range(4, 14)) + [-1, -1]
        assert table[2, :3].tolist() == [2, 14, -1] and table[3, :2].tolist() == [3, -1]
        stack, top = fc.fc_pool_export_state(pool)
        assert top == 25 and stack[:top].tolist() == list(range(39, 14, -1))
        for n_new, code in (([500, 0, 0, 0], fc.FC_EINVAL), ([-1, 0, 0, 0], fc.FC_EINVAL)):
            with pytest.raises(fc.FastCacheError) as e:
                fc.fc_extend_batch(pool, table, lens, np.array(n_new, np.int32))
            assert e.value.code == code
        wide = torch.full((4, 64), -1, dtype=torch.int32, device="cuda:0")
        with pytest.raises(fc.FastCacheError) as e:
            fc.fc_extend_batch(pool, wide, lens, np.array([26 * 16, 0, 0, 0], np.int32))
        assert e.value.code == fc.FC_ENOMEM
        assert lens.tolist() == [32, 160, 17, 16] and fc.fc_pool_num_free(pool) == 25 and (wide == -1).all()
    finally:
        fc.fc_pool_destroy(pool)
