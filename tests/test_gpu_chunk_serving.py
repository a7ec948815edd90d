"""The calls on prompts, chunks and 8-bit pools together, as a server makes them, and in the ways a
server may: captured and replayed, on another stream, many requests, far blocks, rows of any layout."""

import numpy as np
import pytest

from attention_util import Chunk, blocks_for, check
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


def test_a_conversation():
    """Prompts: attention with the window rows' log-sum-exps, K and V into the pool, compression with
    them; the next turn's chunk over the compressed caches; then into an 8-bit pool, a drafted chunk
    and a decode step there.  Every attention against 64 bits over the cache as it is then."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    layers, heads, group, dim, window = 2, 3, 1, 64, 16
    rng = np.random.default_rng(11)
    lens = np.array([70, 200, 33], np.int32)
    n_blocks = 60
    dev = torch.device("cuda:0")
    kv = torch.zeros((layers, n_blocks, 2, heads, 16, dim), dtype=torch.float16, device=dev)
    kv8 = torch.zeros((layers, n_blocks, 32 * heads * (dim + 1)), dtype=torch.uint8, device=dev)
    pool = fc.fc_pool_create(kv, n_blocks, layers, heads, dim)
    pool8 = fc.fc_pool_create(kv8, n_blocks, layers, heads, dim, dtype=fc.FC_DTYPE_E4M3)

    def rows(n):
        x = torch.from_numpy(rng.standard_normal((n, heads * (group + 2), dim)).astype(np.float16)).to(dev)
        return x[:, :heads * group], x[:, heads * group:heads * (group + 1)], x[:, heads * (group + 1):]

    def cached(layer, eight=False):
        t = (table8 if eight else table).cpu().numpy()
        if eight:
            b = kv8[layer].cpu().numpy()
            x = ao.values(b[:, :32 * heads * dim].reshape(-1, 2, heads, 16, dim), b[:, 32 * heads * dim:].reshape(-1, 2, heads, 16))
        else:
            x = kv[layer].cpu().numpy().astype(np.float64)
        n = lens8 if eight else lens
        return [x[t[r, :blocks_for(n[r])]].transpose(1, 2, 0, 3, 4).reshape(2, heads, -1, dim)[:, :, :n[r]] for r in range(3)]

    def compare(out, q, n_new, caches, total):
        out, q, at = out.cpu().numpy(), q.cpu().numpy(), 0
        for r, n in enumerate(n_new):
            for h in range(heads):
                check(q[at:at + n, h], caches[r][0][h], caches[r][1][h], int(total[r]) - int(n), out[at:at + n, h])
            at += n

    try:
        table = torch.full((3, 20), -1, dtype=torch.int32, device=dev)
        start = np.zeros(3, np.int32)
        fc.fc_extend_batch(pool, table, start, lens)
        assert (start == lens).all()
        lse = torch.empty((3, layers, heads, window), device=dev)
        q_window = torch.empty((3, layers, heads, window, dim), dtype=torch.float16, device=dev)
        for layer in range(layers):
            q, k, v = rows(int(lens.sum()))
            out = fc.fc_prefill_attention(pool, layer, q, k, v, lens, lse_out=lse, window=window)
            fc.fc_store_chunk(pool, layer, table, lens, lens, k, v)
            compare(out, q, lens, cached(layer), lens)
            for r, end in enumerate(np.cumsum(lens)):
                q_window[r, layer] = q[end - window:end].transpose(0, 1)
        from_pool = torch.empty_like(lse)
        fc.fc_window_lse(pool, table, lens, q_window, window, None, from_pool)
        assert (lse - from_pool).abs().max() < 1e-4
        budget = np.array([30, 64, 20], np.int32)
        kept = torch.empty(int(budget.sum()) * layers * heads, dtype=torch.int32, device=dev)
        free = fc.fc_pool_num_free(pool)
        fc.fc_compress_batch_lse(pool, table, lens, q_window, lse, window, np.full(3, fc.FC_METHOD_SNAPKV, np.int32), budget,
                                 kept_out=kept)
        assert (lens == budget).all() and fc.fc_pool_num_free(pool) == free + 5 + 13 + 3 - (2 + 4 + 2)
        # the next turn
        turn = np.array([40, 1, 0], np.int32)
        fc.fc_extend_batch(pool, table, lens, turn)
        for layer in range(layers):
            q, k, v = rows(41)
            fc.fc_store_chunk(pool, layer, table, lens, turn, k, v)
            compare(fc.fc_chunk_attention(pool, layer, table, lens, turn, q), q, turn, cached(layer), lens)
        # into 8 bits
        table8 = torch.full((3, 12), -1, dtype=torch.int32, device=dev)
        lens8 = np.zeros(3, np.int32)
        fc.fc_extend_batch(pool8, table8, lens8, lens)
        fc.fc_quantise_batch(pool8, table8, pool, table, lens)
        for layer in range(layers):
            for a, b in zip(cached(layer), cached(layer, True)):
                assert (np.abs(a - b) <= np.maximum(2.0 ** -4 * np.abs(a), 2.0 ** -10 * np.abs(a).max(-1, keepdims=True) / 224)).all()
        for r in range(3):
            fc.fc_pool_free(pool, table[r, :blocks_for(int(lens[r]))].contiguous())
        assert fc.fc_pool_num_free(pool) == n_blocks
        drafts = np.array([5, 5, 5], np.int32)
        fc.fc_extend_batch(pool8, table8, lens8, drafts)
        for layer in range(layers):
            q, k, v = rows(15)
            fc.fc_store_chunk(pool8, layer, table8, lens8, drafts, k, v)
            compare(fc.fc_chunk_attention(pool8, layer, table8, lens8, drafts, q), q, drafts, cached(layer, True), lens8)
        new = torch.from_numpy(rng.standard_normal((3, layers, 2, heads, dim)).astype(np.float16)).to(dev)
        fc.fc_append_batch(pool8, table8, lens8, new)
        q = torch.from_numpy(rng.standard_normal((3, layers, heads, dim)).astype(np.float16)).to(dev)
        got = fc.fc_decode_attention(pool8, table8, lens8, q).cpu().numpy()
        for layer in range(layers):
            for r, x in enumerate(cached(layer, True)):
                for h in range(heads):
                    want = ao.attention(q[r, layer, h].cpu().numpy()[None], x[0][h], x[1][h], int(lens8[r]) - 1)[0][0]
                    assert (np.abs(got[r, layer, h] - want) <= 1e-3 * np.abs(want) + 1e-4).all()
    finally:
        fc.fc_pool_destroy(pool)
        fc.fc_pool_destroy(pool8)


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
def test_captured_calls_replayed(dtype):
    """A graph of store and attention (long caches, split; many and few rows) and, over an 8-bit pool,
    a decode step, replayed between eager calls with other inputs: as the eager calls."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([2100, 60, 700], [1, 50, 3], 1, 2, 128, dtype=dtype)
    try:
        q = c.q_dev.contiguous()
        k, v = c.k_dev.contiguous(), c.v_dev.contiguous()
        out, lse = torch.empty_like(q), torch.empty((3, c.layers, 2, 4), device=c.dev)
        dq = torch.randn((3, c.layers, 1, 128), device=c.dev).half()
        decoded = torch.empty(dq.shape, device=c.dev)

        def step():
            fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, k, v)
            fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q, out=out, lse_out=lse, window=4)
            if dtype == "e4m3":
                fc.fc_decode_attention(c.pool, c.table_dev, c.lens, dq, out=decoded)

        lse.zero_()
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for i in range(4):
            for x in (q, k, v, dq):
                x.copy_(torch.randn(x.shape, device=c.dev).half())
            step()
            torch.cuda.synchronize()
            want = [x.clone() for x in (out, lse[:, 0], c.kv_dev)] + ([decoded.clone()] if dtype == "e4m3" else [])
            out.zero_()
            decoded.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = [out, lse[:, 0], c.kv_dev] + ([decoded] if dtype == "e4m3" else [])
            for a, b in zip(got, want):
                assert torch.equal(a, b), i
    finally:
        c.close()


def test_on_another_stream_and_into_other_layouts():
    """A side stream, ordered by the caller; results into head-major memory and into part of wider
    rows, whose other parts stay."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([90, 33], [90, 2], 2, 2, 64)
    try:
        want = fc.fc_prefill_attention(c.pool, 0, c.q_dev[:90], c.k_dev[:90], c.v_dev[:90], c.lens[:1])
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        wider = torch.full((90, 4, 64 + 8), 3.0, dtype=torch.float16, device=c.dev)
        major = torch.full((4, 90, 64), 3.0, dtype=torch.float16, device=c.dev)
        torch.cuda.synchronize()
        for out in (wider[:, :, :64], major.transpose(0, 1)):
            fc.fc_prefill_attention(c.pool, 0, c.q_dev[:90], c.k_dev[:90], c.v_dev[:90], c.lens[:1], out=out, stream=side)
            side.synchronize()
            assert torch.equal(out, want)
        assert (wider[:, :, 64:] == 3.0).all()
        fc.fc_store_chunk(c.pool, 1, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev, stream=side)
        out = fc.fc_chunk_attention(c.pool, 1, c.table_dev, c.lens, c.news, c.q_dev, stream=side)
        side.synchronize()
        c.check(1, out)
    finally:
        c.close()


def test_broadcast_rows():
    """Strides of zero: every query head the same rows of q, every token the same K and V."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([40], [40], 2, 2, 64)
    try:
        q = c.q_dev[:, :1].expand(40, 4, 64)
        k, v = c.k_dev[:1].expand(40, 2, 64), c.v_dev[:1].expand(40, 2, 64)
        out = fc.fc_prefill_attention(c.pool, 0, q, k, v, c.lens).cpu().numpy()
        for h in range(4):      # equal keys: the mean of equal values
            assert (np.abs(out[:, h] - c.v[0, h // 2].astype(np.float64)) <= 2.0 ** -9 * np.abs(c.v[0, h // 2]) + 2.0 ** -24).all()
    finally:
        c.close()


@pytest.mark.parametrize("dtype", ["f16", "e4m3"])
def test_more_requests_than_fit_the_arguments(dtype):
    lens = [1 + (7 * i) % 60 for i in range(170)]
    news = [0 if i % 5 == 3 else min(n, 1 if i % 3 else 40) for i, n in enumerate(lens)]
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk(lens, news, 1, 1, 64, dtype=dtype, layers=1)
    try:
        fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        lse = torch.zeros((170, 1, 1, 2), device=c.dev)
        out = fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=2)
        c.check(0, out, lse, 2)
        if dtype == "e4m3":
            q = torch.from_numpy(np.random.default_rng(1).standard_normal((170, 1, 1, 64)).astype(np.float16)).to(c.dev)
            got = fc.fc_decode_attention(c.pool, c.table_dev, c.lens, q).cpu().numpy()
            rows = c.pool_rows(0)
            for r in range(170):
                k, v = c.cached(rows, r)
                want = ao.attention(q[r, 0].cpu().numpy(), k[0], v[0], lens[r] - 1)[0]
                assert (np.abs(got[r, 0] - want) <= 1e-3 * np.abs(want) + 1e-4).all()
        else:
            prompts = np.array([n for n in news if n], np.int32)
            pre = fc.fc_prefill_attention(c.pool, 0, c.q_dev, c.k_dev, c.v_dev, prompts).cpu().numpy()
            at = 0
            for n in prompts.tolist():
                check(c.q[at:at + n, 0], c.k[at:at + n, 0], c.v[at:at + n, 0], 0, pre[at:at + n, 0])
                at += n
    finally:
        c.close()


@pytest.mark.parametrize("eight", [False, True])
def test_blocks_behind_four_gigabytes(eight):
    """Layers and blocks whose offsets pass 32 bits, in bytes and in elements."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    heads, dim, layers = 8, 128, 2
    per_block = 32 * heads * (dim + 1) if eight else 64 * heads * dim
    n_blocks = int(4.6 * 2 ** 30 / per_block)
    shape = (layers, n_blocks, per_block) if eight else (layers, n_blocks, 2, heads, 16, dim)
    kv = torch.empty(shape, dtype=torch.uint8 if eight else torch.float16, device="cuda:0")
    pool = fc.fc_pool_create(kv, n_blocks, layers, heads, dim, dtype=fc.FC_DTYPE_E4M3 if eight else fc.FC_DTYPE_F16)
    try:
        rng = np.random.default_rng(2)
        lens = np.array([50, 40], np.int32)
        table = np.full((2, 4), -1, np.int32)
        table[0] = [n_blocks - 1, 0, n_blocks - 3, n_blocks // 2]
        table[1, :3] = [n_blocks - 2, n_blocks - 5, 7]
        table = torch.from_numpy(table).cuda()
        x = rng.standard_normal((90, 3 * heads, dim)).astype(np.float16)
        q, k, v = (torch.from_numpy(x).cuda()[:, i * heads:(i + 1) * heads] for i in range(3))
        fc.fc_store_chunk(pool, 1, table, lens, lens, k, v)
        news = np.array([33, 1], np.int32)
        rows = torch.cat([q[17:50], q[89:]])
        got = fc.fc_chunk_attention(pool, 1, table, lens, news, rows).cpu().numpy()
        if eight:
            steps = fc.fc_decode_attention(pool, table, lens, q[[49, 89]][:, None].expand(2, layers, heads, dim).contiguous())
            steps = steps.cpu().numpy()
        for h in range(heads):
            for first, last, new, at in ((0, 50, 33, 0), (50, 90, 1, 33)):
                kk, vv = x[first:last, heads + h].astype(np.float64), x[first:last, 2 * heads + h].astype(np.float64)
                if eight:
                    kk, vv = (np.stack([ao.values(*(np.array(a)[None] for a in ao.quantise_row(row)))[0] for row in y])
                              for y in (x[first:last, heads + h], x[first:last, 2 * heads + h]))
                check(x[last - new:last, h], kk, vv, last - first - new, got[at:at + new, h])
                if eight:
                    want = ao.attention(x[last - 1:last, h], kk, vv, last - first - 1)[0][0]
                    assert (np.abs(steps[int(at > 0), 1, h] - want) <= 1e-3 * np.abs(want) + 1e-4).all()
    finally:
        fc.fc_pool_destroy(pool)


def test_the_longest_cache():
    """32768 tokens: one new token, and a chunk of 130."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([32768, 32768], [1, 130], 1, 1, 64, layers=1)
    try:
        fc.fc_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, c.k_dev, c.v_dev)
        lse = torch.zeros((2, 1, 1, 130), device=c.dev)
        out = fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev, lse_out=lse, window=130)
        c.check(0, out, lse, 130)
    finally:
        c.close()


def test_what_the_binding_refuses():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Chunk([40, 20], [3, 1], 2, 2, 64)
    try:
        args = (c.pool, 0, c.table_dev, c.lens, c.news)
        for bad in (c.q_dev.float(), c.q_dev[:3], c.q_dev[:, :3], c.q_dev.cpu(), c.q_dev[..., :32],
                    torch.empty((4, 4, 128), dtype=torch.float16, device=c.dev)[..., ::2]):
            with pytest.raises((ValueError, fc.FastCacheError)):
                fc.fc_chunk_attention(*args, bad)
        with pytest.raises(ValueError):
            fc.fc_chunk_attention(*args, c.q_dev, lse_out=torch.zeros((2, 1, 4, 3), device=c.dev), window=3)
        with pytest.raises(ValueError):
            fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news[:1], c.q_dev)
        with pytest.raises(ValueError):
            fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news.astype(np.int64), c.q_dev)
        with pytest.raises(ValueError):
            fc.fc_store_chunk(*args, c.k_dev, c.v_dev[:, :1])
        with pytest.raises(fc.FastCacheError):
            fc.fc_chunk_attention(*args, c.q_dev, out=torch.empty(64, dtype=torch.float16, device=c.dev).expand(4, 4, 64))
        with pytest.raises(fc.FastCacheError):
            fc.fc_quantise_batch(c.pool, c.table_dev, c.pool, c.table_dev, c.lens)
        with pytest.raises(ValueError):
            fc.fc_pool_create(c.kv_dev, c.n_blocks, c.layers, c.heads, c.dim, dtype=fc.FC_DTYPE_E4M3)
    finally:
        c.close()
