"""The calls on rotated rows, pools of fewer bits and selected blocks together, as a server makes them, and in the ways
a server may: captured and replayed, on another stream, with its queries' rows written in place."""

import numpy as np
import pytest

from attention_util import blocks_for, check
from cache_util import Cache, decode_check, dtype_of, rows_of
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


def _angles(rotary, n, dev):
    import torch
    w = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rotary // 2) * 2 / rotary)
    x = np.stack([np.cos(w), np.sin(w)], 1).astype(np.float32)
    return x, torch.from_numpy(x).to(dev)


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
def test_a_conversation(fmt):
    """Prompts with rotated rows into an fp16 pool, compression, what is kept into a pool of `fmt`; the next turn's
    chunk behind its true positions, then single tokens over selected blocks, and a decode step."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    layers, heads, group, dim, rotary = 2, 2, 2, 64, 48
    hq = heads * group
    rng = np.random.default_rng(21)
    lens = np.array([300, 700, 40], np.int32)
    positions = np.zeros(3, np.int32)
    n_blocks, dev = 140, torch.device("cuda:0")
    kv = torch.zeros((layers, n_blocks, 2, heads, 16, dim), dtype=torch.float16, device=dev)
    pool = fc.fc_pool_create(kv, n_blocks, layers, heads, dim)
    per = {"f16": 64 * heads * dim, "e4m3": 32 * heads * (dim + 1), "e2m1": 17 * heads * dim}[fmt]
    kv2 = torch.zeros((layers, n_blocks, 2, heads, 16, dim), dtype=torch.float16, device=dev) if fmt == "f16" else \
        torch.zeros((layers, n_blocks, per), dtype=torch.uint8, device=dev)
    pool2 = fc.fc_pool_create(kv2, n_blocks, layers, heads, dim, dtype=dtype_of(fmt))
    angles, table_of_angles = _angles(rotary, 2000, dev)
    rotation = fc.Rotation(table_of_angles)

    def rows(n):
        x = torch.from_numpy(rng.standard_normal((n, hq + 2 * heads, dim)).astype(np.float16)).to(dev)
        return x[:, :hq], x[:, hq:hq + heads], x[:, hq + heads:]

    def caches(layer, t, n, which=None, f=None):
        x = rows_of((kv2 if which is None else which)[layer].cpu().numpy(), f or fmt, heads, dim)
        t = t.cpu().numpy()
        return [x[t[r, :blocks_for(n[r])]].transpose(1, 2, 0, 3, 4).reshape(2, heads, -1, dim)[:, :, :n[r]] for r in range(3)]

    def turned(q, n_new, first):
        at, q = 0, q.cpu().numpy().copy()
        for n, p in zip(n_new, first):
            for i in range(n):
                q[at] = co.rotate(q[at], angles[p + i, 0], angles[p + i, 1], False)
                at += 1
        return q

    try:
        table = torch.full((3, 50), -1, dtype=torch.int32, device=dev)
        now = np.zeros(3, np.int32)
        fc.fc_extend_batch(pool, table, now, lens)
        q_window = torch.empty((3, layers, heads, 16, dim), dtype=torch.float16, device=dev)
        for layer in range(layers):
            q, k, v = rows(int(lens.sum()))
            want = turned(q, lens, positions)
            q = fc.fc_rotate_store_chunk(pool, layer, table, now, lens, rotation, q, k, v)
            assert (q.cpu().numpy() == want).all()
            out = fc.fc_chunk_attention(pool, layer, table, now, lens, q).cpu().numpy()
            cached, at = caches(layer, table, now, kv, "f16"), 0
            for r, n in enumerate(lens):
                for h in range(hq):
                    some = slice(at, at + min(n, 60))
                    check(want[some, h], cached[r][0][h // group], cached[r][1][h // group], 0, out[some, h])
                at += n
                q_window[r, layer] = q[at - 16:at, ::group].transpose(0, 1)
        positions += lens
        budget = np.array([200, 300, 40], np.int32)
        fc.fc_compress_batch(pool, table, now, q_window, 16, np.full(3, fc.FC_METHOD_SNAPKV, np.int32), budget)
        # what is kept into the other pool
        table2 = torch.full((3, 50), -1, dtype=torch.int32, device=dev)
        lens2 = np.zeros(3, np.int32)
        fc.fc_extend_batch(pool2, table2, lens2, now)
        if fmt == "f16":
            for r in range(3):
                m = blocks_for(now[r])
                kv2[:, table2[r, :m].long()] = kv[:, table[r, :m].long()]
        else:
            fc.fc_quantise_batch(pool2, table2, pool, table, now)
        bounds = torch.zeros((layers, n_blocks, heads, 2, dim), dtype=torch.float16, device=dev)
        for layer in range(layers):
            fc.fc_block_bounds(pool2, layer, table2, lens2, lens2, bounds)
        # the next turn: a chunk, then single tokens that select
        for turn in ([40, 3, 0], [1, 1, 1], [1, 0, 1], [1, 1, 1]):
            turn = np.array(turn, np.int32)
            fc.fc_extend_batch(pool2, table2, lens2, turn)
            for layer in range(layers):
                q, k, v = rows(int(turn.sum()))
                want = turned(q, turn, positions)
                fc.fc_rotate_store_chunk(pool2, layer, table2, lens2, turn, rotation, q, k, v, positions=positions, q_out=q)
                assert (q.cpu().numpy() == want).all()
                fc.fc_block_bounds(pool2, layer, table2, lens2, turn, bounds)
                cached = caches(layer, table2, lens2)
                if turn.max() > 1:
                    out, at = fc.fc_chunk_attention(pool2, layer, table2, lens2, turn, q).cpu().numpy(), 0
                    for r, n in enumerate(turn):
                        for h in range(hq):
                            check(want[at:at + n, h], cached[r][0][h // group], cached[r][1][h // group], int(lens2[r]) - n,
                                  out[at:at + n, h])
                        at += n
                    continue
                selected = torch.empty((int(turn.sum()), heads, 5), dtype=torch.int32, device=dev)
                out = fc.fc_sparse_attention(pool2, layer, table2, lens2, turn, bounds, 5, q, selected=selected).cpu().numpy()
                at = 0
                for r in np.flatnonzero(turn):
                    n = int(lens2[r])
                    for h in range(heads):
                        k_, v_ = cached[r][0][h], cached[r][1][h]
                        blocks = [co.bounds(k_[b * 16:b * 16 + 16]) for b in range(blocks_for(n))]
                        mine = want[at, h * group:(h + 1) * group]
                        keep = co.select([co.score(mine, *b) for b in blocks], 5)
                        assert [b for b in selected[at, h].tolist() if b >= 0] == keep
                        tok = np.concatenate([np.arange(b * 16, min(b * 16 + 16, n)) for b in keep])
                        for j in range(group):
                            check(mine[j:j + 1], k_[tok], v_[tok], len(tok) - 1, out[at:at + 1, h * group + j])
                    at += 1
            positions += turn
        q = rng.standard_normal((3, layers, heads, dim)).astype(np.float16)
        got = fc.fc_decode_attention(pool2, table2, lens2, torch.from_numpy(q).to(dev)).cpu().numpy()
        if fmt != "f16":
            class As:  # what decode_check looks at
                pass
            c = As()
            c.dim, c.layers, c.heads, c.lens = dim, layers, heads, lens2
            c.pool_rows = lambda layer: layer
            c.cached = lambda layer, r: caches(layer, table2, lens2)[r]
            decode_check(c, q, got)
        assert fc.fc_pool_num_free(pool2) == n_blocks - sum(blocks_for(n) for n in lens2)
    finally:
        fc.fc_pool_destroy(pool)
        fc.fc_pool_destroy(pool2)


@pytest.mark.parametrize("fmt", ["f16", "e4m3", "e2m1"])
@pytest.mark.parametrize("lens", [[700, 90], [9000, 20]], ids=str)
def test_captured_and_replayed(fmt, lens):
    """A step in a graph, replayed with other rows, other work and other graphs between, against the eager step."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Cache(lens, [1, 2], 2, 2, 64, fmt=fmt, layers=1)
    try:
        _, table = _angles(64, 10000, c.dev)
        rotation = fc.Rotation(table)
        x = torch.from_numpy(np.concatenate([c.q, c.k, c.v], 1)).to(c.dev)
        q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
        q2 = torch.empty_like(q).contiguous()
        bounds = c.new_bounds()
        fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.lens, bounds)
        selected = torch.empty((3, 2, 6), dtype=torch.int32, device=c.dev)
        out, whole = torch.empty_like(q2), torch.empty_like(q2)
        q_step = torch.from_numpy(np.random.default_rng(3).standard_normal((2, 1, 2, 64)).astype(np.float16)).to(c.dev)
        step = torch.empty((2, 1, 2, 64), device=c.dev)

        def run():
            fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, rotation, q, k, v, q_out=q2)
            fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.news, bounds)
            fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, 6, q2, out=out, selected=selected)
            fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q2, out=whole)
            fc.fc_decode_attention(c.pool, c.table_dev, c.lens, q_step, out=step)
            return [t.clone() for t in (q2, bounds, out, selected, whole, step, c.kv_dev)]

        run()  # (its scratch)
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, rotation, q, k, v, q_out=q2)
                fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.news, bounds)
                fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, 6, q2, out=out, selected=selected)
                fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q2, out=whole)
                fc.fc_decode_attention(c.pool, c.table_dev, c.lens, q_step, out=step)
            graphs.append(g)
        for i in range(5):
            x.copy_(torch.from_numpy(np.random.default_rng(30 + i).standard_normal(tuple(x.shape)).astype(np.float16)))
            want = run()
            for t in (q2, out, whole, step):
                t.fill_(-3)
            selected.fill_(-5)
            torch.cuda.synchronize()
            graphs[i % 2].replay()
            for a, b in zip((q2, bounds, out, selected, whole, step, c.kv_dev), want):
                assert torch.equal(a, b)
    finally:
        c.close()


def test_on_another_stream():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([900, 50, 333], [1, 4, 2], 2, 4, 128, fmt="e2m1", layers=1)
    try:
        _, table = _angles(128, 1000, c.dev)
        rotation = fc.Rotation(table, True)
        bounds = c.new_bounds()
        fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.lens, bounds)
        got = []
        for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
            torch.cuda.synchronize()
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                q = fc.fc_rotate_store_chunk(c.pool, 0, c.table_dev, c.lens, c.news, rotation, c.q_dev, c.k_dev, c.v_dev)
                fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.news, bounds)
                got.append([q, fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, 9, q),
                            fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, q), bounds.clone(), c.kv_dev.clone()])
            torch.cuda.synchronize()
        for other in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    finally:
        c.close()


def test_the_bindings_checks():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    c = Cache([20], [2], 2, 2, 64, fmt="e2m1", layers=1)
    try:
        _, table = _angles(64, 100, c.dev)
        rotation = fc.Rotation(table)
        bounds = c.new_bounds()
        args = (c.pool, 0, c.table_dev, c.lens, c.news)
        for bad in (lambda: fc.Rotation(table[:, 0]), lambda: fc.Rotation(table.double()), lambda: fc.Rotation(table[:, :, ::2]),
                    lambda: fc.fc_rotate_store_chunk(*args, rotation, c.q_dev[:1], c.k_dev, c.v_dev),
                    lambda: fc.fc_rotate_store_chunk(*args, rotation, None, c.k_dev, c.v_dev, q_out=c.q_dev),
                    lambda: fc.fc_rotate_store_chunk(*args, rotation, None, c.k_dev, c.v_dev, positions=np.zeros(2, np.int32)),
                    lambda: fc.fc_rotate_store_chunk(*args, rotation, None, c.k_dev.float(), c.v_dev),
                    lambda: fc.fc_block_bounds(*args, bounds[:, :-1]), lambda: fc.fc_block_bounds(*args, bounds.float()),
                    lambda: fc.fc_sparse_attention(*args, bounds, 3, c.q_dev, selected=torch.empty((2, 2, 4), dtype=torch.int32, device=c.dev)),
                    lambda: fc.fc_pool_create(torch.zeros((1, 4, 2, 2, 16, 64), dtype=torch.float16, device=c.dev), 4, 1, 2, 64,
                                              dtype=fc.FC_DTYPE_E2M1)):
            with pytest.raises(ValueError):
                bad()
        for bad in (lambda: fc.fc_rotate_store_chunk(*args, rotation, None, c.k_dev, c.v_dev, positions=np.array([99], np.int32)),
                    lambda: fc.fc_sparse_attention(*args, bounds, 0, c.q_dev), lambda: fc.fc_sparse_attention(*args, bounds, 3, c.q_dev[:, :3])):
            with pytest.raises(fc.FastCacheError) as e:
                bad()
            assert e.value.code == fc.FC_EINVAL
    finally:
        c.close()
