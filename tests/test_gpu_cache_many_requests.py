"""More requests or new tokens than a kernel's arguments hold, for the calls on rotated rows, 4-bit rows and selected
blocks; and a long chunk of new tokens over selected blocks, against torch in 64 bits."""

import numpy as np
import pytest

from attention_util import blocks_for
from cache_util import Cache, decode_check, encode
from test_gpu_sparse import _bounds, _same, _step

pytestmark = pytest.mark.gpu

MANY = 170


@pytest.mark.parametrize("fmt,group", [("f16", 2), ("e4m3", 1), ("e2m1", 2), ("e2m1", 20)])
def test_single_tokens(fmt, group):
    """Bounds, selection and attention by one launch; over 4 bits of up to 16 rows of a head and of more."""
    c = Cache([1 + 5 * i % 150 for i in range(MANY)], [1 if i % 9 else 0 for i in range(MANY)], 2, group, 64, fmt=fmt, layers=1)
    try:
        assert int((c.news > 0).sum()) > 149
        bounds = c.new_bounds(7.0)
        c.fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.lens, bounds)
        want = np.full(tuple(bounds.shape), 7.0)
        for r, blocks in enumerate(_bounds(c, 0)):
            for b, h in np.ndindex(len(blocks), c.heads):
                want[0, c.table[r, b], h] = blocks[b][h]
        assert _same(bounds.cpu().numpy().astype(np.float64), want)
        _step(c, 0, 4, bounds=bounds)
    finally:
        c.close()


@pytest.mark.parametrize("lens,news,group,n_select", [([6300, 6400, 300, 6250], [40] * 4, 1, 9), ([300] * 80, [2] * 80, 33, 5)], ids=["long", "33 rows"])
def test_tokens_that_select_apart(lens, news, group, n_select):
    """Scores, selection and attention in launches of their own."""
    c = Cache(lens, news, 2, group, 64, fmt="f16", layers=1)
    try:
        assert int(c.news.sum()) > 149
        _step(c, 0, n_select)
    finally:
        c.close()


@pytest.mark.parametrize("longest", [100, 3000])
def test_attention_over_4_bits(longest):
    """Of few rows of every request, heads whole and cut."""
    c = Cache([1 + 7 * i % 100 for i in range(MANY - 1)] + [longest], [1] * MANY, 2, 4, 64, layers=1)
    try:
        c.check(0, c.fc.fc_chunk_attention(c.pool, 0, c.table_dev, c.lens, c.news, c.q_dev))
    finally:
        c.close()


def test_copies_stores_and_appends_into_4_bits():
    import torch
    from paper_2503_08461_amd import fastcache as fc
    heads, dim = 1, 64
    lens = [1 + i % 20 for i in range(MANY)]
    c = Cache(lens, lens, heads, 1, dim, fmt="f16", layers=1)
    kv4 = torch.full((1, 2 * c.n_blocks + MANY, 17 * heads * dim), 0xA5, dtype=torch.uint8, device=c.dev)
    pool4 = fc.fc_pool_create(kv4, kv4.shape[1], 1, heads, dim, dtype=fc.FC_DTYPE_E2M1)

    def rows(table, n):
        """[request] -> (codes, exponents) [2][token][...]"""
        image = kv4[0].cpu().numpy()
        codes = image[:, :16 * heads * dim].reshape(-1, 2, 16, dim // 2)
        exps = image[:, 16 * heads * dim:].reshape(-1, 2, 16, dim // 32)
        out = []
        for r in range(MANY):
            ids = table[r, :blocks_for(n[r])]
            out.append(tuple(x[ids].transpose(1, 0, 2, 3).reshape(2, -1, x.shape[-1])[:, :n[r]] for x in (codes, exps)))
        return out

    try:
        table4 = torch.full((MANY, 3), -1, dtype=torch.int32, device=c.dev)
        lens4 = np.zeros(MANY, np.int32)
        fc.fc_extend_batch(pool4, table4, lens4, c.lens)
        fc.fc_quantise_batch(pool4, table4, c.pool, c.table_dev, c.lens)
        want = []
        for r in range(MANY):
            x = c.kv[0, c.table[r, :blocks_for(lens[r])], :, 0].transpose(1, 0, 2, 3).reshape(2, -1, dim)[:, :lens[r]]
            want.append(encode(x, "e2m1"))
        got = rows(table4.cpu().numpy(), lens)
        assert all((a == b).all() for g, w in zip(got, want) for a, b in zip(g, w))
        # a token more for each, behind the others
        new = np.random.default_rng(5).standard_normal((MANY, 1, 2, heads, dim)).astype(np.float16)
        fc.fc_append_batch(pool4, table4, lens4, torch.from_numpy(new).to(c.dev))
        for r in range(MANY):
            codes, exps = encode(new[r, 0, :, :1], "e2m1")
            want[r] = tuple(np.concatenate([w, x], 1) for w, x in zip(want[r], (codes, exps)))
        got = rows(table4.cpu().numpy(), lens4)
        assert all((a == b).all() for g, w in zip(got, want) for a, b in zip(g, w))
        q = np.random.default_rng(6).standard_normal((MANY, 1, heads, dim)).astype(np.float16)
        table = table4.cpu().numpy()
        c.lens, c.kv_dev, c.fmt, c.table = lens4, kv4, "e2m1", table
        decode_check(c, q, fc.fc_decode_attention(pool4, table4, lens4, torch.from_numpy(q).to(c.dev)).cpu().numpy())
        # the same tokens' rows again as a chunk, other ones
        k, v = (np.random.default_rng(s).standard_normal((int(lens4.sum()), heads, dim)).astype(np.float16) for s in (7, 8))
        fc.fc_store_chunk(pool4, 0, table4, lens4, lens4, torch.from_numpy(k).to(c.dev), torch.from_numpy(v).to(c.dev))
        got, at = rows(table, lens4), 0
        for r, n in enumerate(lens4.tolist()):
            codes, exps = encode(np.stack([k[at:at + n, 0], v[at:at + n, 0]]), "e2m1")
            assert (got[r][0] == codes).all() and (got[r][1] == exps).all()
            at += n
    finally:
        fc.fc_pool_destroy(pool4)
        c.close()


@pytest.mark.parametrize("fmt", ["f16", "e2m1"])
def test_a_long_chunk(fmt):
    """600 new tokens of a cache of 9000, four heads of four: every selection in 64 bits, where no two scores at the
    border are nearer than their sums are rounded, and the attention of some of the tokens."""
    import torch
    from attention_util import check
    heads, group, dim, n, new, n_select = 4, 4, 128, 9000, 600, 40
    c = Cache([n], [new], heads, group, dim, fmt="f16", layers=1, seed=12)
    try:
        if fmt == "e2m1":                                   # (the oracle's rows one by one would take minutes)
            kv4 = torch.zeros((1, c.n_blocks, 17 * heads * dim), dtype=torch.uint8, device=c.dev)
            pool4 = c.fc.fc_pool_create(kv4, c.n_blocks, 1, heads, dim, dtype=c.fc.FC_DTYPE_E2M1)
            c.fc.fc_quantise_batch(pool4, c.table_dev, c.pool, c.table_dev, c.lens)
            c.fc.fc_pool_destroy(c.pool)
            c.pool, c.kv_dev, c.fmt = pool4, kv4, fmt
        bounds = c.new_bounds()
        c.fc.fc_block_bounds(c.pool, 0, c.table_dev, c.lens, c.lens, bounds)
        selected = torch.empty((new, heads, n_select), dtype=torch.int32, device=c.dev)
        out = c.fc.fc_sparse_attention(c.pool, 0, c.table_dev, c.lens, c.news, bounds, n_select, c.q_dev, selected=selected).cpu().numpy()
        got = selected.cpu().numpy()
        nb = blocks_for(n)
        held = bounds[0, torch.from_numpy(c.table[0, :nb].astype(np.int64)).to(c.dev)].double()       # [block][head][2][d]
        k, v = c.cached(c.pool_rows(0), 0)
        seen = n - new + 1 + np.arange(new)
        for h in range(heads):
            q = torch.from_numpy(c.q[:, h * group:(h + 1) * group]).to(c.dev).double().reshape(-1, dim)
            scores = q.clamp(max=0) @ held[:, h, 0].T.contiguous() + q.clamp(min=0) @ held[:, h, 1].T.contiguous()
            scores = scores.reshape(new, group, nb).amax(1).cpu().numpy()
            for t in range(new):
                own = blocks_for(int(seen[t])) - 1
                order = np.argsort(-scores[t, :own], kind="stable")
                edge = scores[t, order[n_select - 2]] - scores[t, order[n_select - 1]]
                assert edge > 1e-9                          # (128 products of some tens: their sums are off by 1e-12)
                assert got[t, h].tolist() == sorted(order[:n_select - 1].tolist()) + [own], (t, h)
            for t in (0, 7, 8, 9, 300, new - 1):
                tok = np.concatenate([np.arange(b * 16, min(b * 16 + 16, seen[t])) for b in got[t, h]])
                for j in range(h * group, (h + 1) * group):
                    check(c.q[t:t + 1, j], k[h][tok], v[h][tok], len(tok) - 1, out[t:t + 1, j])
    finally:
        c.close()
