"""The conversions of 4-bit rows one by one: every fp16 number under every exponent that a group with it can have, every
largest magnitude, and what every code stands for under every exponent, in each of the kernels that read it."""

import numpy as np
import pytest

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu

EXPONENTS = list(range(-23, 14))


def _groups(rng):
    """Groups of 32 numbers: for every exponent all fp16 numbers that it reaches beside 6 * 2^e, and for every
    magnitude one group in which no other is larger."""
    finite = np.arange(0x7c00, dtype=np.uint16).view(np.float16)
    out = []
    for e in EXPONENTS:
        x = finite if e == 13 else finite[finite.astype(np.float64) <= 6 * 2.0 ** e]
        x = np.concatenate([x, -x])
        x = rng.permutation(np.concatenate([x, np.zeros(-len(x) % 31, np.float16)])).reshape(-1, 31)
        out.append(np.concatenate([np.full((len(x), 1), 6 * 2.0 ** e, np.float16), x], 1))
    rest = (rng.uniform(-1, 1, (len(finite), 32)) * finite[:, None].astype(np.float64)).astype(np.float16)
    rest[:, 0] = finite * rng.choice(np.array([-1, 1], np.float16), len(finite))
    out.append(rest)
    x = np.concatenate(out)
    return rng.permuted(x, axis=1)[rng.permutation(len(x))]


def _encode(x):
    """Groups [n][32] -> (codes, exponents + 127), by comparison with every number that a code stands for."""
    x = x.astype(np.float64)
    most = np.abs(x).max(1)
    e = -23 + sum((most > 6 * 2.0 ** k).astype(int) for k in range(-23, 13))
    d = np.abs(co.E2M1 - (np.abs(x) / np.exp2(e)[:, None])[..., None])
    near = d == d.min(-1, keepdims=True)
    code = np.where(near.sum(-1) == 1, near.argmax(-1), (near & (np.arange(8) % 2 == 0)).argmax(-1))
    return (code | np.where(np.signbit(x), 8, 0)).astype(np.uint8), (e + 127).astype(np.uint8)


@pytest.mark.parametrize("dim", [64, 128])
def test_every_number_under_every_exponent(dim):
    import torch
    from paper_2503_08461_amd import fastcache as fc
    rng = np.random.default_rng(dim)
    groups = _groups(rng)
    per = 2 * 16 * dim // 32                                 # groups of a block
    groups = np.concatenate([groups, np.zeros((-len(groups) % per, 32), np.float16)])
    codes, exps = _encode(groups)
    for i in rng.choice(len(groups), 60, replace=False):     # (as the other tests' oracle has it)
        want = co.quantise_row(groups[i])
        assert (want[0] == codes[i]).all() and want[1][0] == exps[i]
    n_blocks, dev = len(groups) // per, torch.device("cuda:0")
    kv = torch.from_numpy(groups.reshape(1, n_blocks, 2, 1, 16, dim)).to(dev)
    kv4 = torch.full((1, n_blocks, 17 * dim), 0xA5, dtype=torch.uint8, device=dev)
    pool = fc.fc_pool_create(kv, n_blocks, 1, 1, dim)
    pool4 = fc.fc_pool_create(kv4, n_blocks, 1, 1, dim, dtype=fc.FC_DTYPE_E2M1)
    try:
        width = 2048
        table = torch.zeros((-(-n_blocks // width), width), dtype=torch.int32, device=dev)
        table.view(-1)[:n_blocks] = torch.arange(n_blocks, dtype=torch.int32, device=dev)
        lens = np.array([16 * min(width, n_blocks - width * r) for r in range(len(table))], np.int32)
        fc.fc_quantise_batch(pool4, table, pool, table, lens)
        want = np.concatenate([co.pack(codes).reshape(n_blocks, -1), exps.reshape(n_blocks, -1)], 1)
        got = kv4[0].cpu().numpy()
        assert got.shape == want.shape and (got == want).all()
        # the rows' way by the store: the first heads' worth, as new tokens
        kv4.fill_(0xA5)
        rows = groups.reshape(n_blocks, 2, 16, dim)
        k, v = (torch.from_numpy(np.ascontiguousarray(rows[:, i]).reshape(-1, 1, dim)).to(dev) for i in range(2))
        fc.fc_store_chunk(pool4, 0, table, lens, lens, k, v)
        assert (kv4[0].cpu().numpy() == want).all()
    finally:
        fc.fc_pool_destroy(pool)
        fc.fc_pool_destroy(pool4)


@pytest.mark.parametrize("dim", [64, 128])
def test_every_code_under_every_exponent(dim):
    """One token a request, whose weight is one: results are its V, bounds its K."""
    import torch
    from paper_2503_08461_amd import fastcache as fc
    dev, n = torch.device("cuda:0"), len(EXPONENTS) + 1
    exps = np.array([e + 127 for e in EXPONENTS] + [255], np.uint8)
    code = np.tile(np.arange(16, dtype=np.uint8), dim // 16)
    image = np.full((1, n, 17 * dim), 0xA5, np.uint8)        # (slots behind the token: anything)
    want = np.zeros((n, dim))
    for r in range(n):
        codes, ex = image[0, r, :16 * dim].reshape(2, 16, dim // 2), image[0, r, 16 * dim:].reshape(2, 16, dim // 32)
        codes[:, 0], ex[:, 0] = co.pack(code), exps[r]
        want[r] = co.values(co.pack(code), np.full(dim // 32, exps[r]))
    kv = torch.from_numpy(image).to(dev)
    pool = fc.fc_pool_create(kv, n, 1, 1, dim, dtype=fc.FC_DTYPE_E2M1)
    try:
        table = torch.arange(n, dtype=torch.int32, device=dev)[:, None].contiguous()
        ones = np.ones(n, np.int32)
        bounds = torch.zeros((1, n, 1, 2, dim), dtype=torch.float16, device=dev)
        fc.fc_block_bounds(pool, 0, table, ones, ones, bounds)
        for side in range(2):
            got = bounds[0, :, 0, side].cpu().numpy().astype(np.float64)
            assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()
        # a key that is not a number is none of its token's: K is 0 from here on
        kv[0, :, :8 * dim] = 0
        kv.view(n, -1)[:, 16 * dim:16 * dim + dim // 2] = 127
        q = torch.ones((n, 1, 1, dim), dtype=torch.float16, device=dev)
        results = [fc.fc_decode_attention(pool, table, ones, q)[:, 0, 0]]
        for group in (1, 20, 64):                            # up to 16 rows, up to 32, more
            out = fc.fc_chunk_attention(pool, 0, table, ones, ones, q[:, 0].expand(n, group, dim).contiguous())
            results += [out[:, 0], out[:, -1]]
        for group in (1, 20):
            out = fc.fc_sparse_attention(pool, 0, table, ones, ones, bounds, 1, q[:, 0].expand(n, group, dim).contiguous())
            results += [out[:, 0], out[:, -1]]
        for x in results:
            got = x.cpu().numpy().astype(np.float64)
            assert ((got == want) | (np.isnan(got) & np.isnan(want))).all()
    finally:
        fc.fc_pool_destroy(pool)
