"""The paged cache, written with the position rotation, held in 4 bits, read block by selected block: the cases that these
operators' speed is measured on, each with its plain form, its required work and its 64-bit definition.

rotate     new tokens' q and k rotated by their positions, k and v written into the paged pool (16, 8 or 4 bits), one layer
chunk4     the same into a 4-bit pool, then the attention of the new tokens over it; a chunk of one token is the decode step
           of a model with grouped heads
decode4    a decode step's attention over a 4-bit pool, all layers at once
quantise4  the cache of a batch copied from an fp16 pool into a 4-bit one
bounds     the smallest and largest value of each channel of K, for every block of a batch's caches, one layer
sparse     a decode step that reads the best blocks only: the bounds of the blocks with new tokens, then the attention of
           each new token over the blocks that its score selects

Rows of 8 bits are e4m3 codes times one power of two: the smallest 2^e that brings the row's largest magnitude to 448 or
less, -15 <= e <= 8.  Rows of 4 bits are e2m1 codes (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign) times one power of two for every
32 channels: the smallest 2^e that brings their largest magnitude to 6 or less, -23 <= e <= 13.  Every value is an fp16
number.  A pool block holds the codes of [K|V][head][slot][channel], of 4 bits two to a byte, the even channel in the low
half, and behind them the exponents, e + 127, of [K|V][head][slot] or of [K|V][head][slot][32 channels].

A rotated row is rounded to 32 and then to 16 bits before anything else is done with it, and both are determined by the
inputs: 64 bits hold the products of 16- and 32-bit numbers exactly, and their sum is rounded once.  So the bytes of a pool
are determined too, and come back as they are where the codes are of 4 bits.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 16


def _case(name, kind, n_req, len_lo, len_hi, heads, q_heads, dim, new_lo=0, new_hi=0, bits=4, layers=1, rotary=0,
          interleaved=False, select=0, shape_seed=1):
    """n_req requests of len_lo..len_hi cached tokens and new_lo..new_hi new ones, drawn from shape_seed; heads: of K and
    V; rotary: channels that are rotated; select: blocks that a query attends to."""
    c = dict(kind=kind, n_req=n_req, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi, heads=heads,
             q_heads=q_heads, dim=dim, bits=bits, layers=layers, rotary=rotary, interleaved=interleaved, select=select,
             shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of a four-head toy model: launches and host time are all there is
        _case("rotate_token", "rotate", 1, 256, 256, 4, 4, 64, 1, 1, 16, rotary=64),
        # a batch of ordinary prompts (benchmark configuration 3), whole
        _case("rotate_prompts", "rotate", 32, 0, 0, 32, 32, 128, 600, 1200, 16, rotary=128),
        # the decode step of a large batch with grouped heads, caches not compressed
        _case("chunk4_tokens", "chunk4", 48, 1280, 7040, 8, 32, 128, 1, 1, rotary=128),
        # the last 2048 tokens of a very long prompt over what is cached of it, half of the channels rotated
        _case("chunk4_long", "chunk4", 1, 30000, 30000, 8, 32, 128, 2048, 2048, rotary=64, interleaved=True),
        # one decode step of a few requests over compressed caches, pool of one layer
        _case("decode4_small", "decode4", 8, 256, 1408, 32, 32, 128),
        # one decode step of a large batch over uncompressed caches
        _case("decode4_full", "decode4", 48, 1280, 7040, 32, 32, 128, layers=2),
        # what the toy configuration keeps of its prompt, 64 tokens
        _case("quantise4_question", "quantise4", 1, 64, 64, 4, 4, 64),
        # the compressed caches of 64 multi-image prompts (configuration 4, 4 of its 32 layers)
        _case("quantise4_batch", "quantise4", 64, 256, 1408, 32, 32, 128, layers=4),
        # the bounds of one single-image prompt of 640 tokens (configuration 2)
        _case("bounds_image", "bounds", 1, 640, 640, 32, 32, 128, bits=16),
        # the bounds of the long prompts of configuration 4, in an 8-bit pool
        _case("bounds_prompts", "bounds", 64, 1280, 7040, 32, 32, 128, bits=8),
        # the decode step of a large batch with grouped heads, 1024 tokens of every cache attended to
        _case("sparse_tokens", "sparse", 48, 1280, 7040, 8, 32, 128, 1, 1, 16, select=64),
        # drafted tokens of two very long caches in 4 bits, 2048 tokens attended to
        _case("sparse_drafts", "sparse", 2, 28000, 30000, 8, 32, 128, 5, 5, 4, select=128),
    ]


_POSITIONS = 65536    # rows of the rotation's table
_MAX_SCORES = 2.2e9   # elements of the padded score matrix of the plain form
_MAX_PADDED = 1.5e9   # elements of the padded keys
_MAX_WORK = 1e12      # flops: no more than the largest listed case
_MAX_BYTES = 4e9


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "rotate", "chunk4", "chunk4", "decode4", "quantise4", "bounds", "sparse", "sparse"])
    dim = rng.choice([64, 128, 128])
    heads, group = rng.choice([(1, 8), (2, 4), (4, 1), (4, 8), (5, 3), (8, 4), (8, 5), (12, 1), (12, 2), (32, 1), (40, 1)])
    if kind in ("decode4", "quantise4", "bounds"):
        group = 1
    len_lo = log_int(1, 12000)
    len_hi = min(30000, len_lo * rng.choice([1, 2, 3]) + rng.randrange(16))
    new_lo = new_hi = 0
    if kind in ("rotate", "chunk4"):
        new_lo = rng.choice([1, 1, 4, log_int(1, 1500)])
        new_hi = min(2048, new_lo * rng.choice([1, 1, 4]) + rng.choice([0, 0, rng.randrange(64)]))
    elif kind == "sparse":
        new_lo = rng.choice([1, 1, 1, rng.randrange(1, 9)])
        new_hi = new_lo + rng.choice([0, 0, rng.randrange(4)])
    c = _case("", kind, log_int(1, 64), len_lo, len_hi, heads, heads * group, dim, new_lo, new_hi,
              4 if kind.endswith("4") else rng.choice([4, 8, 16]),
              rng.choice([1, 2, 4]) if kind in ("decode4", "quantise4") else 1,
              rng.choice([dim, dim, dim // 2, 16 * rng.randrange(1, dim // 16 + 1)]) if kind in ("rotate", "chunk4") else 0,
              rng.choice([False, True]) if kind in ("rotate", "chunk4") else False,
              log_int(1, 256) if kind == "sparse" else 0, rng.randrange(1 << 20))

    def too_much():
        lens, news = _lengths(c)
        rows, keys = max(1, int(news.max())), int((lens + news).max())
        w = work(c)
        scores = c["n_req"] * c["layers"] * c["q_heads"] * rows * keys if kind in ("chunk4", "decode4") else \
            c["n_req"] * rows * keys * c["heads"] * dim // BLOCK if kind == "sparse" else 0
        return (scores > _MAX_SCORES or c["n_req"] * c["layers"] * c["heads"] * keys * dim > _MAX_PADDED or
                w["flops"] > _MAX_WORK or w["bytes"] > _MAX_BYTES)

    while too_much() and c["n_req"] > 1:
        c["n_req"] = c["n_req"] // 2
    while too_much():
        c["len_lo"], c["len_hi"] = max(1, c["len_lo"] // 2), max(1, c["len_hi"] // 2)
        if c["new_lo"]:
            c["new_lo"], c["new_hi"] = max(1, c["new_lo"] // 2), max(1, c["new_hi"] // 2)
    return c


# --- the batch's shape ------------------------------------------------------------------------------------------------


def _lengths(c):
    """(cached tokens before the call, new tokens) of every request, from the case alone."""
    rng = np.random.Generator(np.random.PCG64(c["shape_seed"]))
    lens = rng.integers(c["len_lo"], c["len_hi"] + 1, size=c["n_req"])
    if not c["new_lo"]:
        return lens.astype(np.int64), np.zeros(c["n_req"], np.int64)
    news = np.round(np.exp(rng.uniform(math.log(c["new_lo"]), math.log(c["new_hi"]), size=c["n_req"]))).astype(np.int64)
    return lens.astype(np.int64), news


def _row_bytes(c):
    """Bytes of one row of K or V of one head in the pool."""
    return {16: 2 * c["dim"], 8: c["dim"] + 1, 4: c["dim"] * 17 // 32}[c["bits"]]


def work(c):
    lens, news = _lengths(c)
    h, hq, d, n_l = c["heads"], c["q_heads"], c["dim"], c["layers"]
    new, total = int(news.sum()), int((lens + news).sum())
    if c["kind"] in ("rotate", "chunk4"):  # q, k, v and the table's rows in, q out, k and v written
        w = {"bytes": new * ((2 * hq + 2 * h) * 2 * d + 2 * h * _row_bytes(c) + 4 * c["rotary"]),
             "flops": new * (hq + h) * 3 * c["rotary"]}
        if c["kind"] == "chunk4":  # the cache in, the result out
            seen = int((news * lens + news * (news + 1) // 2).sum())
            w["bytes"] += int(lens.sum()) * 2 * h * _row_bytes(c) + new * hq * 2 * d
            w["flops"] += 4 * d * hq * seen
        return w
    if c["kind"] == "bounds":  # K in, two rows a block out
        blocks = int((-(-lens // BLOCK)).sum())
        return {"bytes": total * h * _row_bytes(c) + blocks * h * 4 * d, "flops": 2 * total * h * d}
    if c["kind"] == "sparse":  # for every token and head the bounds and the blocks selected, q in, the result out
        seen = np.concatenate([n + 1 + np.arange(m) for n, m in zip(lens.tolist(), news.tolist())])
        blocks = -(-seen // BLOCK)
        read = np.minimum(blocks, c["select"])
        rows = int(((read - 1) * BLOCK + (seen - 1) % BLOCK + 1).sum())
        # (the bounds and blocks of a request's tokens that are the same are needed once: those of its last token)
        last = np.cumsum(news) - 1
        rows_once = int(((read - 1) * BLOCK + (seen - 1) % BLOCK + 1)[last].sum())
        return {"bytes": int(blocks[last].sum()) * h * 4 * d + rows_once * 2 * h * _row_bytes(c) + new * hq * 4 * d + new * h * 4 * c["select"],
                "flops": 4 * d * hq * rows + 2 * d * hq * int(blocks.sum())}
    rows = n_l * h * total
    if c["kind"] == "quantise4":
        return {"bytes": rows * 2 * (2 * d + _row_bytes(c)), "flops": rows * 2 * 2 * d}
    return {"bytes": rows * 2 * _row_bytes(c) + c["n_req"] * n_l * h * d * 6, "flops": rows * 4 * d}


# --- the formats ------------------------------------------------------------------------------------------------------


def _power_of_two(exps):
    return (exps.to(torch.int32) << 23).view(torch.float32)


def _quantise8(x):
    """Rows of fp32 values that are fp16 numbers -> (codes, exponents + 127), bytes."""
    top, power = torch.frexp(x.abs().amax(-1))
    e = (power - 9 + (top > 0.875)).clamp(-15, 8)
    most = torch.where(e == 8, 240.0, 448.0)[..., None]  # (256 * 2^8 is no fp16 number)
    scaled = x * _power_of_two(127 - e)[..., None]
    return torch.minimum(torch.maximum(scaled, -most), most).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _quantise4(x):
    """The same in 4 bits: (codes, two to a byte; exponents + 127 of every 32 channels)."""
    g = x.unflatten(-1, (-1, 32))
    top, power = torch.frexp(g.abs().amax(-1))
    e = (power - 3 + (top > 0.75)).clamp(-23, 13)
    s = (g.abs() * _power_of_two(127 - e)[..., None]).flatten(-2)
    # (to the nearest, ties to the even code; what is over 5 is 6)
    code = (s > 0.25).to(torch.uint8) + (s >= 0.75) + (s > 1.25) + (s >= 1.75) + (s > 2.5) + (s >= 3.5) + (s > 5)
    code = code | (torch.signbit(x).to(torch.uint8) << 3)
    return code[..., ::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _parts(kv, c):
    """Codes [...][K|V][head][slot][bytes] and exponents of pool blocks of bytes [...][bytes], views."""
    h, d = c["heads"], c["dim"]
    if c["bits"] == 8:
        return kv[..., :2 * h * BLOCK * d].unflatten(-1, (2, h, BLOCK, d)), kv[..., 2 * h * BLOCK * d:].unflatten(-1, (2, h, BLOCK))
    return kv[..., :h * BLOCK * d].unflatten(-1, (2, h, BLOCK, d // 2)), kv[..., h * BLOCK * d:].unflatten(-1, (2, h, BLOCK, d // 32))


def _values(kv, c):
    """What blocks of the pool stand for, fp32 [...][K|V][head][slot][channel]."""
    if c["bits"] == 16:
        return kv.float()
    codes, exps = _parts(kv, c)
    if c["bits"] == 8:
        return codes.view(torch.float8_e4m3fn).float() * _power_of_two(exps)[..., None]
    of = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=kv.device)
    x = torch.empty(codes.shape + (2,), device=kv.device)
    x[..., 0] = of[(codes & 15).int()]
    x[..., 1] = of[(codes >> 4).int()]
    return (x.flatten(-2).unflatten(-1, (-1, 32)) * _power_of_two(exps)[..., None]).flatten(-2)


# --- inputs -----------------------------------------------------------------------------------------------------------


def _pool(c, bits, n_blocks, gen, loud):
    """A pool full of rows: N(0, 1), four key channels of every head eight times as large."""
    h, d, n_l = c["heads"], c["dim"], c["layers"]
    dev = torch.device("cuda:0")
    kv = torch.empty((n_l, n_blocks, 2, h, BLOCK, d), dtype=torch.float16, device=dev) if bits == 16 else \
        torch.empty((n_l, n_blocks, 2 * h * BLOCK * (d + 1) if bits == 8 else 17 * h * d), dtype=torch.uint8, device=dev)
    step = max(1, (1 << 28) // (2 * h * BLOCK * d))
    for layer in range(n_l):
        for at in range(0, n_blocks, step):
            n = min(step, n_blocks - at)
            x = torch.randn((n, 2, h, BLOCK, d), generator=gen, device=dev)
            x[:, 0] *= loud[:, None, :]
            x = x.half()
            if bits != 16:
                codes, exps = (_quantise8 if bits == 8 else _quantise4)(x.float())
                x = torch.cat([codes.reshape(n, -1), exps.reshape(n, -1)], 1)
            kv[layer, at:at + n] = x
    return kv


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    lens, news = _lengths(c)
    h, hq, d = c["heads"], c["q_heads"], c["dim"]
    s = {"case": c, "lens": (lens + news).astype(np.int32), "news": news.astype(np.int32)}
    loud = 1.0 + 7.0 * (torch.rand((h, d), generator=gen, device=dev).argsort(-1).argsort(-1) < 4)
    need = -(-s["lens"].astype(np.int64) // BLOCK)
    n_blocks = int(math.ceil(int(need.sum()) / 0.9)) + 1
    order = torch.randperm(n_blocks, generator=gen, device=dev).cpu().numpy().astype(np.int32)
    table = np.full((c["n_req"], int(need.max())), -1, np.int32)
    for r, at in enumerate(np.cumsum(need) - need):
        table[r, :need[r]] = order[at:at + need[r]]
    s["table"] = torch.from_numpy(table).to(dev)
    s["kv"] = _pool(c, 16 if c["kind"] == "quantise4" else c["bits"], n_blocks, gen, loud)
    if c["kind"] in ("rotate", "chunk4"):  # what the projection of the new tokens gives: q, k and v of a token side by side
        x = torch.randn((int(news.sum()), hq + 2 * h, d), generator=gen, device=dev)
        x[:, hq:hq + h] *= loud
        x = x.half()
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
        angles = torch.arange(_POSITIONS, device=dev).double()[:, None] * \
            torch.exp2(torch.arange(c["rotary"] // 2, device=dev).double() * (-2.0 / c["rotary"] * math.log2(10000.0)))
        s["angles"] = torch.stack([angles.cos(), angles.sin()], 1).float()  # [position][cosines, sines][pair]
        # (compressed caches are shorter than the positions that they end at)
        ahead = torch.randint(0, 30000, (c["n_req"],), generator=gen, device=dev).cpu().numpy()
        s["positions"] = (lens + np.where(lens > 0, ahead, 0)).astype(np.int32)
    elif c["kind"] == "sparse":
        s["q"] = torch.randn((int(news.sum()), hq, d), generator=gen, device=dev).half()
    elif c["kind"] == "decode4":
        s["q"] = torch.randn((c["n_req"], c["layers"], h, d), generator=gen, device=dev).half()
    elif c["kind"] == "quantise4":
        s["table4"] = torch.from_numpy(np.where(table >= 0, n_blocks - 1 - table, -1).astype(np.int32)).to(dev)
        s["kv4"] = torch.zeros((c["layers"], n_blocks, 17 * h * d), dtype=torch.uint8, device=dev)
    if c["kind"] in ("bounds", "sparse"):
        s["bounds"] = torch.zeros((1, n_blocks, h, 2, d), dtype=torch.float16, device=dev)
    if c["kind"] == "sparse":  # the bounds of what was cached before
        step = max(1, (1 << 26) // (2 * h * BLOCK * d))
        n = torch.from_numpy(s["lens"] - s["news"]).to(dev)
        ids = torch.full((n_blocks,), BLOCK, dtype=torch.int64, device=dev)  # tokens of each block
        cached = s["table"] >= 0
        ids[s["table"][cached].long()] = (n[:, None] - torch.arange(table.shape[1], device=dev) * BLOCK).clamp(1, BLOCK)[cached]
        for at in range(0, n_blocks, step):
            s["bounds"][0, at:at + step] = _bounds_of(_values(s["kv"][0, at:at + step], c)[:, 0], ids[at:at + step]).half()
        s["selected"] = torch.empty((int(news.sum()), h, c["select"]), dtype=torch.int32, device=dev)
    if own:  # the handles of the pools, which a program keeps
        from paper_2503_08461_amd import fastcache as fc
        s["fc"] = fc
        dtypes = {16: fc.FC_DTYPE_F16, 8: fc.FC_DTYPE_E4M3, 4: fc.FC_DTYPE_E2M1}
        bits = 16 if c["kind"] == "quantise4" else c["bits"]
        s["pool"] = _Pool(fc, fc.fc_pool_create(s["kv"], n_blocks, c["layers"], h, d, dtype=dtypes[bits]))
        if "kv4" in s:
            s["pool4"] = _Pool(fc, fc.fc_pool_create(s["kv4"], n_blocks, c["layers"], h, d, dtype=dtypes[4]))
        if "angles" in s:
            s["rotation"] = fc.Rotation(s["angles"], interleaved=c["interleaved"])
    return s


class _Pool:
    """A pool's handle; the library's side of it goes with the object."""

    def __init__(self, fc, handle):
        self.fc, self.handle = fc, handle

    def __del__(self):
        self.fc.fc_pool_destroy(self.handle)


# --- one pass ---------------------------------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "rotate":
        return {"q": _rotate_store(s, c), **_cache(s["kv"], c)}
    if c["kind"] == "chunk4":
        q = _rotate_store(s, c)
        return {"q": q, "out": _chunk(s, c, q), **_cache(s["kv"], c)}
    if c["kind"] == "quantise4":
        _quantise_cache(s, c)
        return {"kv": s["kv4"]}
    if c["kind"] == "decode4":
        return {"out": _decode(s, c)}
    if c["kind"] == "bounds":
        _bounds(s, c)
        return {"bounds": s["bounds"]}
    _bounds(s, c)
    out = _sparse(s, c)
    return {"out": out, "selected": s["selected"], "bounds": s["bounds"]}


def _cache(kv, c):
    if c["bits"] != 8:
        return {"kv": kv}
    codes, exps = _parts(kv, c)
    return {"codes": codes.view(torch.float8_e4m3fn), "exponents": exps}


def _run_own(s, c):
    fc = s["fc"]
    pool = s["pool"].handle
    if c["kind"] == "rotate":
        return {"q": fc.fc_rotate_store_chunk(pool, 0, s["table"], s["lens"], s["news"], s["rotation"], s["q"], s["k"], s["v"],
                                              positions=s["positions"]), **_cache(s["kv"], c)}
    if c["kind"] == "chunk4":
        q = fc.fc_rotate_store_chunk(pool, 0, s["table"], s["lens"], s["news"], s["rotation"], s["q"], s["k"], s["v"],
                                     positions=s["positions"])
        return {"q": q, "out": fc.fc_chunk_attention(pool, 0, s["table"], s["lens"], s["news"], q), **_cache(s["kv"], c)}
    if c["kind"] == "quantise4":
        fc.fc_quantise_batch(s["pool4"].handle, s["table4"], pool, s["table"], s["lens"])
        return {"kv": s["kv4"]}
    if c["kind"] == "decode4":
        return {"out": fc.fc_decode_attention(pool, s["table"], s["lens"], s["q"])}
    if c["kind"] == "bounds":
        fc.fc_block_bounds(pool, 0, s["table"], s["lens"], s["lens"], s["bounds"])
        return {"bounds": s["bounds"]}
    fc.fc_block_bounds(pool, 0, s["table"], s["lens"], s["news"], s["bounds"])
    out = fc.fc_sparse_attention(pool, 0, s["table"], s["lens"], s["news"], s["bounds"], c["select"], s["q"], selected=s["selected"])
    return {"out": out, "selected": s["selected"], "bounds": s["bounds"]}


# The plain form: requests padded to the longest, scores of every pair in fp32, masked, softmax, product.


def _index(counts, dev):
    """For packed rows of `counts` each: the request and the row within it."""
    n = torch.from_numpy(counts.astype(np.int64)).to(dev)
    req = torch.repeat_interleave(torch.arange(len(counts), device=dev), n)
    return req, torch.arange(req.numel(), device=dev) - (n.cumsum(0) - n)[req]


def _device(s, *names):
    return (torch.from_numpy(s[x].astype(np.int64)).to(s["table"].device) for x in names)


def _rotated(x, angles, c):
    """Rows [token][head][channel], their angles' cosines and sines [token][2][pair]."""
    n = c["rotary"]
    cos, sin = angles[:, None, 0].double(), angles[:, None, 1].double()
    y, out = x[..., :n].double(), x.clone()
    if c["interleaved"]:
        a, b = y[..., ::2], y[..., 1::2]
        out[..., :n] = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2).float().half()
    else:
        a, b = y[..., :n // 2], y[..., n // 2:]
        out[..., :n] = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).float().half()
    return out


def _rotate_store(s, c):
    kv, table = s["kv"], s["table"]
    req, row = _index(s["news"], table.device)
    lens, news, positions = _device(s, "lens", "news", "positions")
    angles = s["angles"][positions[req] + row]
    q, k = _rotated(s["q"], angles, c), _rotated(s["k"], angles, c)
    at = (lens - news)[req] + row
    block, slot = table[req, at // BLOCK].long(), at % BLOCK
    new = torch.stack([k, s["v"]], 1)  # [row][K|V][head][channel]
    if c["bits"] == 16:
        kv[0, block, :, :, slot] = new
    else:
        codes, exps = (_quantise8 if c["bits"] == 8 else _quantise4)(new.float())
        to_codes, to_exps = _parts(kv, c)
        to_codes[0, block, :, :, slot] = codes
        to_exps[0, block, :, :, slot] = exps
    return q


def _attend(q, k, v, visible):
    """q [request][head][row][channel], k and v [request][head of K and V][key][channel], fp32; visible: rows' last key."""
    group = q.shape[1] // k.shape[1]
    r, h, n, d = k.shape
    rows = q.shape[2]
    scores = torch.matmul(q.reshape(r, h, group * rows, d), k.transpose(2, 3).contiguous()).reshape(r, h, group, rows, n)
    scores *= 1.0 / math.sqrt(d)
    hidden = torch.arange(n, device=q.device) > visible[:, :, None]  # [request][row][key]
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    scores -= scores.amax(-1, keepdim=True)
    scores.exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.reshape(r, h, group * rows, n), v).reshape(r, h, group, rows, d) / total
    return out.reshape(r, h * group, rows, d)


def _gathered(s, c, blocks, lens):
    """(K, V) of block lists [request][block] of one layer or all, fp32, padded: [request][head][key][channel]."""
    x = _values(blocks, c).permute(2, 0, 3, 1, 4, 5).flatten(3, 4)
    past = torch.arange(x.shape[3], device=x.device) >= lens[:, None]
    return x[0].contiguous(), x[1].masked_fill(past[:, None, :, None], 0.0).contiguous()


def _chunk(s, c, q):
    req, row = _index(s["news"], q.device)
    lens, news = _device(s, "lens", "news")
    k, v = _gathered(s, c, s["kv"][0][s["table"].clamp_min(0).long()], lens)
    longest = int(s["news"].max())
    padded = torch.zeros((c["n_req"], longest) + q.shape[1:], device=q.device)
    padded[req, row] = q.float()
    out = _attend(padded.transpose(1, 2).contiguous(), k, v, (lens - news)[:, None] + torch.arange(longest, device=q.device))
    return out.transpose(1, 2)[req, row].half()


def _decode(s, c):
    """All layers at once: a layer is a request of its own."""
    n, n_l = s["q"].shape[:2]
    t = s["table"].clamp_min(0).long()
    lens, = _device(s, "lens")
    lens = lens.repeat_interleave(n_l)
    k, v = _gathered(s, c, s["kv"][:, t].transpose(0, 1).flatten(0, 1), lens)
    out = _attend(s["q"].float().flatten(0, 1)[:, :, None], k, v, (lens - 1)[:, None])
    return out.reshape(s["q"].shape)


def _quantise_cache(s, c):
    req, row = _index(s["lens"], s["table"].device)
    block, block4, slot = s["table"][req, row // BLOCK].long(), s["table4"][req, row // BLOCK].long(), row % BLOCK
    codes, exps = _quantise4(s["kv"][:, block, :, :, slot].float())  # [row][layer][K|V][head][channel]
    to_codes, to_exps = _parts(s["kv4"], c)
    to_codes[:, block4, :, :, slot] = codes
    to_exps[:, block4, :, :, slot] = exps


def _bounds_of(k, count):
    """[block][2][...]: smallest and largest of the first `count` tokens, k: [block][head][slot][channel]."""
    behind = (torch.arange(BLOCK, device=k.device) >= count[:, None])[:, None, :, None]
    return torch.stack([k.masked_fill(behind, math.inf).amin(2), k.masked_fill(behind, -math.inf).amax(2)], 2)


def _bounds(s, c):
    """Of the blocks that hold the new tokens (all tokens where the case has no new ones)."""
    lens, news = _device(s, "lens", "news" if c["kind"] == "sparse" else "lens")
    first = (lens - news) // BLOCK
    counts = (-(-lens // BLOCK) - first)
    req = torch.repeat_interleave(torch.arange(len(lens), device=lens.device), counts)
    b = torch.arange(req.numel(), device=lens.device) - (counts.cumsum(0) - counts)[req] + first[req]
    ids = s["table"][req, b].long()
    k = _values(s["kv"][0][ids], c)[:, 0]
    s["bounds"][0, ids] = _bounds_of(k, (lens[req] - b * BLOCK).clamp_max(BLOCK)).half()


def _sparse(s, c):
    h, hq, d, n_sel = c["heads"], c["q_heads"], c["dim"], c["select"]
    req, row = _index(s["news"], s["q"].device)
    lens, news = _device(s, "lens", "news")
    seen = (lens - news)[req] + row + 1
    n_blocks = -(-seen // BLOCK)
    t = s["table"].clamp_min(0).long()[req]  # [token][block]
    lo, hi = s["bounds"][0][t].double().permute(3, 0, 2, 1, 4)  # [token][head][block][channel]
    q = s["q"].double().reshape(-1, h, hq // h, d)
    score = (torch.matmul(q.clamp_min(0), hi.transpose(2, 3).contiguous()) + torch.matmul(q.clamp_max(0), lo.transpose(2, 3).contiguous())).amax(2)
    at = torch.arange(t.shape[1], device=t.device)
    score = score.masked_fill((at >= n_blocks[:, None])[:, None], -math.inf).masked_fill((at == n_blocks[:, None] - 1)[:, None], math.inf)
    best = torch.sort(score, descending=True, stable=True)[1][..., :n_sel]
    none = best >= n_blocks[:, None, None]
    best = torch.sort(best.masked_fill(none, 1 << 30), -1)[0]
    none = best == 1 << 30
    s["selected"].fill_(-1)
    s["selected"][..., :best.shape[2]] = best.masked_fill(none, -1).int()
    ids = torch.gather(t[:, None].expand(-1, h, -1), 2, best.masked_fill(none, 0))  # [token][head][selected]
    token = (best[..., None] * BLOCK + torch.arange(BLOCK, device=t.device)).flatten(2)
    hidden = token >= seen[:, None, None]
    head = torch.arange(h, device=t.device)[None, :, None]
    if c["bits"] == 16:
        x = s["kv"][0][ids, :, head].float()  # [token][head][selected][K|V][slot][channel]
    else:
        codes, exps = _parts(s["kv"][0], c)
        one = dict(c, heads=1)
        x = torch.cat([codes[ids, :, head].flatten(3), exps[ids, :, head].flatten(3)], -1)
        x = _values(x, one)[..., 0, :, :]
    x = x.permute(3, 0, 1, 2, 4, 5).flatten(3, 4)
    v = x[1].masked_fill(hidden[..., None], 0.0)
    p = torch.matmul(s["q"].float().reshape(-1, h, hq // h, d), x[0].transpose(2, 3).contiguous()) / math.sqrt(d)
    p = p.masked_fill(hidden[:, :, None], -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp()
    return (torch.matmul(p, v) / p.sum(-1, keepdim=True)).reshape(s["q"].shape).half()


# --- the definition, in 64 bits ---------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions on the same inputs, request by request and head by head, in 64 bits; what is whole numbers is not
    computed.  None where nothing else comes back, or where it takes long."""
    if case["kind"] == "quantise4" or work(case)["flops"] > 6e12:
        return None
    s = prepare(case, seed)
    c = s["case"]
    h, hq, d = c["heads"], c["q_heads"], c["dim"]
    scale = 1.0 / math.sqrt(d)
    dev = s["table"].device

    def number(code):  # what each of 16 codes stands for
        m, e = code & 1, (code >> 1) & 3
        x = (1 + m / 2) * 2.0 ** (e - 1) if e else m / 2
        return -x if code & 8 else x

    numbers = torch.tensor([number(i) for i in range(16)], dtype=torch.float64, device=dev)

    def nearest8(x):
        top = x.abs().amax(-1)
        e = torch.full(top.shape, 8, dtype=torch.int64, device=dev)
        for k in range(7, -16, -1):
            e = torch.where(top <= 448.0 * 2.0 ** k, k, e)
        y = x / torch.exp2(e.double())[..., None]
        _, p = torch.frexp(y.abs())
        step = torch.exp2((p - 1).clamp_min(-6).double() - 3)
        most = torch.where(e == 8, 240.0, 448.0)[..., None].double()
        return (torch.round(y / step) * step).clamp(-most, most), e

    def nearest4(x):
        g = x.unflatten(-1, (-1, 32))
        top = g.abs().amax(-1)
        e = torch.full(top.shape, 13, dtype=torch.int64, device=dev)
        for k in range(12, -24, -1):
            e = torch.where(top <= 6.0 * 2.0 ** k, k, e)
        y = (g / torch.exp2(e.double())[..., None]).clamp(-6, 6)
        _, p = torch.frexp(y.abs())
        step = torch.exp2((p - 1).clamp_min(0).double() - 1)
        return (torch.round(y / step) * step * torch.exp2(e.double())[..., None]).flatten(-2)

    def block_values(ids, layer=0):
        """[block][K|V][head][slot][channel], fp64"""
        x = s["kv"][layer, ids]
        if c["bits"] == 16:
            return x.double()
        codes, exps = _parts(x, c)
        if c["bits"] == 8:
            return codes.view(torch.float8_e4m3fn).double() * torch.exp2(exps.double() - 127)[..., None]
        y = numbers[torch.stack([codes % 16, codes // 16], -1).int()].flatten(-2)
        return (y.unflatten(-1, (-1, 32)) * torch.exp2(exps.double() - 127)[..., None]).flatten(-2)

    def softmax(q, k, v, first):
        """q [row][d] sees keys 0..first + row."""
        t = (q @ k.T.contiguous()) * scale
        t = t.masked_fill(torch.arange(k.shape[0], device=dev) > first + torch.arange(q.shape[0], device=dev)[:, None], -math.inf)
        return torch.softmax(t, -1) @ v

    def cached(r, n, layer=0):
        x = block_values(s["table"][r, :-(-n // BLOCK)].long(), layer).permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n]
        return x[0], x[1]

    def turned(x, first):
        """Rows [token][head][channel] from position `first` on, by complex numbers."""
        n = c["rotary"]
        w = s["angles"][first:first + x.shape[0]].double()
        w = torch.complex(w[:, 0], w[:, 1])[:, None]
        y = x.double()
        a, b = (y[..., :n:2], y[..., 1:n:2]) if c["interleaved"] else (y[..., :n // 2], y[..., n // 2:n])
        z = torch.complex(a.contiguous(), b.contiguous()) * w
        z = torch.stack([z.real, z.imag], -1).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
        return torch.cat([z, y[..., n:]], -1)

    if c["kind"] == "decode4":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=dev)
        for r, n in enumerate(s["lens"].tolist()):
            for layer in range(c["layers"]):
                k, v = cached(r, n, layer)
                t = (k * s["q"][r, layer].double()[:, None, :]).sum(-1) * scale
                out[r, layer] = (torch.softmax(t, -1)[..., None] * v).sum(1)
        return {"out": out}
    if c["kind"] in ("bounds", "sparse"):
        bounds = s["bounds"].double()
        for r, n in enumerate(s["lens"].tolist()):
            first = 0 if c["kind"] == "bounds" else (n - int(s["news"][r])) // BLOCK
            ids = s["table"][r, first:-(-n // BLOCK)].long()
            k = block_values(ids)[:, 0]
            bounds[0, ids] = torch.stack([k.amin(2), k.amax(2)], 2)
            last = k[-1, :, :n - (n - 1) // BLOCK * BLOCK]
            bounds[0, ids[-1]] = torch.stack([last.amin(1), last.amax(1)], 1)
        if c["kind"] == "bounds":
            return {"bounds": bounds}
        out = torch.empty((s["q"].shape[0], hq, d), dtype=torch.float64, device=dev)
        t = 0
        for r, (n, m) in enumerate(zip(s["lens"].tolist(), s["news"].tolist())):
            k, v = cached(r, n)
            lo_hi = bounds[0, s["table"][r, :-(-n // BLOCK)].long()]
            for seen in range(n - m + 1, n + 1):
                nb = -(-seen // BLOCK)
                for j in range(h):
                    q = s["q"][t, j * hq // h:(j + 1) * hq // h].double()
                    prod = q[:, None, None] * lo_hi[None, :nb, j]  # [query head][block][lo, hi][channel]
                    score = prod.amax(2).sum(-1).amax(0)
                    score[nb - 1] = math.inf
                    keep = torch.sort(score, descending=True, stable=True)[1][:c["select"]]
                    tok = (keep[:, None] * BLOCK + torch.arange(BLOCK, device=dev)).flatten()
                    tok = tok[tok < seen]
                    out[t, j * hq // h:(j + 1) * hq // h] = torch.softmax(q @ k[j, tok].T.contiguous() * scale, -1) @ v[j, tok]
                t += 1
        return {"out": out, "selected": None, "bounds": bounds}
    # rotate, chunk4: rows rounded to 16 bits as they are stored, and as they come back
    q = torch.empty((s["q"].shape[0], hq, d), dtype=torch.float64, device=dev)
    out = torch.empty_like(q)
    kv = s["kv"].double() if c["bits"] == 16 else None
    codes8 = _parts(s["kv"], c)[0].view(torch.float8_e4m3fn).double() if c["bits"] == 8 else None
    at = 0
    for r, n in enumerate(s["news"].tolist()):
        first, position = int(s["lens"][r]) - n, int(s["positions"][r])
        q[at:at + n] = turned(s["q"][at:at + n], position)
        k, v = turned(s["k"][at:at + n], position).float().half().double(), s["v"][at:at + n].double()
        tok = first + torch.arange(n, device=dev)
        ids, slot = s["table"][r, tok // BLOCK].long(), tok % BLOCK
        new = torch.stack([k, v], 1)  # [token][K|V][head][channel]
        if c["bits"] == 16:
            kv[0, ids, :, :, slot] = new
        elif c["bits"] == 8:
            codes8[0, ids, :, :, slot] = nearest8(new)[0]
        if c["kind"] == "chunk4":
            k, v = nearest4(new).permute(1, 2, 0, 3)
            old_k, old_v = cached(r, first)
            k, v = torch.cat([old_k, k], 1), torch.cat([old_v, v], 1)
            turned_q = q[at:at + n].float().half().double()
            for j in range(hq):
                out[at:at + n, j] = softmax(turned_q[:, j], k[j * h // hq], v[j * h // hq], first)
        at += n
    found = {"q": q, "out": out} if c["kind"] == "chunk4" else {"q": q}
    return {**found, "codes": codes8, "exponents": None} if c["bits"] == 8 else {**found, "kv": kv}
