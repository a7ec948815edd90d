"""Attention over whole prompts and over chunks of new tokens, and the 8-bit cache: the cases that these operators'
speed is measured on, each with its plain form, its required work and its 64-bit definition.

prefill   causal attention of whole prompts, packed one after the other, q, k and v as views of one projection's rows
chunk     new tokens' K and V written into the paged pool, then their attention over the cache, for one layer; a chunk
          of one token is the decode step of a model with grouped heads; the pool holds fp16 rows or 8-bit ones
quantise  the cache of a batch copied from an fp16 pool into an 8-bit one
decode8   a decode step's attention over an 8-bit pool, all layers at once

An 8-bit row is e4m3 codes times one power of two: the smallest 2^e that brings the row's largest magnitude to 448 or
less, -15 <= e <= 8, so that every value it stands for is an fp16 number.  A pool block holds the codes of
[K|V][head][slot][channel] and behind them the exponents, e + 127, of [K|V][head][slot].
"""

import math

import numpy as np
import torch

own = False

BLOCK = 16


def _case(name, kind, n_req, len_lo, len_hi, heads, q_heads, dim, new_lo=1, new_hi=1, bits=16, layers=1, window=0,
          shape_seed=1):
    """n_req requests of len_lo..len_hi cached tokens (prefill: prompt tokens), new_lo..new_hi new ones (chunk), drawn from
    shape_seed; heads: of K and V; window: the last rows of each request whose log-sum-exp is asked for."""
    c = dict(kind=kind, n_req=n_req, len_lo=len_lo, len_hi=len_hi, new_lo=new_lo, new_hi=new_hi, heads=heads,
             q_heads=q_heads, dim=dim, bits=bits, layers=layers, window=window, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: one short question to a four-head toy model; launches and host time are all there is
        _case("prefill_question", "prefill", 1, 29, 29, 4, 4, 64, window=16),
        # one single-image prompt of 640 tokens (benchmark configuration 2), for compression with its log-sum-exps
        _case("prefill_image", "prefill", 1, 640, 640, 32, 32, 128, window=32),
        # a batch of ordinary prompts of different lengths (configuration 3)
        _case("prefill_packed", "prefill", 32, 600, 1200, 32, 32, 128, window=32),
        # a few multi-image prompts (configuration 4's longest) for a model with four query heads to a key head
        _case("prefill_long", "prefill", 3, 5900, 7040, 8, 32, 128, window=64),
        # the decode step of a large batch with grouped heads, caches not compressed
        _case("chunk_tokens", "chunk", 48, 1280, 7040, 8, 32, 128),
        # a mixed step of a server that splits prompts: chunks of up to 512 tokens next to single tokens
        _case("chunk_mixed", "chunk", 24, 256, 4000, 32, 32, 128, 1, 512),
        # the last 2048 tokens of a very long prompt over what is cached of it
        _case("chunk_long", "chunk", 1, 30000, 30000, 8, 32, 128, 2048, 2048, window=32),
        # drafted tokens over compressed caches in an 8-bit pool
        _case("chunk8_drafts", "chunk", 32, 256, 1408, 8, 32, 128, 5, 5, bits=8),
        # what the toy configuration keeps of its prompt, 64 tokens
        _case("quantise_question", "quantise", 1, 64, 64, 4, 4, 64, bits=8),
        # the compressed caches of 64 multi-image prompts (configuration 4, 4 of its 32 layers)
        _case("quantise_batch", "quantise", 64, 256, 1408, 32, 32, 128, bits=8, layers=4),
        # one decode step of a few requests over compressed caches, pool of one layer
        _case("decode8_small", "decode8", 8, 256, 1408, 32, 32, 128, bits=8),
        # one decode step of a large batch over uncompressed caches
        _case("decode8_full", "decode8", 48, 1280, 7040, 32, 32, 128, bits=8, layers=2),
    ]


_MAX_SEQ = 32768
_MAX_SCORES = 4e9     # elements of the padded score matrix of the plain form
_MAX_PADDED = 1.5e9   # elements of the padded keys
_MAX_WORK = 1e12      # flops and bytes: no more than the largest listed cases
_MAX_BYTES = 4e9


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["prefill", "prefill", "chunk", "chunk", "chunk", "quantise", "decode8"])
    dim = rng.choice([64, 128, 128])
    heads, group = rng.choice([(1, 8), (2, 4), (4, 1), (4, 8), (5, 3), (8, 4), (8, 5), (12, 1), (12, 2), (32, 1), (40, 1)])
    if kind in ("quantise", "decode8"):
        group = 1
    len_lo = log_int(1, 12000)
    len_hi = min(30000, len_lo * rng.choice([1, 2, 3]) + rng.randrange(16))
    new_lo = rng.choice([1, 1, 4, log_int(1, 1500)])
    new_hi = min(2048, new_lo * rng.choice([1, 1, 4]) + rng.choice([0, 0, rng.randrange(64)]))
    if kind == "prefill":
        len_lo, len_hi = min(len_lo, 7040), min(len_hi, 7040)
        new_lo = new_hi = 1
    elif kind != "chunk":
        new_lo = new_hi = 1
    c = _case("", kind, log_int(1, 64), len_lo, len_hi, heads, heads * group, dim, new_lo, new_hi,
              16 if kind == "prefill" else 8 if kind != "chunk" else rng.choice([8, 16]),
              1 if kind in ("prefill", "chunk") else rng.choice([1, 2, 4]),
              rng.choice([0, 16, 32, 64]) if kind in ("prefill", "chunk") else 0, rng.randrange(1 << 20))

    def too_much():
        lens, news = _lengths(c)
        rows = int(news.max()) if kind == "chunk" else int(lens.max()) if kind == "prefill" else 1
        keys = int((lens + news).max()) if kind == "chunk" else int(lens.max())
        w = work(c)
        return (c["n_req"] * c["layers"] * c["q_heads"] * rows * keys > _MAX_SCORES or
                c["n_req"] * c["layers"] * c["heads"] * keys * dim > _MAX_PADDED or
                w["flops"] > _MAX_WORK or w["bytes"] > _MAX_BYTES)

    while too_much() and c["n_req"] > 1:
        c["n_req"] = c["n_req"] // 2
    while too_much():
        c["len_lo"], c["len_hi"] = max(1, c["len_lo"] // 2), max(1, c["len_hi"] // 2)
        c["new_lo"], c["new_hi"] = max(1, c["new_lo"] // 2), max(1, c["new_hi"] // 2)
    return c


# --- the batch's shape ------------------------------------------------------------------------------------------------


def _lengths(c):
    """(cached tokens before the call, new tokens) of every request, from the case alone."""
    rng = np.random.Generator(np.random.PCG64(c["shape_seed"]))
    lens = rng.integers(c["len_lo"], c["len_hi"] + 1, size=c["n_req"])
    news = np.round(np.exp(rng.uniform(math.log(c["new_lo"]), math.log(c["new_hi"]), size=c["n_req"]))).astype(np.int64)
    if c["kind"] != "chunk":
        news = np.zeros(c["n_req"], np.int64)
    return lens.astype(np.int64), news


def _row_bytes(c):
    """Bytes of one row of K or V of one head in the pool."""
    return 2 * c["dim"] if c["bits"] == 16 else c["dim"] + 1


def work(c):
    lens, news = _lengths(c)
    h, hq, d, n_l = c["heads"], c["q_heads"], c["dim"], c["layers"]
    lse = 4 * hq * int(np.minimum(c["window"], lens if c["kind"] == "prefill" else news).sum())
    if c["kind"] == "prefill":  # q, k, v in, the result out; 4 d operations for each query and key that it sees
        return {"bytes": 2 * d * int(lens.sum()) * (2 * hq + 2 * h) + lse, "flops": 4 * d * hq * int((lens * (lens + 1) // 2).sum())}
    if c["kind"] == "chunk":  # new k and v in and written, the cache and the queries in, the result out
        new = int(news.sum())
        seen = int((news * lens + news * (news + 1) // 2).sum())
        return {"bytes": new * (2 * h * (2 * d + _row_bytes(c)) + 2 * hq * 2 * d) + int(lens.sum()) * 2 * h * _row_bytes(c) + lse,
                "flops": 4 * d * hq * seen}
    rows = n_l * h * int(lens.sum())
    if c["kind"] == "quantise":
        return {"bytes": rows * 2 * (2 * d + _row_bytes(c)), "flops": rows * 2 * 2 * d}
    return {"bytes": rows * 2 * _row_bytes(c) + c["n_req"] * n_l * h * d * 6, "flops": rows * 4 * d}


# --- inputs -----------------------------------------------------------------------------------------------------------


def _power_of_two(exps):
    return (exps.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """Rows of fp32 values that are fp16 numbers -> (codes, exponents + 127)."""
    top, power = torch.frexp(x.abs().amax(-1))
    e = (power - 9 + (top > 0.875)).clamp(-15, 8)
    most = torch.where(e == 8, 240.0, 448.0)[..., None]  # (256 * 2^8 is no fp16 number)
    scaled = x * _power_of_two(127 - e)[..., None]
    return torch.minimum(torch.maximum(scaled, -most), most).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _codes(kv8, c):
    """[layer][block][K|V][head][slot][channel] of an 8-bit pool, a view."""
    h, d = c["heads"], c["dim"]
    return kv8[:, :, :2 * h * BLOCK * d].view(torch.float8_e4m3fn).unflatten(2, (2, h, BLOCK, d))


def _exponents(kv8, c):
    """[layer][block][K|V][head][slot] of an 8-bit pool, a view."""
    h, d = c["heads"], c["dim"]
    return kv8[:, :, 2 * h * BLOCK * d:].unflatten(2, (2, h, BLOCK))


def _pool(c, n_blocks, gen):
    """A pool full of rows: N(0, 1), four key channels of every head eight times as large."""
    h, d, n_l = c["heads"], c["dim"], c["layers"]
    dev = torch.device("cuda:0")
    loud = 1.0 + 7.0 * (torch.rand((h, d), generator=gen, device=dev).argsort(-1).argsort(-1) < 4)
    eight = c["bits"] == 8 and c["kind"] != "quantise"
    kv = torch.empty((n_l, n_blocks, 2 * h * BLOCK * (d + 1)), dtype=torch.uint8, device=dev) if eight else \
        torch.empty((n_l, n_blocks, 2, h, BLOCK, d), dtype=torch.float16, device=dev)
    step = max(1, (1 << 28) // (2 * h * BLOCK * d))
    for layer in range(n_l):
        for at in range(0, n_blocks, step):
            n = min(step, n_blocks - at)
            x = torch.randn((n, 2, h, BLOCK, d), generator=gen, device=dev)
            x[:, 0] *= loud[:, None, :]
            if eight:
                codes, exps = _quantise(x.half().float())
                kv[layer, at:at + n] = torch.cat([codes.reshape(n, -1).view(torch.uint8), exps.reshape(n, -1)], 1)
            else:
                kv[layer, at:at + n] = x.half()
    return kv, loud


def prepare(case, seed):
    c = dict(case)
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    lens, news = _lengths(c)
    h, hq, d = c["heads"], c["q_heads"], c["dim"]
    s = {"case": c, "lens": (lens + news).astype(np.int32), "news": news.astype(np.int32)}
    rows = int(lens.sum()) if c["kind"] == "prefill" else int(news.sum())

    def new_rows(loud):  # what the projection of the new tokens gives: q, k and v of a token side by side
        x = torch.randn((rows, hq + 2 * h, d), generator=gen, device=dev)
        x[:, hq:hq + h] *= loud
        x = x.half()
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + h], x[:, hq + h:]
        s["lse"] = torch.zeros((c["n_req"], 1, hq, c["window"]), device=dev) if c["window"] else None

    if c["kind"] == "prefill":
        new_rows(1.0 + 7.0 * (torch.rand((h, d), generator=gen, device=dev).argsort(-1).argsort(-1) < 4))
        n_blocks = 1
        s["kv"] = torch.empty((1, 1, 2, h, BLOCK, d), dtype=torch.float16, device=dev)
    else:
        need = -(-s["lens"].astype(np.int64) // BLOCK)
        n_blocks = int(math.ceil(int(need.sum()) / 0.9)) + 1
        order = torch.randperm(n_blocks, generator=gen, device=dev).cpu().numpy().astype(np.int32)
        table = np.full((c["n_req"], int(need.max())), -1, np.int32)
        for r, at in enumerate(np.cumsum(need) - need):
            table[r, :need[r]] = order[at:at + need[r]]
        s["table"] = torch.from_numpy(table).to(dev)
        s["kv"], loud = _pool(c, n_blocks, gen)
        if c["kind"] == "chunk":
            new_rows(loud)
        elif c["kind"] == "decode8":
            s["q"] = torch.randn((c["n_req"], c["layers"], h, d), generator=gen, device=dev).half()
        else:
            s["table8"] = torch.from_numpy(np.where(table >= 0, n_blocks - 1 - table, -1).astype(np.int32)).to(dev)
            s["kv8"] = torch.zeros((c["layers"], n_blocks, 2 * h * BLOCK * (d + 1)), dtype=torch.uint8, device=dev)
    if own:  # the handles of the pools, which a program keeps
        from paper_2503_08461_amd import fastcache as fc
        s["fc"] = fc
        dtype = fc.FC_DTYPE_E4M3 if s["kv"].dtype == torch.uint8 else fc.FC_DTYPE_F16
        s["pool"] = _Pool(fc, fc.fc_pool_create(s["kv"], n_blocks, c["layers"], h, d, dtype=dtype))
        if "kv8" in s:
            s["pool8"] = _Pool(fc, fc.fc_pool_create(s["kv8"], n_blocks, c["layers"], h, d, dtype=fc.FC_DTYPE_E4M3))
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
    if c["kind"] == "prefill":
        out = _prefill(s, c)
        return {"out": out} if s["lse"] is None else {"out": out, "lse": s["lse"]}
    if c["kind"] == "chunk":
        out = _chunk(s, c)
        return {"out": out, **_cache(s["kv"], c)} if s["lse"] is None else {"out": out, "lse": s["lse"], **_cache(s["kv"], c)}
    if c["kind"] == "quantise":
        _quantise_cache(s, c)
        return _cache(s["kv8"], c)
    return {"out": _decode8(s, c)}


def _cache(kv, c):
    return {"kv": kv} if kv.dtype == torch.float16 else {"codes": _codes(kv, c), "exponents": _exponents(kv, c)}


def _run_own(s, c):
    fc = s["fc"]
    pool = s["pool"].handle
    if c["kind"] == "prefill":
        out = fc.fc_prefill_attention(pool, 0, s["q"], s["k"], s["v"], s["lens"], lse_out=s["lse"], window=c["window"])
        return {"out": out} if s["lse"] is None else {"out": out, "lse": s["lse"]}
    if c["kind"] == "chunk":
        fc.fc_store_chunk(pool, 0, s["table"], s["lens"], s["news"], s["k"], s["v"])
        out = fc.fc_chunk_attention(pool, 0, s["table"], s["lens"], s["news"], s["q"], lse_out=s["lse"], window=c["window"])
        return {"out": out, **_cache(s["kv"], c)} if s["lse"] is None else {"out": out, "lse": s["lse"], **_cache(s["kv"], c)}
    if c["kind"] == "quantise":
        fc.fc_quantise_batch(s["pool8"].handle, s["table8"], pool, s["table"], s["lens"])
        return _cache(s["kv8"], c)
    return {"out": fc.fc_decode_attention(pool, s["table"], s["lens"], s["q"])}


# The plain form: requests padded to the longest, scores of every pair in fp32, masked, softmax, product.


def _index(counts, dev):
    """For packed rows of `counts` each: the request and the row within it."""
    n = torch.from_numpy(counts.astype(np.int64)).to(dev)
    req = torch.repeat_interleave(torch.arange(len(counts), device=dev), n)
    return req, torch.arange(req.numel(), device=dev) - (n.cumsum(0) - n)[req]


def _attend(q, k, v, visible):
    """q [request][head][row][channel], k and v [request][head of K and V][key][channel], fp32; visible: rows' last key.
    (result, log-sum-exp)"""
    group = q.shape[1] // k.shape[1]
    r, h, n, d = k.shape
    rows = q.shape[2]
    scores = torch.matmul(q.reshape(r, h, group * rows, d), k.transpose(2, 3).contiguous()).reshape(r, h, group, rows, n)
    scores *= 1.0 / math.sqrt(d)
    hidden = torch.arange(n, device=q.device) > visible[:, :, None]  # [request][row][key]
    scores.masked_fill_(hidden[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-1e30)
    scores -= top
    scores.exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.reshape(r, h, group * rows, n), v).reshape(r, h, group, rows, d) / total
    return out.reshape(r, h * group, rows, d), (top + total.log()).reshape(r, h * group, rows)


def _padded(x, req, row, n_req, longest):
    """Packed [row][head][channel] -> [request][head][row][channel], fp32."""
    out = torch.zeros((n_req, longest) + x.shape[1:], dtype=torch.float32, device=x.device)
    out[req, row] = x.float()
    return out.transpose(1, 2).contiguous()


def _log_sum_exps(s, c, lse, counts, req, row):
    """The last rows' log-sum-exps into the caller's [request][layer][head][window]."""
    count = torch.from_numpy(counts.astype(np.int64)).to(row.device)[req]
    at = row - count + c["window"]
    keep = at >= 0
    s["lse"][req[keep], 0, :, at[keep]] = lse[req[keep], :, row[keep]]


def _prefill(s, c):
    req, row = _index(s["lens"], s["q"].device)
    n, longest = c["n_req"], int(s["lens"].max())
    q, k, v = (_padded(s[x], req, row, n, longest) for x in ("q", "k", "v"))
    out, lse = _attend(q, k, v, torch.arange(longest, device=q.device).expand(n, longest))
    if c["window"]:
        _log_sum_exps(s, c, lse, s["lens"], req, row)
    return out.transpose(1, 2)[req, row].half()


def _gathered(s, c, kv, table, layer):
    """(K, V) of every request, fp32, padded: [request][head][key][channel]."""
    t = table.clamp_min(0).long()
    if kv.dtype == torch.float16:
        x = kv[layer][t].float()  # [request][block][K|V][head][slot][channel]
    else:
        x = _codes(kv, c)[layer].view(torch.uint8)[t].view(torch.float8_e4m3fn).float() * _power_of_two(_exponents(kv, c)[layer][t])[..., None]
    x = x.permute(2, 0, 3, 1, 4, 5).flatten(3, 4)
    lens = torch.from_numpy(s["lens"].astype(np.int64)).to(t.device)
    past = torch.arange(x.shape[3], device=t.device) >= lens[:, None]
    return x[0].contiguous(), x[1].masked_fill(past[:, None, :, None], 0.0).contiguous()


def _chunk(s, c):
    kv, table = s["kv"], s["table"]
    req, row = _index(s["news"], table.device)
    lens, news = (torch.from_numpy(s[x].astype(np.int64)).to(table.device) for x in ("lens", "news"))
    at = (lens - news)[req] + row
    block, slot = table[req, at // BLOCK].long(), at % BLOCK
    new = torch.stack([s["k"], s["v"]], 1)  # [row][K|V][head][channel]
    if kv.dtype == torch.float16:
        kv[0, block, :, :, slot] = new
    else:
        codes, exps = _quantise(new.float())
        _codes(kv, c).view(torch.uint8)[0, block, :, :, slot] = codes.view(torch.uint8)
        _exponents(kv, c)[0, block, :, :, slot] = exps
    k, v = _gathered(s, c, kv, table, 0)
    longest = int(s["news"].max())
    q = _padded(s["q"], req, row, c["n_req"], longest)
    out, lse = _attend(q, k, v, (lens - news)[:, None] + torch.arange(longest, device=q.device))
    if c["window"]:
        _log_sum_exps(s, c, lse, s["news"], req, row)
    return out.transpose(1, 2)[req, row].half()


def _quantise_cache(s, c):
    req, row = _index(s["lens"], s["table"].device)
    block, block8, slot = s["table"][req, row // BLOCK].long(), s["table8"][req, row // BLOCK].long(), row % BLOCK
    codes, exps = _quantise(s["kv"][:, block, :, :, slot].float())  # [row][layer][K|V][head][channel]
    _codes(s["kv8"], c).view(torch.uint8)[:, block8, :, :, slot] = codes.view(torch.uint8)
    _exponents(s["kv8"], c)[:, block8, :, :, slot] = exps


def _decode8(s, c):
    """All layers at once: a layer is a request of its own."""
    n, n_l = s["q"].shape[:2]
    t = s["table"].clamp_min(0).long()
    codes = _codes(s["kv"], c).view(torch.uint8)[:, t].view(torch.float8_e4m3fn)  # [layer][request][block][K|V][head][slot][channel]
    x = codes.float() * _power_of_two(_exponents(s["kv"], c)[:, t])[..., None]
    x = x.permute(3, 1, 0, 4, 2, 5, 6).flatten(4, 5).flatten(1, 2)  # [K|V][request, layer][head][key][channel]
    lens = torch.from_numpy(s["lens"].astype(np.int64)).to(t.device).repeat_interleave(n_l)
    out, _ = _attend(s["q"].float().flatten(0, 1)[:, :, None], x[0].contiguous(), x[1].contiguous(), (lens - 1)[:, None])
    return out.reshape(s["q"].shape)


# --- the definition, in 64 bits ---------------------------------------------------------------------------------------


def exact(case, seed):
    """The definitions on the same inputs, request by request and head by head, in 64 bits; bytes of a cache as they are.
    None where that takes long."""
    if work(case)["flops"] > 6e12:
        return None
    s = prepare(case, seed)
    c = s["case"]
    h, hq, d = c["heads"], c["q_heads"], c["dim"]
    scale = 1.0 / math.sqrt(d)

    def softmax(q, k, v, first):
        """q [row][d] sees keys 0..first + row."""
        t = (q @ k.T.contiguous()) * scale
        t = t.masked_fill(torch.arange(k.shape[0], device=q.device) > first + torch.arange(q.shape[0], device=q.device)[:, None], -math.inf)
        return torch.softmax(t, -1) @ v, torch.logsumexp(t, -1)

    def codes_of(x):
        """8-bit values and exponents of rows x of fp64, by their definition: the nearest of the 8-bit numbers, ties to even."""
        top = x.abs().amax(-1)
        e = torch.full(top.shape, 8, dtype=torch.int64, device=x.device)
        for k in range(7, -16, -1):
            e = torch.where(top <= 448.0 * 2.0 ** k, k, e)
        y = x / torch.exp2(e.double())[..., None]
        _, p = torch.frexp(y.abs())
        step = torch.exp2((p - 1).clamp_min(-6).double() - 3)
        most = torch.where(e == 8, 240.0, 448.0)[..., None].double()
        return (torch.round(y / step) * step).clamp(-most, most), (e + 127).to(torch.uint8)

    def cached(kv, layer, r, n):
        """(K, V) of a request, [head][token][channel], fp64."""
        ids = s["table"][r, :-(-n // BLOCK)].long()
        if kv.dtype == torch.float16:
            x = kv[layer, ids].double()
        else:
            x = _codes(kv, c)[layer].view(torch.uint8)[ids].view(torch.float8_e4m3fn).double() * torch.exp2(_exponents(kv, c)[layer, ids].double() - 127)[..., None]
        x = x.permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n]
        return x[0], x[1]

    if c["kind"] == "quantise":
        codes, exps = _codes(s["kv8"], c).double(), _exponents(s["kv8"], c).clone()
        for r, n in enumerate(s["lens"].tolist()):
            ids, ids8 = (s[t][r, :-(-n // BLOCK)].long() for t in ("table", "table8"))
            v, e = codes_of(s["kv"][:, ids].double())
            v[:, -1, :, :, (n - 1) % BLOCK + 1:] = 0  # (behind the last token: as they were, zeros)
            e[:, -1, :, :, (n - 1) % BLOCK + 1:] = 0
            codes[:, ids8], exps[:, ids8] = v, e
        return {"codes": codes, "exponents": exps}
    if c["kind"] == "decode8":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
        for r, n in enumerate(s["lens"].tolist()):
            for layer in range(c["layers"]):
                k, v = cached(s["kv"], layer, r, n)
                t = (k * s["q"][r, layer].double()[:, None, :]).sum(-1) * scale
                out[r, layer] = (torch.softmax(t, -1)[..., None] * v).sum(1)
        return {"out": out}
    out = torch.empty((s["q"].shape[0], hq, d), dtype=torch.float64, device=s["q"].device)
    lse = None if s["lse"] is None else s["lse"].double()
    counts = s["lens"] if c["kind"] == "prefill" else s["news"]
    at = 0
    kv = s["kv"]
    for r, n in enumerate(counts.tolist()):
        q = s["q"][at:at + n].double()
        k, v = s["k"][at:at + n].double().transpose(0, 1), s["v"][at:at + n].double().transpose(0, 1)
        first = 0
        if c["kind"] == "chunk":
            first = int(s["lens"][r]) - n
            if kv.dtype == torch.uint8:
                (kc, ke), (vc, ve) = codes_of(k), codes_of(v)
                k, v = (x * torch.exp2(e.double() - 127)[..., None] for x, e in ((kc, ke), (vc, ve)))
            old_k, old_v = cached(kv, 0, r, first)
            k, v = torch.cat([old_k, k], 1), torch.cat([old_v, v], 1)
        for j in range(hq):
            o, e = softmax(q[:, j], k[j * h // hq], v[j * h // hq], first)
            out[at:at + n, j] = o
            if lse is not None:
                w = min(n, c["window"])
                lse[r, 0, j, c["window"] - w:] = e[n - w:]
        at += n
    found = {"out": out} if lse is None else {"out": out, "lse": lse}
    if c["kind"] == "chunk":
        found.update({"kv": None} if kv.dtype == torch.float16 else {"codes": None, "exponents": None})
    return found
