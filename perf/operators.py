"""Operators of a 4-bit paged key/value cache and of what feeds it, each in plain torch and as the framework's call.

    norm_rope   per-head RMSNorm of queries and keys with the position rotation in the same pass
    append      reserve pages, quantise new keys and values to 4 bits, read them back
    attention   attention of the newest tokens over the 4-bit cache
    fork        new rows from old ones: full pages shared, partly filled last pages copied, unused rows freed
    compact     live pages moved into the holes at the front of the pool, page tables rewritten

A page holds `page` tokens of one layer, for every KV head one block of page * (d + 8) bytes:
    K codes   [page][d / 2]                byte i of a token: code 2i (low four bits), code 2i + 1 (high four bits)
    V codes   [page / 2][d / 4][2][2]      token pair, group of 4 dimensions, token of the pair, byte as for K
    K params  [page][2] 16-bit             scale, offset of the token's row
    V params  [page][2] 16-bit
and a code c stands for offset + scale * c.  A row x is stored with offset = min(x), scale = (max(x) - min(x)) / 15
rounded to the storage type, c = (x - offset) / scale to the nearest whole number (ties to even) in 0 .. 15.
"""
import math

import torch

own = False

_T = {"f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one request's decode step, 64 query heads on 8 KV heads: latency
        {"name": "norm_rope decode 1", "op": "norm_rope", "type": "f16", "tokens": 1, "hq": 64, "hkv": 8, "d": 128,
         "rotary": 128, "halves": False, "far": 640},
        # a batch of 16 prompts of 1024 tokens, 40 heads, rotated in halves
        {"name": "norm_rope prompts", "op": "norm_rope", "type": "bf16", "tokens": 16 * 1024, "hq": 40, "hkv": 40,
         "d": 128, "rotary": 128, "halves": True, "far": 1024},
        # a decode step of 16 requests, 40 heads: one new token each
        {"name": "append decode 16", "op": "append", "type": "f16", "rows": 16, "new": 1, "held": 1039, "hkv": 40,
         "d": 128, "page": 64},
        # prompts of up to 1021 tokens for 8 requests, behind 7 tokens that are there already (an odd start)
        {"name": "append prompts", "op": "append", "type": "bf16", "rows": 8, "new": 1021, "held": 7, "hkv": 32,
         "d": 128, "page": 64},
        # one request, short context, grouped heads: latency
        {"name": "attention 1x513", "op": "attention", "type": "f16", "rows": 1, "queries": 1, "longest": 513,
         "hq": 64, "hkv": 8, "d": 128, "page": 64},
        # 16 requests of ragged lengths up to 1279, every head with its own keys
        {"name": "attention 16x1279", "op": "attention", "type": "f16", "rows": 16, "queries": 1, "longest": 1279,
         "hq": 40, "hkv": 40, "d": 128, "page": 64},
        # four drafted tokens verified at once for 8 requests
        {"name": "attention 8x4001 drafts", "op": "attention", "type": "bf16", "rows": 8, "queries": 4,
         "longest": 4001, "hq": 64, "hkv": 8, "d": 128, "page": 16},
        # long contexts, a full batch: bandwidth
        {"name": "attention 64x16384", "op": "attention", "type": "f16", "rows": 64, "queries": 1, "longest": 16384,
         "hq": 64, "hkv": 8, "d": 128, "page": 64},
        # a beam-search step of 4 beams on one small model: latency
        {"name": "fork 4 beams", "op": "fork", "type": "f16", "rows": 4, "kept": 3, "length": 77, "layers": 4,
         "hkv": 4, "d": 64, "page": 16},
        # 8 requests of 8 beams each that share their full pages, 32 layers of 32 heads
        {"name": "fork 64 beams", "op": "fork", "type": "f16", "rows": 64, "kept": 40, "length": 1070, "layers": 32,
         "hkv": 32, "d": 128, "page": 64},
        # a small pool after a few requests have ended
        {"name": "compact small", "op": "compact", "type": "f16", "rows": 5, "length": 130, "spare": 30, "moved": 9,
         "layers": 2, "hkv": 8, "d": 64, "page": 16},
        # 80 layers of 8 heads: a third of the live pages move
        {"name": "compact 80 layers", "op": "compact", "type": "bf16", "rows": 16, "length": 1000, "spare": 120,
         "moved": 85, "layers": 80, "hkv": 8, "d": 128, "page": 64},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind, t = rng.choice(("norm_rope", "append", "attention", "attention", "fork", "compact")), rng.choice(("f16", "bf16"))
    d = rng.choice((64, 128, 128))
    hkv = rng.choice((1, 2, 4, 5, 8, 8, 12, 32, 40))
    page = rng.choice((16, 32, 64, 64, 128))
    if kind == "norm_rope":
        g = rng.choice((1, 1, 2, 3, 4, 8))
        most = max(1, min(16384, 16384 * 80 * 128 // ((g + 1) * hkv * d)))
        return {"op": kind, "type": t, "tokens": _log(rng, 1, most), "hq": g * hkv, "hkv": hkv, "d": d,
                "rotary": rng.choice((d, d, d // 2)), "halves": rng.random() < 0.5, "far": rng.choice((640, 4096, 1000003))}
    if kind == "append":
        rows = _log(rng, 1, 64)
        new = rng.choice((1, _log(rng, 1, max(1, 8 * 1021 * 32 * 128 // (rows * hkv * d)))))
        return {"op": kind, "type": t, "rows": rows, "new": min(new, 8191), "held": _log(rng, 1, 2048) - 1, "hkv": hkv,
                "d": d, "page": page}
    if kind == "attention":
        g = rng.choice((1, 1, 2, 3, 4, 6, 8, 8, 16))
        rows = _log(rng, 1, 64)
        longest = _log(rng, 1, max(1, min(65536, 64 * 16384 * 8 * 128 // (rows * hkv * d))))
        queries = rng.choice((1, 1, 1, 2, 3, 5, 8))
        return {"op": kind, "type": t, "rows": rows, "queries": queries, "longest": longest, "hq": g * hkv, "hkv": hkv,
                "d": d, "page": page}
    layers = rng.choice((1, 3, 4, 32, 40))
    if kind == "fork":
        rows = _log(rng, 2, 64)
        return {"op": kind, "type": t, "rows": rows, "kept": rng.randint(1, rows), "length": _log(rng, 1, 1100),
                "layers": min(layers, 32), "hkv": min(hkv, 32), "d": d, "page": page}
    rows, length = _log(rng, 1, 24), _log(rng, 1, 1000)
    live = rows * -(-length // page)
    room = max(1, 250 * 80 * 8 * 64 * 136 // (layers * hkv * page * (d + 8)))     # pages that cost what the listed ones do
    live_most = max(1, room * 2 // 3)
    while live > live_most and rows > 1:
        rows -= 1
        live = rows * -(-length // page)
    if live > live_most:
        length = max(1, live_most // rows) * page - rng.randint(0, page - 1)
        live = rows * -(-length // page)
    moved = rng.randint(0, max(0, min(live, max(1, room // 3))))
    return {"op": kind, "type": t, "rows": rows, "length": length, "spare": moved + rng.randint(0, 9), "moved": moved,
            "layers": layers, "hkv": hkv, "d": d, "page": page}


# ------------------------------------------------------------------ sizes that a case implies
def _lengths(case):
    """Tokens held by each row: ragged from half the longest up, the second of three or more rows empty."""
    n, top = case["rows"], case["longest"]
    lens = [max(1, top - (top // 2) * b // max(1, n)) for b in range(n)]
    if n > 2:
        lens[1] = 0
    return lens


def _news(case):
    """New tokens of each row of an append: one each, or ragged down to two thirds."""
    return [max(1, case["new"] - (case["new"] // 3) * b // case["rows"]) for b in range(case["rows"])]


def _pages(tokens, page):
    return -(-tokens // page)


def work(case):
    op, d, hkv = case["op"], case["d"], case["hkv"]
    if op == "norm_rope":
        heads = case["hq"] + hkv
        n = case["tokens"] * heads * d
        return {"bytes": 4.0 * n + 4.0 * d + 4.0 * case["rotary"] + 4.0 * case["tokens"], "flops": 9.0 * n}
    if op == "append":
        n = sum(_news(case)) * hkv
        # 16-bit keys and values in, codes and params out; codes and params in again, 16-bit values out
        return {"bytes": n * 2.0 * (2 * d + 2 * (d // 2 + 4) + 2 * d) + 20.0 * sum(_news(case)), "flops": 12.0 * n * d}
    if op == "attention":
        keys, rows = sum(_lengths(case)), case["rows"] * case["queries"]
        return {"bytes": keys * hkv * (d + 8.0) + 4.0 * rows * case["hq"] * d + 4.0 * _pages(keys, case["page"]),
                "flops": 4.0 * keys * case["queries"] * case["hq"] * d}
    if op == "fork":
        tail = case["length"] % case["page"]
        copies = case["rows"] - case["kept"] if tail else 0
        table = 8.0 * case["rows"] * _pages(case["length"], case["page"])
        return {"bytes": 2.0 * copies * tail * hkv * (d + 8) * case["layers"] + table, "flops": 0.0}
    live = case["rows"] * _pages(case["length"], case["page"])
    return {"bytes": 2.0 * case["moved"] * case["page"] * hkv * (d + 8) * case["layers"] + 8.0 * live, "flops": 0.0}


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, t, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(t)


def _pool(gen, layers, n_pages, case):
    """Random pages with the statistics of quantised rows: codes over the whole range, scales of a few tenths."""
    hkv, d, page, t = case["hkv"], case["d"], case["page"], _T[case["type"]]
    block = page * (d + 8)
    pool = torch.randint(0, 256, (layers, n_pages, hkv, block), dtype=torch.uint8, device="cuda", generator=gen)
    if case["op"] == "attention" or case["op"] == "append":
        scale = torch.rand((layers, n_pages, hkv, 2 * page), generator=gen, device="cuda") * 0.2 + 0.2
        off = scale * (torch.randn(scale.shape, generator=gen, device="cuda") * 0.4 - 7.5)
        params = torch.stack([scale, off], -1).to(t).view(torch.uint8).reshape(layers, n_pages, hkv, -1)
        pool[..., page * d:] = params
    return pool.view(layers, n_pages, hkv * block)


def _table(gen, lens, page, extra_pages, max_pages):
    """Pages of all rows in random order out of the pool's; -1 where a row has none.  Returns the table and the pool's size."""
    counts = [_pages(n, page) for n in lens]
    n_pages = sum(counts) + extra_pages
    ids = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, c in enumerate(counts):
        table[r, :c] = ids[at:at + c]
        at += c
    return table, n_pages


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, op, d, hkv = _T[case["type"]], case["op"], case["d"], case["hkv"]
    s = dict(case)
    if op == "norm_rope":
        n, hq = case["tokens"], case["hq"]
        s["qkv"] = _normal(gen, (n, (hq + 2 * hkv) * d), t)          # the fused projection's output; v is not touched
        s["q_gain"] = (1 + torch.randn(d, generator=gen, device="cuda") * 0.1).to(t)
        s["k_gain"] = (1 + torch.randn(d, generator=gen, device="cuda") * 0.1).to(t)
        j = torch.arange(case["rotary"] // 2, device="cuda", dtype=torch.float64)
        s["turns"] = torch.exp(-math.log(10000.0) * 2 * j / case["rotary"]) / (2 * math.pi)
        s["positions"] = torch.randint(0, case["far"], (n,), generator=gen, device="cuda").to(torch.int32)
        return s
    page = case["page"]
    if op == "append":
        news, held = _news(case), case["held"]
        total = sum(news)
        lens = [held] * case["rows"]
        max_pages = _pages(held + max(news), page)
        s["table"], n_pages = _table(gen, lens, page, sum(_pages(held + n, page) - _pages(held, page) for n in news) + 3,
                                     max_pages)
        s["pool"] = _pool(gen, 1, n_pages, case)
        s["lens"], s["add"] = _int(lens), _int(news)
        s["rows_of"] = torch.repeat_interleave(torch.arange(case["rows"], device="cuda"), s["add"].long()).to(torch.int32)
        first = torch.cumsum(s["add"], 0) - s["add"]
        s["positions"] = (torch.arange(total, device="cuda") - first[s["rows_of"].long()] + held).to(torch.int32)
        s["k"], s["v"] = _normal(gen, (total, hkv, d), t), _normal(gen, (total, hkv, d), t)
        return s
    if op == "attention":
        lens = _lengths(case)
        s["table"], n_pages = _table(gen, lens, page, 5, _pages(case["longest"], page) + 1)
        s["pool"] = _pool(gen, 1, n_pages, case)
        s["lens"] = _int(lens)
        s["q"] = _normal(gen, (case["rows"], case["queries"], case["hq"], d), t)
        return s
    lens = [case["length"]] * case["rows"]
    s["lens"] = _int(lens)
    per_row = _pages(case["length"], page)
    if op == "fork":
        # beams of one request (groups of 8 rows) share their full pages; each has its own last page
        rows, full = case["rows"], case["length"] // page
        groups, tails = _pages(rows, 8), per_row - full
        n_pages = groups * full + rows * tails + rows + 2
        ids = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.full((rows, per_row + 2), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :full] = ids[:groups * full].view(groups, full).repeat_interleave(8, 0)[:rows]
        s["table"][:, full:per_row] = ids[groups * full:groups * full + rows * tails].view(rows, tails)
        kept = torch.randperm(case["rows"], generator=gen, device="cuda")[:case["kept"]]
        more = kept[torch.randint(0, case["kept"], (case["rows"] - case["kept"],), generator=gen, device="cuda")]
        mixed = torch.cat([kept, more])
        s["source"] = mixed[torch.randperm(case["rows"], generator=gen, device="cuda")].to(torch.int32)
    else:
        live = case["rows"] * per_row
        n_pages = live + case["spare"]
        front = torch.randperm(live, generator=gen, device="cuda")[case["moved"]:]
        back = live + torch.randperm(case["spare"], generator=gen, device="cuda")[:case["moved"]]
        ids = torch.cat([front, back])
        ids = ids[torch.randperm(live, generator=gen, device="cuda")]
        s["table"] = torch.full((case["rows"], per_row + 1), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :per_row] = ids.view(case["rows"], per_row).to(torch.int32)
    s["pool"] = _pool(gen, case["layers"], n_pages, case)
    return s


# ------------------------------------------------------------------ plain forms
def _rope_plain(x, gain, s):
    rot, t = s["rotary"], x.dtype
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gain.float()
    turn = s["positions"].double()[:, None] * s["turns"]
    angle = (turn - torch.floor(turn)) * (2 * math.pi)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if s["halves"]:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., rot:]], -1)
    return y.to(t)


def _split(s):
    n, hq, hkv, d = s["tokens"], s["hq"], s["hkv"], s["d"]
    q = s["qkv"][:, :hq * d].unflatten(1, (hq, d))
    k = s["qkv"][:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d))
    return q, k


def _quantise_plain(x):
    """(codes, scale, offset) of rows, in 64 bits: a code next to a border must not depend on a rounding."""
    x64 = x.double()
    low, high = x64.amin(-1, keepdim=True), x64.amax(-1, keepdim=True)
    scale = ((high - low) / 15).to(x.dtype).double()
    code = torch.where(scale > 0, torch.round((x64 - low) / scale), torch.zeros_like(x64)).clamp(0, 15)
    return code.to(torch.uint8), scale.to(x.dtype), low.to(x.dtype)


def _value_plain(codes, scale, off):
    return codes.float() * scale.float() + off.float()


def _reserve_plain(s):
    table, lens, add, page, n_pages = s["table"].long(), s["lens"].long(), s["add"].long(), s["page"], s["pool"].shape[1]
    col = torch.arange(table.shape[1], device="cuda")
    have, want = (lens + page - 1) // page, (lens + add + page - 1) // page
    used = torch.where(col < have[:, None], table, torch.full_like(table, n_pages))
    live = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda").index_fill(0, used.flatten(), 1)[:n_pages]
    free = torch.argsort(live, stable=True)
    end = torch.cumsum(want - have, 0)
    fresh = free[(end[:, None] - want[:, None] + col).clamp(0, n_pages - 1)]
    fits = (end <= n_pages - live.sum()) & (want <= table.shape[1])
    new = fits[:, None] & (col >= have[:, None]) & (col < want[:, None])
    return torch.where(new, fresh, table).to(torch.int32), torch.where(fits, lens + add, lens).to(torch.int32), (~fits).sum()


def _bytes_of(page, d, hkv):
    """Index ranges of a page's parts, as a view [hkv][parts]."""
    return (0, page * d // 2), (page * d // 2, page * d), (page * d, page * (d + 4)), (page * (d + 4), page * (d + 8))


def _unpack_plain(pool, s, t):
    """Codes and params of all pages of one layer: K, V codes [pages][hkv][page][d], params [pages][hkv][page][2]."""
    page, d, hkv = s["page"], s["d"], s["hkv"]
    p = pool.view(pool.shape[0], hkv, page * (d + 8))
    (k0, k1), (v0, v1), (a0, a1), (b0, b1) = _bytes_of(page, d, hkv)
    kb = p[..., k0:k1].reshape(-1, hkv, page, d // 2)
    vb = p[..., v0:v1].reshape(-1, hkv, page // 2, d // 4, 2, 2).transpose(-3, -2).reshape(-1, hkv, page, d // 2)
    codes = [torch.stack([b & 15, b >> 4], -1).flatten(-2) for b in (kb, vb)]
    params = [p[..., i:j].contiguous().view(t).view(-1, hkv, page, 2) for i, j in ((a0, a1), (b0, b1))]
    return codes, params


def _append_plain(s):
    page, d, hkv, t = s["page"], s["d"], s["hkv"], s["k"].dtype
    table, lens, refused = _reserve_plain(s)
    pos = s["positions"].long()
    at, slot = table[s["rows_of"].long(), pos // page].long(), pos % page
    pool = s["pool"][0].view(-1, hkv, page * (d + 8))
    for x, part, ppart in ((s["k"], 0, 2), (s["v"], 1, 3)):     # keys, then values
        codes, scale, off = _quantise_plain(x)
        nibbles = codes[..., 0::2] | (codes[..., 1::2] << 4)
        i, j = _bytes_of(page, d, hkv)[part]
        if part == 0:
            pool[..., i:j].view(-1, hkv, page, d // 2)[at, :, slot] = nibbles
        else:
            pool[..., i:j].view(-1, hkv, page // 2, d // 4, 2, 2)[at, :, slot // 2, :, slot % 2] = \
                nibbles.view(-1, hkv, d // 4, 2)
        i, j = _bytes_of(page, d, hkv)[ppart]
        pool[..., i:j].view(-1, hkv, page, 4)[at, :, slot] = torch.cat([scale, off], -1).contiguous().view(torch.uint8)
    codes, params = _unpack_plain(s["pool"][0], s, t)
    k, v = (_value_plain(c[at, :, slot], p[at, :, slot][..., :1], p[at, :, slot][..., 1:]).to(t) for c, p in zip(codes, params))
    return {"k": k, "v": v, "table": table, "lens": lens, "refused": refused}


def _attention_plain(s):
    q, page, d, hkv = s["q"], s["page"], s["d"], s["hkv"]
    b, n, hq = q.shape[:3]
    g = hq // hkv
    codes, params = _unpack_plain(s["pool"][0], s, q.dtype)
    at = s["table"].long().clamp(min=0)
    k, v = (_value_plain(c[at], p[at][..., :1], p[at][..., 1:]).transpose(1, 2).flatten(2, 3) for c, p in zip(codes, params))
    t = k.shape[2]
    qf = q.float().view(b, n, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, n * g, d)
    score = (qf @ k.transpose(-1, -2)) / math.sqrt(d)
    limit = s["lens"][:, None] - (n - 1) + torch.arange(n, device="cuda", dtype=torch.int32)       # [b][n]
    seen = torch.arange(t, device="cuda") < limit[:, :, None]
    seen = seen[:, None, :, None].expand(b, hkv, n, g, t).reshape(b, hkv, n * g, t)
    score = torch.where(seen, score, torch.full_like(score, -math.inf))
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    w = torch.exp(score - top)
    total = w.sum(-1, keepdim=True)
    o = (w @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.view(b, hkv, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, hq, d).to(q.dtype)


def _copy_plain(s, src, dst, tokens, on):
    """Pages src -> dst of every layer where `on`, the filled groups of 16 tokens of each."""
    page, d, hkv = s["page"], s["d"], s["hkv"]
    pool = s["pool"].view(s["pool"].shape[0], s["pool"].shape[1], hkv, page * (d + 8))
    byte = torch.arange(page * (d + 8), device="cuda")
    in_k, in_v = byte < page * d // 2, byte < page * d
    token = torch.where(in_k, byte // (d // 2), torch.where(in_v, (byte - page * d // 2) // d * 2, (byte - page * d) // 4 % page))
    filled = (token // 16 * 16)[None, :] < tokens[:, None]                                            # [moves][bytes]
    filled = (filled & on[:, None])[None, :, None, :]
    pool[:, dst] = torch.where(filled, pool[:, src], pool[:, dst])


def _fork_plain(s):
    table, lens, src, page = s["table"].long(), s["lens"].long(), s["source"].long(), s["page"]
    rows, n_pages = table.shape[0], s["pool"].shape[1]
    me = torch.arange(rows, device="cuda")
    col = torch.arange(table.shape[1], device="cuda")
    have = (lens + page - 1) // page
    used = torch.where(col < have[:, None], table, torch.full_like(table, n_pages))
    live = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda").index_fill(0, used.flatten(), 1)[:n_pages]
    free = torch.argsort(live, stable=True)
    taken = src >= 0
    from_ = src.clamp(min=0)
    n = torch.where(taken, lens[from_], torch.zeros_like(lens[from_]))
    # the row that keeps the partly filled page: the source itself where it stays, else the first of its heirs
    stays = (src == me)[from_] & taken
    heirs = (src[None, :] == src[:, None])
    first = torch.where(heirs, me[None, :], torch.full_like(heirs, rows, dtype=torch.int64)).amin(1)
    keeps = torch.where(stays, from_ == me, first == me)
    needs = taken & (n % page > 0) & ~keeps
    rank = torch.cumsum(needs.long(), 0) - 1
    fits = ~needs | (rank < n_pages - live.sum())
    copies = needs & fits
    fresh = free[rank.clamp(0, n_pages - 1)]
    last = (n // page).clamp(max=table.shape[1] - 1)
    old = table[from_, last].clamp(min=0)
    spare = free[(n_pages - live.sum() - 1).clamp(min=0)]     # a row that copies nothing names a page that is free
    _copy_plain(s, torch.where(copies, old, spare), torch.where(copies, fresh, spare), n % page, copies)
    n = torch.where(fits, n, torch.zeros_like(n))
    out = torch.where(col < ((n + page - 1) // page)[:, None], table[from_], torch.full_like(table, -1))
    out = torch.where(copies[:, None] & (col == last[:, None]), fresh[:, None], out)
    return {"pool": s["pool"], "table": out.to(torch.int32), "lens": n.to(torch.int32), "refused": (~fits).sum()}


def _compact_plain(s):
    table, lens, page = s["table"].long(), s["lens"].long(), s["page"]
    n_pages = s["pool"].shape[1]
    col = torch.arange(table.shape[1], device="cuda")
    have = (lens + page - 1) // page
    held = (lens[:, None] - col * page).clamp(0, page)                                                # tokens on each page
    used = torch.where(col < have[:, None], table, torch.full_like(table, n_pages))
    fill = torch.zeros(n_pages + 1, dtype=torch.int64, device="cuda").scatter_reduce(0, used.flatten(), held.flatten(), "amax")[:n_pages]
    live = fill > 0
    count = live.sum()
    ids = torch.arange(n_pages, device="cuda")
    holes = torch.argsort((live | (ids >= count)).int(), stable=True)             # free ids below the count come first
    moves = live & (ids >= count)
    rank = (torch.cumsum(moves.long(), 0) - 1).clamp(min=0)
    new = torch.where(moves, holes[rank], ids)
    src = torch.argsort((~moves).int(), stable=True)[:s["moved"]]                 # the moving pages first
    _copy_plain(s, src, new[src], fill[src], moves[src])
    out = torch.where(col < have[:, None], new[table.clamp(min=0)], torch.full_like(table, -1))
    return {"pool": s["pool"], "table": out.to(torch.int32), "live": count}


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["op"]
    if not own:
        if op == "norm_rope":
            q, k = _split(s)
            return {"q": _rope_plain(q, s["q_gain"], s), "k": _rope_plain(k, s["k_gain"], s)}
        return {"append": _append_plain, "attention": _attention_plain, "fork": _fork_plain, "compact": _compact_plain}[op](s)
    from paper_2605_25655_b200 import thinfer
    if op == "norm_rope":
        q, k = _split(s)
        q, k = thinfer.op_qk_norm_rope(q, k, s["q_gain"], s["k_gain"], 1e-6, s["turns"], s["positions"], halves=s["halves"])
        return {"q": q, "k": k}
    if op == "append":
        pool = s["pool"][0]
        lens, refused = thinfer.op_kv4_reserve(s["table"], s["lens"], s["add"], pool.shape[0], s["page"])
        thinfer.op_kv4_append(pool, s["table"], s["k"], s["v"], s["rows_of"], s["positions"], s["page"])
        k, v = thinfer.op_kv4_read(pool, s["table"], s["rows_of"], s["positions"], s["page"], s["d"], s["k"].dtype)
        return {"k": k, "v": v, "table": s["table"], "lens": lens, "refused": refused.view(())}
    if op == "attention":
        return thinfer.op_kv4_attention(s["q"], s["pool"][0], s["table"], s["lens"], s["page"])
    if op == "fork":
        table, lens, refused = thinfer.op_kv4_fork(s["pool"], s["table"], s["lens"], s["source"], s["page"], s["d"])
        return {"pool": s["pool"], "table": table, "lens": lens, "refused": refused.view(())}
    table, live = thinfer.op_kv4_compact(s["pool"], s["table"], s["lens"], s["page"], s["d"])
    return {"pool": s["pool"], "table": table, "live": live.view(())}


# ------------------------------------------------------------------ the definition in 64 bits
def _row_of_cache(s, row, n, which):
    """Keys (0) or values (1) of the first n tokens of a row, [n][hkv][d], byte by byte from the page layout."""
    page, d, hkv = s["page"], s["d"], s["hkv"]
    t = torch.arange(n, device="cuda")
    block = page * (d + 8)
    base = (s["table"][row].long()[t // page] * hkv * block)[:, None, None] + (torch.arange(hkv, device="cuda") * block)[:, None]
    j, slot = torch.arange(d, device="cuda"), (t % page)[:, None, None]
    if which == 0:
        at = slot * (d // 2) + j // 2
    else:
        at = page * d // 2 + slot // 2 * d + j // 4 * 4 + slot % 2 * 2 + j % 4 // 2
    flat = s["pool"].flatten()
    code = (flat[base + at].long() >> (4 * (j % 2))) & 15
    par = page * d + which * page * 4 + slot * 4
    half = (flat[base + par + torch.arange(4, device="cuda")]).contiguous().view(_T[s["type"]]).double()     # scale, offset
    return half[..., 1:] + half[..., :1] * code


def exact(case, seed):
    s = prepare(case, seed)
    op, d, hkv = case["op"], case["d"], case["hkv"]
    if op == "norm_rope":
        got = {}
        for name, x, gain in zip(("q", "k"), _split(s), (s["q_gain"], s["k_gain"])):
            x = x.double()
            x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.double()
            angle = 2 * math.pi * torch.remainder(s["positions"].double()[:, None, None] * s["turns"], 1.0)
            rot = case["rotary"]
            i = torch.arange(rot // 2, device="cuda")
            first, second = (i, i + rot // 2) if case["halves"] else (2 * i, 2 * i + 1)
            z = torch.polar(torch.ones_like(angle), angle) * torch.complex(x[..., first], x[..., second])
            y = x.clone()
            y[..., first], y[..., second] = z.real, z.imag
            got[name] = y
        return got
    if op == "append":
        got = {"table": None, "lens": None, "refused": None}
        for name in ("k", "v"):
            x = s[name].double()
            low = x.min(-1, keepdim=True).values
            step = ((x.max(-1, keepdim=True).values - low) / 15).to(s[name].dtype).double()
            c = torch.floor(torch.where(step > 0, (x - low) / step, 0 * x) + 0.5)
            tie = torch.where(step > 0, ((x - low) / step) % 1 == 0.5, False)
            c = torch.where(tie & (c % 2 == 1), c - 1, c)
            got[name] = low + step * c.clamp(max=15)
        return got
    if op == "attention":
        if sum(_lengths(case)) * hkv * d > 1.5e9:
            return None
        n, g = case["queries"], case["hq"] // hkv
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for row, held in enumerate(_lengths(case)):
            if held == 0:
                continue
            k, v = _row_of_cache(s, row, held, 0), _row_of_cache(s, row, held, 1)
            for i in range(n):
                m = held - (n - 1 - i)
                if m <= 0:
                    continue
                q = s["q"][row, i].double().view(hkv, g, d)
                p = torch.softmax(torch.einsum("hgd,thd->hgt", q, k[:m]) / math.sqrt(d), -1)
                out[row, i] = torch.einsum("hgt,thd->hgd", p, v[:m]).reshape(-1, d)
        return out
    return None
