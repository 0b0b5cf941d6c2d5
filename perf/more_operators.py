"""Operators that cut a decode step's weight bytes and get several tokens out of one, in plain torch and as the framework's calls.

    quantise    16-bit weights to 4 bits with a scale and a zero point per row and group of columns, and back
    linear      products of few token rows with such weights
    probs       probabilities of FP32 logits at a temperature per row (not positive: all of it on the lowest largest index)
    verify      which drafted tokens stay, given both models' probabilities and uniform random numbers, and the token behind them

Packed weights of n rows and k columns in groups of G: three regions of bytes.  Rows come in tiles of 16, columns in blocks
of 128 (both padded with zeros); row 8 i + g of a tile, column 32 q + 8 t + 4 s + 2 b + e of a block:
    codes    [tile][block][q / 2][g][t][q % 2][s][e][b]     byte: row g's code in the low, row 8 + g's in the high four bits
    scales   [tile][block][g][group of the block][i]        16-bit
    zeros    [tile][block][g][group of the block]           byte as for the codes
and a code c stands for scale * (c - zero).
"""
import math

import torch

own = False

_T = {"f16": torch.float16, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # weights of an odd small layer, once
        {"name": "quantise small", "op": "quantise", "type": "bf16", "n": 1001, "k": 1000, "group": 32},
        # the gate projection of the largest configuration
        {"name": "quantise gate", "op": "quantise", "type": "f16", "n": 28672, "k": 8192, "group": 128},
        # one request's output projection, 32 heads: latency
        {"name": "linear 1x4096x4096", "op": "linear", "type": "f16", "rows": 1, "n": 4096, "k": 4096, "group": 128, "fp32": False},
        # a batch of four, the gate projection of the largest configuration: bandwidth
        {"name": "linear 4x28672x8192", "op": "linear", "type": "f16", "rows": 4, "n": 28672, "k": 8192, "group": 128, "fp32": False},
        # a full batch of 16 on the down projection of the 40-head model
        {"name": "linear 16x5120x13824", "op": "linear", "type": "bf16", "rows": 16, "n": 5120, "k": 13824, "group": 64, "fp32": False},
        # the vocabulary projection of 4 requests with 5 drafted tokens each and one more: FP32 logits
        {"name": "linear head 24", "op": "linear", "type": "f16", "rows": 24, "n": 32000, "k": 8192, "group": 32, "fp32": True},
        # the most rows a decode step has
        {"name": "linear 64x28672x8192", "op": "linear", "type": "bf16", "rows": 64, "n": 28672, "k": 8192, "group": 128, "fp32": False},
        # one request's next token: latency
        {"name": "probs 1x32000", "op": "probs", "rows": 1, "vocab": 32000},
        # 64 requests, four drafts and one more each, a large vocabulary: bandwidth
        {"name": "probs 320x128000", "op": "probs", "rows": 320, "vocab": 128000},
        # one request, four drafts: latency
        {"name": "verify 1x4", "op": "verify", "batch": 1, "drafts": 4, "vocab": 32000, "sure": False, "ragged": False},
        # drafts looked up in the prompt, which have no probabilities; up to 7 a request, an odd vocabulary
        {"name": "verify 16x7 lookup", "op": "verify", "batch": 16, "drafts": 7, "vocab": 100003, "sure": True, "ragged": True},
        # 64 requests with four drafts each, a large vocabulary
        {"name": "verify 64x4", "op": "verify", "batch": 64, "drafts": 4, "vocab": 128000, "sure": False, "ragged": False},
    ]


def _log(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("quantise", "linear", "linear", "linear", "probs", "verify", "verify"))
    t = rng.choice(("f16", "bf16"))
    if kind in ("quantise", "linear"):
        most = 28672 * 8192
        k = rng.choice((4096, 5120, 8192, 11008, 13824, 28672, 8 * _log(rng, 4, 3584)))
        n = rng.choice((1024, 4096, 8192, _log(rng, 16, 32000), _log(rng, 16, 32000)))
        n = max(1, min(n, most // k))
        case = {"op": kind, "type": t, "n": n, "k": k, "group": rng.choice((32, 64, 128, 128))}
        return case if kind == "quantise" else {**case, "rows": _log(rng, 1, 64), "fp32": rng.random() < 0.3}
    vocab = rng.choice((32000, 128000, _log(rng, 2, 160000), _log(rng, 1000, 160000)))
    if kind == "probs":
        return {"op": kind, "rows": _log(rng, 1, max(1, min(1024, 320 * 128000 // vocab))), "vocab": vocab}
    return {"op": kind, "batch": _log(rng, 1, max(1, min(256, 64 * 128000 // vocab))), "drafts": rng.randint(0, 8) if vocab <= 32000 else rng.randint(0, 4),
            "vocab": vocab, "sure": rng.random() < 0.3, "ragged": rng.random() < 0.5}


# ------------------------------------------------------------------ sizes that a case implies
def _up(a, b):
    return -(-a // b)


def _packed_sizes(n, k, group):
    """Tiles, blocks, groups of a block; bytes of codes, scales, zeros."""
    tiles, blocks, per = _up(n, 16), _up(k, 128), 128 // group
    return (tiles, blocks, per), (tiles * blocks * 1024, tiles * blocks * per * 32, tiles * blocks * per * 8)


def work(case):
    op = case["op"]
    if op in ("quantise", "linear"):
        n, k = case["n"], case["k"]
        packed = n * k / 2.0 + n * _up(k, case["group"]) * 2.5
        if op == "quantise":
            return {"bytes": 4.0 * n * k + 2.0 * packed, "flops": 8.0 * n * k}
        rows = case["rows"]
        return {"bytes": packed + 2.0 * rows * k + (4.0 if case["fp32"] else 2.0) * rows * n, "flops": 2.0 * rows * n * k}
    if op == "probs":
        return {"bytes": 8.0 * case["rows"] * case["vocab"], "flops": 6.0 * case["rows"] * case["vocab"]}
    # a row of the target's probabilities for each request, and one of the draft's for the three quarters that reject one
    n = case["batch"] * case["vocab"]
    return {"bytes": (4.0 if case["sure"] or case["drafts"] == 0 else 7.0) * n, "flops": 3.0 * n}


# ------------------------------------------------------------------ inputs
def _pack(codes, scales, zeros, group):
    """codes uint8 [n][k], scales 16-bit [n][groups], zeros uint8 [n][groups] -> the packed bytes."""
    n, k = codes.shape
    (tiles, blocks, per), _ = _packed_sizes(n, k, group)

    def padded(x, cols):
        return torch.nn.functional.pad(x, (0, cols - x.shape[1], 0, tiles * 16 - n))

    c = padded(codes, blocks * 128).view(tiles, 2, 8, blocks, 2, 2, 4, 2, 2, 2)            # tile i g block q/2 q%2 t s b e
    c = c.permute(0, 3, 4, 2, 6, 5, 7, 9, 8, 1)                                            # tile block q/2 g t q%2 s e b i
    c = c[..., 0] | (c[..., 1] << 4)
    s = padded(scales.view(torch.int16), blocks * per).view(tiles, 2, 8, blocks, per).permute(0, 3, 2, 4, 1).contiguous()
    z = padded(zeros, blocks * per).view(tiles, 2, 8, blocks, per).permute(0, 3, 2, 4, 1)
    z = z[..., 0] | (z[..., 1] << 4)
    return torch.cat([c.reshape(-1), s.view(torch.uint8).reshape(-1), z.reshape(-1)])


def _normal(gen, shape, t, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(t)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    op = case["op"]
    if op == "quantise":
        s["w"] = _normal(gen, (case["n"], case["k"]), _T[case["type"]], 0.02)
    elif op == "linear":
        n, k, group = case["n"], case["k"], case["group"]
        shape = (n, _up(k, group))
        codes = torch.randint(0, 16, (n, k), dtype=torch.uint8, device="cuda", generator=gen)
        scales = (0.004 + 0.004 * torch.rand(shape, generator=gen, device="cuda")).to(_T[case["type"]])
        zeros = torch.randint(5, 11, shape, dtype=torch.uint8, device="cuda", generator=gen)
        s["packed"] = _pack(codes, scales, zeros, group)
        s["x"] = _normal(gen, (case["rows"], k), _T[case["type"]])
    elif op == "probs":
        s["logits"] = torch.randn((case["rows"], case["vocab"]), generator=gen, device="cuda") * 4
        warm = 0.5 + torch.rand(case["rows"], generator=gen, device="cuda")
        s["temperature"] = torch.where(torch.arange(case["rows"], device="cuda") % 8 == 5, torch.zeros_like(warm), warm)   # some greedy
    else:
        b, n, v = case["batch"], case["drafts"], case["vocab"]
        logits = torch.randn((b, n + 1, v), generator=gen, device="cuda") * (6 if case["sure"] else 3)
        s["p"] = torch.softmax(logits, -1)
        near = logits[:, :n] + torch.randn((b, n, v), generator=gen, device="cuda") * 0.8      # a draft that agrees four times in five
        s["q"] = None if case["sure"] or n == 0 else torch.softmax(near, -1)
        # drafts drawn from the draft's probabilities, or the likeliest token of a model like the target
        noise = 0 if case["sure"] else -torch.log(-torch.log(torch.rand((b, n, v), generator=gen, device="cuda").clamp(1e-20, 1 - 1e-7)))
        s["tokens"] = (near + noise).argmax(-1).to(torch.int32)
        s["uniforms"] = torch.rand((b, n + 1), generator=gen, device="cuda")
        s["counts"] = torch.randint(0, n + 1, (b,), generator=gen, device="cuda").to(torch.int32) if case["ragged"] else None
    return s


# ------------------------------------------------------------------ plain forms
def _quantise_plain(w, group):
    """(codes, scales, zeros) of rows, in 64 bits: a code next to a border must not depend on a rounding."""
    n, k = w.shape
    x = torch.nn.functional.pad(w, (0, _up(k, group) * group - k)).view(n, -1, group).double()
    low, high = x.amin(-1).clamp(max=0), x.amax(-1).clamp(min=0)
    scale = ((high - low) / 15).to(w.dtype)
    by = torch.where(scale > 0, scale.double(), torch.full_like(low, math.inf))
    zero = torch.round(-low / by).clamp(0, 15)
    code = (torch.round(x / by[..., None]) + zero[..., None]).clamp(0, 15)
    return code, scale, zero


def _unpack_plain(packed, n, k, group, t):
    """scale * (code - zero) of all weights, FP32 [n][k]."""
    (tiles, blocks, per), (nc, ns, nz) = _packed_sizes(n, k, group)
    c = packed[:nc].view(tiles, blocks, 2, 8, 4, 2, 2, 2, 2)
    s = packed[nc:nc + ns].view(t).view(tiles, blocks, 8, per, 2).float()
    z = packed[nc + ns:nc + ns + nz].view(tiles, blocks, 8, per)
    c = torch.stack([c & 15, c >> 4], -1).permute(0, 9, 3, 1, 2, 5, 4, 6, 8, 7).reshape(tiles, 2, 8, blocks, per, group)
    z = torch.stack([z & 15, z >> 4], -1).permute(0, 4, 2, 1, 3)
    w = (c.float() - z.float()[..., None]) * s.permute(0, 4, 2, 1, 3)[..., None]
    return w.reshape(tiles * 16, blocks * 128)[:n, :k]


def _probs_plain(s):
    x, temp = s["logits"], s["temperature"][:, None]
    w = torch.exp((x - x.amax(-1, keepdim=True)) / torch.where(temp > 0, temp, torch.ones_like(temp)))
    w = w / w.sum(-1, keepdim=True)
    one = (torch.arange(x.shape[1], device="cuda") == x.argmax(-1, keepdim=True)).float()
    return torch.where(temp > 0, w, one)


def _verify_plain(s):
    p, q, tokens, u, n = s["p"], s["q"], s["tokens"].long(), s["uniforms"].double(), s["drafts"]
    b, v = p.shape[0], p.shape[2]
    at = torch.arange(n + 1, device="cuda")
    count = torch.full((b,), n, device="cuda") if s["counts"] is None else s["counts"].long()
    pt = p[:, :n].gather(2, tokens[..., None])[..., 0].double()
    qt = torch.ones_like(pt) if q is None else q.gather(2, tokens[..., None])[..., 0].double()
    stays = (u[:, :n] * qt < pt) & (at[:n] < count[:, None])
    stays = torch.cat([stays, torch.zeros((b, 1), dtype=torch.bool, device="cuda")], 1)
    kept = torch.cumprod(stays.long(), 1).sum(1)
    row = torch.arange(b, device="cuda")
    r = p[row, kept].double()
    if n > 0:
        last = kept.clamp(max=n - 1)
        if q is None:
            other = (torch.arange(v, device="cuda") == tokens[row, last][:, None]).double()
        else:
            other = q[row, last].double()
        left = (r - other).clamp(min=0)
        r = torch.where(((kept < count) & (left.sum(-1) > 0))[:, None], left, r)
    total = torch.cumsum(r, -1)
    token = (total <= u[:, n:] * total[:, -1:]).sum(-1)
    padded = torch.cat([tokens, torch.zeros_like(tokens[:, :1]) if n else torch.zeros((b, 1), dtype=torch.int64, device="cuda")], 1)
    out = torch.where(at < kept[:, None], padded, torch.where(at == kept[:, None], token[:, None], torch.full_like(padded, -1)))
    return {"tokens": out.to(torch.int32), "accepted": kept.to(torch.int32)}


# ------------------------------------------------------------------ one pass
def run(s):
    op = s["op"]
    if not own:
        if op == "quantise":
            code, scale, zero = _quantise_plain(s["w"], s["group"])
            back = ((code - zero[..., None]).float() * scale.float()[..., None]).flatten(1)[:, :s["k"]]
            return back.to(s["w"].dtype)
        if op == "linear":
            y = s["x"].float() @ _unpack_plain(s["packed"], s["n"], s["k"], s["group"], s["x"].dtype).T
            return y if s["fp32"] else y.to(s["x"].dtype)
        return _probs_plain(s) if op == "probs" else _verify_plain(s)
    from paper_2605_25655_b200 import thinfer
    if op == "quantise":
        packed = thinfer.op_w4_quantize(s["w"], s["group"])
        return thinfer.op_w4_read(packed, s["n"], s["k"], s["group"], s["w"].dtype)
    if op == "linear":
        return thinfer.op_w4_linear(s["x"], s["packed"], s["n"], s["group"], out_fp32=s["fp32"])
    if op == "probs":
        return thinfer.op_token_probs(s["logits"], s["temperature"])
    tokens, accepted = thinfer.op_verify_drafts(s["p"], s["q"], s["tokens"], s["uniforms"], s["counts"])
    return {"tokens": tokens, "accepted": accepted}


# ------------------------------------------------------------------ the definition in 64 bits
def _weights_of_rows(s, rows):
    """scale * (code - zero) of some rows, FP64, byte by byte from the layout."""
    n, k, group = s["n"], s["k"], s["group"]
    (_, blocks, per), (nc, ns, _) = _packed_sizes(n, k, group)
    col = torch.arange(k, device="cuda")
    tile, i, g = (rows // 16)[:, None], (rows % 16 // 8)[:, None], (rows % 8)[:, None]
    block, c = col // 128, col % 128
    q, t, st, b, e = c // 32, c % 32 // 8, c % 8 // 4, c % 4 // 2, c % 2
    at = (tile * blocks + block) * 1024 + q // 2 * 512 + g * 64 + t * 16 + q % 2 * 8 + st * 4 + e * 2 + b
    flat = s["packed"]
    code = flat[at].long() >> (4 * i) & 15
    pair = ((tile * blocks + block) * 8 + g) * per + c // group
    zero = flat[nc + ns + pair].long() >> (4 * i) & 15
    scale = flat[nc:nc + ns].view(s["x"].dtype)[2 * pair + i].double()
    return scale * (code - zero)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantise":
        w, group = s["w"].double(), case["group"]
        parts = []
        for part in torch.split(w, group, 1):
            low, high = part.min(1).values.clamp(max=0), part.max(1).values.clamp(min=0)
            step = ((high - low) / 15).to(s["w"].dtype).double()[:, None]
            zero = torch.clamp(torch.round(torch.nan_to_num(-low[:, None] / step)), 0, 15)
            code = torch.clamp(torch.round(torch.nan_to_num(part / step)) + zero, 0, 15)
            parts.append(step * (code - zero))
        return torch.cat(parts, 1)
    if op == "linear":
        x = s["x"].double()
        return torch.cat([x @ _weights_of_rows(s, rows).T for rows in torch.arange(case["n"], device="cuda").split(2048)], 1)
    if op == "probs":
        x, temp = s["logits"].double(), s["temperature"].double()
        y = torch.softmax(x / torch.where(temp > 0, temp, 1.0)[:, None], -1)
        greedy = torch.zeros_like(y).scatter_(1, x.argmax(1, keepdim=True), 1.0)
        return torch.where((temp > 0)[:, None], y, greedy)
    return None
