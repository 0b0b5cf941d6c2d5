"""Float64 definitions of the per-head norm with rotation and of the 4-bit paged cache (numpy, plain loops).

Independent of csrc/: a page is taken apart byte by byte from its documented layout, page tables are Python lists, and
nothing is done in a way chosen for speed.  `dt` is the storage type: numpy float16, or "bf16" for BF16 held as float32.
"""
import numpy as np


def round_to(x, dt):
    """float64 -> the values of the storage type, nearest, ties to even."""
    x = np.asarray(x, dtype=np.float64)
    if dt != "bf16":
        return x.astype(np.float16).astype(np.float64)
    with np.errstate(over="ignore"):
        f = x.astype(np.float32)
    # double rounding through float32 only matters within 2^-24 of a tie: put those on the side of the float64 value
    u = f.view(np.uint32)
    near = np.where(np.abs(f.astype(np.float64)) > np.abs(x), u - np.uint32(1), u)
    tie = (u & np.uint32(0xFFFF)) == 0x8000
    up = np.abs(x) > np.abs(f.astype(np.float64))
    out = ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000))
    out = np.where(tie & up, (u & np.uint32(0xFFFF0000)) + np.uint32(0x10000), out)
    out = np.where(tie & (near != u), u & np.uint32(0xFFFF0000), out)
    return out.astype(np.uint32).view(np.float32).astype(np.float64)


def qk_norm_rope(x, gain, eps, turns, positions, halves):
    """x [tokens][heads][d] -> normalised and rotated, float64, unrounded."""
    x = np.asarray(x, dtype=np.float64)
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    out = y.copy()
    n = len(turns)
    for j in range(n):
        a, b = (j, j + n) if halves else (2 * j, 2 * j + 1)
        angle = 2 * np.pi * np.mod(np.asarray(positions, dtype=np.float64) * turns[j], 1.0)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
    return out


def quantise(x, dt):
    """One row -> (codes, scale, offset)."""
    x = np.asarray(x, dtype=np.float64)
    if not np.all(np.isfinite(x)):
        return np.zeros(x.shape, np.int64), np.nan, np.nan
    off = x.min()
    scale = float(round_to((x.max() - off) / 15.0, dt))
    if scale == 0:
        return np.zeros(x.shape, np.int64), scale, off
    return np.clip(np.rint((x - off) / scale), 0, 15).astype(np.int64), scale, off


class Pool:
    """One layer's pages as bytes, read and written token by token."""

    def __init__(self, data, n_kv, d, page, dt):
        self.data, self.n_kv, self.d, self.page, self.dt = data, n_kv, d, page, dt   # data: uint8 [n_pages][page bytes]
        self.block = page * (d + 8)

    def _code_at(self, which, slot, e):
        if which == 0:
            return slot * (self.d // 2) + e // 2, 4 * (e % 2)
        return self.page * self.d // 2 + (slot // 2) * self.d + (e // 4) * 4 + (slot % 2) * 2 + (e % 4) // 2, 4 * (e % 2)

    def _param_at(self, which, slot):
        return self.page * self.d + which * self.page * 4 + slot * 4

    def read(self, page_id, slot, head, which):
        """Values of one row, float64."""
        if not 0 <= page_id < len(self.data):
            return np.full(self.d, np.nan)
        b = self.data[page_id][head * self.block:(head + 1) * self.block]
        at, sh = zip(*(self._code_at(which, slot, e) for e in range(self.d)))
        codes = (b[list(at)].astype(np.int64) >> np.array(sh)) & 15
        raw = b[self._param_at(which, slot):][:4].copy().view(np.uint16)
        if self.dt == "bf16":
            s, o = (raw.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
        else:
            s, o = raw.view(np.float16).astype(np.float64)
        return o + s * codes

    def write(self, page_id, slot, head, which, x):
        if not 0 <= page_id < len(self.data):
            return
        codes, scale, off = quantise(x, self.dt)
        b = self.data[page_id][head * self.block:(head + 1) * self.block]
        for e in range(self.d):
            at, sh = self._code_at(which, slot, e)
            b[at] = (int(b[at]) & (0xF0 if sh == 0 else 0x0F)) | (int(codes[e]) << sh)
        pair = np.array([scale, off])
        if self.dt == "bf16":
            raw = (pair.astype(np.float32).view(np.uint32) >> np.uint32(16)).astype(np.uint16)
        else:
            raw = pair.astype(np.float16).view(np.uint16)
        b[self._param_at(which, slot):][:4] = raw.view(np.uint8)


def keys_values(pool, table_row, n):
    """K, V [n][n_kv][d] of the first n tokens of a row."""
    out = np.zeros((2, n, pool.n_kv, pool.d))
    for t in range(n):
        col = t // pool.page
        page_id = table_row[col] if col < len(table_row) else -1
        for which in (0, 1):
            for h in range(pool.n_kv):
                out[which, t, h] = pool.read(page_id, t % pool.page, h, which)
    return out


def attention(q, kv, n_keys, limit_shift):
    """q [hq][d] over the first n_keys - limit_shift keys of kv = (K, V); also sum_t p_t (|v_t - middle of the row| + 1/28 of
    its range) and max_t sum |q k| / sqrt d: what rounding the weights, and the scores, can move."""
    hq, d = q.shape
    k, v = kv
    m = n_keys - limit_shift
    out, spread, mag = np.zeros((hq, d)), np.zeros((hq, d)), np.zeros((hq, 1))
    if m <= 0:
        return out, spread, mag
    g = hq // k.shape[1]
    for h in range(hq):
        kh, vh = k[:m, h // g], v[:m, h // g]
        s = kh @ q[h].astype(np.float64) / np.sqrt(d)
        p = np.exp(s - s.max()) if np.all(np.isfinite(s)) else np.full(m, np.nan)
        p = p / p.sum()
        low, high = vh.min(-1, keepdims=True), vh.max(-1, keepdims=True)
        out[h], spread[h] = p @ vh, p @ (np.abs(vh - (low + high) / 2) + (high - low) / 28)
        mag[h] = np.max(np.abs(kh) @ np.abs(q[h].astype(np.float64))) / np.sqrt(d)
    return out, spread, mag


# ------------------------------------------------------------------ page tables
def _pages(n, page):
    return -(-max(n, 0) // page)


def in_use(table, lens, page, n_pages):
    return sorted({p for row, n in zip(table, lens) for p in row[:_pages(n, page)] if 0 <= p < n_pages})


def reserve(table, lens, add, n_pages, page):
    """-> (table, lens, refused), Python lists."""
    table, lens = [list(r) for r in table], list(lens)
    used = set(in_use(table, lens, page, n_pages))
    free = [p for p in range(n_pages) if p not in used]
    at, refused, out = 0, 0, []
    for r, n in enumerate(lens):
        have = max(n, 0)
        first, last = _pages(have, page), _pages(have + max(add[r], 0), page)
        end = at + last - first
        if have > len(table[r]) * page or (last > first and (end > len(free) or last > len(table[r]))):
            refused += 1
            out.append(n)
        else:
            table[r][first:last] = free[at:end]
            out.append(have + max(add[r], 0))
        at = end
    return table, out, refused


def fork(table, lens, source, n_pages, page):
    """-> (table, lens, refused, copies [(src, dst, tokens)])."""
    rows, width = len(table), len(table[0])
    used = set(in_use(table, lens, page, n_pages))
    free = [p for p in range(n_pages) if p not in used]
    new_table, new_lens, copies, refused, asked = [], [], [], 0, 0
    for r, s in enumerate(source):
        if s < 0 or s >= rows:
            refused += s >= rows
            new_table.append([-1] * width)
            new_lens.append(0)
            continue
        n = min(max(lens[s], 0), width * page)
        row = list(table[s][:_pages(n, page)])
        heirs = [i for i, x in enumerate(source) if x == s]
        keeper = s if s in heirs else heirs[0]
        if n % page and r != keeper and 0 <= row[-1] < n_pages:
            if asked < len(free):
                copies.append((row[-1], free[asked], n % page))
                row[-1] = free[asked]
            else:
                refused, row, n = refused + 1, [], 0
            asked += 1
        new_table.append(row + [-1] * (width - len(row)))
        new_lens.append(n)
    return new_table, new_lens, refused, copies


def compact(table, lens, n_pages, page):
    """-> (table, live, moves [(src, dst, tokens)])."""
    live = in_use(table, lens, page, n_pages)
    holes = [p for p in range(len(live)) if p not in set(live)]
    moving = [p for p in live if p >= len(live)]
    new = dict(zip(moving, holes))
    fill = dict.fromkeys(moving, 0)
    out = []
    for row, n in zip(table, lens):
        n = min(max(n, 0), len(row) * page)
        used = row[:_pages(n, page)]
        for c, p in enumerate(used):
            if p in fill:
                fill[p] = max(fill[p], min(page, n - c * page))
        out.append([new.get(p, p) for p in used] + [-1] * (len(row) - len(used)))
    return out, len(live), [(p, new[p], fill[p]) for p in moving]


def copied(data, moves, n_kv, d, page):
    """Pool bytes [layers][n_pages][page bytes] after moving the filled tokens, in groups of 16, of every (src, dst, tokens)."""
    out = data.copy()
    view = out.reshape(out.shape[0], out.shape[1], n_kv, page * (d + 8))
    old = data.reshape(view.shape)
    for src, dst, tokens in moves:
        f = min(page, -(-tokens // 16) * 16)
        for a, b in ((0, f * d // 2), (page * d // 2, page * d // 2 + f * d // 2), (page * d, page * d + 4 * f),
                     (page * (d + 4), page * (d + 4) + 4 * f)):
            view[:, dst, :, a:b] = old[:, src, :, a:b]
    return out
