"""Float64 definitions of the weights in 4 bits with group scales (numpy).

Independent of csrc/: packed bytes are addressed one number at a time from their documented layout.  `dt` is the storage
type: numpy float16, or "bf16".
"""
import numpy as np

from oracle.kv4 import round_to


def quantise(w, group, dt):
    """w [n][k] -> (codes [n][k], scales [n][groups], zeros [n][groups])."""
    w = np.asarray(w, dtype=np.float64)
    n, k = w.shape
    groups = -(-k // group)
    codes, scales, zeros = np.zeros((n, k), np.int64), np.zeros((n, groups)), np.zeros((n, groups), np.int64)
    for j in range(groups):
        part = w[:, j * group:(j + 1) * group]
        ok = np.isfinite(part).all(1)
        x = np.where(ok[:, None], part, 0.0)
        lo, hi = np.minimum(x.min(1), 0), np.maximum(x.max(1), 0)
        scale = round_to((hi - lo) / 15.0, dt)
        by = np.where(scale > 0, scale, 1.0)
        zero = np.where(scale > 0, np.clip(np.rint(-lo / by), 0, 15), 0)
        code = np.clip(np.rint(x / by[:, None]) + zero[:, None], 0, 15)
        codes[:, j * group:(j + 1) * group] = np.where((scale > 0)[:, None], code, 0)
        scales[:, j], zeros[:, j] = np.where(ok, scale, np.nan), zero
    return codes, scales, zeros


def values(codes, scales, zeros, group):
    """scale * (code - zero), float64, unrounded."""
    of = np.arange(codes.shape[1]) // group
    return scales[:, of] * (codes - zeros[:, of])


def sizes(n, k, group):
    tiles, blocks, per = -(-n // 16), -(-k // 128), 128 // group
    return tiles, blocks, per, (tiles * blocks * 1024, tiles * blocks * per * 32, tiles * blocks * per * 8)


def code_at(row, col, n, k, group):
    """(byte, shift) of a code."""
    _, blocks, _, _ = sizes(n, k, group)
    tile, i, g = row // 16, row % 16 // 8, row % 8
    block, c = col // 128, col % 128
    q, t, s, b, e = c // 32, c % 32 // 8, c % 8 // 4, c % 4 // 2, c % 2
    at = tile * blocks + block
    for size, index in ((2, q // 2), (8, g), (4, t), (2, q % 2), (2, s), (2, e), (2, b)):
        at = at * size + index
    return at, 4 * i


def param_at(row, j, n, k, group):
    """(index of the 16-bit scale, byte of the zero behind the scales, shift of the zero) of group j of a row."""
    _, blocks, per, _ = sizes(n, k, group)
    pair = ((row // 16 * blocks + j // per) * 8 + row % 8) * per + j % per
    return 2 * pair + row % 16 // 8, pair, 4 * (row % 16 // 8)


def pack(codes, scales, zeros, group, dt):
    """The packed bytes."""
    n, k = codes.shape
    _, _, _, (nc, ns, nz) = sizes(n, k, group)
    out = np.zeros(nc + ns + nz, np.uint8)
    rows, cols = np.meshgrid(np.arange(n), np.arange(k), indexing="ij")
    at, shift = code_at(rows, cols, n, k, group)
    np.add.at(out, at.ravel(), (codes << shift).astype(np.uint8).ravel())
    rows, js = np.meshgrid(np.arange(n), np.arange(scales.shape[1]), indexing="ij")
    si, zi, zs = param_at(rows, js, n, k, group)
    half = np.zeros(ns // 2, np.uint16)
    half[si] = bits(scales, dt)
    out[nc:nc + ns] = half.view(np.uint8)
    np.add.at(out, (nc + ns + zi).ravel(), (zeros << zs).astype(np.uint8).ravel())
    return out


def bits(x, dt):
    """The 16 bits of values of the storage type (any NaN: 0x7FFF)."""
    x = np.asarray(x, dtype=np.float64)
    b = (x.astype(np.float32).view(np.uint32) >> 16).astype(np.uint16) if dt == "bf16" else x.astype(np.float16).view(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FFF), b)


def linear(x, w):
    """x [rows][k] times w [n][k] transposed, and the sum of the sizes of its terms."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    return x @ w.T, np.abs(x) @ np.abs(w).T
