"""Microscaled 4-bit matrices, 8-bit checkpoints and the layers on them, from their definitions in 64 bits (numpy, CPU).

Test infrastructure: nothing here comes from the library.  Layouts are written as index formulas, element by element.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _fmix32(h):
    h = np.atleast_1d(np.asarray(h, np.uint32))
    h = (h ^ (h >> np.uint32(16))) * np.uint32(0x85EBCA6B)
    h = (h ^ (h >> np.uint32(13))) * np.uint32(0xC2B2AE35)
    return h ^ (h >> np.uint32(16))


def draws(rows, cols, seed):
    """The 16-bit draw of every element."""
    key = _fmix32(np.uint32(seed & 0xFFFFFFFF) ^ _fmix32(np.uint32((seed >> 32) & 0xFFFFFFFF) ^ np.uint32(0x9E3779B9)))
    r, c = np.arange(rows, dtype=np.uint64)[:, None], np.arange(cols, dtype=np.uint64)[None, :]
    h = _fmix32((r * np.uint64((cols + 1) // 2) + c // 2).astype(np.uint32) ^ key)
    return np.where(c % 2 == 0, h >> np.uint32(16), h & np.uint32(0xFFFF)).astype(np.int64)


def _in_blocks(x, fill=0.0):
    rows, cols = x.shape
    out = np.full((rows, -(-cols // BLOCK) * BLOCK), fill, np.float64)
    out[:, :cols] = x
    return out.reshape(rows, -1, BLOCK)


def _bytes(top, below):
    """Scale bytes of blocks with the largest magnitudes `top` (fp64, exact)."""
    with np.errstate(all="ignore"):
        e = np.where(top > 0, np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 1, -10000)
    return np.where(np.isfinite(top), np.clip(e - below + 127, 1, 254), 255).astype(np.int64)


def mx4_codes(x, stochastic=False, seed=0, transpose=False):
    """(codes [R, blocks, 32] 0 .. 15, scale bytes [R, blocks]) of fp32/bf16 values x; R counts columns of x when `transpose`."""
    x = np.asarray(x, np.float64)
    u = draws(*x.shape, seed) if stochastic else np.zeros(x.shape, np.int64)
    if transpose:
        x, u = x.T, u.T
    b, u = _in_blocks(x), _in_blocks(u)
    top = np.abs(b).max(axis=2)
    top = np.where(np.isnan(b).any(axis=2), np.nan, top)
    byte = _bytes(top, 2)
    if stochastic:
        with np.errstate(invalid="ignore"):
            byte = np.where((byte < 255) & (top > 6 * np.exp2(byte - 127.0)), byte + 1, byte)
    codes = np.zeros(b.shape, np.int64)
    ok = byte < 255
    t = np.abs(b[ok]) / np.exp2(byte[ok] - 127.0)[:, None]
    if stochastic:
        low = np.searchsorted(GRID, t, side="right") - 1
        high = np.minimum(low + 1, 7)
        gap = np.where(high > low, GRID[high] - GRID[low], 1.0)
        c = np.where(np.floor((t - GRID[low]) / gap * 65536) > u[ok], high, low)
    else:
        middle = (GRID[1:] + GRID[:-1]) / 2
        c = np.searchsorted(middle, t, side="left")
        tie = (c < 7) & (t == middle[np.minimum(c, 6)])
        c = np.where(tie & (c % 2 == 1), c + 1, c)
    codes[ok] = c + 8 * (np.signbit(b[ok]) & (np.abs(b[ok]) >= 0))
    return codes, byte


def mx4_values(codes, byte, cols):
    v = np.where(codes >= 8, -1.0, 1.0) * GRID[codes & 7] * np.where(byte == 255, np.nan, np.exp2(byte - 127.0))[:, :, None]
    return v.reshape(v.shape[0], -1)[:, :cols]


def mx4_buffer(codes, byte):
    """The packed buffer, by the index formulas of the layout."""
    R, nb, _ = codes.shape
    blocks, groups = -(-R // 32), -(-nb // 8)
    off = blocks * groups * 4096
    buf = np.zeros(off + blocks * groups * 256, np.uint8)
    r, b = np.arange(R)[:, None], np.arange(nb)[None, :]
    at = (((r // 32) * (4 * groups) + b // 2) * 2 + b % 2) * 512 + (r % 32) * 16
    for j in range(16):
        buf[at + j] = codes[:, :, 2 * j] | (codes[:, :, 2 * j + 1] << 4)
    buf[off + (((r // 32) * groups + b // 8) * 2 + b % 2) * 128 + (r % 32) * 4 + (b // 2) % 4] = byte
    return buf


def ckpt8_codes(x, parts=1):
    """(codes [rows * parts, blocks, 32], scale bytes [rows * parts, blocks])."""
    x = np.asarray(x, np.float64)
    b = _in_blocks(x.reshape(x.shape[0] * parts, -1))
    top = np.where(np.isnan(b).any(axis=2), np.nan, np.abs(b).max(axis=2))
    byte = _bytes(top, 6)
    codes = np.zeros(b.shape, np.int64)
    ok = byte < 255
    codes[ok] = np.clip(np.rint(b[ok] / np.exp2(byte[ok] - 127.0)[:, None]), -127, 127)
    return codes, byte


def ckpt8_values(codes, byte, rows, cols, parts=1):
    v = codes * np.where(byte == 255, np.nan, np.exp2(byte - 127.0))[:, :, None]
    return v.reshape(rows * parts, -1)[:, :cols].reshape(rows, parts * cols)


def ckpt8_buffer(codes, byte):
    n, nb, _ = codes.shape
    off = -(-n * nb * 32 // 256) * 256
    buf = np.zeros(off + -(-n * nb // 256) * 256, np.uint8)
    buf[:n * nb * 32] = codes.astype(np.int8).ravel().view(np.uint8)
    buf[off:off + n * nb] = byte.astype(np.uint8).ravel()
    return buf


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(x, name):
    """(f(x), f'(x)) for "silu" and "gelu"."""
    x = np.asarray(x, np.float64)
    if name == "silu":
        s = 1 / (1 + np.exp(-x))
        return x * s, s + x * s * (1 - s)
    cdf = 0.5 * _erfc(-x / math.sqrt(2))   # (1 + erf cancels far below zero)
    return x * cdf, cdf + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
