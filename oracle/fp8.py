"""8-bit floating point matrices, routing and experts' products, from their definitions in 64 bits (numpy, CPU).

Test infrastructure: nothing here comes from the library.  Layouts are written as index formulas, element by element.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
# the values of the codes 0 .. 126: exponent field 0 counts in steps of 2^-9, others are 2^(e - 7) * (1 + m / 8); 127 is NaN
GRID = np.array([m * 2.0 ** -9 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8) for e in range(16) for m in range(8)][:127])


def scale_byte(top):
    """The byte of a block with the largest magnitude `top`: the smallest 2^(byte - 127), byte >= 1, of which it is at most 448."""
    if not np.isfinite(top):
        return 255
    byte = 1
    if top > 448 * 2.0 ** -126:
        byte = max(1, int(np.ceil(np.log2(top / 448))) + 126)
        while top > 448 * 2.0 ** (byte - 127):
            byte += 1
    return byte


def nearest(t):
    """Codes 0 .. 126 of magnitudes t <= 448, ties to the even code."""
    hi = np.clip(np.searchsorted(GRID, t), 1, 126)
    lo = hi - 1
    down, up = t - GRID[lo], GRID[hi] - t
    return np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)


def _codes(block, byte):
    if byte == 255:
        return np.full(block.shape, 127, np.uint8)
    return (nearest(np.abs(block) / 2.0 ** (byte - 127)) | np.where(np.signbit(block), 128, 0)).astype(np.uint8)


def quantize(x):
    """(codes [rows, cols], scale bytes [rows, blocks]) with blocks along the rows of x."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    codes, byte = np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // BLOCK)), np.int64)
    for b in range(byte.shape[1]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        top = np.where(np.isfinite(part).all(1), np.abs(part).max(1), np.nan)
        byte[:, b] = [scale_byte(v) for v in top]
        for k in np.unique(byte[:, b]):
            r = byte[:, b] == k
            codes[r, b * BLOCK:(b + 1) * BLOCK] = _codes(part[r], k)
    return codes, byte


def quantize_weights(w):
    """The same with one scale for a tile of 128 x 128."""
    w = np.asarray(w, np.float64)
    rows, cols = w.shape
    codes, byte = np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // BLOCK)), np.int64)
    for r in range(0, rows, BLOCK):
        for b in range(byte.shape[1]):
            part = w[r:r + BLOCK, b * BLOCK:(b + 1) * BLOCK]
            k = scale_byte(np.abs(part).max() if np.isfinite(part).all() else np.nan)
            byte[r:r + BLOCK, b] = k
            codes[r:r + BLOCK, b * BLOCK:(b + 1) * BLOCK] = _codes(part, k)
    return codes, byte


def transposed_weights(codes, byte):
    """Codes and scale bytes of the transposed matrix: the same tiles."""
    rows, cols = codes.shape
    t = np.empty((cols, -(-rows // BLOCK)), np.int64)
    for c in range(cols):
        for b in range(t.shape[1]):
            t[c, b] = byte[b * BLOCK, c // BLOCK]
    return codes.T.copy(), t


def values(codes, byte):
    with np.errstate(invalid="ignore"):
        v = np.where(codes % 128 == 127, np.nan, GRID[np.minimum(codes % 128, 126)])
        v = np.where(codes >= 128, -v, v)
        s = np.where(byte == 255, np.nan, 2.0 ** (np.minimum(byte, 254) - 127.0))
        return v * np.repeat(s, BLOCK, axis=1)[:, :codes.shape[1]]


def buffer(codes, byte):
    """(bytes of the packed matrix, which of them are defined)."""
    rows, cols = codes.shape
    pitch = -(-cols // BLOCK) * BLOCK
    off = -(-rows * pitch // 256) * 256
    words = -(-cols // 512)
    out = np.zeros(off + -(-words * rows * 4 // 256) * 256, np.uint8)
    known = np.zeros(out.size, bool)
    known[:rows * pitch] = True
    known[off:off + words * rows * 4] = True
    for r in range(rows):
        out[r * pitch:r * pitch + cols] = codes[r]
        if byte[r, -1] == 255:
            out[r * pitch + cols:(r + 1) * pitch] = 127        # padding is what a zero there would be
        for b in range(byte.shape[1]):
            out[off + ((b // 4) * rows + r) * 4 + b % 4] = byte[r, b]
    return out, known


# ------------------------------------------------------------------------------------------------ routing
def scores(logits, kind):
    x = np.asarray(logits, np.float64)
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return np.where(np.isneginf(x), 0.0, np.where(x >= 0, 1 / (1 + np.exp(-x)), np.exp(x) / (1 + np.exp(x))))
        e = np.exp(x - np.where(np.isneginf(x).all(1, keepdims=True), 0.0, x.max(1, keepdims=True)))
        total = e.sum(1, keepdims=True)
        return np.where(total == 0, 0.0, e / np.where(total == 0, 1.0, total))


def _shares(x, s, e, kind):
    """The scores of a token's experts `e` for their renormalised weights, which depend on these alone: of a softmax those of the row without the others,
    which 64 bits hold however far below them they are."""
    if kind == "sigmoid":
        return s
    return scores(np.where(np.isin(np.arange(len(x)), e), x, -np.inf)[None], kind)[0]


def _best(c, n):
    """The indices of the n largest, in descending order, the lowest of equals first; -infinity is never taken."""
    order = sorted((i for i in range(len(c)) if c[i] > -np.inf), key=lambda i: (-c[i], i))[:n]
    return order


def route(logits, picks, kind, bias=None, groups=1, top_groups=1, renormalize=True, scale=1.0):
    x = np.asarray(logits, np.float64)
    T, E = x.shape
    s = scores(x, kind)
    weights, chosen = np.zeros((T, picks)), np.full((T, picks), -1, np.int64)
    for t in range(T):
        c = s[t] + (0 if bias is None else np.asarray(bias, np.float64))
        c = np.where(np.isneginf(x[t]), -np.inf, c)
        if np.isnan(c).any() or np.isnan(x[t]).any() or (kind == "softmax" and np.isposinf(x[t]).any()):
            weights[t] = np.nan
            continue
        if groups > 1:
            by = c.reshape(groups, -1)
            total = [sum(sorted((v for v in g if v > -np.inf), reverse=True)[:2]) if (g > -np.inf).any() else -np.inf for g in by]
            stay = _best(np.array(total), top_groups)
            c = np.where(np.isin(np.arange(E) // (E // groups), stay), c, -np.inf)
        best = _best(c, picks)
        chosen[t, :len(best)] = best
        weights[t, :len(best)] = s[t, best]
        if renormalize:
            weights[t, :len(best)] = _shares(x[t], s[t], best, kind)[best]
            total = weights[t].sum()
            weights[t] = weights[t] / total if total > 0 else 0
        weights[t] *= scale
    return weights, chosen


def route_backward(dweights, logits, chosen, kind, renormalize=True, scale=1.0):
    """Through the Jacobian of each token's weights by its logits."""
    x, g = np.asarray(logits, np.float64), np.asarray(dweights, np.float64)
    T, E = x.shape
    s, out = scores(x, kind), np.zeros((T, E))
    for t in range(T):
        at = [j for j in range(chosen.shape[1]) if chosen[t, j] >= 0]
        if not at:
            continue
        e = chosen[t, at]
        ds = np.zeros(E)
        if renormalize:
            s[t] = _shares(x[t], s[t], e, kind)
            total = s[t, e].sum()
            if total > 0:
                for j, k in zip(at, e):
                    ds[k] += scale * (g[t, j] - (g[t, at] * s[t, e]).sum() / total) / total
        else:
            for j, k in zip(at, e):
                ds[k] += scale * g[t, j]
        if kind == "sigmoid":
            with np.errstate(all="ignore"):
                rest = np.where(x[t] >= 0, np.exp(-x[t]) / (1 + np.exp(-x[t])), 1 / (1 + np.exp(x[t])))
            out[t] = np.where(ds != 0, ds * s[t] * rest, 0.0)
        else:
            out[t] = s[t] * (ds - (ds * s[t]).sum())
    return out


def plan(chosen, experts):
    """(counts, table, rows, place)."""
    T, k = chosen.shape
    flat = [int(e) for e in chosen.reshape(-1)]
    lists = [[i for i, e in enumerate(flat) if e == x] for x in range(experts)]
    counts = [len(l) for l in lists]
    rows = [i for l in lists for i in l]
    place = np.full(T * k, -1, np.int64)
    place[rows] = np.arange(len(rows))
    table = np.zeros((4, experts + 1), np.int64)
    for q, n in enumerate((1, 256, 128, 64)):
        table[q, 1:] = np.cumsum([-(-c // n) for c in counts])
    return np.array(counts), table, np.array(rows + [-1] * (T * k - len(rows)), np.int64), place.reshape(T, k)


def columns(tokens, picks, experts):
    """Columns of the rows in blocks of 128 that begin anew with every expert: the most that any choice needs."""
    slots = tokens * picks
    return (slots + 127 * min(experts, slots)) // 128 * 128
