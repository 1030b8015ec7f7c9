"""Plain 64-bit numpy forms of the 4-bit tables and of the rows sorted by
expert, written from their definitions and used by the tests alone."""
import math

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])
BLOCK = 32


def encode(x):
    """Scale bytes [rows, blocks] and rounded values in units of the scale [rows,
    cols] of a float64 table; a block with a NaN or an infinity: 255 and zeros."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    scale = np.full((rows, blocks), 127, np.int64)
    units = np.zeros((rows, cols))
    for r in range(rows):
        for b in range(blocks):
            v = x[r, b * BLOCK:(b + 1) * BLOCK]
            if not np.isfinite(v).all():
                scale[r, b] = 255
                continue
            most = np.abs(v).max()
            if most == 0:
                units[r, b * BLOCK:(b + 1) * BLOCK] = v
                continue
            e = max(math.frexp(most / 6)[1], -127)  # 6 * 2^e > most / 2
            while most > 6 * 2.0 ** e:
                e += 1
            while e > -127 and most <= 6 * 2.0 ** (e - 1):
                e -= 1
            scale[r, b] = e + 127
            u = v / 2.0 ** e
            step = np.where(np.abs(u) < 2, 0.5, np.where(np.abs(u) < 4, 1, 2))
            units[r, b * BLOCK:(b + 1) * BLOCK] = np.copysign(np.round(np.abs(u) / step) * step, u)  # ties to even
    return scale, units


def halves(codes, cols):
    """The codes of uint8 [rows, ld] one by one, [rows, cols]."""
    c = np.arange(cols)
    return (codes[:, c // 2] >> (4 * (c % 2)).astype(np.uint8)) & 15


def scale_bytes(scales, cols):
    """[groups, rows, 4] as [rows, blocks]."""
    blocks = -(-cols // BLOCK)
    return scales.transpose(1, 0, 2).reshape(scales.shape[1], -1)[:, :blocks].astype(np.int64)


def values(codes, scales, cols):
    if cols == 0:
        return np.zeros((codes.shape[0], 0))
    s = np.repeat(scale_bytes(scales, cols), BLOCK, axis=1)[:, :cols]
    return np.where(s == 255, np.nan, GRID[halves(codes, cols)] * np.ldexp(1.0, s - 127))


def route(chosen, experts):
    """offsets, place, source."""
    rows, k = chosen.shape
    order = [(e, t, j) for t in range(rows) for j in range(k) for e in [int(chosen[t, j])] if 0 <= e < experts]
    order.sort()
    place = np.full((rows, k), -1, np.int64)
    source = np.full(rows * k, -1, np.int64)
    offsets = np.zeros(experts + 1, np.int64)
    for i, (e, t, j) in enumerate(order):
        place[t, j], source[i] = i, t
        offsets[e + 1] += 1
    return np.cumsum(offsets), place, source


def route_fast(chosen, experts):
    """The same for many entries."""
    rows, k = chosen.shape
    flat = chosen.reshape(-1).astype(np.int64)
    kind = np.where((flat >= 0) & (flat < experts), flat, experts)
    order = np.argsort(kind, kind="stable")
    kept = kind[order] < experts
    place = np.empty(rows * k, np.int64)
    place[order] = np.where(kept, np.arange(rows * k), -1)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(kind, minlength=experts + 1)[:experts])])
    return offsets, place.reshape(rows, k), np.where(kept, order // k, -1)


def combine(y, place, weights):
    """out, and the magnitudes summed."""
    at = np.maximum(place, 0)
    terms = np.where(place >= 0, weights, 0.0)[:, :, None] * np.where((place >= 0)[:, :, None], y[at], 0.0)
    return terms.sum(1), np.abs(terms).sum(1)


def combine_backward(dout, y, place, weights):
    """dy, dweights, and the magnitudes summed in dweights."""
    dy = np.zeros_like(y)
    there = place >= 0
    dy[place[there]] = (weights[:, :, None] * dout[:, None, :])[there]
    terms = np.where(there[:, :, None], dout[:, None, :] * y[np.maximum(place, 0)], 0.0)
    return dy, terms.sum(2), np.abs(terms).sum(2)
