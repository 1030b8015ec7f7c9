"""Plain 64-bit numpy forms of the dense operators, written from their
definitions and used by the tests alone."""
import math

import numpy as np

BLOCK = 128
# mantissa bits, least normal exponent, largest value
FORMATS = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0)}


def encode(x, fmt):
    """Scale exponents [blocks, rows] and rounded values in units of the scale
    [rows, cols] (NaN where the format holds NaN) of a float64 table."""
    bits, least, top = FORMATS[fmt]
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    exps = np.zeros((blocks, rows), np.int64)
    units = np.zeros((rows, cols))
    for b in range(blocks):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        most = np.max(np.where(np.isfinite(v), np.abs(v), 0.0), axis=1)
        for r in range(rows):
            if most[r] == 0:
                continue
            e = -127
            if most[r] > top * 2.0 ** -127:
                e = math.frexp(most[r] / top)[1]  # top * 2^e >= most
                while most[r] <= top * 2.0 ** (e - 1) and e > -127:
                    e -= 1
            exps[b, r] = e
        u = v / np.ldexp(1.0, exps[b])[:, None]
        with np.errstate(invalid="ignore", divide="ignore"):
            size = np.maximum(np.abs(u), 2.0 ** least)
            step = np.exp2(np.floor(np.frexp(size)[1] - 1.0) - bits)
            rounded = np.round(u / step) * step  # ties to even
        if fmt == "e4m3":
            rounded = np.where(np.isinf(v), np.nan, rounded)
        else:
            rounded = np.where(np.isinf(v), v, rounded)
        units[:, b * BLOCK:(b + 1) * BLOCK] = rounded
    return exps, units


def decode_codes(codes, fmt):
    """Unscaled float64 values of uint8 codes."""
    bits, least, _ = FORMATS[fmt]
    c = codes.astype(np.int64)
    field, mant = (c >> bits) & ((1 << (7 - bits)) - 1), (c & ((1 << bits) - 1)).astype(np.float64)
    v = np.where(field == 0, np.ldexp(mant, least - bits), np.ldexp(1 + mant / (1 << bits), field + least - 1))
    if fmt == "e4m3":
        v = np.where((c & 127) == 127, np.nan, v)
    else:
        v = np.where((c & 127) == 124, np.inf, np.where((c & 127) > 124, np.nan, v))
    return np.where(c >= 128, -v, v)


def values(codes, scales, cols, fmt):
    """float64 [rows, cols] of packed codes [rows, ld] and scale bytes [blocks, rows]."""
    block = np.arange(cols) // BLOCK
    return decode_codes(codes[:, :cols], fmt) * np.ldexp(1.0, scales.astype(np.int64)[block].T - 127)


def act(z, kind):
    """Value and slope."""
    if kind == "relu":
        return np.where(z > 0, z, 0 * z), (z > 0).astype(np.float64)
    if kind == "silu":
        p = 1 / (1 + np.exp(-z))
        return z * p, p + z * p * (1 - p)
    if kind == "gelu":
        erf = np.vectorize(math.erf, otypes=[np.float64])
        p = 0.5 * (1 + erf(z / math.sqrt(2)))
        return z * p, p + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return z, np.ones_like(z)


def norm(x, groups, weight, bias, eps, kind, offsets):
    """y, mean, rstd, xh, z of float64 x."""
    rows, channels = x.shape
    per = channels // groups
    segments = len(offsets) - 1
    mean, rstd = np.zeros((segments, groups)), np.full((segments, groups), 1 / np.sqrt(eps) if eps else np.inf)
    xh = np.zeros_like(x)
    for s in range(segments):
        b, e = offsets[s], offsets[s + 1]
        if e <= b:
            continue
        v = x[b:e].reshape(e - b, groups, per)
        mean[s] = v.mean(axis=(0, 2))
        rstd[s] = 1 / np.sqrt(((v - mean[s][None, :, None]) ** 2).mean(axis=(0, 2)) + eps)
        xh[b:e] = ((v - mean[s][None, :, None]) * rstd[s][None, :, None]).reshape(e - b, channels)
    w = 1.0 if weight is None else weight
    z = xh * w + (0.0 if bias is None else bias)
    return act(z, kind)[0], mean, rstd, xh, z


def norm_backward(dy, x, mean, rstd, groups, weight, bias, kind, offsets):
    """dx, dweight, dbias and, for tolerances, the magnitudes summed in each."""
    rows, channels = x.shape
    per = channels // groups
    w = np.ones(channels) if weight is None else weight
    seg = np.repeat(np.arange(len(offsets) - 1), np.diff(offsets))
    spread = lambda v: np.repeat(v[seg], per, axis=1)  # noqa: E731
    xh = (x - spread(mean)) * spread(rstd)
    z = xh * w + (0.0 if bias is None else bias)
    dz = dy * act(z, kind)[1]
    dh = dz * w
    count = np.maximum(np.diff(offsets), 1)[:, None] * per

    def means(v):
        out = np.zeros((len(offsets) - 1, groups))
        np.add.at(out, seg, v.reshape(rows, groups, per).sum(axis=2))
        return out / count

    dx = spread(rstd) * (dh - spread(means(dh)) - xh * spread(means(dh * xh)))
    size = spread(rstd) * (np.abs(dy * w) + spread(means(np.abs(dy * w))) +
                           np.abs(xh) * spread(means(np.abs(dy * w * xh))))
    return dx, (dz * xh).sum(0), dz.sum(0), size, np.abs(dy * xh).sum(0), np.abs(dy).sum(0), z
