"""Operator cases: the dense operators around the sparse products, over the
sizes they are used at.

Every case names an operator and the sizes of one call.

Operators:
* ``norm``      group norm with an activation over segments of rows, channels
                last; forward alone;
* ``train``     the same as a training step uses it: forward, then the gradients
                from a given output gradient, the input kept as it is or in
                8 bits (``keep``) between the two;
* ``pack``      activations to 8 bits with one power-of-two scale for each row
                and block of 128 columns, and back;
* ``gradient``  the weight gradient X^T.G from activations kept in 8 bits;
* ``product``   X.W^T of two such 8-bit operands, with a bias where one is given.

All inputs are drawn on the GPU from the seed with torch.
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 128  # columns that share a scale
# 8-bit formats: torch's type, the largest value as mantissa * 2^exponent
# (mantissa in [0.5, 1), as frexp gives it), mantissa bits, least exponent
FORMATS = {"e4m3": (torch.float8_e4m3fn, 0.875, 9, 3, -6), "e5m2": (torch.float8_e5m2, 0.875, 16, 2, -14)}
EPS = 1e-5


# ------------------------------------------------------------------ cases ---
def listed():
    return [
        # the node features of one small graph in a forward pass: launch latency
        {"name": "norm_one_graph", "op": "norm", "rows": 37, "channels": 64, "groups": 8, "segments": 1,
         "ragged": False, "dtype": "f32", "act": "relu"},
        # a batch of a few thousand small graphs, each normalised by itself
        {"name": "norm_batch", "op": "norm", "rows": 100003, "channels": 96, "groups": 6, "segments": 3001,
         "ragged": True, "dtype": "bf16", "act": "gelu"},
        # a training step of one layer on a middling graph, its input kept in 8 bits
        {"name": "train_262k", "op": "train", "rows": 1 << 18, "channels": 128, "groups": 8, "segments": 1,
         "ragged": False, "dtype": "f32", "act": "silu", "keep": "e4m3"},
        # the same on the largest graph, where the node tables pass every cache
        {"name": "train_2m4", "op": "train", "rows": 2400000, "channels": 128, "groups": 8, "segments": 1,
         "ragged": False, "dtype": "f32", "act": "silu", "keep": "e4m3"},
        # an odd feature table of a small graph, with the wide-range format
        {"name": "pack_odd", "op": "pack", "rows": 4999, "cols": 601, "dtype": "f16", "format": "e5m2"},
        # a layer's activations on a middling graph
        {"name": "pack_262k", "op": "pack", "rows": 1 << 18, "cols": 128, "dtype": "f32", "format": "e4m3"},
        # the last layer's weight gradient on a middling graph, from a full-precision output gradient
        {"name": "gradient_262k", "op": "gradient", "rows": 1 << 18, "cols": 128, "n": 64, "dtype": "f32",
         "format": "e4m3"},
        # the first layer's on odd, wide features
        {"name": "gradient_odd", "op": "gradient", "rows": 50021, "cols": 601, "n": 129, "dtype": "bf16",
         "format": "e4m3"},
        # one node through a wide layer: the weights are read once, latency counts
        {"name": "product_one_row", "op": "product", "rows": 1, "cols": 4096, "n": 4096, "dtype": "bf16",
         "x_format": "e4m3", "w_format": "e4m3", "bias": True},
        # a layer's transform on a middling graph, into the type the sparse product takes
        {"name": "product_262k", "op": "product", "rows": 1 << 18, "cols": 128, "n": 128, "dtype": "f32",
         "x_format": "e4m3", "w_format": "e4m3", "bias": False},
        # an output gradient in the wide-range format through odd sizes
        {"name": "product_odd", "op": "product", "rows": 5003, "cols": 601, "n": 47, "dtype": "f16",
         "x_format": "e5m2", "w_format": "e4m3", "bias": True},
        # wide layers over many nodes: bound by the matrix units
        {"name": "product_large", "op": "product", "rows": 8192, "cols": 8192, "n": 8192, "dtype": "bf16",
         "x_format": "e4m3", "w_format": "e4m3", "bias": False},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(low * (high / low) ** rng.random()))))


def draw(rng):
    op = rng.choice(("norm", "train", "pack", "gradient", "product"))
    dtype = rng.choice(("f32", "f32", "bf16", "f16"))
    if op in ("norm", "train"):
        groups = rng.choice((1, 2, 4, 5, 8, 16, 32))
        channels = groups * _log_int(rng, 1, 512 // groups)
        rows = _log_int(rng, 1, min(1 << 21, (1 << 28) // channels))
        ragged = rng.random() < 0.5
        if ragged:
            segments = _log_int(rng, 1, max(1, rows // 3))
        else:
            segments = _log_int(rng, 1, rows)
            rows = segments * max(1, rows // segments)
        case = {"op": op, "rows": rows, "channels": channels, "groups": groups, "segments": segments,
                "ragged": ragged, "dtype": dtype}
        if op == "norm":
            case["act"] = rng.choice(("none", "relu", "silu", "gelu"))
        else:
            # relu's derivative jumps: its gradient at a value within rounding of 0 is not comparable
            case["act"] = rng.choice(("none", "silu", "gelu"))
            case["keep"] = rng.choice(("none", "e4m3", "e5m2"))
        return case
    if op == "pack":
        cols = _log_int(rng, 1, 4096)
        return {"op": op, "rows": _log_int(rng, 1, min(1 << 21, (1 << 28) // cols)), "cols": cols, "dtype": dtype,
                "format": rng.choice(("e4m3", "e5m2"))}
    cols, n = _log_int(rng, 16, 4096), _log_int(rng, 8, 4096)
    if op == "gradient":
        rows = _log_int(rng, 1, min(1 << 21, (1 << 28) // max(cols, n), 200_000_000_000 // (cols * n)))
        return {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "format": rng.choice(("e4m3", "e5m2"))}
    rows = _log_int(rng, 1, min(1 << 21, (1 << 28) // max(cols, n), 500_000_000_000 // (cols * n)))
    return {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "x_format": rng.choice(("e4m3", "e5m2")),
            "w_format": "e4m3", "bias": rng.random() < 0.5}


# ----------------------------------------------------------------- inputs ---
def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _offsets(case, seed):
    """Row offsets of the segments: lengths around a mean, one in sixteen empty."""
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(0.5 * torch.randn(case["segments"], generator=g, dtype=torch.float64).clamp(-2, 2))
    if case["segments"] > 1:
        w[torch.rand(case["segments"], generator=g) < 1 / 16] = 0
        w[0] = max(float(w[0]), 1.0)
    at = torch.cat([torch.zeros(1, dtype=torch.float64), torch.cumsum(w, 0)])
    off = torch.floor(at * (case["rows"] / float(at[-1]))).to(torch.int32)
    off[-1] = case["rows"]
    return off, int((off[1:] - off[:-1]).max())


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    op, rows = case["op"], case["rows"]
    state = dict(case)
    if op in ("norm", "train"):
        c, dtype = case["channels"], DTYPES[case["dtype"]]
        # sums over neighbours: a mean and a spread of each channel's own
        x = _normal(g, rows, c) * (0.5 + torch.rand(c, generator=g, device=DEV)) + _normal(g, c)
        state["x"] = x.to(dtype)
        del x
        state["weight"] = 1 + 0.2 * _normal(g, c)
        state["shift"] = 0.2 * _normal(g, c)
        state["offsets"], state["longest"] = None, rows // case["segments"]
        if case["ragged"]:
            off, state["longest"] = _offsets(case, int(seed))
            state["offsets"] = off.to(DEV)
        if op == "train":
            state["dy"] = (_normal(g, rows, c) * 0.1).to(dtype)
        return state
    if op == "pack":
        # magnitudes that differ from row to row, some entries cut to 0 by an activation
        x = _normal(g, rows, case["cols"]) * torch.exp(_normal(g, rows, 1))
        x[:, ::3] = x[:, ::3].clamp_min(0)
        state["x"] = x.to(DTYPES[case["dtype"]])
        return state
    if op == "gradient":
        state["x"] = _quantised(_normal(g, rows, case["cols"]) * torch.exp(0.5 * _normal(g, rows, 1)), case["format"])
        state["g"] = (0.1 * _normal(g, rows, case["n"])).to(DTYPES[case["dtype"]])
        return state
    state["x"] = _quantised(_normal(g, rows, case["cols"]) * torch.exp(0.5 * _normal(g, rows, 1)), case["x_format"])
    state["w"] = _quantised(_normal(g, case["n"], case["cols"]) * case["cols"] ** -0.5, case["w_format"])
    state["b"] = _normal(g, case["n"]) if case["bias"] else None
    return state


def _blocks(cols):
    return -(-cols // BLOCK)


def _quantised(x, fmt):
    """8-bit codes [rows, cols up to a multiple of 16, zeros there] and scale
    exponents [blocks, rows], 127 for a scale of 1."""
    kind, top, shift, _, _ = FORMATS[fmt]
    rows, cols = x.shape
    padded = torch.zeros(rows, _blocks(cols) * BLOCK, device=DEV)
    padded[:, :cols] = x
    v = padded.view(rows, _blocks(cols), BLOCK)
    finite = torch.where(torch.isfinite(v), v.abs(), torch.zeros_like(v))
    mant, e = torch.frexp(finite.amax(2))
    e = torch.where(mant == 0, torch.zeros_like(e), e - shift + (mant > top).to(e.dtype)).clamp(-127, 127)
    inverse = ((127 - e).clamp(0, 254).to(torch.int32) << 23).view(torch.float32)
    inverse = torch.where(e == 127, torch.full_like(inverse, 2.0 ** -127), inverse)
    codes = (v * inverse[:, :, None]).to(kind).view(torch.uint8).view(rows, -1)
    return codes[:, : -(-cols // 16) * 16].contiguous(), (e + 127).to(torch.uint8).t().contiguous()


def _values(codes, scales, cols, fmt):
    """The numbers that codes and scales stand for, in 32 bits."""
    rows = codes.shape[0]
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    s = torch.where(scales == 0, torch.full_like(s, 2.0 ** -127), s)
    v = codes.view(FORMATS[fmt][0]).to(torch.float32)[:, :cols]
    return v * s.t().repeat_interleave(BLOCK, 1)[:, :cols].view(rows, cols)


# ------------------------------------------------------------- plain forms ---
def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (0.5 / 3.141592653589793) ** 0.5
    return torch.ones_like(z)


def _spread(v, state):
    """[rows, C] as [segments, longest, groups, C / groups] with the mask of
    the rows that are there (None where all are)."""
    s, groups = state["segments"], state["groups"]
    if state["offsets"] is None:
        return v.view(s, -1, groups, v.shape[1] // groups), None
    off = state["offsets"].long()
    at = off[:-1, None] + torch.arange(state["longest"], device=DEV)
    mask = at < off[1:, None]
    return v[at.clamp(max=v.shape[0] - 1)].view(s, -1, groups, v.shape[1] // groups), mask


def _gather(v, mask, shape):
    return (v if mask is None else v[mask]).reshape(shape)


def _mean(v, mask):
    if mask is None:
        return v.mean((1, 3), keepdim=True)
    count = mask.sum(1).clamp(min=1) * v.shape[3]
    v = torch.where(mask[:, :, None, None], v, torch.zeros_like(v))
    return v.sum((1, 3), keepdim=True) / count.to(v.dtype).view(-1, 1, 1, 1)


def _plain_norm(state):
    x = state["x"].to(torch.float32)
    v, mask = _spread(x, state)
    mean = _mean(v, mask)
    rstd = 1 / torch.sqrt(_mean((v - mean) ** 2, mask) + EPS)
    z = _gather((v - mean) * rstd, mask, x.shape) * state["weight"] + state["shift"]
    return _act(z, state["act"]).to(state["x"].dtype), mean, rstd


def _plain_train(state):
    y, mean, rstd = _plain_norm(state)
    x = state["x"].to(torch.float32)
    if state["keep"] != "none":
        x = _values(*_quantised(x, state["keep"]), x.shape[1], state["keep"])
    v, mask = _spread(x, state)
    xh = _gather((v - mean) * rstd, mask, x.shape)
    dz = state["dy"].to(torch.float32) * _act_slope(xh * state["weight"] + state["shift"], state["act"])
    xs, _ = _spread(xh, state)
    dh, _ = _spread(dz * state["weight"], state)
    dx = rstd * (dh - _mean(dh, mask) - xs * _mean(dh * xs, mask))
    return {"y": y, "dx": _gather(dx, mask, x.shape).to(state["x"].dtype), "dweight": (dz * xh).sum(0),
            "dbias": dz.sum(0)}


def _plain(state):
    op = state["op"]
    if op == "norm":
        y, mean, rstd = _plain_norm(state)
        return {"y": y, "mean": mean.view(state["segments"], -1), "rstd": rstd.view(state["segments"], -1)}
    if op == "train":
        return _plain_train(state)
    if op == "pack":
        x = state["x"].to(torch.float32)
        return _values(*_quantised(x, state["format"]), x.shape[1], state["format"]).to(torch.bfloat16)
    if op == "gradient":
        return _values(*state["x"], state["cols"], state["format"]).t() @ state["g"].to(torch.float32)
    y = _values(*state["x"], state["cols"], state["x_format"]) @ \
        _values(*state["w"], state["cols"], state["w_format"]).t()
    return (y if state["b"] is None else y + state["b"]).to(DTYPES[state["dtype"]])


def run(state):
    if not own:
        return _plain(state)
    from paper_2608_05033_amd import dense

    op = state["op"]
    if op in ("norm", "train"):
        shape = {"groups": state["groups"], "weight": state["weight"], "bias": state["shift"], "eps": EPS,
                 "activation": state["act"], "segments": state["segments"], "offsets": state["offsets"],
                 "longest": state["longest"]}
        keep = state.get("keep", "none")
        out = dense.group_norm(state["x"], keep=None if keep == "none" else keep, **shape)
        if op == "norm":
            return {"y": out.y, "mean": out.mean, "rstd": out.rstd}
        dx, dweight, dbias = dense.group_norm_backward(state["dy"], out.x, out.mean, out.rstd, **shape)
        return {"y": out.y, "dx": dx, "dweight": dweight, "dbias": dbias}
    if op == "pack":
        return dense.unpack(dense.pack(state["x"], state["format"]), torch.bfloat16)
    x = dense.Packed(*state["x"], state["cols"], state["format" if op == "gradient" else "x_format"])
    if op == "gradient":
        return dense.weight_gradient(x, state["g"])
    w = dense.Packed(*state["w"], state["cols"], state["w_format"])
    return dense.product(x, w, state["b"], DTYPES[state["dtype"]])


# ------------------------------------------------------------------- work ---
def work(case):
    op, rows, d = case["op"], case["rows"], BYTES[case["dtype"]]
    if op in ("norm", "train"):
        c, s = case["channels"], case["segments"]
        stats = 8.0 * s * case["groups"] + 8.0 * c + (4.0 * s if case["ragged"] else 0)
        if op == "norm":
            return {"bytes": 2.0 * d * rows * c + stats, "flops": 12.0 * rows * c}
        kept = d * rows * c if case["keep"] == "none" else rows * c + rows * _blocks(c)
        # x read, y and the kept input written; dy and the kept input read, dx written
        written = 0 if case["keep"] == "none" else kept
        return {"bytes": 4.0 * d * rows * c + written + kept + 2 * stats + 8.0 * c, "flops": 36.0 * rows * c}
    cols = case["cols"]
    packed = 1.0 * rows * cols + rows * _blocks(cols)
    if op == "pack":
        return {"bytes": (d + 2.0) * rows * cols + 2 * packed, "flops": 4.0 * rows * cols}
    n = case["n"]
    if op == "gradient":
        return {"bytes": packed + 1.0 * d * rows * n + 4.0 * cols * n, "flops": 2.0 * rows * cols * n}
    return {"bytes": packed + n * cols + n * _blocks(cols) + (4.0 * n if case["bias"] else 0) + 1.0 * d * rows * n,
            "flops": 2.0 * rows * cols * n}


# ------------------------------------------------------------------ exact ---
def _power(e):
    """2^e in 64 bits, for whole numbers e of any type (pow need not be exact)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(x, fmt):
    """What 64-bit `x` becomes in 8 bits, from the definition: the least power of
    two that brings a block's largest value into range, then the nearest of the
    format's numbers, ties to even."""
    _, top, shift, bits, least = FORMATS[fmt]
    out = torch.empty_like(x)
    for b in range(_blocks(x.shape[1])):
        v = x[:, b * BLOCK:(b + 1) * BLOCK]
        most = v.abs().amax(1, keepdim=True)
        limit = torch.tensor(top * 2.0 ** shift, dtype=torch.float64, device=DEV)
        e = torch.ceil(torch.log2(most / limit)).clamp(-127, 127)
        e = torch.where(most > limit * _power(e), e + 1, e)
        e = torch.where(most <= limit * _power(e - 1), e - 1, e).clamp(-127, 127)
        e = torch.where(most == 0, torch.zeros_like(e), e)
        u = v / _power(e)
        step = _power(torch.frexp(u.abs().clamp(min=2.0 ** least))[1] - 1 - bits)
        out[:, b * BLOCK:(b + 1) * BLOCK] = torch.round(u / step) * step * _power(e)
    return out


def _exact_from_codes(codes, scales, cols, fmt):
    """64-bit values of codes, field by field."""
    _, _, _, bits, least = FORMATS[fmt]
    c = codes[:, :cols].to(torch.int64)
    field, mant = (c >> bits) & ((1 << (7 - bits)) - 1), (c & ((1 << bits) - 1)).double()
    v = torch.where(field == 0, mant * 2.0 ** (least - bits),
                    (1 + mant * 2.0 ** -bits) * _power(field + (least - 1)))
    v = torch.where(c >= 128, -v, v)
    block = torch.arange(cols, device=DEV) // BLOCK
    return v * _power(scales.t()[:, block].to(torch.int64) - 127)


def exact(case, seed):
    state = prepare(case, seed)
    op = state["op"]
    if op == "pack":
        return _exact_values(state["x"].double(), case["format"])
    if op == "gradient":
        x = _exact_from_codes(*state["x"], case["cols"], case["format"])
        return x.t().contiguous() @ state["g"].double()
    if op == "product":
        y = _exact_from_codes(*state["x"], case["cols"], case["x_format"]) @ \
            _exact_from_codes(*state["w"], case["cols"], case["w_format"]).t().contiguous()
        return y if state["b"] is None else y + state["b"].double()
    x, rows, groups, s = state["x"].double(), case["rows"], case["groups"], case["segments"]
    c = case["channels"]
    # segment of each row, and sums over segments through running sums' differences where they are ragged
    if state["offsets"] is None:
        off = torch.arange(s + 1, device=DEV) * (rows // s)
    else:
        off = state["offsets"].long()
    length = off[1:] - off[:-1]
    of_row = torch.repeat_interleave(torch.arange(s, device=DEV), length)
    count = (length.clamp(min=1) * (c // groups)).double()[:, None]

    def sums(v):  # [rows, C] -> [segments, groups]
        v = v.reshape(rows, groups, -1).sum(2)
        if s == 1:
            return v.sum(0, keepdim=True)
        return torch.zeros(s, groups, dtype=torch.float64, device=DEV).index_add_(0, of_row, v)

    def rows_of(v):  # [segments, groups] -> [rows, C]
        return (v.expand(rows, -1) if s == 1 else v[of_row]).repeat_interleave(c // groups, 1)

    mean = sums(x) / count
    var = sums((x - rows_of(mean)) ** 2) / count
    rstd = (var + EPS) ** -0.5
    w, b = state["weight"].double(), state["shift"].double()
    act = case["act"]

    def value_and_slope(z):
        if act == "relu":
            return z * (z > 0), (z > 0).double()
        if act == "silu":
            p = torch.sigmoid(z)
            return z * p, p + z * p * (1 - p)
        if act == "gelu":
            p = 0.5 * torch.erfc(-z / 2.0 ** 0.5)
            return z * p, p + z * torch.exp(-z * z / 2) / (2 * 3.141592653589793) ** 0.5
        return z, torch.ones_like(z)

    y = value_and_slope((x - rows_of(mean)) * rows_of(rstd) * w + b)[0]
    if op == "norm":
        return {"y": y, "mean": mean, "rstd": rstd}
    kept = x if case["keep"] == "none" else _exact_values(x, case["keep"])
    xh = (kept - rows_of(mean)) * rows_of(rstd)
    dz = state["dy"].double() * value_and_slope(xh * w + b)[1]
    dh = dz * w
    dx = rows_of(rstd) * (dh - rows_of(sums(dh) / count) - xh * rows_of(sums(dh * xh) / count))
    return {"y": y, "dx": dx, "dweight": (dz * xh).sum(0), "dbias": dz.sum(0)}
