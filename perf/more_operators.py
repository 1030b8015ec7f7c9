"""Operator cases: 4-bit tables and their products, and rows sorted by expert.

Every case names an operator and the sizes of one call.

Operators:
* ``pack``      a table to 4 bits with a power-of-two scale for each row and 32
                columns, and back;
* ``product``   X.W^T of two such tables, with a bias where one is given;
* ``linear``    a layer's transform in 4 bits as a training step uses it: X.W, and
                from a given output gradient the gradients of X and W, every
                operand rounded to 4 bits along the sum;
* ``experts``   rows of a 4-bit table, each through the 4-bit weights of the
                experts chosen for it;
* ``exchange``  rows sorted by expert and the experts' results brought back with
                weights: forward, or (``train``) forward and all gradients.

All inputs are drawn on the GPU from the seed with torch.
"""
from __future__ import annotations

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 32  # columns that share a scale
GROUP = 128  # columns whose four scales lie together
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of the codes 0 to 7; 8 to 15 are negative


# ------------------------------------------------------------------ cases ---
def listed():
    return [
        # an odd feature table of a small graph
        {"name": "pack_odd", "op": "pack", "rows": 4999, "cols": 601, "dtype": "f16"},
        # a layer's activations on a middling graph
        {"name": "pack_262k", "op": "pack", "rows": 1 << 18, "cols": 128, "dtype": "f32"},
        # one node through a wide layer: the weights are read once, latency counts
        {"name": "product_one_row", "op": "product", "rows": 1, "cols": 4096, "n": 4096, "dtype": "bf16",
         "bias": True},
        # the last layer of a small graph with odd features and classes
        {"name": "product_odd", "op": "product", "rows": 5003, "cols": 601, "n": 47, "dtype": "f16", "bias": True},
        # wide layers over many nodes: bound by the matrix units
        {"name": "product_large", "op": "product", "rows": 8192, "cols": 8192, "n": 8192, "dtype": "bf16",
         "bias": False},
        # a training step of one layer's transform on a middling graph
        {"name": "linear_262k", "op": "linear", "rows": 1 << 18, "cols": 256, "n": 128, "dtype": "f32"},
        # one row through 8 of 64 experts, as an answer to one request: their weights are read once
        {"name": "experts_one_row", "op": "experts", "rows": 1, "k": 8, "experts": 64, "cols": 2048, "n": 1024,
         "dtype": "bf16", "bias": False},
        # nodes of eight types that differ in number, odd sizes, a bias for each type
        {"name": "experts_odd", "op": "experts", "rows": 5003, "k": 1, "experts": 8, "cols": 601, "n": 257,
         "dtype": "f32", "bias": True},
        # a batch through two of sixteen wide experts: bound by the matrix units
        {"name": "experts_large", "op": "experts", "rows": 16384, "k": 2, "experts": 16, "cols": 4096, "n": 4096,
         "dtype": "bf16", "bias": False},
        # a handful of rows to their experts and back: launch latency
        {"name": "exchange_few", "op": "exchange", "rows": 37, "k": 2, "experts": 16, "cols": 64, "dtype": "bf16",
         "train": False, "drop": False},
        # a training step on a middling graph, two experts a row
        {"name": "exchange_262k", "op": "exchange", "rows": 1 << 18, "k": 2, "experts": 8, "cols": 128,
         "dtype": "f32", "train": True, "drop": False},
        # a training step of odd width through many experts, some of which are full and turn rows away
        {"name": "exchange_odd", "op": "exchange", "rows": 20011, "k": 4, "experts": 60, "cols": 601,
         "dtype": "bf16", "train": True, "drop": True},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(low * (high / low) ** rng.random()))))


def draw(rng):
    op = rng.choice(("pack", "product", "linear", "experts", "exchange"))
    dtype = rng.choice(("f32", "bf16", "f16"))
    if op == "pack":
        cols = _log_int(rng, 1, 4096)
        return {"op": op, "rows": _log_int(rng, 1, min(1 << 21, (1 << 28) // cols)), "cols": cols, "dtype": dtype}
    if op == "exchange":
        experts = _log_int(rng, 1, 256)
        k = rng.randint(1, min(8, experts))
        cols = _log_int(rng, 1, 2048)
        return {"op": op, "rows": _log_int(rng, 1, min(1 << 19, (1 << 26) // (cols * k))), "k": k,
                "experts": experts, "cols": cols, "dtype": dtype, "train": rng.random() < 0.5,
                "drop": rng.random() < 0.5}
    if op == "linear":
        cols, n = _log_int(rng, 16, 1024), _log_int(rng, 8, 1024)
        return {"op": op, "rows": _log_int(rng, 1, min(1 << 19, (1 << 26) // max(cols, n))), "cols": cols, "n": n,
                "dtype": dtype}
    cols, n = _log_int(rng, 16, 4096), _log_int(rng, 8, 4096)
    if op == "product":
        rows = _log_int(rng, 1, min(1 << 21, (1 << 28) // max(cols, n), 500_000_000_000 // (cols * n)))
        return {"op": op, "rows": rows, "cols": cols, "n": n, "dtype": dtype, "bias": rng.random() < 0.5}
    experts = _log_int(rng, 1, max(1, min(128, (1 << 28) // (cols * n))))
    k = rng.randint(1, min(8, experts))
    rows = _log_int(rng, 1, max(1, min(1 << 18, (1 << 27) // (k * max(cols, n)), 500_000_000_000 // (k * cols * n))))
    return {"op": op, "rows": rows, "k": k, "experts": experts, "cols": cols, "n": n, "dtype": dtype,
            "bias": rng.random() < 0.5}


# ----------------------------------------------------------------- inputs ---
def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _chosen(g, case):
    """The k experts of each row that score highest, some experts more in demand than others."""
    scores = _normal(g, case["rows"], case["experts"]) + 0.5 * _normal(g, case["experts"])
    return torch.topk(scores, case["k"], dim=1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    op, rows, cols = case["op"], case["rows"], case["cols"]
    state, dtype = dict(case), DTYPES[case["dtype"]]
    if op == "pack":
        # magnitudes that differ from row to row, some entries cut to 0 by an activation
        x = _normal(g, rows, cols) * torch.exp(_normal(g, rows, 1))
        x[:, ::3] = x[:, ::3].clamp_min(0)
        state["x"] = x.to(dtype)
        return state
    if op == "exchange":
        scores, chosen = _chosen(g, case)
        if case["drop"]:
            chosen = torch.where(torch.rand(chosen.shape, generator=g, device=DEV) < 1 / 16,
                                 torch.full_like(chosen, -1), chosen)
        state["chosen"] = chosen.contiguous()
        state["weights"] = torch.softmax(scores, 1).contiguous()
        state["x"] = _normal(g, rows, cols, dtype=dtype)
        state["y"] = _normal(g, rows * case["k"], cols, dtype=dtype)
        if case["train"]:
            state["dsorted"] = (0.1 * _normal(g, rows * case["k"], cols)).to(dtype)
            state["dout"] = (0.1 * _normal(g, rows, cols)).to(dtype)
        return state
    if op == "linear":
        state["x"] = (_normal(g, rows, cols) * torch.exp(0.5 * _normal(g, rows, 1))).to(dtype)
        state["w"] = _normal(g, cols, case["n"]) * cols ** -0.5
        state["dz"] = 0.1 * _normal(g, rows, case["n"])
        return state
    state["x"] = _quantised(_normal(g, rows, cols) * torch.exp(0.5 * _normal(g, rows, 1)))
    if op == "product":
        state["w"] = _quantised(_normal(g, case["n"], cols) * cols ** -0.5)
        state["b"] = _normal(g, case["n"]) if case["bias"] else None
        return state
    state["w"] = _quantised(_normal(g, case["experts"] * case["n"], cols) * cols ** -0.5)
    state["b"] = _normal(g, case["experts"], case["n"]) if case["bias"] else None
    state["chosen"] = _chosen(g, case)[1].contiguous()
    return state


def _ceil(a, b):
    return -(-a // b)


def _quantised(x):
    """Codes [rows, bytes up to a multiple of 16], two in a byte, the even column
    in its lower half, and scale bytes [groups of 128 columns, rows, 4], 127 for a
    scale of 1 and past the last block."""
    rows, cols = x.shape
    groups = _ceil(cols, GROUP)
    padded = torch.zeros(rows, groups * GROUP, device=DEV)
    padded[:, :cols] = x
    v = padded.view(rows, groups * 4, BLOCK)
    most = v.abs().amax(2)
    # the least e with most <= 6 * 2^e; 6 is 0.75 * 2^3
    mant, e = torch.frexp(most)
    e = torch.where(mant == 0, torch.zeros_like(e), e - 3 + (mant > 0.75).to(e.dtype)).clamp(min=-127)
    # in two steps: 2^-e itself need not fit 32 bits
    half = torch.div(e, 2, rounding_mode="floor")
    u = torch.ldexp(torch.ldexp(v, -half[:, :, None]), (half - e)[:, :, None])
    a = u.abs()
    # between neighbours ties go to the even code
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75).to(torch.uint8) + (a > 1.25).to(torch.uint8) + \
        (a >= 1.75).to(torch.uint8) + (a > 2.5).to(torch.uint8) + (a >= 3.5).to(torch.uint8) + (a > 5).to(torch.uint8)
    code = code + 8 * torch.signbit(u).to(torch.uint8)
    bad = ~torch.isfinite(most)
    code = torch.where(bad[:, :, None], torch.zeros_like(code), code).view(rows, -1, 2)
    s = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    codes = (code[:, :, 0] + 16 * code[:, :, 1])[:, : _ceil(cols, BLOCK) * 16].contiguous()
    return codes, s.view(rows, groups, 4).transpose(0, 1).contiguous()


def _values(codes, scales, cols):
    """The numbers that codes and scales stand for, in 32 bits."""
    rows = codes.shape[0]
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=DEV)
    both = torch.stack([codes & 15, codes >> 4], 2).view(rows, -1)[:, :cols]
    v = grid[both.to(torch.int32)]
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    s = torch.where(scales == 0, torch.full_like(s, 2.0 ** -127), s)
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return v * s.transpose(0, 1).reshape(rows, -1).repeat_interleave(BLOCK, 1)[:, :cols]


# ------------------------------------------------------------- plain forms ---
def _plain_route(chosen, experts):
    """offsets [experts + 1], place [rows, k] and source [rows * k]: entries in
    the order of their experts, those of an expert in the order of their rows."""
    rows, k = chosen.shape
    flat = chosen.reshape(-1)
    key = torch.where((flat >= 0) & (flat < experts), flat, torch.full_like(flat, experts))
    ordered, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(ordered, torch.arange(experts + 1, device=DEV)).to(torch.int32)
    there = ordered < experts
    place = torch.empty_like(order)
    place[order] = torch.where(there, torch.arange(rows * k, device=DEV), torch.full_like(order, -1))
    source = torch.where(there, order // k, torch.full_like(order, -1))
    return offsets, place.view(rows, k).to(torch.int32), source.to(torch.int32)


def _take(v, at):
    """Rows of v in 32 bits, zeros where `at` is negative."""
    out = v.to(torch.float32)[at.clamp(min=0).long()]
    return torch.where(at[:, None] >= 0, out, torch.zeros_like(out))


def _plain_exchange(state):
    chosen, w, dtype, k = state["chosen"], state["weights"], DTYPES[state["dtype"]], state["k"]
    offsets, place, source = _plain_route(chosen, state["experts"])
    y = state["y"]
    out = sum(w[:, j:j + 1] * _take(y, place[:, j]) for j in range(k)).to(dtype)
    res = {"offsets": offsets, "place": place, "source": source, "sorted": _take(state["x"], source).to(dtype),
           "out": out}
    if state["train"]:
        dout = state["dout"].to(torch.float32)
        res["dx"] = sum(_take(state["dsorted"], place[:, j]) for j in range(k)).to(dtype)
        res["dweights"] = torch.stack([(dout * _take(y, place[:, j])).sum(1) for j in range(k)], 1)
        dy = torch.zeros(y.shape, device=DEV)
        for j in range(k):
            there = place[:, j] >= 0
            dy[place[:, j][there].long()] = (w[:, j:j + 1] * dout)[there]
        res["dy"] = dy.to(dtype)
    return res


def _plain_experts(state):
    n, cols = state["n"], state["cols"]
    offsets, _, source = _plain_route(state["chosen"], state["experts"])
    x, w = _values(*state["x"], cols), _values(*state["w"], cols)
    y = torch.empty(source.numel(), n, dtype=DTYPES[state["dtype"]], device=DEV)
    off = offsets.tolist()
    for e in range(state["experts"]):
        rows = slice(off[e], off[e + 1])
        if rows.start < rows.stop:
            part = x[source[rows].long()] @ w[e * n:(e + 1) * n].t()
            y[rows] = (part if state["b"] is None else part + state["b"][e]).to(y.dtype)
    return y


def _plain_linear(state):
    x, w, dz = state["x"].to(torch.float32), state["w"], state["dz"]

    def rounded(v):
        return _values(*_quantised(v), v.shape[1])

    z = rounded(x) @ rounded(w.t()).t()
    dx = rounded(dz) @ rounded(w).t()
    dw = rounded(x.t()) @ rounded(dz.t()).t()
    return {"z": z, "dx": dx.to(state["x"].dtype), "dw": dw}


def _plain(state):
    op = state["op"]
    if op == "exchange":
        return _plain_exchange(state)
    if op == "experts":
        return _plain_experts(state)
    if op == "linear":
        return _plain_linear(state)
    if op == "pack":
        x = state["x"].to(torch.float32)
        return _values(*_quantised(x), x.shape[1]).to(torch.bfloat16)
    y = _values(*state["x"], state["cols"]) @ _values(*state["w"], state["cols"]).t()
    return (y if state["b"] is None else y + state["b"]).to(DTYPES[state["dtype"]])


def run(state):
    if not own:
        return _plain(state)
    from paper_2608_05033_amd import dense, experts, gcn

    op = state["op"]
    if op == "pack":
        return dense.unpack4(dense.pack4(state["x"]), torch.bfloat16)
    if op == "linear":
        x, w = state["x"].detach().requires_grad_(), state["w"].detach().requires_grad_()
        z = gcn.transform4(x, w)
        dx, dw = torch.autograd.grad(z, (x, w), state["dz"])
        return {"z": z.detach(), "dx": dx, "dw": dw}
    if op == "exchange":
        route = experts.route(state["chosen"], state["experts"])
        res = {"offsets": route.offsets, "place": route.place, "source": route.source}
        x, y, w = state["x"], state["y"], state["weights"]
        if state["train"]:
            x, y, w = x.detach().requires_grad_(), y.detach().requires_grad_(), w.detach().requires_grad_()
        there, out = experts.dispatch(x, route), experts.combine(y, route, w)
        res.update({"sorted": there.detach(), "out": out.detach()})
        if state["train"]:
            res["dx"], res["dy"], res["dweights"] = torch.autograd.grad((there, out), (x, y, w),
                                                                        (state["dsorted"], state["dout"]))
        return res
    x, w = dense.Packed4(*state["x"], state["cols"]), dense.Packed4(*state["w"], state["cols"])
    if op == "product":
        return dense.product4(x, w, state["b"], DTYPES[state["dtype"]])
    route = experts.route(state["chosen"], state["experts"])
    return experts.product(x, w, route, state["b"], DTYPES[state["dtype"]])


# ------------------------------------------------------------------- work ---
def _packed(rows, cols):
    return 0.5 * rows * cols + 1.0 * rows * _ceil(cols, BLOCK)


def work(case):
    op, rows, cols, d = case["op"], case["rows"], case["cols"], BYTES[case["dtype"]]
    if op == "pack":
        return {"bytes": (d + 2.0) * rows * cols + 2 * _packed(rows, cols), "flops": 4.0 * rows * cols}
    if op == "exchange":
        k = case["k"]
        table = 1.0 * d * rows * cols
        # experts read; offsets, places and sources written; x read, its copies written; results read, sums written
        total = (8.0 + 4 + 4) * rows * k + 4.0 * (case["experts"] + 1) + 4.0 * rows * k + table * (2 + 2 * k)
        if case["train"]:  # the sorted copies' gradients read, dx written; the sums' gradient read, dy and dw written
            total += table * (k + 1) + table * (1 + k) + 4.0 * rows * k
        return {"bytes": total, "flops": (2.0 + (4.0 if case["train"] else 0)) * rows * k * cols}
    n = case["n"]
    if op == "linear":
        return {"bytes": 2.0 * d * rows * cols + 8.0 * rows * n + 8.0 * cols * n, "flops": 6.0 * rows * cols * n}
    if op == "product":
        return {"bytes": _packed(rows, cols) + _packed(n, cols) + (4.0 * n if case["bias"] else 0) + d * rows * n,
                "flops": 2.0 * rows * cols * n}
    k, experts = case["k"], case["experts"]
    used = min(experts, rows * k)
    return {"bytes": _packed(rows, cols) + _packed(used * n, cols) + (4.0 * used * n if case["bias"] else 0) +
            1.0 * d * rows * k * n + (8.0 + 4 + 4) * rows * k, "flops": 2.0 * rows * k * cols * n}


# ------------------------------------------------------------------ exact ---
def _power(e):
    """2^e in 64 bits, for whole numbers e of any type (pow need not be exact)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(x):
    """What 64-bit `x` becomes in 4 bits, from the definition: the least power of
    two that brings a block's largest value to at most 6, then the nearest of the
    format's numbers (halves up to 2, whole ones up to 4, even ones up to 6),
    ties to even."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], BLOCK):
        v = x[:, c:c + BLOCK]
        most = v.abs().amax(1, keepdim=True)
        e = torch.ceil(torch.log2(most / 6.0)).clamp(-127, 127)
        e = torch.where(most > 6.0 * _power(e), e + 1, e)
        e = torch.where(most <= 6.0 * _power(e - 1), e - 1, e).clamp(-127, 127)
        e = torch.where(most == 0, torch.zeros_like(e), e)
        u = v / _power(e)
        a = u.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
        out[:, c:c + BLOCK] = torch.round(u / step) * step * _power(e)
    return out


def _exact_from_codes(codes, scales, cols):
    """64-bit values of codes, field by field."""
    c = torch.arange(cols, device=DEV)
    half = (codes[:, c // 2].to(torch.int64) >> (4 * (c % 2))) & 15
    field, mant = (half >> 1) & 3, (half & 1).double()
    v = torch.where(field == 0, 0.5 * mant, (1 + 0.5 * mant) * _power(field - 1))
    v = torch.where(half >= 8, -v, v)
    s = scales[c // GROUP, :, (c // BLOCK) % 4].t().to(torch.int64)
    return torch.where(s == 255, torch.full_like(v, float("nan")), v * _power(s - 127))


def _exact_order(chosen, experts):
    """Sorted entries as a list of (row, slot), and where each expert's begin, from a walk on the host."""
    lists = [[] for _ in range(experts)]
    for t, row in enumerate(chosen.tolist()):
        for j, e in enumerate(row):
            if 0 <= e < experts:
                lists[e].append((t, j))
    begin = [0]
    for entries in lists:
        begin.append(begin[-1] + len(entries))
    return [entry for entries in lists for entry in entries], begin


def exact(case, seed):
    state = prepare(case, seed)
    op, cols = state["op"], case["cols"]
    if op == "pack":
        return _exact_values(state["x"].double())
    if op == "product":
        y = _exact_from_codes(*state["x"], cols) @ _exact_from_codes(*state["w"], cols).t().contiguous()
        return y if state["b"] is None else y + state["b"].double()
    if op == "linear":
        x, w, dz = state["x"].double(), state["w"].double(), state["dz"].double()
        q = _exact_values
        return {"z": q(x) @ q(w.t().contiguous()).t().contiguous(), "dx": q(dz) @ q(w).t().contiguous(),
                "dw": q(x.t().contiguous()) @ q(dz.t().contiguous()).t().contiguous()}
    order, begin = _exact_order(state["chosen"], case["experts"])
    at = torch.tensor(order, dtype=torch.int64).view(-1, 2).to(DEV)
    row, slot, total = at[:, 0], at[:, 1], case["rows"] * case["k"]
    if op == "experts":
        n = case["n"]
        x, y = _exact_from_codes(*state["x"], cols), torch.zeros(total, n, dtype=torch.float64, device=DEV)
        for e in range(case["experts"]):
            b, end = begin[e], begin[e + 1]
            if b < end:
                w = _exact_from_codes(state["w"][0][e * n:(e + 1) * n],
                                      state["w"][1][:, e * n:(e + 1) * n], cols)
                y[b:end] = x[row[b:end]] @ w.t().contiguous()
                if state["b"] is not None:
                    y[b:end] += state["b"][e].double()
        return y
    have, y, w = len(order), state["y"].double(), state["weights"].double()
    out = torch.zeros(case["rows"], cols, dtype=torch.float64, device=DEV)
    out.index_add_(0, row, w[row, slot][:, None] * y[:have])
    there = torch.zeros(total, cols, dtype=torch.float64, device=DEV)
    there[:have] = state["x"].double()[row]
    res = {"offsets": None, "place": None, "source": None, "sorted": there, "out": out}
    if case["train"]:
        dout = state["dout"].double()
        res["dx"] = torch.zeros_like(out).index_add_(0, row, state["dsorted"].double()[:have])
        res["dweights"] = torch.zeros(case["rows"], case["k"], dtype=torch.float64, device=DEV)
        res["dweights"][row, slot] = (dout[row] * y[:have]).sum(1)
        res["dy"] = torch.zeros_like(there)
        res["dy"][:have] = w[row, slot][:, None] * dout[row]
    return res
