"""Rows through the experts (or by the types) that were chosen for them.

    r = route(chosen, experts)              chosen [rows, k]: entries sorted by expert
    xs = dispatch(x, r)                     the rows in that order          (gradients)
    out = combine(ys, r, weights)           the results back, weighted      (gradients)
    ys = product(pack4(x), W4, r)           all experts' products in 4 bits, from the
                                            unsorted rows; W4 = pack4(W.view(experts * n, cols))

Arguments are checked here and in the library; every call runs on the current
stream of its tensors' device, and results and workspaces are torch tensors of
that stream.  `dispatch` and `combine` record gradients where torch does; a step that
is captured into a graph takes leaves of its own (x.detach().requires_grad_()), since
torch ties a leaf to the stream that it was first used on.  Forward derivatives are
refused.  A trace (torch.jit.trace) holds `dispatch` and `combine` with the route that
they were given; `route` and `product` are not for one.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import _check, _lib, sd_route_t
from .autograd import first_derivatives_only
from .dense import TYPES, Packed4, _float32, _on_its_device, _raw_stream, _table, _uint8

_int32 = torch.int32
_forward = torch.autograd.forward_ad
_tracing = torch._C._get_tracing_state
_INDEX_BYTES = {torch.int32: 4, torch.int64: 8}


class Route:
    """Entries (t, j) of a table [rows, k] of chosen experts, sorted by expert, then
    t, then j: offsets int32 [experts + 1] (expert e has the entries from offsets[e]
    to offsets[e + 1]), place int32 [rows, k] (an entry's place among them, -1
    without an expert) and source int32 [rows * k] (the row of the i-th entry, -1
    behind the last)."""

    __slots__ = ("_offsets", "_place", "_source", "_store", "rows", "k", "experts", "index", "c")

    def __init__(self, offsets, place, source):
        index = offsets.get_device()
        for v, what, dims in ((offsets, "offsets", 1), (place, "place", 2), (source, "source", 1)):
            if v.dtype != _int32 or v.dim() != dims or v.get_device() != index or index < 0 or not v.is_contiguous():
                raise ValueError(f"{what} must be a contiguous int32 tensor of {dims} dimensions, all on one GPU")
        rows, k = place.shape
        if k < 1 or offsets.numel() < 2 or source.numel() != rows * k:
            raise ValueError(f"offsets, place and source must be [experts + 1], [rows, k] and [rows * k], got "
                             f"{tuple(offsets.shape)}, {tuple(place.shape)} and {tuple(source.shape)}")
        _fits(k, offsets.numel() - 1)
        self._offsets, self._place, self._source, self._store = offsets, place, source, None
        self.rows, self.k, self.experts, self.index = rows, k, offsets.numel() - 1, index
        self.c = sd_route_t(rows, k, self.experts, offsets.data_ptr(), place.data_ptr(), source.data_ptr())

    @classmethod
    def empty(cls, rows: int, k: int, experts: int, like):
        """A new one on the device of the tensor `like`: one allocation, whose parts
        become tensors of their own when they are asked for."""
        store = like.new_empty(experts + 1 + 2 * rows * k, dtype=_int32)
        r, at = cls.__new__(cls), store.data_ptr()
        r._offsets, r._place, r._source, r._store = None, None, None, store
        r.rows, r.k, r.experts, r.index = rows, k, experts, store.get_device()
        place = at + 4 * (experts + 1)
        r.c = sd_route_t(rows, k, experts, at, place, place + 4 * rows * k)
        return r

    def kept(self):
        """The tensors that hold it, for autograd to watch."""
        return (self._offsets, self._place, self._source) if self._store is None else (self._store,)

    @property
    def offsets(self):
        if self._offsets is None:
            self._offsets = self._store.as_strided((self.experts + 1,), (1,))
        return self._offsets

    @property
    def place(self):
        if self._place is None:
            self._place = self._store.as_strided((self.rows, self.k), (self.k, 1), self.experts + 1)
        return self._place

    @property
    def source(self):
        if self._source is None:
            entries = self.rows * self.k
            self._source = self._store.as_strided((entries,), (1,), self.experts + 1 + entries)
        return self._source

    @property
    def device(self):
        return (self._offsets if self._store is None else self._store).device

    def get_device(self) -> int:
        return self.index


def _fits(k, experts):
    """Both are 32 bits wide in the library, and ctypes would cut off what is above."""
    if not (k < 1 << 31 and -(1 << 31) <= experts < 1 << 31):
        raise ValueError(f"the experts of a row and all experts must be fewer than 2^31, got {k} and {experts}")


@functools.lru_cache(maxsize=4096)
def _route_size(rows, k, experts):
    _fits(k, experts)
    size = ctypes.c_size_t()
    _check(_lib.sd_route_size(rows, k, experts, size), "sd_route_size")
    return size.value


@_on_its_device
def route(chosen, experts: int) -> Route:
    """chosen: int32 or int64 [rows, k] on the GPU (as torch.topk gives it); numbers
    outside [0, experts) are entries without an expert.  experts: at most 4095."""
    if chosen.dim() != 2 or chosen.dtype not in _INDEX_BYTES or not chosen.is_cuda or not chosen.is_contiguous() or \
            chosen.shape[1] < 1:
        raise ValueError(f"chosen must be a contiguous int32 or int64 [rows, k] on the GPU, got {chosen.dtype} "
                         f"{tuple(chosen.shape)} on {chosen.device}")
    rows, k = chosen.shape
    size = _route_size(rows, k, experts)
    r = Route.empty(rows, k, experts, chosen)
    work = chosen.new_empty(size, dtype=_uint8) if size else None  # lives until the call has been enqueued
    _check(_lib.sd_route(chosen.data_ptr(), _INDEX_BYTES[chosen.dtype], r.c, work.data_ptr() if size else None, size,
                         _raw_stream(r.index)), "sd_route")
    return r


def _rows_of(x, rows, route, what):
    stride = _table(x, what)
    if x.shape[0] != rows or x.get_device() != route.index:
        raise ValueError(f"{what} must have {rows} rows on {route.device}, got {tuple(x.shape)} on {x.device}")
    return stride


@_on_its_device
def _dispatch(x, route):
    stride = _rows_of(x, route.rows, route, "x")
    cols = x.shape[1]
    y = x.new_empty((route.rows * route.k, cols))
    _check(_lib.sd_dispatch(route.c, x.data_ptr(), TYPES[x.dtype], cols, stride, y.data_ptr(), cols,
                            _raw_stream(route.index)), "sd_dispatch")
    return y


def _weights_of(weights, route):
    if weights is None:
        return None
    if weights.shape != (route.rows, route.k) or weights.dtype != _float32 or weights.get_device() != route.index or \
            not weights.is_contiguous():
        raise ValueError(f"weights must be contiguous float32 [{route.rows}, {route.k}] on {route.device}, got "
                         f"{weights.dtype} {tuple(weights.shape)} on {weights.device}")
    return weights.data_ptr()


@_on_its_device
def _combine(y, route, weights):
    stride = _rows_of(y, route.rows * route.k, route, "y")
    weights = _weights_of(weights, route)
    cols = y.shape[1]
    out = y.new_empty((route.rows, cols))
    _check(_lib.sd_combine(route.c, y.data_ptr(), TYPES[y.dtype], cols, stride, weights, out.data_ptr(), cols,
                           _raw_stream(route.index)), "sd_combine")
    return out


@_on_its_device
def combine_backward(dout, y, route: Route, weights=None, need_dy: bool = True, need_dweights: bool = True):
    """(dy, dweights) of `combine` from its result's gradient, None where not needed;
    y is read for dweights alone and may be None without them."""
    stride = _rows_of(dout, route.rows, route, "dout")
    cols, total = dout.shape[1], route.rows * route.k
    at = _weights_of(weights, route)
    y_at, y_stride = None, 0
    if need_dweights:
        y_stride = _rows_of(y, total, route, "y")
        if y.dtype != dout.dtype or y.shape[1] != cols:
            raise ValueError(f"y must be {dout.dtype} [{total}, {cols}], got {y.dtype} {tuple(y.shape)}")
        y_at = y.data_ptr()
    dy = dout.new_empty((total, cols)) if need_dy else None
    dweights = dout.new_empty((route.rows, route.k), dtype=_float32) if need_dweights else None
    _check(_lib.sd_combine_backward(route.c, dout.data_ptr(), TYPES[dout.dtype], cols, stride, y_at, y_stride, at,
                                    dy.data_ptr() if need_dy else None, cols,
                                    dweights.data_ptr() if need_dweights else None, _raw_stream(route.index)),
           "sd_combine_backward")
    return dy, dweights


# A route is kept whole, and its tensors as saved ones: one that was written to in
# the meantime is found when they are asked for.
class _Dispatch(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, route):
        ctx.route = route
        ctx.save_for_backward(*route.kept())
        return _dispatch(x, route)

    @staticmethod
    def backward(ctx, dy):
        ctx.saved_tensors
        return combine(dy.contiguous(), ctx.route), None


class _Sum(torch.autograd.Function):
    """combine without weights."""

    @staticmethod
    def forward(ctx, y, route):
        ctx.route = route
        ctx.save_for_backward(*route.kept())
        return _combine(y, route, None)

    @staticmethod
    def backward(ctx, dout):
        ctx.saved_tensors
        return dispatch(dout.contiguous(), ctx.route), None


class _WeightedSum(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, weights, route):
        ctx.route = route
        ctx.save_for_backward(weights if ctx.needs_input_grad[0] else None, y if ctx.needs_input_grad[1] else None,
                              *route.kept())
        return _combine(y, route, weights)

    @staticmethod
    @first_derivatives_only
    def backward(ctx, kept, dout):
        weights, y = kept[:2]
        need_dy, need_dweights = ctx.needs_input_grad[:2]
        return *combine_backward(dout.contiguous(), y, ctx.route, weights, need_dy, need_dweights), None


def _watched():
    """Whether torch may be following tensors by other ways than gradients: inside a
    level of forward derivatives, which it refuses here, or in a trace.  Asked for in
    0.2 us, a tensor for its tangent in 0.4."""
    return getattr(_forward, "_current_level", 0) >= 0 or _tracing() is not None


def dispatch(x: torch.Tensor, route: Route) -> torch.Tensor:
    """x's rows in the order of the route, [rows * k, cols]; zeros behind the last entry."""
    if x.requires_grad and torch.is_grad_enabled() or _watched():
        return _Dispatch.apply(x, route)
    return _dispatch(x, route)


def combine(y: torch.Tensor, route: Route, weights=None) -> torch.Tensor:
    """out[t] = the sum over j of weights[t, j] times the row of y that entry (t, j) is
    sorted to (weights None: 1), [rows, cols] in y's type, summed in 32 bits.  Gradients
    for y and for weights, which are float32 [rows, k]; with weights no second ones."""
    if torch.is_grad_enabled() and (y.requires_grad or weights is not None and weights.requires_grad) or \
            _watched():
        return _Sum.apply(y, route) if weights is None else _WeightedSum.apply(y, weights, route)
    return _combine(y, route, weights)


@_on_its_device
def product(x: Packed4, w: Packed4, route: Route, bias=None, dtype=torch.float32, sorted: bool = False) -> torch.Tensor:
    """Each entry's row of x through its expert's weights, [rows * k, n] in the order of
    the route: x [rows, cols] (or, with sorted=True, [rows * k, cols] in that order)
    and w [experts * n, cols] in 4 bits, bias float32 [experts, n]; zeros behind the
    last entry."""
    total = route.rows * route.k
    if x.index != w.index or x.index != route.index or x.cols != w.cols or w.rows % route.experts or \
            x.rows != (total if sorted else route.rows):
        raise ValueError(f"x, w and the route must fit on one device: {total if sorted else route.rows} rows of x and "
                         f"{route.experts} times as many of w as columns in the result, got {x.rows} x {x.cols} on "
                         f"{x.device}, {w.rows} x {w.cols} on {w.device} and {route.device}")
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    n = w.rows // route.experts
    if bias is not None and (bias.shape != (route.experts, n) or bias.dtype != _float32 or
                             bias.get_device() != x.index or not bias.is_contiguous()):
        raise ValueError(f"bias must be contiguous float32 [{route.experts}, {n}] on {x.device}")
    y = x.new_empty((total, n), dtype=dtype)
    _check(_lib.sd_expert_product(x.c, w.c, route.c, int(sorted), None if bias is None else bias.data_ptr(),
                                  y.data_ptr(), TYPES[dtype], n, _raw_stream(x.index)), "sd_expert_product")
    return y
