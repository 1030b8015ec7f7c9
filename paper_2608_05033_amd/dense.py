"""The dense operators of a graph network's layer, on GPU tensors.

    X8 = pack(X); W8 = pack(W, transpose=True)       8 bits, a scale per row and 128 columns
    Z  = product(X8, W8)                             X.W on the matrix units
    out = group_norm(A, groups, w, b, activation="relu", keep="e4m3", pack_y="e4m3", dense_y=False)
    dW = weight_gradient(X8, dZ)                     X^T.dZ from the 8-bit copy
    dA, dw, db = group_norm_backward(dH, out.x, out.mean, out.rstd, groups, w, b, activation="relu")

Arguments are checked here and in the library; every call runs on the current
stream of its tensors' device, and results and workspaces are torch tensors of
that stream.  Nothing here records gradients; gcn.py builds the autograd
functions of a whole layer from these calls.
"""
from __future__ import annotations

import torch

from . import (ACTIVATIONS, PACK_FORMATS, SD_TYPE_BF16, SD_TYPE_F16, SD_TYPE_F32, sd_group_norm,
               sd_group_norm_backward, sd_group_norm_size, sd_norm_t, sd_pack, sd_pack_gradient,
               sd_pack_gradient_size, sd_pack_product, sd_packed_t, sd_unpack)

BLOCK = 128  # columns that share a scale
TYPES = {torch.float32: SD_TYPE_F32, torch.float16: SD_TYPE_F16, torch.bfloat16: SD_TYPE_BF16}


def _table(x, what):
    """Row stride of a two-dimensional GPU tensor whose columns lie next to each other."""
    if x.dim() != 2 or x.dtype not in TYPES or not x.is_cuda:
        raise ValueError(f"{what} must be a float32, float16 or bfloat16 matrix on the GPU, got "
                         f"{x.dtype} {tuple(x.shape)} on {x.device}")
    rows, cols = x.shape
    if cols > 1 and x.stride(1) != 1 or rows > 1 and x.stride(0) < cols:
        raise ValueError(f"{what}: columns must lie next to each other and rows must not overlap, got strides "
                         f"{x.stride()}")
    return x.stride(0) if rows > 1 else cols


def _vector(v, n, like, what):
    if v is not None and (v.shape != (n,) or v.dtype != torch.float32 or v.device != like.device or
                          not v.is_contiguous()):
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} on {like.device}")
    return v


class _On:
    """Makes a tensor's device current where it is not, and names its current stream."""

    def __init__(self, x):
        self.device = x.device
        self.other = None

    def __enter__(self):
        index = self.device.index
        if index != torch.cuda.current_device():
            self.other = torch.cuda.device(index)
            self.other.__enter__()
        return torch.cuda.current_stream(index).cuda_stream

    def __exit__(self, *e):
        if self.other is not None:
            self.other.__exit__(*e)


class Packed:
    """A rows x cols table in 8 bits: codes uint8 [rows, ld] (ld a multiple of
    16, zeros from cols to the next multiple of 16) and scales uint8
    [ceil(cols / 128), rows], a code's value times 2^(scale - 127)."""

    __slots__ = ("codes", "scales", "rows", "cols", "format", "c")

    def __init__(self, codes, scales, cols: int, format: str = "e4m3"):
        rows = codes.shape[0]
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8 or codes.dim() != 2 or not codes.is_cuda or \
                codes.device != scales.device:
            raise ValueError("codes and scales must be uint8 tensors on one GPU")
        if format not in PACK_FORMATS:
            raise ValueError(f"format must be one of {sorted(PACK_FORMATS)}, got {format!r}")
        ld = codes.stride(0) if rows > 1 and cols else -(-cols // 16) * 16
        if cols < 0 or codes.shape[1] < -(-cols // 16) * 16 or codes.shape[1] > 1 and codes.stride(1) != 1:
            raise ValueError(f"codes must hold {cols} columns, rounded up to 16, next to each other")
        if scales.shape != (-(-cols // BLOCK), rows) or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous [{-(-cols // BLOCK)}, {rows}], got {tuple(scales.shape)}")
        self.codes, self.scales, self.rows, self.cols, self.format = codes, scales, rows, cols, format
        self.c = sd_packed_t(rows, cols, ld, PACK_FORMATS[format], 0, codes.data_ptr(), scales.data_ptr())

    @property
    def device(self):
        return self.codes.device

    @classmethod
    def empty(cls, rows: int, cols: int, format: str, device):
        """One allocation for codes and scales."""
        ld = -(-cols // 16) * 16
        blocks = -(-cols // BLOCK)
        store = torch.empty(rows * ld + blocks * rows, dtype=torch.uint8, device=device)
        return cls(store[:rows * ld].view(rows, ld), store[rows * ld:].view(blocks, rows), cols, format)


def pack(x, format: str = "e4m3", transpose: bool = False) -> Packed:
    """x in 8 bits (of x^T with transpose=True: a weight [k, n] as product's
    second operand).  Any strides."""
    if x.dim() != 2 or x.dtype not in TYPES or not x.is_cuda:
        raise ValueError(f"x must be a float32, float16 or bfloat16 matrix on the GPU, got {x.dtype} "
                         f"{tuple(x.shape)} on {x.device}")
    if transpose:
        x = x.t()
    rows, cols = x.shape
    with _On(x) as stream:
        out = Packed.empty(rows, cols, format, x.device)
        sd_pack(x, TYPES[x.dtype], x.stride(0), 1 if cols == 1 else x.stride(1), out.c, stream)
    return out


def unpack(x: Packed, dtype=torch.float32) -> torch.Tensor:
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    with _On(x) as stream:
        y = torch.empty((x.rows, x.cols), dtype=dtype, device=x.device)
        sd_unpack(x.c, y, TYPES[dtype], x.cols, stream)
    return y


def product(x: Packed, w: Packed, bias=None, dtype=torch.float32) -> torch.Tensor:
    """x.w^T (+ bias), [x.rows, w.rows], summed in 32 bits and rounded once to dtype."""
    if x.cols != w.cols or x.device != w.device:
        raise ValueError(f"operands must have the same columns on one device, got {x.cols} on {x.device} and "
                         f"{w.cols} on {w.device}")
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    _vector(bias, w.rows, x, "bias")
    with _On(x) as stream:
        y = torch.empty((x.rows, w.rows), dtype=dtype, device=x.device)
        sd_pack_product(x.c, w.c, bias, y, TYPES[dtype], w.rows, stream)
    return y


def weight_gradient(x: Packed, g) -> torch.Tensor:
    """x^T.g in float32, [x.cols, g.shape[1]]."""
    stride = _table(g, "g")
    if g.shape[0] != x.rows or g.device != x.device:
        raise ValueError(f"g must have {x.rows} rows on {x.device}, got {tuple(g.shape)} on {g.device}")
    n = g.shape[1]
    with _On(x) as stream:
        dw = torch.empty((x.cols, n), dtype=torch.float32, device=x.device)
        size = sd_pack_gradient_size(x.rows, x.cols, n)
        work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
        sd_pack_gradient(x.c, g, TYPES[g.dtype], n, stride, dw, work, size, stream)
    return dw


class NormOut:
    """What group_norm leaves: y (None without it), y_packed, x (what the
    backward pass takes: the input itself or its 8-bit copy), mean, rstd."""

    __slots__ = ("y", "y_packed", "x", "mean", "rstd")

    def __init__(self, y, y_packed, x, mean, rstd):
        self.y, self.y_packed, self.x, self.mean, self.rstd = y, y_packed, x, mean, rstd


def _norm_of(like, rows, channels, dtype, groups, weight, bias, eps, activation, segments, offsets, longest):
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {activation!r}")
    if groups < 1 or channels < 1 or channels % groups:
        raise ValueError(f"{channels} channels cannot be cut into {groups} equal groups")
    _vector(weight, channels, like, "weight")
    _vector(bias, channels, like, "bias")
    if offsets is not None:
        if offsets.dim() != 1 or offsets.dtype != torch.int32 or offsets.device != like.device or \
                not offsets.is_contiguous() or offsets.numel() < 1:
            raise ValueError(f"offsets must be a contiguous int32 vector on {like.device}")
        if segments not in (None, offsets.numel() - 1):
            raise ValueError(f"{segments} segments need {segments + 1} offsets, got {offsets.numel()}")
        segments = offsets.numel() - 1
    else:
        segments = 1 if segments is None else segments
    if segments < 0 or rows and (segments < 1 or offsets is None and rows % segments):
        raise ValueError(f"{rows} rows cannot be cut into {segments} equal segments")
    return sd_norm_t(rows, segments, offsets.data_ptr() if offsets is not None else None, longest, channels, groups,
                     TYPES[dtype], ACTIVATIONS[activation], eps, 0, weight.data_ptr() if weight is not None else None,
                     bias.data_ptr() if bias is not None else None)


def group_norm(x, groups: int, weight=None, bias=None, eps: float = 1e-5, activation: str = "none", segments=None,
               offsets=None, longest: int = 0, keep=None, pack_y=None, dense_y: bool = True) -> NormOut:
    """act(group norm(x) * weight + bias) over segments of x's rows.

    segments: that many of equal length (default one); or offsets: int32
    [segments + 1] on the GPU, with longest the rows of the longest segment
    where the caller knows it.  keep: format of an 8-bit copy of x for the
    backward pass (default: x itself).  pack_y: format of an 8-bit copy of y;
    dense_y=False leaves out y itself."""
    stride = _table(x, "x")
    rows, channels = x.shape
    d = _norm_of(x, rows, channels, x.dtype, groups, weight, bias, eps, activation, segments, offsets, longest)
    if not dense_y and pack_y is None:
        raise ValueError("dense_y=False needs pack_y")
    with _On(x) as stream:
        y = torch.empty((rows, channels), dtype=x.dtype, device=x.device) if dense_y else None
        xp = Packed.empty(rows, channels, keep, x.device) if keep is not None else None
        yp = Packed.empty(rows, channels, pack_y, x.device) if pack_y is not None else None
        stats = torch.empty((2, d.segments, groups), dtype=torch.float32, device=x.device)
        mean, rstd = stats[0], stats[1]
        size = sd_group_norm_size(d)[0]
        work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
        sd_group_norm(d, x, stride, y, channels, xp.c if xp else None, yp.c if yp else None, mean, rstd, work, size,
                      stream)
    return NormOut(y, yp, x if xp is None else xp, mean, rstd)


def group_norm_backward(dy, x, mean, rstd, groups: int, weight=None, bias=None, eps: float = 1e-5,
                        activation: str = "none", segments=None, offsets=None, longest: int = 0):
    """(dx, dweight, dbias) from dy and what group_norm left: x (dense or
    Packed), mean and rstd; the other arguments as there."""
    stride = _table(dy, "dy")
    rows, channels = dy.shape
    packed = isinstance(x, Packed)
    if packed:
        if (x.rows, x.cols) != (rows, channels) or x.device != dy.device:
            raise ValueError(f"x must be {rows} x {channels} on {dy.device}, got {x.rows} x {x.cols} on {x.device}")
    else:
        x_stride = _table(x, "x")
        if x.shape != dy.shape or x.dtype != dy.dtype or x.device != dy.device:
            raise ValueError(f"x must be {dy.dtype} {tuple(dy.shape)} on {dy.device}, got {x.dtype} "
                             f"{tuple(x.shape)} on {x.device}")
    d = _norm_of(dy, rows, channels, dy.dtype, groups, weight, bias, eps, activation, segments, offsets, longest)
    for v, what in ((mean, "mean"), (rstd, "rstd")):
        if v.shape != (d.segments, groups) or v.dtype != torch.float32 or v.device != dy.device or \
                not v.is_contiguous():
            raise ValueError(f"{what} must be contiguous float32 [{d.segments}, {groups}] on {dy.device}")
    with _On(dy) as stream:
        dx = torch.empty((rows, channels), dtype=dy.dtype, device=dy.device)
        dparam = torch.empty((2, channels), dtype=torch.float32, device=dy.device)
        size = sd_group_norm_size(d)[1]
        work = torch.empty(size, dtype=torch.uint8, device=dy.device) if size else None
        sd_group_norm_backward(d, dy, stride, None if packed else x, 0 if packed else x_stride,
                               x.c if packed else None, mean, rstd, dx, channels, dparam[0], dparam[1], work, size,
                               stream)
    return dx, dparam[0], dparam[1]
