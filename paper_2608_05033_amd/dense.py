"""The dense operators of a graph network's layer, on GPU tensors.

    X8 = pack(X); W8 = pack(W, transpose=True)       8 bits, a scale per row and 128 columns
    Z  = product(X8, W8)                             X.W on the matrix units
    out = group_norm(A, groups, w, b, activation="relu", keep="e4m3", pack_y="e4m3", dense_y=False)
    dW = weight_gradient(X8, dZ)                     X^T.dZ from the 8-bit copy
    dA, dw, db = group_norm_backward(dH, out.x, out.mean, out.rstd, groups, w, b, activation="relu")
    Z  = product4(pack4(X), pack4(W, transpose=True))    the same in 4 bits, a scale per row and 32 columns

Arguments are checked here and in the library; every call runs on the current
stream of its tensors' device, and results and workspaces are torch tensors of
that stream.  Nothing here records gradients; gcn.py builds the autograd
functions of a whole layer from these calls.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import (ACTIVATIONS, PACK_FORMATS, SD_TYPE_BF16, SD_TYPE_F16, SD_TYPE_F32, _check, _lib, sd_nibble_t, sd_norm_t,
               sd_packed_t)

BLOCK = 128  # columns that share a scale
TYPES = {torch.float32: SD_TYPE_F32, torch.float16: SD_TYPE_F16, torch.bfloat16: SD_TYPE_BF16}
# Small calls take a few microseconds on the GPU, so the way there is kept short:
# the library is called with plain addresses, and the raw handle of the current
# stream is asked for where torch gives it without making a stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_uint8, _float32 = torch.uint8, torch.float32


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


def _vector(v, n, index, what):
    """The address of a float32 vector of n on GPU `index`, or None."""
    if v is None:
        return None
    if v.shape != (n,) or v.dtype != _float32 or v.get_device() != index or not v.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 vector of {n} on cuda:{index}")
    return v.data_ptr()


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_its_device(call):
    """Runs call(first, ...) with the first argument's device as the current one."""

    @functools.wraps(call)
    def wrapped(first, *args, **kw):
        index = first.get_device()
        if index < 0 or index == _current_device():
            return call(first, *args, **kw)
        with torch.cuda.device(index):
            return call(first, *args, **kw)

    return wrapped


class Packed:
    """A rows x cols table in 8 bits: codes uint8 [rows, ld] (ld a multiple of
    16, zeros from cols to the next multiple of 16) and scales uint8
    [ceil(cols / 128), rows], a code's value times 2^(scale - 127)."""

    __slots__ = ("codes", "scales", "rows", "cols", "format", "index", "c")

    def __init__(self, codes, scales, cols: int, format: str = "e4m3"):
        index = codes.get_device()
        if codes.dtype != _uint8 or scales.dtype != _uint8 or codes.dim() != 2 or index < 0 or \
                index != scales.get_device():
            raise ValueError("codes and scales must be uint8 tensors on one GPU")
        if format not in PACK_FORMATS:
            raise ValueError(f"format must be one of {sorted(PACK_FORMATS)}, got {format!r}")
        rows, width = codes.shape
        ld, step = codes.stride()
        need = (cols + 15) // 16 * 16
        if cols < 0 or width < need or width > 1 and step != 1:
            raise ValueError(f"codes must hold {cols} columns, rounded up to 16, next to each other")
        if scales.shape != ((cols + 127) // BLOCK, rows) or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous [{-(-cols // BLOCK)}, {rows}], got {tuple(scales.shape)}")
        self.codes, self.scales, self.rows, self.cols, self.format, self.index = codes, scales, rows, cols, format, index
        self.c = sd_packed_t(rows, cols, ld if rows > 1 and cols else need, PACK_FORMATS[format], 0, codes.data_ptr(),
                             scales.data_ptr())

    @property
    def device(self):
        return self.codes.device

    def get_device(self) -> int:
        return self.index

    @classmethod
    def empty(cls, rows: int, cols: int, format: str, like):
        """A new one on the device of the tensor `like`: one allocation for codes and scales."""
        if format not in PACK_FORMATS:
            raise ValueError(f"format must be one of {sorted(PACK_FORMATS)}, got {format!r}")
        ld, blocks = (cols + 15) // 16 * 16, (cols + 127) // BLOCK
        size = rows * ld
        store = like.new_empty(size + blocks * rows, dtype=_uint8)
        p, at = cls.__new__(cls), store.data_ptr()
        p.codes, p.scales = store.as_strided((rows, ld), (ld, 1)), store.as_strided((blocks, rows), (rows, 1), size)
        p.rows, p.cols, p.format, p.index = rows, cols, format, store.get_device()
        p.c = sd_packed_t(rows, cols, ld, PACK_FORMATS[format], 0, at, at + size)
        return p


@_on_its_device
def pack(x, format: str = "e4m3", transpose: bool = False) -> Packed:
    """x in 8 bits (of x^T with transpose=True: a weight [k, n] as product's
    second operand).  Any strides."""
    if x.dim() != 2 or x.dtype not in TYPES or not x.is_cuda:
        raise ValueError(f"x must be a float32, float16 or bfloat16 matrix on the GPU, got {x.dtype} "
                         f"{tuple(x.shape)} on {x.device}")
    (rows, cols), (down, right) = x.shape, x.stride()
    if transpose:
        rows, cols, down, right = cols, rows, right, down
    out = Packed.empty(rows, cols, format, x)
    _check(_lib.sd_pack(x.data_ptr(), TYPES[x.dtype], down, 1 if cols == 1 else right, out.c,
                        _raw_stream(x.get_device())), "sd_pack")
    return out


@_on_its_device
def unpack(x: Packed, dtype=torch.float32) -> torch.Tensor:
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    y = x.codes.new_empty((x.rows, x.cols), dtype=dtype)
    _check(_lib.sd_unpack(x.c, y.data_ptr(), TYPES[dtype], x.cols, _raw_stream(x.index)), "sd_unpack")
    return y


@_on_its_device
def product(x: Packed, w: Packed, bias=None, dtype=torch.float32) -> torch.Tensor:
    """x.w^T (+ bias), [x.rows, w.rows], summed in 32 bits and rounded once to dtype."""
    if x.cols != w.cols or x.index != w.index:
        raise ValueError(f"operands must have the same columns on one device, got {x.cols} on {x.device} and "
                         f"{w.cols} on {w.device}")
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    n = w.rows
    bias = _vector(bias, n, x.index, "bias")
    y = x.codes.new_empty((x.rows, n), dtype=dtype)
    _check(_lib.sd_pack_product(x.c, w.c, bias, y.data_ptr(), TYPES[dtype], n, _raw_stream(x.index)),
           "sd_pack_product")
    return y


@_on_its_device
def weight_gradient(x: Packed, g) -> torch.Tensor:
    """x^T.g in float32, [x.cols, g.shape[1]]."""
    stride = _table(g, "g")
    rows, n = g.shape
    if rows != x.rows or g.get_device() != x.index:
        raise ValueError(f"g must have {x.rows} rows on {x.device}, got {tuple(g.shape)} on {g.device}")
    dw = g.new_empty((x.cols, n), dtype=_float32)
    size = ctypes.c_size_t()
    _check(_lib.sd_pack_gradient_size(rows, x.cols, n, size), "sd_pack_gradient_size")
    work = g.new_empty(size.value, dtype=_uint8) if size.value else None
    _check(_lib.sd_pack_gradient(x.c, g.data_ptr(), TYPES[g.dtype], n, stride, dw.data_ptr(),
                                 None if work is None else work.data_ptr(), size, _raw_stream(x.index)),
           "sd_pack_gradient")
    return dw


class Packed4:
    """A rows x cols table in 4 bits: codes uint8 [rows, ld], two in a byte, the
    even column in the lower half (ld a multiple of 16, 16 bytes for every 32
    columns begun, zeros past cols), and scales uint8 [ceil(cols / 128), rows, 4].
    A code's value is e2m1(code) times 2^(scale - 127); 255 makes a block NaN."""

    __slots__ = ("_codes", "_scales", "store", "rows", "cols", "index", "c")

    def __init__(self, codes, scales, cols: int):
        index = codes.get_device()
        if codes.dtype != _uint8 or scales.dtype != _uint8 or codes.dim() != 2 or index < 0 or \
                index != scales.get_device():
            raise ValueError("codes and scales must be uint8 tensors on one GPU")
        rows, width = codes.shape
        ld, step = codes.stride()
        need = (cols + 31) // 32 * 16
        if cols < 0 or width < need or width > 1 and step != 1:
            raise ValueError(f"codes must hold {cols} columns, two in a byte and rounded up to 32, next to each other")
        if scales.shape != ((cols + 127) // 128, rows, 4) or not scales.is_contiguous():
            raise ValueError(f"scales must be contiguous [{-(-cols // 128)}, {rows}, 4], got {tuple(scales.shape)}")
        self._codes, self._scales, self.store, self.rows, self.cols, self.index = codes, scales, None, rows, cols, index
        self.c = sd_nibble_t(rows, cols, ld if rows > 1 and cols else need, 0, codes.data_ptr(), scales.data_ptr())

    @classmethod
    def empty(cls, rows: int, cols: int, like):
        """A new one on the device of the tensor `like`: one allocation for codes and
        scales, which become tensors of their own when they are asked for."""
        size = rows * ((cols + 31) // 32 * 16)
        return cls._laid_out(like.new_empty(size + (cols + 127) // 128 * rows * 4, dtype=_uint8), rows, cols)

    @classmethod
    def of(cls, store, rows: int, cols: int):
        """The one whose codes and, behind them, scales are `store`, the `store` of
        another of this size (or a copy of it)."""
        size = rows * ((cols + 31) // 32 * 16) + (cols + 127) // 128 * rows * 4
        if store.dtype != _uint8 or not store.is_cuda or store.shape != (size,) or not store.is_contiguous():
            raise ValueError(f"store must be {size} uint8 in a row on the GPU, got {store.dtype} {tuple(store.shape)} "
                             f"on {store.device}")
        return cls._laid_out(store, rows, cols)

    @classmethod
    def _laid_out(cls, store, rows, cols):
        ld = (cols + 31) // 32 * 16
        p, at = cls.__new__(cls), store.data_ptr()
        p._codes, p._scales, p.store, p.rows, p.cols, p.index = None, None, store, rows, cols, store.get_device()
        p.c = sd_nibble_t(rows, cols, ld, 0, at, at + rows * ld)
        return p

    @property
    def codes(self):
        if self._codes is None:
            ld = self.c.ld
            self._codes = self.store.as_strided((self.rows, ld), (ld, 1))
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            shape = (self.cols + 127) // 128, self.rows, 4
            self._scales = self.store.as_strided(shape, (self.rows * 4, 4, 1), self.rows * self.c.ld)
        return self._scales

    def new_empty(self, *args, **kw):
        return (self._codes if self.store is None else self.store).new_empty(*args, **kw)

    @property
    def device(self):
        return (self._codes if self.store is None else self.store).device

    def get_device(self) -> int:
        return self.index


@_on_its_device
def pack4(x, transpose: bool = False) -> Packed4:
    """x in 4 bits (of x^T with transpose=True: a weight [k, n] as product4's
    second operand).  Any strides."""
    if x.dim() != 2 or x.dtype not in TYPES or not x.is_cuda:
        raise ValueError(f"x must be a float32, float16 or bfloat16 matrix on the GPU, got {x.dtype} "
                         f"{tuple(x.shape)} on {x.device}")
    (rows, cols), (down, right) = x.shape, x.stride()
    if transpose:
        rows, cols, down, right = cols, rows, right, down
    out = Packed4.empty(rows, cols, x)
    _check(_lib.sd_nibble_pack(x.data_ptr(), TYPES[x.dtype], down, 1 if cols == 1 else right, out.c,
                               _raw_stream(x.get_device())), "sd_nibble_pack")
    return out


@_on_its_device
def pack4_both(x):
    """(pack4(x), pack4(x, transpose=True)), from one reading of x where that is faster."""
    if x.dim() != 2 or x.dtype not in TYPES or not x.is_cuda:
        raise ValueError(f"x must be a float32, float16 or bfloat16 matrix on the GPU, got {x.dtype} "
                         f"{tuple(x.shape)} on {x.device}")
    (rows, cols), (down, right) = x.shape, x.stride()
    out, out_t = Packed4.empty(rows, cols, x), Packed4.empty(cols, rows, x)
    _check(_lib.sd_nibble_pack_both(x.data_ptr(), TYPES[x.dtype], down if rows > 1 else cols, 1 if cols == 1 else right,
                                    out.c, out_t.c, _raw_stream(x.get_device())), "sd_nibble_pack_both")
    return out, out_t


@_on_its_device
def unpack4(x: Packed4, dtype=torch.float32) -> torch.Tensor:
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    y = x.new_empty((x.rows, x.cols), dtype=dtype)
    _check(_lib.sd_nibble_unpack(x.c, y.data_ptr(), TYPES[dtype], x.cols, _raw_stream(x.index)), "sd_nibble_unpack")
    return y


@functools.lru_cache(maxsize=4096)
def _product4_size(rows, cols, n, index):
    """The workspace in bytes on GPU `index`, which is the current one."""
    size = ctypes.c_size_t()
    _check(_lib.sd_nibble_product_size(rows, cols, n, size), "sd_nibble_product_size")
    return size.value


@_on_its_device
def product4(x: Packed4, w: Packed4, bias=None, dtype=torch.float32) -> torch.Tensor:
    """x.w^T (+ bias), [x.rows, w.rows], summed in 32 bits and rounded once to dtype."""
    if x.cols != w.cols or x.index != w.index:
        raise ValueError(f"operands must have the same columns on one device, got {x.cols} on {x.device} and "
                         f"{w.cols} on {w.device}")
    if dtype not in TYPES:
        raise ValueError(f"dtype must be one of {list(TYPES)}, got {dtype}")
    n = w.rows
    bias = _vector(bias, n, x.index, "bias")
    y = x.new_empty((x.rows, n), dtype=dtype)
    size = _product4_size(x.rows, x.cols, n, x.index)
    work = y.new_empty(size, dtype=_uint8) if size else None  # lives until the call has been enqueued
    _check(_lib.sd_nibble_product(x.c, w.c, bias, y.data_ptr(), TYPES[dtype], n, work.data_ptr() if size else None, size,
                                  _raw_stream(x.index)), "sd_nibble_product")
    return y


class NormOut:
    """What group_norm leaves: y (None without it), y_packed, x (what the
    backward pass takes: the input itself or its 8-bit copy), mean, rstd."""

    __slots__ = ("y", "y_packed", "x", "mean", "rstd")

    def __init__(self, y, y_packed, x, mean, rstd):
        self.y, self.y_packed, self.x, self.mean, self.rstd = y, y_packed, x, mean, rstd


def _norm_of(index, rows, channels, dtype, groups, weight, bias, eps, activation, segments, offsets, longest):
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {activation!r}")
    if groups < 1 or channels < 1 or channels % groups:
        raise ValueError(f"{channels} channels cannot be cut into {groups} equal groups")
    at = None
    if offsets is not None:
        if offsets.dim() != 1 or offsets.dtype != torch.int32 or offsets.get_device() != index or \
                not offsets.is_contiguous() or offsets.numel() < 1:
            raise ValueError(f"offsets must be a contiguous int32 vector on cuda:{index}")
        if segments not in (None, offsets.numel() - 1):
            raise ValueError(f"{segments} segments need {segments + 1} offsets, got {offsets.numel()}")
        segments, at = offsets.numel() - 1, offsets.data_ptr()
    elif segments is None:
        segments = 1
    if segments < 0 or rows and (segments < 1 or at is None and rows % segments):
        raise ValueError(f"{rows} rows cannot be cut into {segments} equal segments")
    return sd_norm_t(rows, segments, at, longest, channels, groups, TYPES[dtype], ACTIVATIONS[activation], eps, 0,
                     _vector(weight, channels, index, "weight"), _vector(bias, channels, index, "bias"))


@_on_its_device
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
    index = x.get_device()
    d = _norm_of(index, rows, channels, x.dtype, groups, weight, bias, eps, activation, segments, offsets, longest)
    if not dense_y and pack_y is None:
        raise ValueError("dense_y=False needs pack_y")
    y = x.new_empty((rows, channels)) if dense_y else None
    xp = Packed.empty(rows, channels, keep, x) if keep is not None else None
    yp = Packed.empty(rows, channels, pack_y, x) if pack_y is not None else None
    mean, rstd = x.new_empty((2, d.segments, groups), dtype=_float32).unbind(0)
    size = ctypes.c_size_t()
    _check(_lib.sd_group_norm_size(d, size, None), "sd_group_norm_size")
    work = x.new_empty(size.value, dtype=_uint8) if size.value else None
    _check(_lib.sd_group_norm(d, x.data_ptr(), stride, y.data_ptr() if dense_y else None, channels,
                              xp.c if xp else None, yp.c if yp else None, mean.data_ptr(), rstd.data_ptr(),
                              None if work is None else work.data_ptr(), size, _raw_stream(index)),
           "sd_group_norm")
    return NormOut(y, yp, x if xp is None else xp, mean, rstd)


@_on_its_device
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
    index = dy.get_device()
    d = _norm_of(index, rows, channels, dy.dtype, groups, weight, bias, eps, activation, segments, offsets, longest)
    for v, what in ((mean, "mean"), (rstd, "rstd")):
        if v.shape != (d.segments, groups) or v.dtype != _float32 or v.get_device() != index or not v.is_contiguous():
            raise ValueError(f"{what} must be contiguous float32 [{d.segments}, {groups}] on cuda:{index}")
    dx = dy.new_empty((rows, channels))
    dweight, dbias = dy.new_empty((2, channels), dtype=_float32).unbind(0)
    size = ctypes.c_size_t()
    _check(_lib.sd_group_norm_size(d, None, size), "sd_group_norm_size")
    work = dy.new_empty(size.value, dtype=_uint8) if size.value else None
    _check(_lib.sd_group_norm_backward(d, dy.data_ptr(), stride, None if packed else x.data_ptr(),
                                       0 if packed else x_stride, x.c if packed else None, mean.data_ptr(),
                                       rstd.data_ptr(), dx.data_ptr(), channels, dweight.data_ptr(), dbias.data_ptr(),
                                       None if work is None else work.data_ptr(), size,
                                       _raw_stream(index)), "sd_group_norm_backward")
    return dx, dweight, dbias
