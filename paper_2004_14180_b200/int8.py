"""Products of rows in 8 bits, with weights in 8 bits or as a worker holds them (include/qadam.h).

A layer y = x W^T with 8-bit weights w = quantize_rows(W), or with held weights, and its gradients:

    y  = int8_matmul(quantize_rows(x), w)                                   held_matmul(quantize_rows(x), wcodes, ...)
    dx = int8_matmul(quantize_rows(dy, columns=w.scale), w, transpose=True)  held_matmul(quantize_rows(dy), wcodes, ..., transpose=True)
    dW = int8_matmul(quantize_columns(dy), quantize_columns(x), out_dtype=torch.float32)

All calls run on the current stream of their operands' device.  None of them is recorded by autograd; it is told that `out` is
written.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from .adamw import _need_cuda, stream_of, written
from .binding import PRODUCT_ARGS, _check, load_library
from .embedding import _elsewhere, _row_stride, _status, _type


class Int8Rows:
    """Rows in 8 bits: q[i, k] is worth scale[i]; sums[i] (None if not known) is the sum of q[i, :].

    q: [rows, width] int8 whose rows begin on 16 bytes, a multiple of 16 bytes apart; scale: [rows] float32; sums: [rows] int32.
    What quantize_rows, quantize_columns, held_rows and layer_norm give is so (one allocation; the three are views of it, made when
    they are asked for); q of one's own may be laid out by `empty_rows`."""

    __slots__ = ("rows", "width", "stride", "device", "q_at", "scale_at", "sums_at", "_q", "_scale", "_sums", "_buffer")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, sums: Optional[torch.Tensor] = None):
        if not q.is_cuda or q.dim() != 2 or q.dtype is not torch.int8:
            _need_cuda()
            raise ValueError("q must be a CUDA tensor [rows, width] of int8; there is no CPU path")
        self.rows, self.width = q.shape
        self.device = q.device
        if scale.device != q.device or scale.dtype is not torch.float32 or scale.shape != (self.rows,) or not scale.is_contiguous():
            raise ValueError(f"scale must be {self.rows} contiguous float32 on {q.device}")
        if sums is not None and (sums.device != q.device or sums.dtype is not torch.int32 or sums.shape != (self.rows,) or
                                 not sums.is_contiguous()):
            raise ValueError(f"sums must be {self.rows} contiguous int32 on {q.device}")
        row, column = q.stride()
        if self.width > 1 and column != 1:
            raise ValueError("a row's elements must be next to each other")
        self.stride = row if self.rows > 1 else (self.width + 15) // 16 * 16
        self.q_at = q.data_ptr()
        if self.stride % 16 or self.stride < self.width or self.q_at % 16:
            raise ValueError("rows must begin on 16 bytes, a multiple of 16 bytes apart (empty_rows lays them out so)")
        self.scale_at, self.sums_at = scale.data_ptr(), None if sums is None else sums.data_ptr()
        self._q, self._scale, self._sums, self._buffer = q, scale, sums, None

    @classmethod
    def _make(cls, rows: int, width: int, device: torch.device, sums: bool) -> "Int8Rows":
        """Room for so many rows, in one allocation: [q, rows on 16 bytes][scale][sums]."""
        self = cls.__new__(cls)
        self.rows, self.width, self.device = rows, width, device
        self.stride = stride = (width + 15) // 16 * 16
        self._buffer = buffer = torch.empty(rows * (stride + (8 if sums else 4)), dtype=torch.uint8, device=device)
        self.q_at = at = buffer.data_ptr()
        self.scale_at = at + rows * stride
        self.sums_at = self.scale_at + 4 * rows if sums else None
        self._q = self._scale = self._sums = None
        return self

    def _at(self):
        """q, q_stride, scale, sums"""
        return self.q_at, self.stride, self.scale_at, self.sums_at

    @property
    def q(self) -> torch.Tensor:
        if self._q is None:
            self._q = self._buffer[:self.rows * self.stride].view(torch.int8).view(self.rows, self.stride)[:, :self.width]
        return self._q

    @property
    def scale(self) -> torch.Tensor:
        if self._scale is None:
            first = self.rows * self.stride
            self._scale = self._buffer[first:first + 4 * self.rows].view(torch.float32)
        return self._scale

    @property
    def sums(self) -> Optional[torch.Tensor]:
        if self._sums is None and self.sums_at is not None:
            self._sums = self._buffer[self.rows * (self.stride + 4):].view(torch.int32)
        return self._sums

    def values(self) -> torch.Tensor:
        """What the rows stand for, float32 (by torch's operations)."""
        return self.q.float() * self.scale[:, None]

    def __repr__(self) -> str:
        return f"Int8Rows({self.rows} x {self.width} on {self.device})"


def empty_rows(rows: int, width: int, device: torch.device) -> torch.Tensor:
    """[rows, width] int8, rows on 16 bytes."""
    pitch = (width + 15) // 16 * 16
    q = torch.empty(rows, pitch, dtype=torch.int8, device=device)
    return q if pitch == width else q[:, :width]


def quantize_rows(x: torch.Tensor, columns: Optional[torch.Tensor] = None, sums: bool = True) -> Int8Rows:
    """x [..., width] (float32, bfloat16 or float16, rows at equal distances) as rows in 8 bits, leading dimensions joined.

    columns ([width] float32): factors of the columns, multiplied in before."""
    if not x.is_cuda or x.dim() < 1:
        _need_cuda()
        raise ValueError("x: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = x.device, x.shape[-1]
    if _elsewhere(device):
        with torch.cuda.device(device):
            return quantize_rows(x, columns, sums)
    if width < 1:
        raise ValueError("x: rows of no elements")
    if columns is not None and (columns.device != device or columns.dtype is not torch.float32 or columns.shape != (width,) or
                                not columns.is_contiguous()):
        raise ValueError(f"columns: {width} contiguous float32 on {device} are needed")
    stride = width if x.is_contiguous() else _row_stride(x, "x", x.shape, device)
    rows = x.numel() // width
    r = Int8Rows._make(rows, width, device, sums)
    rc = load_library().qadam_quantize_rows(x.data_ptr(), _type(x, "x"), stride, None if columns is None else columns.data_ptr(), rows, width,
                                            r.q_at, r.stride, r.scale_at, r.sums_at, stream_of(device))
    if rc:
        _check(rc, "qadam_quantize_rows")
    return r


@functools.lru_cache(maxsize=256)
def _column_workspace(rows: int, width: int) -> int:
    size = C.c_size_t()
    _check(load_library().qadam_quantize_columns_query_sizes(rows, width, C.byref(size)), "qadam_quantize_columns_query_sizes")
    return size.value


def quantize_columns(x: torch.Tensor) -> Int8Rows:
    """The columns of x [..., width] (leading dimensions joined, at least one row) as rows in 8 bits: q is [width, rows]."""
    if not x.is_cuda or x.dim() < 1:
        _need_cuda()
        raise ValueError("x: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = x.device, x.shape[-1]
    if _elsewhere(device):
        with torch.cuda.device(device):
            return quantize_columns(x)
    if x.numel() == 0:
        raise ValueError("x: no elements")
    stride = width if x.is_contiguous() else _row_stride(x, "x", x.shape, device)
    rows = x.numel() // width
    r = Int8Rows._make(width, rows, device, False)
    size = _column_workspace(rows, width)
    scratch = torch.empty(size, dtype=torch.uint8, device=device)
    rc = load_library().qadam_quantize_columns(x.data_ptr(), _type(x, "x"), stride, rows, width, r.q_at, r.stride, r.scale_at,
                                               scratch.data_ptr(), size, stream_of(device))
    if rc:
        _check(rc, "qadam_quantize_columns")
    return r


def _check_codes(wcodes: torch.Tensor) -> None:
    if not wcodes.is_cuda:
        _need_cuda()
    if not wcodes.is_cuda or wcodes.dtype != torch.uint8 or not wcodes.is_contiguous():
        raise ValueError("wcodes: a contiguous CUDA tensor of uint8 is needed; there is no CPU path")


def held_rows(wcodes: torch.Tensor, kx: int, rows: int, width: int, first: int = 0) -> Int8Rows:
    """Elements [first, first + rows * width) of the weights that a worker holds (see held_lookup), kx = 0 .. 6, as rows in 8
    bits: levels, each worth 2^-(kx + 1)."""
    _check_codes(wcodes)
    device = wcodes.device
    if _elsewhere(device):
        with torch.cuda.device(device):
            return held_rows(wcodes, kx, rows, width, first)
    if rows < 0 or width < 1:
        raise ValueError(f"no table of {rows} rows of {width}")
    r = Int8Rows._make(rows, width, device, False)
    rc = load_library().qadam_held_rows(wcodes.data_ptr(), wcodes.numel(), kx, first, rows, width, r.q_at, r.stride, r.scale_at,
                                        stream_of(device))
    if rc:
        _check(rc, "qadam_held_rows")
    return r


def _output(rows, channels, out, out_dtype, accumulate, bias, device):
    """-> out, its row stride, pointer and type of bias"""
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if out is None:
        out, stride = torch.empty(rows, channels, dtype=out_dtype or torch.bfloat16, device=device), channels
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise ValueError(f"out is {out.dtype}, {out_dtype} was asked for")
        stride = _row_stride(out, "out", (rows, channels), device)
    if bias is None:
        return out, stride, 0, 0
    if bias.device != device or bias.shape != (channels,) or not bias.is_contiguous():
        raise ValueError(f"bias: {channels} contiguous elements on {device} are needed")
    return out, stride, bias.data_ptr(), _type(bias, "bias")


def int8_matmul(a: Int8Rows, b: Int8Rows, bias: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                out: Optional[torch.Tensor] = None, accumulate: bool = False, transpose: bool = False,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T + bias: [rows of a, rows of b], rounded once to out_dtype (bfloat16 if not given), or into `out`, or added to it.

    The sums over the common width (at most 131072) are exact.  transpose: a b instead, [rows of a, width of b]; b's scales belong
    to the axis that is then summed over and are not applied: quantize a with columns=b.scale.
    status: one int32 on the device that gets ST_TIMEOUT if a wait inside the kernel gives up; part of the result is then not written, and
    without it nothing says so."""
    return _product(a, b, None, bias, out_dtype, out, accumulate, transpose, status)


def _product(a, b, worth, bias, out_dtype, out, accumulate, transpose, status):
    """int8_matmul; worth: what all of b's numbers are worth, in place of its scales."""
    device, rows, depth = a.device, a.rows, a.width
    if _elsewhere(device):
        with torch.cuda.device(device):
            return _product(a, b, worth, bias, out_dtype, out, accumulate, transpose, status)
    if b.device != device:
        raise ValueError(f"a on {device}, b on {b.device}")
    common, channels = (b.rows, b.width) if transpose else (b.width, b.rows)
    if depth != common:
        raise ValueError(f"a [{rows}, {depth}] and b [{b.rows}, {b.width}] have no common axis{' (transposed)' if transpose else ''}")
    given = out is not None
    out, out_stride, bias_at, bias_type = _output(rows, channels, out, out_dtype, accumulate, bias, device)
    rc = load_library().qadam_row_product(PRODUCT_ARGS.pack(
        a.q_at, a.stride, a.scale_at, 0, rows, depth, b.q_at, b.stride, 0 if transpose or worth is not None else b.scale_at, channels, bias_at,
        out.data_ptr(), out_stride, 0 if status is None else _status(status, device), 0, 0, transpose, bias_type, _type(out, "out"), accumulate, 0, 0, 0,
        1.0 if worth is None else worth), stream_of(device))
    if rc:
        _check(rc, "qadam_row_product")
    if given:
        written(out)
    return out


def held_matmul(a: Int8Rows, wcodes: torch.Tensor, kx: int, rows: int, width: int, first: int = 0, bias: Optional[torch.Tensor] = None,
                out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None, accumulate: bool = False,
                transpose: bool = False, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a W^T + bias, or a W with transpose, for the table W [rows, width] of the weights that a worker holds (see held_lookup;
    kx = 0 .. 6).  As int8_matmul, and a needs its sums.

    Codes of one byte (kx = 6) whose rows begin on 16 bytes are multiplied as they lie; others are laid out as rows in 8 bits
    first, by a launch that writes rows * width bytes."""
    device, a_rows, depth = a.device, a.rows, a.width
    _check_codes(wcodes)
    if wcodes.device != device:
        raise ValueError(f"a on {device}, wcodes on {wcodes.device}")
    if _elsewhere(device):
        with torch.cuda.device(device):
            return held_matmul(a, wcodes, kx, rows, width, first, bias, out_dtype, out, accumulate, transpose, status)
    if depth != (rows if transpose else width):
        raise ValueError(f"a [{a_rows}, {depth}] and W [{rows}, {width}] have no common axis{' (transposed)' if transpose else ''}")
    if kx != 6 or width % 16 or first % 16:
        w = held_rows(wcodes, kx, rows, width, first)
        return _product(a, w, 2.0 ** -(kx + 1), bias, out_dtype, out, accumulate, transpose, status)
    if a.sums_at is None:
        raise ValueError("a: the sums of its rows are needed")
    channels = width if transpose else rows
    given = out is not None
    out, out_stride, bias_at, bias_type = _output(a_rows, channels, out, out_dtype, accumulate, bias, device)
    rc = load_library().qadam_held_product(PRODUCT_ARGS.pack(
        a.q_at, a.stride, a.scale_at, a.sums_at, a_rows, depth, wcodes.data_ptr(), 0, 0, channels, bias_at, out.data_ptr(), out_stride,
        0 if status is None else _status(status, device), first, wcodes.numel(), transpose, bias_type, _type(out, "out"), accumulate, kx, 0, 0, 0.0),
        stream_of(device))
    if rc:
        _check(rc, "qadam_held_product")
    if given:
        written(out)
    return out
