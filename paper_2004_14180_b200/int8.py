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
from typing import NamedTuple, Optional

import torch

from .adamw import TYPES, _need_cuda, element_type, stream_of, written
from .binding import _check, load_library
from .embedding import _elsewhere, _row_stride, _status, _type


class Int8Rows(NamedTuple):
    """Rows in 8 bits: q[i, k] is worth scale[i]; sums[i] (if there) is the sum of q[i, :].

    q: [rows, width] int8 whose rows begin on 16 bytes, a multiple of 16 bytes apart; scale: [rows] float32; sums: [rows] int32.
    What quantize_rows, quantize_columns, held_rows and layer_norm give is so; q of one's own may be laid out by `empty_rows`."""
    q: torch.Tensor
    scale: torch.Tensor
    sums: Optional[torch.Tensor] = None

    def values(self) -> torch.Tensor:
        """What the rows stand for, float32 (by torch's operations)."""
        return self.q.float() * self.scale[:, None]


def empty_rows(rows: int, width: int, device: torch.device) -> torch.Tensor:
    """[rows, width] int8, rows on 16 bytes."""
    pitch = (width + 15) // 16 * 16
    q = torch.empty(rows, pitch, dtype=torch.int8, device=device)
    return q if pitch == width else q[:, :width]


def _rows_of(a: Int8Rows, what: str):
    """-> rows, width, stride of a.q, all checked but for the alignment, which the library looks at."""
    q, scale = a.q, a.scale
    if not q.is_cuda or q.dim() != 2 or q.dtype != torch.int8:
        _need_cuda()
        raise ValueError(f"{what}: q must be a CUDA tensor [rows, width] of int8; there is no CPU path")
    rows, width = q.shape
    if scale.device != q.device or scale.dtype != torch.float32 or scale.shape != (rows,) or not scale.is_contiguous():
        raise ValueError(f"{what}: scale must be {rows} contiguous float32 on {q.device}")
    if width > 1 and q.stride(1) != 1:
        raise ValueError(f"{what}: a row's elements must be next to each other")
    stride = q.stride(0) if rows > 1 else (width + 15) // 16 * 16
    if stride % 16 or stride < width or (rows and q.data_ptr() % 16):
        raise ValueError(f"{what}: rows must begin on 16 bytes, a multiple of 16 bytes apart (empty_rows lays them out so)")
    return rows, width, stride


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
    if columns is not None and (columns.device != device or columns.dtype != torch.float32 or columns.shape != (width,) or
                                not columns.is_contiguous()):
        raise ValueError(f"columns: {width} contiguous float32 on {device} are needed")
    stride = _row_stride(x, "x", x.shape, device)
    rows = x.numel() // width
    q = empty_rows(rows, width, device)
    scale = torch.empty(rows, dtype=torch.float32, device=device)
    total = torch.empty(rows, dtype=torch.int32, device=device) if sums else None
    rc = load_library().qadam_quantize_rows(
        x.data_ptr(), _type(x, "x"), stride, None if columns is None else columns.data_ptr(), rows, width, q.data_ptr(),
        (width + 15) // 16 * 16, scale.data_ptr(), None if total is None else total.data_ptr(), stream_of(device))
    if rc:
        _check(rc, "qadam_quantize_rows")
    return Int8Rows(q, scale, total)


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
    stride = _row_stride(x, "x", x.shape, device)
    rows = x.numel() // width
    q = empty_rows(width, rows, device)
    scale = torch.empty(width, dtype=torch.float32, device=device)
    size = _column_workspace(rows, width)
    scratch = torch.empty(size, dtype=torch.uint8, device=device)
    rc = load_library().qadam_quantize_columns(x.data_ptr(), _type(x, "x"), stride, rows, width, q.data_ptr(), (rows + 15) // 16 * 16,
                                               scale.data_ptr(), scratch.data_ptr(), size, stream_of(device))
    if rc:
        _check(rc, "qadam_quantize_columns")
    return Int8Rows(q, scale)


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
    q = empty_rows(rows, width, device)
    rc = load_library().qadam_held_rows(wcodes.data_ptr(), wcodes.numel(), kx, first, rows, width, q.data_ptr(), (width + 15) // 16 * 16,
                                        stream_of(device))
    if rc:
        _check(rc, "qadam_held_rows")
    return Int8Rows(q, torch.full((rows,), 2.0 ** -(kx + 1), dtype=torch.float32, device=device))


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
        return out, stride, None, 0
    if bias.device != device or bias.shape != (channels,) or not bias.is_contiguous():
        raise ValueError(f"bias: {channels} contiguous elements on {device} are needed")
    return out, stride, bias.data_ptr(), _type(bias, "bias")


def int8_matmul(a: Int8Rows, b: Int8Rows, bias: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                out: Optional[torch.Tensor] = None, accumulate: bool = False, transpose: bool = False,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """a b^T + bias: [rows of a, rows of b], rounded once to out_dtype (bfloat16 if not given), or into `out`, or added to it.

    The sums over the common width (at most 131072) are exact.  transpose: a b instead, [rows of a, width of b]; b's scales belong
    to the axis that is then summed over and are not applied: quantize a with columns=b.scale.
    status: one int32 on the device that gets ST_TIMEOUT if a wait inside the kernel gives up."""
    rows, depth, a_stride = _rows_of(a, "a")
    device = a.q.device
    if _elsewhere(device):
        with torch.cuda.device(device):
            return int8_matmul(a, b, bias, out_dtype, out, accumulate, transpose, status)
    b_rows, b_width, b_stride = _rows_of(b, "b")
    if b.q.device != device:
        raise ValueError(f"a on {device}, b on {b.q.device}")
    if depth != (b_rows if transpose else b_width):
        raise ValueError(f"a [{rows}, {depth}] and b [{b_rows}, {b_width}] have no common axis{' (transposed)' if transpose else ''}")
    channels = b_width if transpose else b_rows
    given = out is not None
    out, out_stride, bias_at, bias_type = _output(rows, channels, out, out_dtype, accumulate, bias, device)
    rc = load_library().qadam_row_product(
        a.q.data_ptr(), a_stride, a.scale.data_ptr(), rows, depth, b.q.data_ptr(), b_stride, b.scale.data_ptr(), channels, int(transpose),
        bias_at, bias_type, out.data_ptr(), _type(out, "out"), out_stride, int(accumulate),
        None if status is None else _status(status, device), stream_of(device))
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
    a_rows, depth, a_stride = _rows_of(a, "a")
    _check_codes(wcodes)
    device = a.q.device
    if wcodes.device != device:
        raise ValueError(f"a on {device}, wcodes on {wcodes.device}")
    if _elsewhere(device):
        with torch.cuda.device(device):
            return held_matmul(a, wcodes, kx, rows, width, first, bias, out_dtype, out, accumulate, transpose, status)
    if depth != (rows if transpose else width):
        raise ValueError(f"a [{a_rows}, {depth}] and W [{rows}, {width}] have no common axis{' (transposed)' if transpose else ''}")
    if kx != 6 or width % 16 or first % 16 or wcodes.data_ptr() % 16:
        w = held_rows(wcodes, kx, rows, width, first)
        if transpose:              # the weights' worth is the same for all: it goes to a
            a = Int8Rows(a.q, a.scale * 2.0 ** -(kx + 1))
        return int8_matmul(a, w, bias, out_dtype, out, accumulate, transpose, status)
    sums = a.sums
    if sums is None or sums.device != device or sums.dtype != torch.int32 or sums.shape != (a_rows,) or not sums.is_contiguous():
        raise ValueError(f"a: sums ({a_rows} contiguous int32 on {device}) are needed")
    channels = width if transpose else rows
    given = out is not None
    out, out_stride, bias_at, bias_type = _output(a_rows, channels, out, out_dtype, accumulate, bias, device)
    rc = load_library().qadam_held_product(
        a.q.data_ptr(), a_stride, a.scale.data_ptr(), sums.data_ptr(), a_rows, depth, wcodes.data_ptr(), wcodes.numel(), kx, first,
        channels, int(transpose), bias_at, bias_type, out.data_ptr(), _type(out, "out"), out_stride, int(accumulate),
        None if status is None else _status(status, device), stream_of(device))
    if rc:
        _check(rc, "qadam_held_product")
    if given:
        written(out)
    return out
