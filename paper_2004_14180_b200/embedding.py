"""Rows of an embedding table, dense or as a worker holds them, and the table's gradient (include/qadam.h).

All calls run on the current stream of the table's device.  `status`, where given, is one int32 on the
device that gets ST_INDEX if a token is not below the number of rows; the caller clears and reads it.
None of them is recorded by autograd: the gradient of a lookup is embedding_grad.  It is told that `out` is written.
"""
from __future__ import annotations

import ctypes as C
import functools
from typing import Optional

import torch

from .adamw import TYPES, _need_cuda, element_type, stream_of, written
from .binding import _check, load_library


def _elsewhere(device: torch.device) -> bool:
    """Whether another device than `device` is the current one (torch.cuda.device(device) costs 3 us when it is not)."""
    return torch.cuda.current_device() != device.index


def _type(t: torch.Tensor, what: str) -> int:
    ty = TYPES.get(t.dtype)
    return ty if ty is not None else element_type(t.dtype, what)


def _tokens(ids: torch.Tensor, device: torch.device) -> torch.Tensor:
    if ids.dtype is not torch.int64 and ids.dtype is not torch.int32:
        raise ValueError(f"ids: int64 or int32 is needed, got {ids.dtype}")
    if ids.device != device:
        raise ValueError(f"ids on {ids.device}, table on {device}")
    return ids if ids.is_contiguous() else ids.contiguous()


def _row_stride(t: torch.Tensor, what: str, shape, device: torch.device) -> int:
    """Elements from one row of `t` to the next, its columns being next to each other."""
    if t.device != device or t.shape != shape:
        raise ValueError(f"{what}: {tuple(shape)} on {device} is needed, got {tuple(t.shape)} on {t.device}")
    width = shape[-1]
    if t.is_contiguous():
        return max(width, 1)
    try:
        flat = t.view(-1, width)
    except RuntimeError:
        raise ValueError(f"{what}: its rows must lie at equal distances") from None
    if (width > 1 and flat.stride(1) != 1) or (flat.shape[0] > 1 and flat.stride(0) < width):
        raise ValueError(f"{what}: a row's elements must be next to each other, and rows must not overlap")
    return flat.stride(0) if flat.shape[0] > 1 else max(width, 1)


def _status(status: Optional[torch.Tensor], device: torch.device):
    if status is None:
        return None
    if status.device != device or status.dtype != torch.int32 or status.numel() != 1:
        raise ValueError(f"status: one int32 on {device} is needed")
    return status.data_ptr()


def _out(shape, out, dtype, device):
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if dtype is not None and out.dtype != dtype:
        raise ValueError(f"out is {out.dtype}, {dtype} was asked for")
    return out


@functools.lru_cache(maxsize=256)
def _grad_workspace(count: int, rows: int, width: int) -> int:
    size = C.c_size_t()
    _check(load_library().qadam_embedding_grad_query_sizes(count, rows, width, C.byref(size)), "qadam_embedding_grad_query_sizes")
    return size.value


def embedding_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                     out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[..., :] = scale * table[ids[...], :], rounded once to out_dtype (the table's, if not given).

    table: [rows, width]; ids: int32 or int64 of any shape; a negative id gives a row of zeros, and so does one that is
    not below the number of rows, which sets ST_INDEX in `status` too."""
    if not table.is_cuda or table.dim() != 2:
        _need_cuda()
        raise ValueError("table: a CUDA tensor [rows, width] is needed; there is no CPU path")
    device = table.device
    if _elsewhere(device):
        with torch.cuda.device(device):
            return embedding_lookup(table, ids, scale, out_dtype, out, status)
    ids = _tokens(ids, device)
    n, width = table.shape
    shape = ids.shape + (width,)
    stride = width if table.is_contiguous() else _row_stride(table, "table", table.shape, device)
    given = out is not None
    if not given:
        out, out_stride = torch.empty(*shape, dtype=out_dtype or table.dtype, device=device), width
    else:
        out, out_stride = _out(shape, out, out_dtype, device), _row_stride(out, "out", shape, device)
    rc = load_library().qadam_embedding_lookup(
        table.data_ptr(), _type(table, "table"), n, width, stride, ids.data_ptr(), 64 if ids.dtype is torch.int64 else 32,
        ids.numel(), scale, out.data_ptr(), _type(out, "out"), out_stride, None if status is None else _status(status, device),
        stream_of(device))
    if rc:
        _check(rc, "qadam_embedding_lookup")
    if given:
        written(out)
    return out


def held_lookup(wcodes: torch.Tensor, kx: int, ids: torch.Tensor, rows: int, width: int, scale: float = 1.0,
                out_dtype: torch.dtype = torch.bfloat16, first: int = 0, out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The same from the weights that a worker holds: wcodes is the packed broadcast Q_x(x) (uint8) of a problem with weight
    quantizer kx, the table its elements [first, first + rows * width); for a tensor of a parameter vector, first is its
    seg_off.  (QAdam.lookup fills these in.)"""
    if not wcodes.is_cuda:
        _need_cuda()
    if not wcodes.is_cuda or wcodes.dtype != torch.uint8 or not wcodes.is_contiguous():
        raise ValueError("wcodes: a contiguous CUDA tensor of uint8 is needed; there is no CPU path")
    device = wcodes.device
    if _elsewhere(device):
        with torch.cuda.device(device):
            return held_lookup(wcodes, kx, ids, rows, width, scale, out_dtype, first, out, status)
    ids = _tokens(ids, device)
    shape = ids.shape + (width,)
    given = out is not None
    if not given:
        out, out_stride = torch.empty(*shape, dtype=out_dtype, device=device), width
    else:
        out_stride = _row_stride(out, "out", shape, device)
    rc = load_library().qadam_held_lookup(
        wcodes.data_ptr(), wcodes.numel(), kx, first, rows, width, ids.data_ptr(), 64 if ids.dtype is torch.int64 else 32, ids.numel(),
        scale, out.data_ptr(), _type(out, "out"), out_stride, None if status is None else _status(status, device), stream_of(device))
    if rc:
        _check(rc, "qadam_held_lookup")
    if given:
        written(out)
    return out


def embedding_grad(ids: torch.Tensor, dy: torch.Tensor, rows: int, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                   out: Optional[torch.Tensor] = None, accumulate: bool = False, padding: int = -1,
                   status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of embedding_lookup(table, ids, scale) with respect to the table, for the gradient dy of its rows.

    dy: [..., width], rows at equal distances that do not overlap (make an expanded gradient contiguous first).
    -> [rows, width] of `dtype` (dy's, if not given), or `out`: overwritten, or added to where accumulate is true (rows
    without a token are then not touched).  `out` may be a part of a larger buffer, such as a worker's gradient of one tensor
    in the padded layout.  Tokens that are negative or equal to `padding` have no gradient; one that is not below `rows` has
    none either and sets ST_INDEX in `status`.  The sums are binary32 and the same bits every time."""
    if not dy.is_cuda or dy.dim() < 1:
        _need_cuda()
        raise ValueError("dy: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = dy.device, dy.shape[-1]
    if _elsewhere(device):
        with torch.cuda.device(device):
            return embedding_grad(ids, dy, rows, scale, dtype, out, accumulate, padding, status)
    ids = _tokens(ids, device)
    count = ids.numel()
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    given = out is not None
    out = _out((rows, width), out, dtype if dtype is not None or out is not None else dy.dtype, device)
    dy_stride = _row_stride(dy, "dy", ids.shape + (width,), device)
    out_stride = _row_stride(out, "out", (rows, width), device)
    size = _grad_workspace(count, rows, width)
    scratch = torch.empty(size, dtype=torch.uint8, device=device)     # (torch's blocks are 512-byte aligned)
    rc = load_library().qadam_embedding_grad(
        ids.data_ptr(), 64 if ids.dtype is torch.int64 else 32, count, dy.data_ptr(), _type(dy, "dy"), dy_stride, scale, padding,
        out.data_ptr(), _type(out, "out"), rows, width, out_stride, int(accumulate), scratch.data_ptr(), size,
        None if status is None else _status(status, device), stream_of(device))
    if rc:
        _check(rc, "qadam_embedding_grad")
    if given:
        written(out)
    return out
