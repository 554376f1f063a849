"""Rows of an embedding table, dense or as a worker holds them, and the table's gradient (include/qadam.h).

All calls run on the current stream of the table's device.  `status`, where given, is one int32 on the
device that gets ST_INDEX if a token is not below the number of rows; the caller clears and reads it.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .adamw import _need_cuda, element_type, stream_of
from .binding import _check, load_library


def _tokens(ids: torch.Tensor, device: torch.device) -> torch.Tensor:
    if ids.dtype not in (torch.int64, torch.int32):
        raise ValueError(f"ids: int64 or int32 is needed, got {ids.dtype}")
    if ids.device != device:
        raise ValueError(f"ids on {ids.device}, table on {device}")
    return ids.contiguous()


def _rows(t: torch.Tensor, what: str, shape, device: torch.device) -> torch.Tensor:
    """`t` as [rows, width] with its columns next to each other; a view, never a copy."""
    if t.device != device or tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: {tuple(shape)} on {device} is needed, got {tuple(t.shape)} on {t.device}")
    try:
        flat = t.view(-1, shape[-1])
    except RuntimeError:
        raise ValueError(f"{what}: its rows must lie at equal distances") from None
    if (flat.shape[-1] > 1 and flat.stride(-1) != 1) or (flat.shape[0] > 1 and flat.stride(0) < flat.shape[1]):
        raise ValueError(f"{what}: a row's elements must be next to each other, and rows must not overlap")
    return flat


def _stride(flat: torch.Tensor) -> int:
    return flat.stride(0) if flat.shape[0] > 1 else max(flat.shape[1], 1)


def _status(status: Optional[torch.Tensor], device: torch.device):
    if status is None:
        return None
    if status.device != device or status.dtype != torch.int32 or status.numel() != 1:
        raise ValueError(f"status: one int32 on {device} is needed")
    return status.data_ptr()


def _out(ids, width, out, dtype, device):
    shape = tuple(ids.shape) + (width,)
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if dtype is not None and out.dtype != dtype:
        raise ValueError(f"out is {out.dtype}, out_dtype {dtype}")
    return out


def embedding_lookup(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out_dtype: Optional[torch.dtype] = None,
                     out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[..., :] = scale * table[ids[...], :], rounded once to out_dtype (the table's, if not given).

    table: [rows, width]; ids: int32 or int64 of any shape; a negative id gives a row of zeros, and so does one that is
    not below the number of rows, which sets ST_INDEX in `status` too."""
    _need_cuda()
    if not table.is_cuda or table.dim() != 2:
        raise ValueError("table: a CUDA tensor [rows, width] is needed; there is no CPU path")
    device = table.device
    ids = _tokens(ids, device)
    n, width = table.shape
    flat = _rows(table, "table", table.shape, device)
    dtype = out_dtype if out_dtype is not None or out is not None else table.dtype
    out = _out(ids, width, out, dtype, device)
    o = _rows(out, "out", tuple(ids.shape) + (width,), device)
    with torch.cuda.device(device):
        _check(load_library().qadam_embedding_lookup(
            table.data_ptr(), element_type(table.dtype, "table"), n, width, _stride(flat), ids.data_ptr(), 8 * ids.element_size(),
            ids.numel(), scale, out.data_ptr(), element_type(out.dtype, "out"), _stride(o), _status(status, device),
            stream_of(device)), "qadam_embedding_lookup")
    return out


def held_lookup(wcodes: torch.Tensor, kx: int, ids: torch.Tensor, rows: int, width: int, scale: float = 1.0,
                out_dtype: torch.dtype = torch.bfloat16, first: int = 0, out: Optional[torch.Tensor] = None,
                status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The same from the weights that a worker holds: wcodes is the packed broadcast Q_x(x) (uint8) of a problem with weight
    quantizer kx, the table its elements [first, first + rows * width); for a tensor of a parameter vector, first is its
    seg_off.  (QAdam.lookup fills these in.)"""
    _need_cuda()
    if not wcodes.is_cuda or wcodes.dtype != torch.uint8 or not wcodes.is_contiguous():
        raise ValueError("wcodes: a contiguous CUDA tensor of uint8 is needed; there is no CPU path")
    device = wcodes.device
    ids = _tokens(ids, device)
    out = _out(ids, width, out, None if out is not None else out_dtype, device)
    o = _rows(out, "out", tuple(ids.shape) + (width,), device)
    with torch.cuda.device(device):
        _check(load_library().qadam_held_lookup(
            wcodes.data_ptr(), wcodes.numel(), kx, first, rows, width, ids.data_ptr(), 8 * ids.element_size(), ids.numel(), scale,
            out.data_ptr(), element_type(out.dtype, "out"), _stride(o), _status(status, device), stream_of(device)),
            "qadam_held_lookup")
    return out


def embedding_grad(ids: torch.Tensor, dy: torch.Tensor, rows: int, scale: float = 1.0, dtype: Optional[torch.dtype] = None,
                   out: Optional[torch.Tensor] = None, accumulate: bool = False, padding: int = -1,
                   status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradient of embedding_lookup(table, ids, scale) with respect to the table, for the gradient dy of its rows.

    -> [rows, width] of `dtype` (dy's, if not given), or `out`: overwritten, or added to where accumulate is true (rows
    without a token are then not touched).  `out` may be a part of a larger buffer, such as a worker's gradient of one tensor
    in the padded layout.  Tokens that are negative or equal to `padding` have no gradient; one that is not below `rows` has
    none either and sets ST_INDEX in `status`.  The sums are binary32 and the same bits every time."""
    _need_cuda()
    if not dy.is_cuda or dy.dim() < 1:
        raise ValueError("dy: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = dy.device, dy.shape[-1]
    ids = _tokens(ids, device)
    if accumulate and out is None:
        raise ValueError("accumulate needs out")
    if out is None:
        out = torch.empty(rows, width, dtype=dtype if dtype is not None else dy.dtype, device=device)
    elif dtype is not None and out.dtype != dtype:
        raise ValueError(f"out is {out.dtype}, dtype {dtype}")
    d = _rows(dy, "dy", tuple(ids.shape) + (width,), device)
    o = _rows(out, "out", (rows, width), device)
    L, size = load_library(), C.c_size_t()
    _check(L.qadam_embedding_grad_query_sizes(ids.numel(), rows, width, C.byref(size)), "qadam_embedding_grad_query_sizes")
    with torch.cuda.device(device):
        scratch = torch.empty(size.value, dtype=torch.uint8, device=device)     # (torch's blocks are 512-byte aligned)
        _check(L.qadam_embedding_grad(
            ids.data_ptr(), 8 * ids.element_size(), ids.numel(), dy.data_ptr(), element_type(dy.dtype, "dy"), _stride(d), scale, padding,
            out.data_ptr(), element_type(out.dtype, "out"), rows, width, _stride(o), int(accumulate), scratch.data_ptr(), size.value,
            _status(status, device), stream_of(device)), "qadam_embedding_grad")
    return out
