"""Layer norm of token rows and its gradients (include/qadam.h).

Calls run on the current stream of x's device.  Neither is recorded by autograd: the gradients are layer_norm_grad.
"""
from __future__ import annotations

import ctypes as C
import functools
from math import inf
from typing import NamedTuple, Optional, Tuple

import torch

from .adamw import _need_cuda, stream_of, written
from .binding import LAYER_NORM_ARGS, LAYER_NORM_GRAD_ARGS, _check, load_library
from .embedding import _elsewhere, _row_stride, _type
from .int8 import Int8Rows


MOST_F32 = 3.4028234663852886e38      # beyond it struct raises an error of its own


class Normed(NamedTuple):
    """out: the normed rows (None if not asked for); sum: x + residual, rounded (x itself without a residual); mean, rstd: of the
    rows, float32, flat; rows: out in 8 bits before its rounding (None if not asked for)."""
    out: Optional[torch.Tensor]
    sum: torch.Tensor
    mean: torch.Tensor
    rstd: torch.Tensor
    rows: Optional[Int8Rows]


def _like(x: torch.Tensor, whole: bool) -> torch.Tensor:
    """A contiguous tensor of x's shape and type (empty_like of a contiguous one is: 1.3 us, not 3.5)."""
    return torch.empty_like(x) if whole else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def _parameter(t: Optional[torch.Tensor], what: str, width: int, device: torch.device):
    if t is None:
        return 0, 0
    if t.device != device or t.shape != (width,) or not t.is_contiguous():
        raise ValueError(f"{what}: {width} contiguous elements on {device} are needed")
    return t.data_ptr(), _type(t, what)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               residual: Optional[torch.Tensor] = None, dense: bool = True, int8: bool = False) -> Normed:
    """Layer norm over the last dimension of x [..., width] (float32, bfloat16 or float16; rows at equal distances), of x + residual if
    a residual is given (x's shape and type).

    weight, bias: [width], of any of the three types each.  dense: give `out`, of x's type; int8: give `rows`, for a product in 8 bits."""
    if not x.is_cuda or x.dim() < 1:
        _need_cuda()
        raise ValueError("x: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = x.device, x.shape[-1]
    if _elsewhere(device):
        with torch.cuda.device(device):
            return layer_norm(x, weight, bias, eps, residual, dense, int8)
    if width < 1:
        raise ValueError("x: rows of no elements")
    n = x.numel() // width
    kind = _type(x, "x")
    whole = x.is_contiguous()
    stride = width if whole else _row_stride(x, "x", x.shape, device)
    weight_at, weight_type = _parameter(weight, "weight", width, device)
    bias_at, bias_type = _parameter(bias, "bias", width, device)
    total, residual_at, residual_stride = x, 0, 0
    if residual is not None:
        if residual.dtype != x.dtype:
            raise ValueError(f"residual is {residual.dtype}, x {x.dtype}")
        residual_at, residual_stride = residual.data_ptr(), _row_stride(residual, "residual", x.shape, device)
        total = _like(x, whole)
    out = _like(x, whole) if dense else None
    mean = torch.empty(n, dtype=torch.float32, device=device)
    rstd = torch.empty(n, dtype=torch.float32, device=device)
    rows = Int8Rows._make(n, width, device, True) if int8 else None
    if n:
        rc = load_library().qadam_layer_norm(LAYER_NORM_ARGS.pack(
            x.data_ptr(), stride, residual_at, residual_stride, weight_at, bias_at, n, width, 0 if residual is None else total.data_ptr(), width,
            0 if out is None else out.data_ptr(), width, mean.data_ptr(), rstd.data_ptr(), *((0, 0, 0, 0) if rows is None else rows._at()),
            kind, weight_type, bias_type, eps if -MOST_F32 <= eps <= MOST_F32 else inf), stream_of(device))
        if rc:
            _check(rc, "qadam_layer_norm")
    return Normed(out, total, mean, rstd, rows)


@functools.lru_cache(maxsize=256)
def _grad_workspace(rows: int, width: int) -> int:
    size = C.c_size_t()
    _check(load_library().qadam_layer_norm_grad_query_sizes(rows, width, C.byref(size)), "qadam_layer_norm_grad_query_sizes")
    return size.value


def layer_norm_grad(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                    dsum: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                    accumulate: bool = False, grad_dtype: torch.dtype = torch.float32) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """-> (dx, dweight, dbias) from dy, the gradient of layer_norm's out; x: what was normed (`sum`); mean, rstd: as it gave them.

    dsum: the gradient that reaches `sum` by other ways: dx is then the gradient of x and of the residual both.  dy, x and dsum have one
    type and one shape.  dweight, dbias: buffers ([width], contiguous, of one type) to overwrite, or to add to with accumulate, such as a
    worker's gradient of one tensor in the padded layout; made here, of grad_dtype, if not given (accumulate needs both).  The
    sums over rows are binary32 and the same bits every time."""
    if not x.is_cuda or x.dim() < 1:
        _need_cuda()
        raise ValueError("x: a CUDA tensor [..., width] is needed; there is no CPU path")
    device, width = x.device, x.shape[-1]
    if _elsewhere(device):
        with torch.cuda.device(device):
            return layer_norm_grad(dy, x, mean, rstd, weight, dsum, dweight, dbias, accumulate, grad_dtype)
    if width < 1:
        raise ValueError("x: rows of no elements")
    n = x.numel() // width
    kind = _type(x, "x")
    for t, what in ((dy, "dy"), (dsum, "dsum")):
        if t is not None and t.dtype != x.dtype:
            raise ValueError(f"{what} is {t.dtype}, x {x.dtype}")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        if t.device != device or t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{what}: {n} contiguous float32 on {device} are needed")
    if accumulate and (dweight is None or dbias is None):
        raise ValueError("accumulate needs dweight and dbias")
    given = [t for t in (dweight, dbias) if t is not None]
    if given:
        grad_dtype = given[0].dtype
    dweight = torch.empty(width, dtype=grad_dtype, device=device) if dweight is None else dweight
    dbias = torch.empty(width, dtype=grad_dtype, device=device) if dbias is None else dbias
    dw_at, dw_type = _parameter(dweight, "dweight", width, device)
    db_at, db_type = _parameter(dbias, "dbias", width, device)
    if dw_type != db_type:
        raise ValueError(f"dweight is {dweight.dtype}, dbias {dbias.dtype}")
    weight_at, weight_type = _parameter(weight, "weight", width, device)
    whole = x.is_contiguous()
    x_stride, dy_stride = width if whole else _row_stride(x, "x", x.shape, device), _row_stride(dy, "dy", x.shape, device)
    ds_at, ds_stride = (0, 0) if dsum is None else (dsum.data_ptr(), _row_stride(dsum, "dsum", x.shape, device))
    dx = _like(x, whole)
    size = _grad_workspace(n, width)
    scratch = torch.empty(size, dtype=torch.uint8, device=device)
    rc = load_library().qadam_layer_norm_grad(LAYER_NORM_GRAD_ARGS.pack(
        dy.data_ptr(), dy_stride, x.data_ptr(), x_stride, mean.data_ptr(), rstd.data_ptr(), weight_at, ds_at, ds_stride, n, width, dx.data_ptr(), width,
        dw_at, db_at, scratch.data_ptr(), size, kind, weight_type, dw_type, int(accumulate)), stream_of(device))
    if rc:
        _check(rc, "qadam_layer_norm_grad")
    for t in given:
        written(t)
    return dx, dweight, dbias
