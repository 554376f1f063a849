"""Layer norm with weight and bias of types of their own, wherever they lie, on every route of the norm and of its gradient."""
import pytest
import torch

from _layer import DTYPES, U, gen_of, grad64, norm64, randn
from test_gpu_layer_norm import near

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


def parameter(values, kind, left):
    """`values` in a type, `left` elements from 16 bytes, NaN around them."""
    room = torch.full((values.numel() + left + 8,), float("nan"), dtype=DTYPES[kind], device="cuda")
    room[left:left + values.numel()] = values
    return room[left:left + values.numel()]


# a warp to a row, rows that a warp goes along, a group of warps, rows read again; pieces of 16 bytes and elements
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(3, 8), (5, 768), (5, 769), (15000, 72), (15000, 71), (40, 1032), (40, 4096), (7, 4097), (5, 16384), (2, 20000)])
@pytest.mark.parametrize("w_kind,w_left,b_kind,b_left", [("f32", 0, "bf16", 0), ("bf16", 0, "f32", 0), ("f16", 1, "f16", 0), ("f32", 1, "f32", 3), ("bf16", 3, None, 0),
                                                         (None, 0, "f16", 1)])
def test_parameters_of_any_type_anywhere(rows, width, kind, w_kind, w_left, b_kind, b_left):
    gen = gen_of(rows, width, w_left, 71)
    x = (randn(gen, rows, width) + randn(gen, rows, 1)).to(DTYPES[kind])
    w = None if w_kind is None else parameter(1 + 0.2 * randn(gen, width), w_kind, w_left)
    b = None if b_kind is None else parameter(0.2 * randn(gen, width), b_kind, b_left)
    got = qb.layer_norm(x, w, b, int8=True)
    want, mean, rstd, off, mean_off, rstd_off = norm64(x.double(), w, b, 1e-5)
    near(got.out, want, off, kind)
    near(got.mean, mean, mean_off, "f32")
    near(got.rstd, rstd, rstd_off, "f32")
    step = want.abs().amax(1, keepdim=True) / 127
    assert bool(((got.rows.values().double() - want).abs() <= step * 0.5 * (1 + 2.0 ** -20) + 2 * off.amax(1, keepdim=True)).all())
    if w is None:
        return
    dy = (randn(gen, rows, width) * 1e-2).to(DTYPES[kind])
    dx, dw, db = qb.layer_norm_grad(dy, x, got.mean, got.rstd, w)
    wx, ww, wb, off, sw, sb = grad64(dy, x, got.mean, got.rstd, w, None)
    near(dx, wx, off, kind)
    few = 3 + min(rows, rows / 64 + 80)
    near(dw, ww, few * U * sw, "f32")
    near(db, wb, few * U * sb, "f32")
