"""Refusals of layer norm, rows in 8 bits and products in 8 bits, on the host: the C interface checks its arguments before any
CUDA call, so none of this needs a GPU."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2004_14180_b200 as qb
from paper_2004_14180_b200 import build as qbuild
from paper_2004_14180_b200.binding import LAYER_NORM_ARGS, LAYER_NORM_GRAD_ARGS, PRODUCT_ARGS, PackedArgs

NULL, SIZE, LEVEL, ALIGN, WORKSPACE, HYPER, TYPE = -1, -2, -3, -4, -5, -8, -12
A = 1 << 20                                    # an aligned address; nothing here follows it


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    return qb.load_library()


def call(fn, names, base, **kw):
    args = dict(base, **kw)
    if not isinstance(names, PackedArgs):
        assert set(args) == set(names), set(args) ^ set(names)
        return fn(*[args[n] for n in names])
    stream = args.pop("stream")
    assert set(args) <= set(names.fields), set(args) - set(names.fields)
    return fn(names.pack(*[args.get(n) or 0 for n in names.fields]), stream)


@pytest.mark.parametrize("name,packed", [("qadam_layer_norm_args", LAYER_NORM_ARGS), ("qadam_layer_norm_grad_args", LAYER_NORM_GRAD_ARGS),
                                         ("qadam_product_args", PRODUCT_ARGS)])
def test_packed_arguments_are_those_of_the_header(name, packed):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "qadam.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = text[:text.index("} " + name + ";")]
    body = body[body.rindex("typedef struct {") + len("typedef struct {"):]
    names, wide = [], True
    for declaration in body.split(";"):
        if not declaration.strip():
            continue
        fields = declaration.split(",")
        kind = fields[0].split()[0] if "*" not in fields[0] else "*"
        small = kind in ("int32_t", "float")
        assert wide or small                                      # (8 bytes first)
        wide = wide and not small
        names += [f.split()[-1].strip("*") for f in fields]
    assert tuple(names) == packed.fields


def test_no_arguments(lib):
    for fn in (lib.qadam_layer_norm, lib.qadam_layer_norm_grad, lib.qadam_row_product, lib.qadam_held_product):
        assert fn(None, None) == NULL


NORM = LAYER_NORM_ARGS
NORM_BASE = dict(x=A, type=1, x_stride=768, residual=None, residual_stride=0, weight=A, weight_type=0, bias=A, bias_type=0, rows=0, width=768,
                 eps=1e-5, sum=None, sum_stride=0, out=A, out_stride=768, mean=A, rstd=A, q=None, q_stride=0, scale=None, sums=None, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(x=None), 0), (dict(rows=5, x=None), NULL), (dict(rows=-1), SIZE), (dict(rows=1 << 31), SIZE), (dict(width=0), SIZE),
    (dict(width=(1 << 24) + 1, x_stride=1 << 30, out_stride=1 << 30), SIZE), (dict(x_stride=767), SIZE), (dict(out_stride=700), SIZE),
    (dict(type=3), TYPE), (dict(weight_type=7), TYPE), (dict(bias_type=-1), TYPE), (dict(weight=None, weight_type=9), 0),
    (dict(eps=-1e-5), HYPER), (dict(eps=float("nan")), HYPER), (dict(eps=float("inf")), HYPER),
    (dict(residual=A, residual_stride=768), NULL), (dict(sum=A, sum_stride=768), NULL),
    (dict(residual=A, residual_stride=768, sum=A, sum_stride=5), SIZE), (dict(residual=A, residual_stride=7, sum=A, sum_stride=768), SIZE),
    (dict(out=None, mean=None, rstd=None), NULL), (dict(out=None), 0), (dict(q=A, q_stride=768), NULL),
    (dict(q=A, q_stride=768, scale=A), 0), (dict(q=A, q_stride=760, scale=A), SIZE), (dict(q=A, q_stride=776, scale=A), ALIGN),
    (dict(q=A + 8, q_stride=768, scale=A), ALIGN), (dict(x=A + 1), ALIGN), (dict(weight=A + 2), ALIGN), (dict(weight=A + 2, weight_type=1), 0),
    (dict(mean=A + 2), ALIGN), (dict(out=A + 1), ALIGN),
])
def test_layer_norm(lib, kw, code):
    assert call(lib.qadam_layer_norm, NORM, NORM_BASE, **kw) == code


GRAD = LAYER_NORM_GRAD_ARGS
GRAD_BASE = dict(dy=A, type=1, dy_stride=768, x=A, x_stride=768, mean=A, rstd=A, weight=A, weight_type=0, dsum=None, dsum_stride=0, rows=0,
                 width=768, dx=A, dx_stride=768, dweight=None, dbias=None, grad_type=0, accumulate=0, workspace=A, workspace_bytes=1 << 24,
                 stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(grad_type=9), 0), (dict(dweight=A, grad_type=9), TYPE), (dict(dbias=A, accumulate=1, workspace=None, workspace_bytes=0), 0),
    (dict(rows=9, dy=None), NULL), (dict(rows=9, x=None), NULL), (dict(rows=9, mean=None), NULL), (dict(rows=9, rstd=None), NULL),
    (dict(rows=9, dx=None), NULL), (dict(rows=9, dweight=A, workspace=None), NULL), (dict(rows=9, dweight=A, workspace_bytes=64), WORKSPACE),
    (dict(rows=9, dbias=A, workspace=A + 128), ALIGN), (dict(accumulate=2), SIZE), (dict(width=0), SIZE), (dict(rows=-2), SIZE),
    (dict(dy_stride=5), SIZE), (dict(dsum=A, dsum_stride=5), SIZE), (dict(dx_stride=0), SIZE), (dict(type=-1), TYPE), (dict(weight_type=3), TYPE),
    (dict(dweight=A + 2), ALIGN), (dict(dweight=A + 2, grad_type=1, accumulate=1), 0), (dict(mean=A + 1), ALIGN), (dict(dy=A + 1), ALIGN),
])
def test_layer_norm_grad(lib, kw, code):
    assert call(lib.qadam_layer_norm_grad, GRAD, GRAD_BASE, **kw) == code


def test_workspaces(lib):
    size = C.c_size_t()
    for rows, width in ((0, 8), (1, 1), (8192, 768), (30011, 2049), (5, 40001), ((1 << 31) - 1, 8192)):
        assert lib.qadam_layer_norm_grad_query_sizes(rows, width, C.byref(size)) == 0
        assert size.value % 256 == 0 and size.value <= 4096 * 2 * 4 * max(width, 64)
        assert lib.qadam_quantize_columns_query_sizes(rows, width, C.byref(size)) == 0 and size.value % 256 == 0
    assert lib.qadam_layer_norm_grad_query_sizes(1, 0, C.byref(size)) == SIZE
    assert lib.qadam_layer_norm_grad_query_sizes(-1, 8, None) == SIZE
    assert lib.qadam_quantize_columns_query_sizes(1, (1 << 24) + 1, None) == SIZE


ROWS = "x type x_stride columns rows width q q_stride scale sums stream".split()
ROWS_BASE = dict(x=A, type=0, x_stride=100, columns=None, rows=0, width=100, q=A, q_stride=112, scale=A, sums=None, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(rows=3, x=None), NULL), (dict(rows=3, q=None), NULL), (dict(rows=3, scale=None), NULL), (dict(type=5), TYPE), (dict(width=0), SIZE),
    (dict(x_stride=99), SIZE), (dict(q_stride=96), SIZE), (dict(q_stride=104), ALIGN), (dict(q=A + 4), ALIGN), (dict(columns=A + 1), ALIGN),
    (dict(x=A + 2), ALIGN), (dict(sums=A + 2), ALIGN), (dict(rows=1 << 31), SIZE),
])
def test_quantize_rows(lib, kw, code):
    assert call(lib.qadam_quantize_rows, ROWS, ROWS_BASE, **kw) == code


COLUMNS = "x type x_stride rows width q q_stride scale workspace workspace_bytes stream".split()
COLUMNS_BASE = dict(x=A, type=0, x_stride=100, rows=33, width=100, q=A, q_stride=48, scale=A, workspace=A, workspace_bytes=0, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, WORKSPACE), (dict(rows=0), SIZE), (dict(q_stride=32), SIZE), (dict(q_stride=50), ALIGN), (dict(x=None), NULL), (dict(q=None), NULL),
    (dict(scale=None), NULL), (dict(workspace=None), NULL), (dict(workspace=A + 16), ALIGN), (dict(type=3), TYPE), (dict(x_stride=10), SIZE),
    (dict(width=0), SIZE), (dict(q=A + 8), ALIGN),
])
def test_quantize_columns(lib, kw, code):
    assert call(lib.qadam_quantize_columns, COLUMNS, COLUMNS_BASE, **kw) == code


HELD = "wcodes wcode_bytes kx first rows width q q_stride scale stream".split()
HELD_BASE = dict(wcodes=A, wcode_bytes=1280, kx=6, first=0, rows=0, width=100, q=A, q_stride=112, scale=None, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(kx=7), LEVEL), (dict(kx=-1), LEVEL), (dict(wcodes=None), NULL), (dict(rows=2, q=None), NULL), (dict(rows=13), SIZE),
    (dict(rows=12, first=100), SIZE), (dict(first=-1), SIZE), (dict(first=1281), SIZE), (dict(wcode_bytes=1281), SIZE), (dict(q_stride=100), SIZE),
    (dict(q_stride=120), ALIGN), (dict(wcodes=A + 8), ALIGN), (dict(q=A + 8), ALIGN), (dict(scale=A + 2), ALIGN), (dict(width=0), SIZE),
])
def test_held_rows(lib, kw, code):
    assert call(lib.qadam_held_rows, HELD, HELD_BASE, **kw) == code


PRODUCT = PRODUCT_ARGS
PRODUCT_BASE = dict(a=A, a_stride=64, a_scale=A, rows=0, depth=64, b=A, b_stride=64, b_scale=A, b_worth=1.0, channels=10, transposed=0, bias=None,
                    bias_type=0, out=A, out_type=1, out_stride=10, accumulate=0, status=None, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(b_scale=None), 0), (dict(rows=4, a=None), NULL), (dict(rows=4, a_scale=None), NULL), (dict(rows=4, out=None), NULL),
    (dict(rows=4, b=None), NULL), (dict(rows=(1 << 31) - 511), SIZE), (dict(channels=1 << 31, out_stride=1 << 31), SIZE), (dict(depth=0), SIZE), (dict(depth=131073, a_stride=131088, b_stride=131088), SIZE),
    (dict(channels=0), SIZE), (dict(a_stride=48), SIZE), (dict(a_stride=72), ALIGN), (dict(b_stride=48), SIZE), (dict(b_stride=68), ALIGN),
    (dict(a=A + 8), ALIGN), (dict(b=A + 8), ALIGN), (dict(transposed=2), SIZE), (dict(transposed=1), SIZE), (dict(transposed=1, b_scale=None), 0),
    (dict(transposed=1, b_scale=None, b_stride=0), SIZE), (dict(accumulate=-1), SIZE), (dict(out_type=3), TYPE), (dict(bias=A, bias_type=4), TYPE),
    (dict(bias=A + 2), ALIGN), (dict(out=A + 1), ALIGN), (dict(out_stride=9), SIZE), (dict(status=A + 2), ALIGN), (dict(a_scale=A + 2), ALIGN),
])
def test_row_product(lib, kw, code):
    assert call(lib.qadam_row_product, PRODUCT, PRODUCT_BASE, **kw) == code


HELD_PRODUCT = PRODUCT_ARGS
HELD_PRODUCT_BASE = dict(a=A, a_stride=64, a_scale=A, a_sums=A, rows=0, depth=64, b=A, wcode_bytes=1280, kx=6, first=0, channels=20, transposed=0,
                         bias=None, bias_type=0, out=A, out_type=1, out_stride=20, accumulate=0, status=None, stream=None)


@pytest.mark.parametrize("kw,code", [
    ({}, 0), (dict(kx=5), LEVEL), (dict(kx=14), LEVEL), (dict(b=None), NULL), (dict(rows=2, a_sums=None), NULL), (dict(channels=21, out_stride=21), SIZE),
    (dict(first=128), SIZE), (dict(first=128, channels=18), 0), (dict(first=8), ALIGN), (dict(first=-16), SIZE), (dict(b=A + 4), ALIGN),
    (dict(depth=50), ALIGN), (dict(transposed=1), ALIGN), (dict(transposed=1, channels=16), 0), (dict(transposed=1, channels=32, out_stride=32), SIZE),
    (dict(a_sums=A + 1), ALIGN), (dict(a_stride=32), SIZE),
])
def test_held_product(lib, kw, code):
    assert call(lib.qadam_held_product, HELD_PRODUCT, HELD_PRODUCT_BASE, **kw) == code


def test_there_is_no_cpu_path(lib):
    x, q = torch.ones(4, 16), torch.ones(4, 16, dtype=torch.int8)
    codes = torch.zeros(128, dtype=torch.uint8)
    for f in (lambda: qb.layer_norm(x), lambda: qb.layer_norm_grad(x, x, x[:, 0], x[:, 0]), lambda: qb.quantize_rows(x), lambda: qb.quantize_columns(x),
              lambda: qb.Int8Rows(q, x[:, 0].clone()), lambda: qb.held_rows(codes, 6, 2, 16)):
        with pytest.raises((RuntimeError, ValueError)):
            f()
