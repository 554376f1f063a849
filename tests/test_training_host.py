"""Refusals of the operators around the quantized step, on the host: the C interface checks its arguments before any CUDA
call, so none of this needs a GPU."""
import ctypes as C

import pytest
import torch

import paper_2004_14180_b200 as qb
from paper_2004_14180_b200 import build as qbuild
from paper_2004_14180_b200.binding import AdamWBuffers, AdamWConfig, TensorList

NULL, SIZE, ALIGN, WORKSPACE, STEP, LEVEL, HYPER, TYPE = -1, -2, -4, -5, -6, -3, -8, -12
A = 1 << 20                                    # an aligned address; nothing here follows it


@pytest.fixture(scope="module")
def lib():
    qbuild.build()
    return qb.load_library()


def _i64(*v):
    return (C.c_int64 * len(v))(*v)


def _i32(*v):
    return (C.c_int32 * len(v))(*v)


def _f32(*v):
    return (C.c_float * len(v))(*v)


def _cfg(**kw):
    base = dict(num_tensors=3, state_bits=32, len=_i64(5, 0, 300), weight_type=None, grad_type=None, decay=None, beta1=0.9,
                beta2=0.999, eps=1e-8, lr=1e-3, master=0, reserved=0, seed=0)
    base.update(kw)
    return AdamWConfig(**base)


def test_error_text(lib):
    assert qb.qadam_strerror(TYPE) == "element type, code width or state width not offered"


def test_adamw_sizes_and_layout(lib):
    D, off, size = C.c_int64(), (C.c_int64 * 3)(), C.c_size_t()
    assert lib.qadam_adamw_query_sizes(C.byref(_cfg()), C.byref(D), off, C.byref(size)) == 0
    assert D.value == 128 + 0 + 384 and list(off) == [0, 128, 128] and size.value % 256 == 0
    assert lib.qadam_adamw_query_sizes(C.byref(_cfg()), None, None, None) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(num_tensors=0), SIZE), (dict(num_tensors=(1 << 20) + 1), SIZE), (dict(reserved=1), SIZE), (dict(len=None), NULL),
    (dict(len=_i64(5, -1, 2)), SIZE), (dict(len=_i64(1 << 41, 1, 1)), SIZE), (dict(state_bits=16), TYPE), (dict(state_bits=0), TYPE),
    (dict(weight_type=_i32(0, 3, 0)), TYPE), (dict(grad_type=_i32(0, 0, -1)), TYPE), (dict(master=2), SIZE),
    (dict(beta1=1.0), HYPER), (dict(beta1=float("nan")), HYPER), (dict(beta2=-0.1), HYPER), (dict(eps=0.0), HYPER), (dict(eps=1e-31), HYPER),
    (dict(eps=float("inf")), HYPER), (dict(lr=-1.0), HYPER), (dict(lr=float("nan")), HYPER),
    (dict(decay=_f32(0.0, -1.0, 0.0)), HYPER), (dict(decay=_f32(0.0, float("inf"), 0.0)), HYPER),
])
def test_adamw_configurations_are_refused(lib, kw, code):
    cfg = _cfg(**kw)
    assert lib.qadam_adamw_query_sizes(C.byref(cfg), None, None, None) == code
    ctx = C.c_void_p(5)
    bufs = AdamWBuffers()
    assert lib.qadam_adamw_create(C.byref(cfg), C.byref(bufs), C.byref(ctx)) == code and not ctx.value


def _bufs(**kw):
    w = (C.c_void_p * 3)(A, None, A + 4096)
    base = dict(weights=w, master=None, m=A, v=A, m_scale=None, r_scale=None, count=A, workspace=A, workspace_bytes=1 << 20, status=A)
    base.update(kw)
    return AdamWBuffers(**base)


@pytest.mark.parametrize("cfg,kw,code", [
    ({}, dict(weights=None), NULL), ({}, dict(m=None), NULL), ({}, dict(v=None), NULL), ({}, dict(status=None), NULL),
    ({}, dict(count=None), NULL), ({}, dict(workspace=None), NULL), (dict(master=1), {}, NULL), (dict(state_bits=8), {}, NULL),
    (dict(state_bits=8), dict(m_scale=A), NULL), ({}, dict(weights=(C.c_void_p * 3)(A, None, None)), NULL),
    ({}, dict(weights=(C.c_void_p * 3)(A, None, A + 2)), ALIGN), ({}, dict(m=A + 8), ALIGN), ({}, dict(v=A + 4), ALIGN),
    (dict(master=1), dict(master=A + 4), ALIGN), (dict(state_bits=8), dict(m_scale=A, r_scale=A + 4), ALIGN),
    ({}, dict(count=A + 4), ALIGN), ({}, dict(status=A + 1), ALIGN), ({}, dict(workspace=A + 128), ALIGN),
    ({}, dict(workspace_bytes=255), WORKSPACE),
])
def test_adamw_buffers_are_refused(lib, cfg, kw, code):
    ctx = C.c_void_p()
    assert lib.qadam_adamw_create(C.byref(_cfg(**cfg)), C.byref(_bufs(**kw)), C.byref(ctx)) == code and not ctx.value


def test_null_contexts(lib):
    assert lib.qadam_adamw_create(None, None, None) == NULL
    assert lib.qadam_adamw_bind(None, (C.c_void_p * 1)(A)) == NULL
    assert lib.qadam_adamw_step(None, 1, 0.1, None, None) == NULL
    assert lib.qadam_adamw_step_counted(None, None, None, None) == NULL
    assert lib.qadam_adamw_moments(None, A, A, None) == NULL
    assert lib.qadam_adamw_poll_status(None, None, None) == NULL
    assert lib.qadam_adamw_destroy(None) == NULL and lib.qadam_adamw_launch_count(None) == NULL
    assert lib.qadam_norm_bind(None, None) == NULL and lib.qadam_norm_run(None, 1.0, A, None) == NULL
    assert lib.qadam_norm_destroy(None) == NULL and lib.qadam_norm_launch_count(None) == NULL


def test_norm_lists(lib):
    size, ctx = C.c_size_t(), C.c_void_p()
    ok = TensorList(2, 0, _i64(5, 9000), _i32(0, 1))
    assert lib.qadam_norm_query_sizes(C.byref(ok), C.byref(size)) == 0 and size.value % 256 == 0
    assert lib.qadam_norm_create(C.byref(ok), None, size.value, C.byref(ctx)) == NULL
    assert lib.qadam_norm_create(C.byref(ok), A + 64, size.value, C.byref(ctx)) == ALIGN
    assert lib.qadam_norm_create(C.byref(ok), A, size.value - 1, C.byref(ctx)) == WORKSPACE
    assert lib.qadam_norm_create(C.byref(ok), A, size.value, None) == NULL
    for bad, code in ((TensorList(0, 0, _i64(1), None), SIZE), (TensorList(1, 1, _i64(1), None), SIZE), (TensorList(1, 0, None, None), NULL),
                      (TensorList(1, 0, _i64(-1), None), SIZE), (TensorList(1, 0, _i64(1), _i32(7)), TYPE)):
        assert lib.qadam_norm_query_sizes(C.byref(bad), None) == code
        assert lib.qadam_norm_create(C.byref(bad), A, 1 << 20, C.byref(ctx)) == code and not ctx.value
    assert lib.qadam_norm_query_sizes(None, None) == NULL


def _lookup(lib, **kw):
    a = dict(table=A, type=0, rows=10, width=8, stride=8, ids=A, id_bits=64, count=4, scale=1.0, out=A, out_type=0, out_stride=8,
             status=None)
    a.update(kw)
    return lib.qadam_embedding_lookup(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), NULL), (dict(ids=None), NULL), (dict(out=None), NULL), (dict(type=3), TYPE), (dict(out_type=-1), TYPE),
    (dict(id_bits=16), TYPE), (dict(rows=0), SIZE), (dict(width=0), SIZE), (dict(stride=7), SIZE), (dict(out_stride=7), SIZE),
    (dict(count=-1), SIZE), (dict(scale=float("nan")), HYPER), (dict(table=A + 2), ALIGN), (dict(type=1, table=A + 1), ALIGN),
    (dict(ids=A + 4), ALIGN), (dict(out=A + 2), ALIGN), (dict(status=A + 2), ALIGN), (dict(count=0), 0),
])
def test_lookup_is_refused(lib, kw, code):
    assert _lookup(lib, **kw) == code


def _held(lib, **kw):
    a = dict(wcodes=A, bytes=160, kx=6, first=0, rows=10, width=16, ids=A, id_bits=64, count=4, scale=1.0, out=A, out_type=0,
             out_stride=16, status=None)
    a.update(kw)
    return lib.qadam_held_lookup(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(wcodes=None), NULL), (dict(kx=-1), LEVEL), (dict(kx=15), LEVEL), (dict(wcodes=A + 4), ALIGN), (dict(bytes=159), SIZE),
    (dict(rows=11), SIZE), (dict(first=1), SIZE), (dict(first=-1), SIZE), (dict(first=1 << 60), SIZE), (dict(bytes=0), SIZE),
    (dict(rows=1 << 40, width=1 << 24, out_stride=1 << 24), SIZE), (dict(width=0), SIZE), (dict(out=None), NULL), (dict(count=0), 0),
])
def test_held_lookup_is_refused(lib, kw, code):
    assert _held(lib, **kw) == code


def _grad(lib, **kw):
    a = dict(ids=A, id_bits=64, count=4, dy=A, dy_type=0, dy_stride=8, scale=1.0, padding=-1, grad=A, grad_type=0, rows=10, width=8,
             grad_stride=8, accumulate=1, workspace=A, bytes=1 << 30, status=None)
    a.update(kw)
    return lib.qadam_embedding_grad(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(ids=None), NULL), (dict(dy=None), NULL), (dict(grad=None), NULL), (dict(workspace=None), NULL), (dict(id_bits=8), TYPE),
    (dict(dy_type=3), TYPE), (dict(grad_type=3), TYPE), (dict(count=-1), SIZE), (dict(count=(1 << 30) + 1), SIZE), (dict(rows=0), SIZE),
    (dict(rows=0x7FFFFFFF), SIZE), (dict(width=0), SIZE), (dict(width=(1 << 22) + 1, dy_stride=1 << 23, grad_stride=1 << 23), SIZE),
    (dict(dy_stride=7), SIZE), (dict(grad_stride=7), SIZE), (dict(accumulate=2), SIZE), (dict(scale=float("inf")), HYPER),
    (dict(grad=A + 2), ALIGN), (dict(dy=A + 2), ALIGN), (dict(ids=A + 4), ALIGN), (dict(workspace=A + 128), ALIGN),
    (dict(status=A + 1), ALIGN), (dict(bytes=256), WORKSPACE), (dict(count=0, workspace=None, ids=None, dy=None), 0),
])
def test_gradient_is_refused(lib, kw, code):
    assert _grad(lib, **kw) == code


def test_gradient_workspace_grows_with_the_batch(lib):
    size, last = C.c_size_t(), 0
    for count in (0, 1, 1000, 100000):
        assert lib.qadam_embedding_grad_query_sizes(count, 30522, 768, C.byref(size)) == 0 and size.value >= last
        last = size.value
    assert lib.qadam_embedding_grad_query_sizes(-1, 10, 10, C.byref(size)) == SIZE


def test_no_cpu_path():
    w = torch.zeros(4, 8)
    ids = torch.zeros(3, dtype=torch.int64)
    error = ValueError if torch.cuda.is_available() else RuntimeError
    for call in (lambda: qb.AdamW([w], [w]), lambda: qb.GradNorm([w]), lambda: qb.embedding_lookup(w, ids),
                 lambda: qb.held_lookup(w.to(torch.uint8), 6, ids, 4, 8), lambda: qb.embedding_grad(ids, torch.zeros(3, 8), 4)):
        with pytest.raises(error):
            call()
