"""Layer norm, its gradients, and rows and columns in 8 bits against plain statements in binary64."""
import pytest
import torch

from _layer import DTYPES, HALF, TINY, U, gen_of, grad64, norm64, randn, rows8

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

WIDTHS = [1, 7, 8, 130, 256, 257, 512, 768, 771, 1000, 1024, 1025, 1032, 2049, 4096, 8200, 16384, 16392, 20001, 32776, 40001]


def near(got, want, off, kind):
    """The error is at most `off`, and the rounding to the type."""
    err = (got.double() - want).abs()
    assert bool((err <= off + HALF[kind] * (want.abs() + off) + TINY[kind]).all()), float((err - off - HALF[kind] * want.abs()).max())


def same(a, b):
    """Equal, NaN where the other is NaN."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(nan=7.0), b.nan_to_num(nan=7.0))


def inputs(gen, rows, width, kind, offset=1.0):
    return (randn(gen, rows, width) + offset * randn(gen, rows, 1)).to(DTYPES[kind])


@pytest.mark.parametrize("kind,w_kind", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("width", WIDTHS)
def test_norm(width, kind, w_kind):
    gen = gen_of(width, len(kind), 3)
    for rows in (1, 9):
        x = inputs(gen, rows, width, kind)
        w, b = (1 + 0.2 * randn(gen, width)).to(DTYPES[w_kind]), (0.2 * randn(gen, width)).to(DTYPES[w_kind])
        for args in ((w, b), (None, b), (w, None), (None, None)):
            got = qb.layer_norm(x, *args, eps=1e-5)
            want, mean, rstd, off, mean_off, rstd_off = norm64(x.double(), *args, 1e-5)
            assert got.sum is x and got.rows is None
            near(got.out, want, off, kind)
            near(got.mean, mean, mean_off, "f32")
            near(got.rstd, rstd, rstd_off, "f32")


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [5, 768, 1001, 4096, 33000])
def test_norm_of_a_sum_and_in_8_bits(width, kind):
    gen = gen_of(width, len(kind), 5)
    x, r = inputs(gen, 6, width, kind), inputs(gen, 6, width, kind)
    w, b = 1 + 0.2 * randn(gen, width), 0.2 * randn(gen, width)
    got = qb.layer_norm(x, w, b, eps=1e-12, residual=r, int8=True)
    h = (x.float() + r.float()).to(x.dtype)
    assert torch.equal(got.sum, h)
    want, _, _, off, _, _ = norm64(h.double(), w, b, 1e-12)
    near(got.out, want, off, kind)
    # quantized from binary32: the largest value is off by `off`, and each value by half a step and by its own
    step = want.abs().amax(1, keepdim=True) / 127
    err = (got.rows.values().double() - want).abs()
    assert bool((err <= step * 0.5 * (1 + 2.0 ** -20) + 2 * off.amax(1, keepdim=True)).all())
    assert bool((got.rows.q.abs().amax(1) == 127).all()) and torch.equal(got.rows.sums, got.rows.q.sum(1, dtype=torch.int32))
    only = qb.layer_norm(x, w, b, eps=1e-12, residual=r, int8=True, dense=False)
    assert only.out is None and torch.equal(only.rows.q, got.rows.q) and torch.equal(only.rows.scale, got.rows.scale)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 7), (700, 8), (50, 130), (3001, 768), (1203, 1000), (40, 1024), (901, 1025), (17, 2049),
                                        (310, 4096), (5, 8192), (30, 8200), (3, 40001)])
def test_norm_grad(rows, width, kind):
    gen = gen_of(rows, width, len(kind))
    x = inputs(gen, rows, width, kind)
    w = (1 + 0.2 * randn(gen, width)).to(DTYPES["bf16" if kind == "bf16" else "f32"])
    ran = qb.layer_norm(x, w, eps=1e-5)
    dy, ds = ((randn(gen, rows, width) * 1e-2).to(DTYPES[kind]) for _ in range(2))
    for weight, more in ((w, None), (None, ds), (w, ds)):
        dx, dw, db = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, weight, dsum=more)
        wx, ww, wb, off, sw, sb = grad64(dy, x, ran.mean, ran.rstd, weight, more)
        assert dx.dtype == x.dtype and dw.dtype == torch.float32
        near(dx, wx, off, kind)
        # a row's term has 3 roundings; a sum of so many terms in any order is off by no more than rows - 1 roundings of the sum of
        # magnitudes, and no thread adds more than its share of the rows, a 64th or more of them being shared out, and 80
        few = 3 + min(rows, rows / 64 + 80)
        near(dw, ww, few * U * sw, "f32")
        near(db, wb, few * U * sb, "f32")
        again = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, weight, dsum=more)
        assert torch.equal(again[1], dw) and torch.equal(again[2], db)


def test_norm_grad_by_differences():
    gen = gen_of(77)
    x, w, b, dy = randn(gen, 3, 96), 1 + 0.2 * randn(gen, 96), 0.2 * randn(gen, 96), randn(gen, 3, 96)
    ran = qb.layer_norm(x, w, b, eps=1e-3)
    dx, dw, db = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, w)

    def loss(x, w, b):
        return float((norm64(x, w, b, 1e-3)[0] * dy.double()).sum())
    h = 1e-5                                    # differences in binary64: off by h^2 and 1e-16 / h
    for grad, at in ((dx, 0), (dw, 1), (db, 2)):
        args = [x.double(), w.double(), b.double()]
        for i in (0, 50, 95):
            for sign in (1, -1):
                moved = [a.clone() for a in args]
                moved[at].view(-1)[i] += sign * h
                up = loss(*moved) if sign > 0 else up
                down = loss(*moved)
            assert abs((up - down) / (2 * h) - float(grad.view(-1)[i])) < 1e-5 * max(1.0, float(grad.abs().max()))


@pytest.mark.parametrize("kind,g_kind", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f16")])
def test_norm_grad_into_a_workers_gradient(kind, g_kind):
    gen = gen_of(91, len(g_kind))
    rows, width = 333, 768
    x, dy = inputs(gen, rows, width, kind), (randn(gen, rows, width) * 1e-2).to(DTYPES[kind])
    ran = qb.layer_norm(x)
    room = (randn(gen, 5000)).to(DTYPES[g_kind])
    before = room.clone()
    dw, db = room[128:128 + width], room[1025:1025 + width]
    out = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, dweight=dw, dbias=db, accumulate=True)
    assert out[1] is dw and out[2] is db
    _, ww, wb, _, sw, sb = grad64(dy, x, ran.mean, ran.rstd, None, None)
    few = 90
    near(dw, ww + before[128:128 + width].double(), few * U * sw + U * ww.abs(), g_kind)
    near(db, wb + before[1025:1025 + width].double(), few * U * sb + U * wb.abs(), g_kind)
    mask = torch.ones(5000, dtype=torch.bool, device="cuda")
    mask[128:128 + width] = mask[1025:1025 + width] = False
    assert torch.equal(room[mask], before[mask])


def test_norm_empty_shapes_and_strides():
    gen = gen_of(13)
    none = qb.layer_norm(torch.empty(0, 768, device="cuda"), int8=True)
    assert none.out.shape == (0, 768) and none.mean.shape == (0,) and none.rows.q.shape == (0, 768)
    empty = torch.empty(0, 768, device="cuda")
    dx, dw, db = qb.layer_norm_grad(empty, empty, none.mean, none.rstd)
    assert dx.shape == (0, 768) and not dw.any() and not db.any()
    kept = torch.ones(768, device="cuda")
    qb.layer_norm_grad(empty, empty, none.mean, none.rstd, dweight=kept, dbias=kept.clone(), accumulate=True)
    assert bool((kept == 1).all())
    big = randn(gen, 2, 3, 900)
    for x in (big[..., 3:3 + 768], big[..., 4:4 + 768], big[..., :768]):
        got = qb.layer_norm(x)
        assert got.out.shape == (2, 3, 768) and got.mean.shape == (6,)
        assert torch.equal(got.out, qb.layer_norm(x.contiguous()).out) or x.data_ptr() % 16
        want, _, _, off, _, _ = norm64(x.reshape(6, 768).double(), None, None, 1e-5)
        near(got.out.view(6, 768), want, off, "f32")
        dy = torch.flip(big, (0, 1))[..., 5:5 + 768]
        got = qb.layer_norm_grad(dy, x, got.mean, got.rstd, dsum=x)
        want = grad64(dy.reshape(6, 768), x.reshape(6, 768), *[t for t in qb.layer_norm(x)[2:4]], None, x.reshape(6, 768))
        near(got[0].view(6, 768), want[0], want[3], "f32")


def test_rows_of_one_value_and_rows_that_are_not_finite():
    x = torch.full((4, 512), 3.0, device="cuda")
    x[1, 7], x[2, 9] = float("inf"), float("nan")
    got = qb.layer_norm(x, int8=True)
    assert not got.out[0].any() and not got.out[3].any()                 # no spread: xhat = 0
    assert bool(got.out[1].isnan().any()) and bool(got.out[2].isnan().all())
    assert bool(got.rows.scale[1:3].isnan().all()) and bool(torch.isfinite(got.rows.scale[[0, 3]]).all())
    q = qb.quantize_rows(x)
    want, scale = rows8(x)
    assert torch.equal(q.q, want) and same(q.scale, scale)
    c = qb.quantize_columns(x)
    want, scale = rows8(x.T)
    assert torch.equal(c.q, want) and same(c.scale, scale)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_rows_in_8_bits(width, kind):
    gen = gen_of(width, len(kind), 21)
    x = (randn(gen, 11, width) * torch.exp2(8 * randn(gen, 11, 1))).to(DTYPES[kind])
    x[3] = 0
    x[4, 0] = 2.0 ** -24                                                 # alone, or far below the others
    columns = torch.exp2(randn(gen, width))
    for factors in (None, columns):
        got = qb.quantize_rows(x, columns=factors)
        q, scale = rows8(x, factors)
        assert torch.equal(got.q, q) and same(got.scale, scale) and torch.equal(got.sums, q.sum(1, dtype=torch.int32))
        assert got.q.stride(0) % 16 == 0 and got.q.data_ptr() % 16 == 0
    tiny = torch.full((2, width), 1e-42, device="cuda")
    assert not qb.quantize_rows(tiny).q.any()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 768), (5, 64), (130, 63), (128, 256), (200, 1000), (4099, 264), (33, 2049)])
def test_columns_in_8_bits(rows, width, kind):
    gen = gen_of(rows, width, len(kind), 4)
    x = (randn(gen, rows, width) * torch.exp2(4 * randn(gen, 1, width))).to(DTYPES[kind])
    x[:, width // 2] = 0
    got = qb.quantize_columns(x)
    q, scale = rows8(x.T)
    assert got.q.shape == (width, rows) and torch.equal(got.q, q) and same(got.scale, scale) and got.sums is None
    wide = torch.zeros(rows, width + 3, dtype=DTYPES[kind], device="cuda")
    wide[:, 1:1 + width] = x
    again = qb.quantize_columns(wide[:, 1:1 + width])
    assert torch.equal(again.q, q) and same(again.scale, scale)
