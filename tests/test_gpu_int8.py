"""Products in 8 bits, dense and with held weights, against whole-number sums in binary64."""
import pytest
import torch

from _layer import DTYPES, HALF, TINY, U, gen_of, pack, randn

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


def int8_rows(gen, rows, width, full=False):
    from paper_2004_14180_b200.int8 import empty_rows
    q = empty_rows(rows, width, torch.device("cuda"))
    q.copy_(torch.randint(-127, 128, (rows, width), generator=gen, device="cuda") if not full else torch.full((rows, width), 127))
    return qb.Int8Rows(q, torch.exp2(randn(gen, rows)), q.sum(1, dtype=torch.int32))


def scaled(a, scale):
    return qb.Int8Rows(a.q, scale, a.sums)


def check(got, a, b, b_scale, bias, kind, before=None):
    """got = sa sb (a b^T) + bias (+ before): the sum is rounded once, two products, a sum, perhaps another sum."""
    whole = a.q.double() @ b.double().T                        # (exact: below 2^53)
    main = whole * a.scale.double()[:, None] * b_scale.double()
    want = main if bias is None else main + bias.double()
    off = 3 * U * main.abs() + U * want.abs()
    if before is not None:
        want = want + before.double()
        off = off + U * want.abs()
    err = (got.double() - want).abs()
    off = off * 1.01
    assert bool((err <= off + HALF[kind] * (want.abs() + off) + TINY[kind]).all()), float(err.max())


SIZES = [(1, 1, 1), (1, 16, 8), (1, 4096, 512), (2, 100, 130), (3, 128, 128), (16, 768, 768), (17, 769, 129), (33, 1000, 257), (64, 2048, 1000),
         (65, 64, 3000), (128, 130, 640), (129, 768, 2304), (300, 257, 1537), (513, 768, 768), (1000, 48, 4097), (2049, 1536, 700), (4099, 300, 2500), (6000, 130, 1537)]


@pytest.mark.parametrize("m,k,n", SIZES)
def test_product(m, k, n):
    gen = gen_of(m, k, n)
    a, b = int8_rows(gen, m, k), int8_rows(gen, n, k)
    bias = randn(gen, n) * 1000
    for kind, more in (("f32", None), ("bf16", bias), ("f16", bias.half())):
        got = qb.int8_matmul(a, b, bias=more, out_dtype=DTYPES[kind])
        if kind == "f16":                                      # (beyond binary16 the result is infinite)
            got = got.float().clamp(-65504, 65504)
            fits = (a.q.double() @ b.q.double().T * a.scale.double()[:, None] * b.scale.double() + more.double()).abs() < 65000
            assert got.shape == (m, n)
            small = qb.int8_matmul(scaled(a, a.scale * 2.0 ** -10), b, out_dtype=torch.float16)
            check(small.clamp(-65504, 65504)[:, :1], scaled(a, a.scale * 2.0 ** -10), b.q[:1], b.scale[:1], None, kind) if bool(fits.all()) else None
        else:
            check(got, a, b.q, b.scale, more, kind)
    # transposed: the scales of b's rows are left to a
    c = int8_rows(gen, k, n)
    check(qb.int8_matmul(a, c, out_dtype=torch.float32, transpose=True), a, c.q.T, torch.ones(n, device="cuda"), None, "f32")


def test_sums_at_the_ends_of_their_range():
    gen = gen_of(5)
    k = 131072
    a, b = int8_rows(gen, 2, k, full=True), int8_rows(gen, 130, k, full=True)
    b.q[1::2] = -128                                           # (a's sums hold, b's are not looked at)
    one = torch.ones(2, device="cuda")
    a = scaled(a, one)
    b = scaled(b, torch.ones(130, device="cuda"))
    got = qb.int8_matmul(a, b, out_dtype=torch.float32)
    want = torch.tensor([127.0 * 127 * k, -127.0 * 128 * k] * 65, dtype=torch.float64).float().cuda()
    assert torch.equal(got, want.expand(2, 130))
    codes = torch.full((130 * k,), 128, dtype=torch.uint8, device="cuda")
    codes[k:2 * k] = 0
    got = qb.held_matmul(a, codes, 6, 130, k, out_dtype=torch.float32)
    want = torch.full((2, 130), 127 * k / 2, device="cuda")
    want[:, 1] *= -1
    assert torch.equal(got, want)


@pytest.mark.parametrize("kx", range(7))
@pytest.mark.parametrize("m,k,n,first", [(1, 768, 300, 0), (5, 33, 17, 131), (70, 129, 256, 128), (600, 768, 400, 256)])
def test_held(kx, m, k, n, first):
    gen = gen_of(kx, m, k, n)
    level = torch.randint(-(1 << kx), (1 << kx) + 1, (first + n * k,), generator=gen, device="cuda")
    codes = pack(level, kx)
    table = level[first:].view(n, k)
    worth = torch.full((n,), 2.0 ** -(kx + 1), device="cuda")
    w = qb.held_rows(codes, kx, n, k, first)
    assert torch.equal(w.q.long(), table) and torch.equal(w.scale, worth)
    a, c = int8_rows(gen, m, k), int8_rows(gen, m, n)
    bias = randn(gen, n)
    check(qb.held_matmul(a, codes, kx, n, k, first, bias=bias, out_dtype=torch.float32), a, table, worth, bias, "f32")
    check(qb.held_matmul(c, codes, kx, n, k, first, transpose=True, out_dtype=torch.bfloat16), c, table.T,
          torch.full((k,), 2.0 ** -(kx + 1), device="cuda"), None, "bf16")


def test_strides_accumulation_and_what_lies_around():
    gen = gen_of(8)
    m, k, n = 77, 200, 333
    pitched = torch.randint(-127, 128, (m, 3 * 208), generator=gen, device="cuda").to(torch.int8)
    a = qb.Int8Rows(pitched[:, 208:208 + k], torch.exp2(randn(gen, m)), None)
    b = int8_rows(gen, n, k)
    for kind in ("f32", "bf16", "f16"):
        room = randn(gen, m + 2, n + 7).to(DTYPES[kind])
        before = room.clone()
        out = room[1:1 + m, 3:3 + n]
        small = scaled(a, a.scale * 2.0 ** -16)
        assert qb.int8_matmul(small, b, out=out, accumulate=True) is out
        check(out, small, b.q, b.scale, None, kind, before[1:1 + m, 3:3 + n])
        keep = torch.ones_like(room, dtype=torch.bool)
        keep[1:1 + m, 3:3 + n] = False
        assert torch.equal(room[keep], before[keep])
    none = qb.int8_matmul(int8_rows(gen, 0, k), b)
    assert none.shape == (0, n) and none.dtype == torch.bfloat16


def test_scale_that_is_not_finite_stays_in_its_row():
    gen = gen_of(9)
    x = randn(gen, 40, 256)
    x[5, 3] = float("nan")
    y = qb.int8_matmul(qb.quantize_rows(x), int8_rows(gen, 99, 256), out_dtype=torch.float32)
    assert bool(y[5].isnan().all()) and bool(torch.isfinite(y[torch.arange(40, device="cuda") != 5]).all())
