"""Products in 8 bits with results in binary16, every value of them, and results at the ends of a type's range."""
import pytest
import torch

from _layer import gen_of, pack, randn
from test_gpu_int8 import check, int8_rows, scaled

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


# results in boxes, with two boxes to a warp (sums of less than 16 blocks of 128) and with one; rows that do not begin on 16 bytes; few tokens
@pytest.mark.parametrize("m,k,n", [(1, 4096, 512), (17, 769, 129), (64, 2048, 1000), (129, 768, 2304), (300, 257, 1537), (300, 2048, 512), (300, 1920, 514),
                                   (513, 4096, 264), (1000, 48, 4096), (2049, 2304, 776), (4099, 300, 2500), (700, 2049, 97)])
def test_results_in_binary16(m, k, n):
    gen = gen_of(m, k, n, 7)
    a, b, bias = int8_rows(gen, m, k), int8_rows(gen, n, k), randn(gen, n)
    # sums of k products are below 5 sqrt(k) 74^2 or so, scales below 2^5 each: times 2^-17 all of it is in range
    a = scaled(a, a.scale * 2.0 ** -17)
    for more in (None, bias, bias.half()):
        got = qb.int8_matmul(a, b, bias=more, out_dtype=torch.float16)
        assert bool(torch.isfinite(got).all())
        check(got, a, b.q, b.scale, more, "f16")
    c = int8_rows(gen, k, n)
    got = qb.int8_matmul(a, c, out_dtype=torch.float16, transpose=True)
    assert bool(torch.isfinite(got).all())
    check(got, a, c.q.T, torch.ones(n, device="cuda"), None, "f16")


@pytest.mark.parametrize("kx", [2, 6])
@pytest.mark.parametrize("m,k,n", [(20, 768, 300), (600, 768, 400), (600, 2304, 272)])
def test_held_results_in_binary16(kx, m, k, n):
    gen = gen_of(kx, m, k, n, 8)
    level = torch.randint(-(1 << kx), (1 << kx) + 1, (n * k,), generator=gen, device="cuda")
    codes, table = pack(level, kx), level.view(n, k)
    a, c = int8_rows(gen, m, k), int8_rows(gen, m, n)
    a, c = scaled(a, a.scale * 2.0 ** -8), scaled(c, c.scale * 2.0 ** -8)
    for got, rows, weights in ((qb.held_matmul(a, codes, kx, n, k, out_dtype=torch.float16), a, table),
                               (qb.held_matmul(c, codes, kx, n, k, out_dtype=torch.float16, transpose=True), c, table.T)):
        assert bool(torch.isfinite(got).all())
        check(got, rows, weights, torch.full((weights.shape[0],), 2.0 ** -(kx + 1), device="cuda"), None, "f16")


@pytest.mark.parametrize("m", [40, 300])
@pytest.mark.parametrize("n", [256, 259])
def test_what_is_beyond_binary16_is_infinite(m, n):
    gen = gen_of(m, n, 9)
    a, b = int8_rows(gen, m, 512), int8_rows(gen, n, 512)
    one = torch.ones(n, device="cuda")
    a, b = scaled(a, torch.ones(m, device="cuda")), scaled(b, one)
    # whole numbers below 2^24: exact, rounded once to binary16
    want = (a.q.double() @ b.q.double().T).float().half()
    assert bool(want.isinf().any()) and bool(want.isfinite().any())
    assert torch.equal(qb.int8_matmul(a, b, out_dtype=torch.float16), want)


@pytest.mark.parametrize("m,left", [(16, 0), (300, 0), (300, 1)])
def test_sums_that_are_added_to_keep_numbers_below_the_normal_ones(m, left):
    # few tokens, boxes, elements; kept, added and what is left of normal numbers: as a binary32 sum has it
    q = torch.zeros(m, 64, dtype=torch.int8, device="cuda")
    q[:, 0] = 1
    a = qb.Int8Rows(q, torch.ones(m, device="cuda"))
    least = 2.0 ** -126
    for before, more in ((1e-41, 0.0), (0.0, 1e-41), (1.5 * least, -least), (1e-41, 2e-41), (-1e-41, least), (least, 2.0 ** -140)):
        b = qb.Int8Rows(q[:1].expand(300, 64).contiguous(), torch.full((300,), more, device="cuda"))
        out = torch.full((m, 304), before, device="cuda")[:, left:left + 300]
        want = (out.double() + b.scale.double()).float()
        assert torch.equal(qb.int8_matmul(a, b, out=out, accumulate=True), want) and bool((want != 0).all())
