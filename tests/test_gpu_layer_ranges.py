"""Layer norm and its gradients at the ends of what binary32 holds, against plain statements in binary64."""
import pytest
import torch

from _layer import DTYPES, gen_of, grad64, randn
from test_gpu_layer_norm import near

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


# every way that a row's elements are dealt out, with threads or elements beyond the row: a warp to a row, a group of warps, rows read again,
# pieces of 16 bytes and elements
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", [7, 128, 200, 520, 521, 769, 1032, 1537, 3000, 5128, 7008, 7009, 8200])
def test_gradient_of_rows_whose_mean_times_rstd_is_beyond_binary32(width, kind):
    gen = gen_of(width, len(kind), 61)
    x = torch.full((9, width), 3e33, device="cuda").to(DTYPES[kind])
    mean, rstd = x[:, 0].float().contiguous(), torch.full((9,), 1e6, device="cuda")          # (3e39 is infinite)
    dy, ds = ((randn(gen, 9, width) * 1e-2).to(DTYPES[kind]) for _ in range(2))
    w = 1 + 0.2 * randn(gen, width)
    for weight, more in ((None, None), (w, ds)):
        dx, dw, db = qb.layer_norm_grad(dy, x, mean, rstd, weight, dsum=more)
        want, _, wb, off, _, sb = grad64(dy, x, mean, rstd, weight, more)
        near(dx, want, off, kind)
        assert not dw.any()                                                     # x is its row's mean: xhat = 0
        near(db, wb, 9 * 2.0 ** -24 * sb, "f32")                                # nine terms in any order


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(3, 41), (3, 896), (3, 1000), (8000, 1000), (3, 3584), (2000, 3584), (3, 7001), (2, 20001)])
def test_rows_of_one_whole_number_have_no_spread(rows, width, kind):
    # The sum is a whole number below 2^24, so exact, and the mean is the value: xhat = 0, and rstd = 1 / sqrt(eps), of which quotient, sum, root and
    # reciprocal leave 3 halves of a step: the root's argument is eps itself.
    x = torch.arange(1, rows + 1, device="cuda").remainder(256).to(DTYPES[kind])[:, None].repeat(1, width)
    b = torch.full((width,), 0.75, device="cuda")
    for eps in (1e-12, 1e-5):
        got = qb.layer_norm(x, None, b, eps=eps, int8=True)
        assert torch.equal(got.mean, x[:, 0].float())
        want = 1 / torch.tensor(eps, dtype=torch.float32, device="cuda").double().sqrt()
        assert bool(((got.rstd.double() - want).abs() <= 3 * 2.0 ** -24 * want).all())
        assert bool((got.out == 0.75).all()) and bool((got.rows.q == 127).all())
    # and the gradient of equal gradients is nothing: g is its own mean
    dy = torch.full_like(x, 3.0)
    dx, dw, db = qb.layer_norm_grad(dy, x, got.mean, got.rstd)
    assert not dx.any() and not dw.any() and torch.equal(db, torch.full_like(db, 3.0 * rows))


@pytest.mark.parametrize("width", [3, 41, 896, 1000, 1025, 3584, 7001, 16384, 20001])
def test_means_of_whole_numbers_are_rounded_once(width):
    # sums of whole numbers below 2^24 are exact in any order, and the mean is the quotient, correctly rounded (as torch's division is)
    gen = gen_of(width, 62)
    x = torch.randint(-300, 701, (500, width), generator=gen, device="cuda").float()
    got = qb.layer_norm(x)
    assert torch.equal(got.mean, x.double().sum(1).float() / torch.full((500,), float(width), device="cuda"))
    big = torch.full((2, width), 3e38, device="cuda")                             # sums beyond binary32: as sum / width has it
    assert bool(qb.layer_norm(big).mean.isinf().all())


@pytest.mark.parametrize("eps", [1e39, -1e39, float("inf"), float("nan"), -1e-5])
def test_an_eps_that_is_not_one_is_refused(eps):
    with pytest.raises(qb.QAdamError) as e:
        qb.layer_norm(torch.ones(2, 8, device="cuda"), eps=eps)
    assert e.value.code == -8
