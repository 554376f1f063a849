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
