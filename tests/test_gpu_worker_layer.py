"""The operators as a worker of the quantized step uses them: rows of the embedding that it holds, a layer norm, a layer on the 8-bit
weights that it holds, the gradients of all of them into its part of g, and the step."""
import pytest
import torch

from _layer import rows8

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

ROWS, WIDTH, OUT, TOKENS = 200, 96, 48, 500
SEG = [ROWS * WIDTH, WIDTH, WIDTH, OUT * WIDTH, OUT]


def problem(kx):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x1 = torch.randn(sum(SEG), generator=gen, device="cuda") * 0.1
    x1[SEG[0]:SEG[0] + WIDTH] = 0.45                              # the norm's weight: the grid ends at 1/2
    q = qb.QAdam(SEG, 2, kg=0, kx=kx, x1=x1, lr=1e-3)
    ids = torch.randint(0, ROWS, (TOKENS,), generator=gen, device="cuda")
    target = torch.randn(TOKENS, OUT, generator=gen, device="cuda")
    return q, ids, target


def held(q, segment):
    """A tensor as the workers hold it."""
    n = SEG[segment]
    return q.lookup(segment, n, torch.zeros(1, dtype=torch.int64, device="cuda"), out_dtype=torch.float32)[0]


def gradient(q, ids, target, g):
    """Of sum (y - target)^2 / (2 tokens), into g [D].  -> what the comparison needs"""
    views = [g[o:o + n] for o, n in zip(q.seg_off, SEG)]
    gamma, beta, bias = held(q, 1), held(q, 2), held(q, 4)
    x = q.lookup(0, WIDTH, ids, scale=8.0, out_dtype=torch.float32)
    r = qb.layer_norm(x, gamma, beta, eps=1e-5, int8=True)
    y = q.matmul(3, WIDTH, r.rows, bias=bias, out_dtype=torch.float32)
    dy = (y - target) / TOKENS
    rows = qb.quantize_rows(dy)
    dxn = q.matmul(3, WIDTH, rows, transpose=True, out_dtype=torch.float32)
    dx, _, _ = qb.layer_norm_grad(dxn, x, r.mean, r.rstd, gamma, dweight=views[1], dbias=views[2])
    dyc, xc = qb.quantize_columns(dy), qb.quantize_columns(r.out)
    qb.int8_matmul(dyc, xc, out=views[3].view(OUT, WIDTH))
    views[4].copy_(dy.sum(0))
    qb.embedding_grad(ids, dx, ROWS, scale=8.0, out=views[0].view(ROWS, WIDTH))
    return views, x, r, y, dy, rows, dxn, dx, dyc, xc


@pytest.mark.parametrize("kx", [6, 4])
def test_a_workers_gradient(kx):
    q, ids, target = problem(kx)
    g = torch.zeros(q.D, device="cuda")
    views, x, r, y, dy, rows, dxn, dx, dyc, xc = gradient(q, ids, target, g)
    # each part in binary64 from what the part before has given, quantized as stated
    weight, gamma, beta = held(q, 3).double().view(OUT, WIDTH), held(q, 1).double(), held(q, 2).double()
    table = held(q, 0).double().view(ROWS, WIDTH)
    assert torch.equal(x.double(), table[ids] * 8)
    h = x.double()
    xn = (h - h.mean(1, keepdim=True)) / torch.sqrt(h.var(1, correction=0, keepdim=True) + 1e-5) * gamma + beta
    # binary32: a few dozen roundings of 2^-24, relative to the largest values
    assert float((r.out.double() - xn).abs().max()) <= 64 * 2.0 ** -24 * float(xn.abs().max())
    assert float((r.rows.values().double() - xn).abs().max()) <= float(xn.abs().max()) / 127 * 0.5 * (1 + 1e-4)
    want = r.rows.values().double() @ weight.T + held(q, 4).double()
    # one rounding of the scale (2^-24 of each value), then three of the result
    assert float((y.double() - want).abs().max()) <= 5 * 2.0 ** -24 * float((r.rows.values().double().abs() @ weight.abs().T).max() + 1)
    assert torch.equal(rows.q, rows8(dy)[0])
    want = rows.values().double() @ weight
    assert float((dxn.double() - want).abs().max()) <= 5 * 2.0 ** -24 * float((rows.values().double().abs() @ weight.abs()).max())
    xhat = (h - r.mean.double()[:, None]) * r.rstd.double()[:, None]
    d = dxn.double() * gamma
    want = r.rstd.double()[:, None] * (d - d.mean(1, keepdim=True) - xhat * (d * xhat).mean(1, keepdim=True))
    assert float((dx.double() - want).abs().max()) <= 64 * 2.0 ** -24 * float(want.abs().max()) * 4
    for got, terms in ((views[1], dxn.double() * xhat), (views[2], dxn.double())):
        assert float((got.double() - terms.sum(0)).abs().max()) <= 100 * 2.0 ** -24 * float(terms.abs().sum(0).max())
    want = dyc.values().double() @ xc.values().double().T
    size = dyc.values().double().abs() @ xc.values().double().abs().T
    assert float((views[3].view(OUT, WIDTH).double() - want).abs().max()) <= 5 * 2.0 ** -24 * float(size.max())
    # 8 bits along 500 tokens: each value off by at most half a step of its column's 127
    whole, step = dy.double().T @ r.out.double(), 0.5 * 1.01
    may = step * (dyc.scale.double()[:, None] * r.out.double().abs().sum(0) + xc.scale.double() * dyc.values().double().abs().sum(1)[:, None])
    assert bool(((views[3].view(OUT, WIDTH).double() - whole).abs() <= may).all())
    total = torch.zeros(ROWS, WIDTH, dtype=torch.float64, device="cuda").index_add_(0, ids, dx.double() * 8)
    assert float((views[0].view(ROWS, WIDTH).double() - total).abs().max()) <= 64 * 2.0 ** -24 * float(total.abs().max()) * 4
    mask = torch.ones(q.D, dtype=torch.bool, device="cuda")
    for o, n in zip(q.seg_off, SEG):
        mask[o:o + n] = False
    assert not g[mask].any()                                      # pads stay zero
    q.close()


def test_steps_on_these_gradients():
    q, ids, target = problem(6)
    g = torch.zeros(2, q.D, device="cuda")
    first = None
    for t in range(1, 4):
        for i in range(2):
            _, _, _, y, dy, *_ = gradient(q, ids, target, g[i])
            g[i].mul_(1 if i else 0.5)
        first = y.clone() if first is None else first
        q.step(t, g)
    assert q.poll_status() == 0 and not torch.equal(gradient(q, ids, target, g[0])[3], first)
    with pytest.raises(ValueError):
        q.matmul(3, WIDTH + 1, qb.quantize_rows(target))
    q.close()
    plain = qb.QAdam([OUT * WIDTH], 1, kx=-1)
    with pytest.raises(ValueError):
        plain.matmul(0, WIDTH, qb.quantize_rows(target))
    plain.close()
