"""What layer norm, rows in 8 bits and their products promise beside their values: refusals, streams, captured calls, what is left
alone, what autograd is told, results added to in every way that there is."""
import numpy as np
import pytest
import torch

from _layer import DTYPES, U, gen_of, grad64, randn
from test_gpu_int8 import check, int8_rows, scaled
from test_gpu_layer_norm import near, norm64

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402
from paper_2004_14180_b200.int8 import empty_rows  # noqa: E402


def test_refusals():
    x, w = torch.ones(4, 32, device="cuda"), torch.ones(32, device="cuda")
    r = qb.layer_norm(x)
    q = qb.quantize_rows(x)
    codes = torch.zeros(1024, dtype=torch.uint8, device="cuda")
    for f in (lambda: qb.layer_norm(x.cpu()), lambda: qb.layer_norm(x.double()), lambda: qb.layer_norm(x, w[:31]), lambda: qb.layer_norm(x, w.cpu()),
              lambda: qb.layer_norm(x, w.double()), lambda: qb.layer_norm(x, residual=x.half()), lambda: qb.layer_norm(x, residual=x[:3]),
              lambda: qb.layer_norm(x.t()), lambda: qb.layer_norm(torch.ones(4, 0, device="cuda")), lambda: qb.layer_norm(x[:1].expand(4, 32)),
              lambda: qb.layer_norm(x, torch.ones(64, device="cuda")[::2]),
              lambda: qb.layer_norm_grad(x.half(), x, r.mean, r.rstd), lambda: qb.layer_norm_grad(x, x, r.mean[:3], r.rstd),
              lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd.double()), lambda: qb.layer_norm_grad(x[:3], x, r.mean, r.rstd),
              lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd, accumulate=True), lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd, dweight=w[:5]),
              lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd, dweight=w.clone(), dbias=w.half()), lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd, dsum=x.half()),
              lambda: qb.quantize_rows(x.long()), lambda: qb.quantize_rows(x, columns=w.half()), lambda: qb.quantize_rows(x, columns=w[:4]),
              lambda: qb.quantize_columns(x[:0]), lambda: qb.quantize_columns(x.bool()),
              lambda: qb.Int8Rows(q.q, q.scale[:3]), lambda: qb.Int8Rows(q.q, q.scale.half()), lambda: qb.Int8Rows(q.q.float(), q.scale),
              lambda: qb.Int8Rows(q.q, q.scale, q.scale), lambda: qb.Int8Rows(torch.zeros(4, 33, dtype=torch.int8, device="cuda"), q.scale),
              lambda: qb.Int8Rows(torch.zeros(200, dtype=torch.int8, device="cuda")[8:136].view(4, 32), q.scale),
              lambda: qb.Int8Rows(q.q, q.scale.cpu()), lambda: qb.Int8Rows(q.q.t(), torch.ones(32, device="cuda")),
              lambda: qb.int8_matmul(q, qb.quantize_rows(x[:, :16])), lambda: qb.int8_matmul(q, q, transpose=True),
              lambda: qb.int8_matmul(q, q, accumulate=True), lambda: qb.int8_matmul(q, q, out=torch.zeros(4, 5, device="cuda")),
              lambda: qb.int8_matmul(q, q, bias=w), lambda: qb.int8_matmul(q, q, out_dtype=torch.float64),
              lambda: qb.int8_matmul(q, q, out=torch.zeros(4, 4, device="cuda"), out_dtype=torch.float16),
              lambda: qb.int8_matmul(q, q, status=torch.zeros(1, device="cuda")), lambda: qb.int8_matmul(q, q, out=torch.zeros(4, 8, device="cuda")[:, ::2]),
              lambda: qb.held_matmul(q, codes, 6, 4, 16), lambda: qb.held_matmul(qb.Int8Rows(q.q, q.scale), codes, 6, 4, 32),
              lambda: qb.held_matmul(q, codes.int(), 6, 4, 32), lambda: qb.held_rows(codes, 6, -1, 32), lambda: qb.held_rows(codes, 6, 1, 0)):
        with pytest.raises(ValueError):
            f()
    for f, code in ((lambda: qb.held_matmul(q, codes, 7, 4, 32), -3), (lambda: qb.held_matmul(q, codes, 6, 33, 32), -2),
                    (lambda: qb.held_rows(codes, 6, 2, 32, first=1000), -2), (lambda: qb.layer_norm(x, eps=-1.0), -8),
                    (lambda: qb.held_matmul(q, torch.zeros(1040, dtype=torch.uint8, device="cuda")[8:1032], 6, 4, 32), -4),
                    (lambda: qb.int8_matmul(int8_rows(gen_of(1), 1, 131088), int8_rows(gen_of(1), 1, 131088)), -2)):
        with pytest.raises(qb.QAdamError) as e:
            f()
        assert e.value.code == code


def chain(x, dy, w, b, weights, grad):
    """A norm, a layer, its gradients."""
    r = qb.layer_norm(x, w, b, int8=True)
    y = qb.int8_matmul(r.rows, weights, out_dtype=torch.float32)
    dxn = qb.int8_matmul(qb.quantize_rows(dy, columns=weights.scale), weights, out_dtype=torch.bfloat16, transpose=True)
    dx, dw, db = qb.layer_norm_grad(dxn, x, r.mean, r.rstd, w)
    qb.int8_matmul(qb.quantize_columns(dy), qb.quantize_columns(r.out), out=grad)
    return y, dx, dw, db, grad


def chain_inputs(seed, tokens=700, width=264, n=400):
    gen = gen_of(seed, 41)
    x, dy = randn(gen, tokens, width).bfloat16(), (randn(gen, tokens, n) * 1e-2).bfloat16()
    return x, dy, 1 + 0.1 * randn(gen, width), 0.1 * randn(gen, width), int8_rows(gen, n, width), torch.empty(n, width, device="cuda")


def copied(rows):
    q = empty_rows(rows.rows, rows.width, rows.device)
    q.copy_(rows.q)
    return qb.Int8Rows(q, rows.scale.clone())


def same(a, b):
    return all(torch.equal(s, t) for s, t in zip(a, b))


def test_another_stream_waits_for_nothing_but_its_own():
    args = chain_inputs(1)
    want = [t.clone() for t in chain(*args)]
    busy = torch.ones(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        torch.mm(busy, busy)
    with torch.cuda.stream(s):
        args[-1].zero_()
        got = chain(*args)
        s.synchronize()
        assert same(got, want)
    torch.cuda.synchronize()


def test_captured_calls_replay_on_new_inputs():
    args = [chain_inputs(seed) for seed in (2, 3, 4)]
    want = [[t.clone() for t in chain(*a)] for a in args]
    graphs, outs = [], []
    held = [[t.clone() if isinstance(t, torch.Tensor) else copied(t) for t in args[0]] for _ in range(2)]
    for h in held:                                              # two graphs, by turns
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(chain(*h))
        graphs.append(g)
    for i in (0, 1, 2, 0):
        for k in (0, 1):
            for t, new in zip(held[k], args[(i + k) % 3]):
                if isinstance(t, torch.Tensor):
                    t.copy_(new)
            weights = args[(i + k) % 3][4]
            held[k][4].q.copy_(weights.q)
            held[k][4].scale.copy_(weights.scale)
            graphs[k].replay()
            torch.cuda.synchronize()
            assert same(outs[k], want[(i + k) % 3])


def test_calls_in_inference_mode_and_empty_batches():
    with torch.inference_mode():
        x = torch.randn(5, 48, device="cuda")
        r = qb.layer_norm(x, int8=True)
        out = torch.zeros(5, 5, device="cuda")
        assert qb.int8_matmul(r.rows, r.rows, out=out) is out and bool(out.any())
    none = torch.empty(0, 48, device="cuda")
    q = qb.quantize_rows(none)
    assert q.q.shape == (0, 48) and q.scale.shape == (0,) and q.sums.shape == (0,)
    assert qb.int8_matmul(q, r.rows).shape == (0, 5)
    codes = torch.zeros(256, dtype=torch.uint8, device="cuda")
    assert qb.held_matmul(q, codes, 6, 5, 48).shape == (0, 5) and qb.held_rows(codes, 3, 0, 48).q.shape == (0, 48)


@pytest.mark.parametrize("call", ["product", "held", "norm grad"])
def test_a_backward_pass_through_an_overwritten_result_is_refused(call):
    x = torch.ones(4, 32, device="cuda")
    q, codes, r = qb.quantize_rows(x), torch.zeros(128, dtype=torch.uint8, device="cuda"), qb.layer_norm(x)
    out, s = torch.empty(32 if call == "norm grad" else (4, 4), device="cuda"), torch.ones(1, device="cuda", requires_grad=True)
    run = {"product": lambda: qb.int8_matmul(q, q, out=out), "held": lambda: qb.held_matmul(q, codes, 6, 4, 32, out=out),
           "norm grad": lambda: qb.layer_norm_grad(x, x, r.mean, r.rstd, dbias=out)[2]}[call]
    y = (s * run()).sum()
    run()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n,left,gap", [(1, 300, 40, 0, 0), (20, 1500, 130, 1, 3), (100, 2048, 256, 0, 0), (300, 130, 520, 0, 0), (300, 130, 515, 4, 1),
                                            (1100, 64, 700, 8, 4)])
def test_results_are_added_to(m, k, n, left, gap, kind):
    gen = gen_of(m, k, n)
    a, b = int8_rows(gen, m, k), int8_rows(gen, n, k)
    a = scaled(a, a.scale * 2.0 ** -17)
    bias = randn(gen, n)
    room = randn(gen, m + 2, left + n + gap).to(DTYPES[kind])
    before, out = room.clone(), room[1:1 + m, left:left + n]
    qb.int8_matmul(a, b, bias=bias, out=out, accumulate=True)
    check(out, a, b.q, b.scale, bias, kind, before[1:1 + m, left:left + n])
    keep = torch.ones_like(room, dtype=torch.bool)
    keep[1:1 + m, left:left + n] = False
    assert torch.equal(room[keep], before[keep])


def test_what_is_added_to_keeps_numbers_below_the_normal_ones():
    q = qb.Int8Rows(torch.zeros(300, 64, dtype=torch.int8, device="cuda"), torch.ones(300, device="cuda"))
    out = torch.full((300, 300), 1e-41, device="cuda")
    qb.int8_matmul(q, q, out=out, accumulate=True)
    assert torch.equal(out, torch.full((300, 300), 1e-41, device="cuda"))


@pytest.mark.parametrize("wide", [False, True])
def test_offsets_beyond_32_bits(wide):
    # 2^31 elements and more between the first row and the last: of x, and of a result
    if wide:
        x = torch.empty(2, 1 << 31, dtype=torch.bfloat16, device="cuda")[:, :1024]
        x.copy_(torch.randn(2, 1024, device="cuda"))
        want, _, _, off, _, _ = norm64(x.double(), None, None, 1e-5)
        got = qb.layer_norm(x, int8=True)
        near(got.out, want, off, "bf16")
        out = torch.empty(2, 1 << 31, dtype=torch.bfloat16, device="cuda")[:, :40]
        b = int8_rows(gen_of(3), 40, 1024)
        check(qb.int8_matmul(got.rows, b, out=out), got.rows, b.q, b.scale, None, "bf16")
        return
    tokens, n = 70000, 31000                                    # 2.17 x 10^9 results
    gen = gen_of(5)
    a, b = int8_rows(gen, tokens, 48), int8_rows(gen, n, 48)
    y = qb.int8_matmul(a, b)
    for rows in (slice(0, 3), slice(tokens - 3, tokens)):
        part = qb.Int8Rows(a.q[rows].clone(), a.scale[rows].clone())
        check(y[rows], part, b.q, b.scale, None, "bf16")
    assert bool(torch.isfinite(y[35000:35010].float()).all())


def test_a_long_batch_of_short_rows_and_a_short_batch_of_long_ones():
    # every route of the norm that goes by the number of rows
    gen = gen_of(31)
    for rows, width in ((20000, 24), (15000, 300), (15000, 761), (14300, 1000), (3, 17000), (2, 70001)):
        x = randn(gen, rows, width).bfloat16()
        w, b = 1 + 0.1 * randn(gen, width), 0.1 * randn(gen, width)
        got = qb.layer_norm(x, w, b, residual=x, int8=True)
        want, _, _, off, _, _ = norm64(got.sum.double(), w, b, 1e-5)
        near(got.out, want, off, "bf16")
        one = qb.layer_norm(x[-1:].contiguous(), w, b, residual=x[-1:].contiguous(), int8=True)
        step = float(want[-1].abs().max()) / 127
        assert float((one.rows.values() - got.rows.values()[-1:]).abs().max()) <= step * 1.01 and int(got.rows.sums[0]) == int(got.rows.q[0].sum(dtype=torch.int32))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,width", [(9000, 250), (5000, 513), (700, 1536), (260, 2304), (200, 5119), (150, 5120), (40, 6145), (33, 7008), (20, 8191)])
def test_gradients_by_every_number_of_warps_to_a_row(rows, width, kind):
    gen = gen_of(rows, width, 2)
    x, dy, ds = ((randn(gen, rows, width) * f).to(DTYPES[kind]) for f in (1.0, 1e-2, 1e-2))
    w = 1 + 0.1 * randn(gen, width)
    ran = qb.layer_norm(x, w)
    dx, dw, db = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, w, dsum=ds)
    wx, ww, wb, off, sw, sb = grad64(dy, x, ran.mean, ran.rstd, w, ds)
    near(dx, wx, off, kind)
    few = 3 + min(rows, rows / 64 + 80)                          # (as in the test of the gradient)
    near(dw, ww, few * U * sw, "f32")
    near(db, wb, few * U * sb, "f32")


def among_nans(t, left, gap):
    """The same rows, `left` elements from 16 bytes and `gap` apart, with NaN before, between and behind them."""
    rows, width = t.shape
    room = torch.full((left + rows * (width + gap) + 16,), float("nan"), dtype=t.dtype, device="cuda")
    r = room[left:left + rows * (width + gap)].view(rows, width + gap)[:, :width]
    r.copy_(t)
    return r


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(4000, 1025), (3500, 1535), (16000, 3), (16000, 255), (16000, 767), (2500, 2303), (700, 8191), (4000, 1)])
def test_rows_anywhere_among_numbers_that_are_not_theirs(rows, width, kind):
    # many rows to a place in shared memory, each as far from 16 bytes as it happens to lie
    gen = gen_of(rows, width, 3)
    x, dy, ds = ((randn(gen, rows, width)).to(DTYPES[kind]) for _ in range(3))
    w = 1 + 0.1 * randn(gen, width)
    ran = qb.layer_norm(x, w, residual=ds, int8=True)
    want = qb.layer_norm_grad(dy, x, ran.mean, ran.rstd, w, dsum=ds)
    for left, gap in ((1, 0), (3, 1), (5, 2), (7, 3), (2, 4)):
        a, b, c = among_nans(x, left, gap), among_nans(dy, left + 1, gap), among_nans(ds, left, gap + 1)
        here = qb.layer_norm(a, w, residual=c, int8=True)
        assert torch.equal(here.out, ran.out) and torch.equal(here.sum, ran.sum) and torch.equal(here.mean, ran.mean) and torch.equal(here.rstd, ran.rstd)
        assert torch.equal(here.rows.q, ran.rows.q) and torch.equal(here.rows.sums, ran.rows.sums)
        for got, wanted in zip(qb.layer_norm_grad(b, a, ran.mean, ran.rstd, w, dsum=c), want):
            assert torch.equal(got, wanted)


def test_bytes_behind_rows_are_not_read():
    gen = gen_of(12)
    for k in (5, 100, 131):
        a, b = int8_rows(gen, 40, k), int8_rows(gen, 150, k)
        want = qb.int8_matmul(a, b, out_dtype=torch.float32)
        for r in (a, b):
            whole = torch.as_strided(r.q, (r.rows, r.stride), (r.stride, 1))
            whole[:, k:] = 77
        assert torch.equal(qb.int8_matmul(a, b, out_dtype=torch.float32), want)


def test_values_of_rows():
    q = qb.quantize_rows(torch.tensor([[1.0, -2.0, 0.5], [0.0, 0.0, 0.0]], device="cuda"))
    assert np.allclose(q.values().cpu().numpy(), [[1.0, -2.0, 0.5], [0, 0, 0]], atol=2.0 / 254) and "2 x 3" in repr(q)
