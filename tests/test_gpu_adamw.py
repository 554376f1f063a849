"""AdamW over many tensors and the gradient norm against plain numpy: bit for bit with the binary32 statement,
within its roundings of the binary64 one."""
import numpy as np
import pytest
import torch

from _training import adamw32, adamw64, adamw8, adamw_constants, code_values, decode_m, decode_r

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}       # half a step, relative
TINY = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8, lr=1e-3)
RAGGED = [1, 0, 3, 127, 128, 129, 255, 256, 257, 384, 2047, 2048, 2049, 5003]


def _tensors(lens, dtype, gen, sigma, shift=0):
    """Tensors in one buffer with room between them (filled with 7), `shift` elements off alignment."""
    dtypes = dtype if isinstance(dtype, list) else [dtype] * len(lens)
    room, out = [], []
    for n, d in zip(lens, dtypes):
        buf = torch.full((n + 64,), 7.0, dtype=d, device="cuda")
        t = buf[16 + shift:16 + shift + n]
        t.copy_(torch.randn(n, generator=gen, device="cuda") * sigma)
        room.append(buf)
        out.append(t)
    return out, room


def _untouched(room, lens, shift=0):
    for buf, n in zip(room, lens):
        rest = torch.cat([buf[:16 + shift], buf[16 + shift + n:]])
        assert bool((rest == 7.0).all())


def _np(t):
    return t.detach().float().cpu().numpy()


def _bits(a):
    return np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)


def _same(a, b):
    a, b = np.asarray(a, dtype=np.float32), np.asarray(b, dtype=np.float32)
    nan = np.isnan(a) & np.isnan(b)
    return bool(np.all(nan | (_bits(a).reshape(a.shape) == _bits(b).reshape(b.shape)) | ((a == 0) & (b == 0))))


def _pad(a, n=None):
    out = np.zeros(-(-a.size // 128) * 128, dtype=a.dtype)
    out[:a.size] = a
    return out


def _run(lens, w, g, bits, master, steps=3, shift=0, scale=None, decay=0.01, missing=(), seed=5):
    """Steps of the library beside the plain statement, every tensor compared after every step."""
    gen = torch.Generator(device="cuda").manual_seed(sum(lens) + bits)
    weights, wroom = _tensors(lens, w, gen, 0.05, shift)
    grads, groom = _tensors(lens, g, gen, 0.01, shift)
    decays = [decay if i % 2 else 0.0 for i in range(len(lens))]
    opt = qb.AdamW(weights, grads, state_bits=bits, master=master, weight_decay=decays, seed=seed, **HYPER)
    if missing:
        opt.bind([None if i in missing else t for i, t in enumerate(grads)])
    assert opt.D == sum(-(-n // 128) * 128 for n in lens)
    state = []
    for wt in weights:
        x = _pad(_np(wt))
        rows = x.size // 128
        state.append([x, np.zeros(x.size, np.uint8), np.zeros(rows, np.float32), np.zeros(x.size, np.uint8), np.zeros(rows, np.float32)]
                     if bits == 8 else [x, np.zeros_like(x), np.zeros_like(x)])
    factor = None if scale is None else torch.tensor([scale], device="cuda")
    for t in range(1, steps + 1):
        for gt in grads:
            gt.copy_(torch.randn(gt.numel(), generator=gen, device="cuda") * 0.01)
        opt.step(t, grad_scale=factor)
        for i, (wt, gt, n, off) in enumerate(zip(weights, grads, lens, opt.off)):
            k = adamw_constants(HYPER["beta1"], HYPER["beta2"], HYPER["lr"], decays[i], t)
            s, gp = state[i], _pad(_np(gt))
            if i not in missing and n:
                before = [a.copy() for a in s]
                if bits == 8:
                    s[:] = adamw8(s[0], s[1], s[2], s[3], s[4], gp, k, HYPER["eps"], off, t, seed, scale)
                else:
                    s[:] = adamw32(s[0], s[1], s[2], gp, k, HYPER["eps"], scale)
                    (x64, m64, v64), (ex, em, ev) = adamw64(before[0], before[1], before[2], gp, HYPER["beta1"], HYPER["beta2"],
                                                            HYPER["lr"], decays[i], t, HYPER["eps"], 1.0 if scale is None else np.float32(scale))
                    for got, want, tol in ((s[0], x64, ex), (s[1], m64, em), (s[2], v64, ev)):
                        assert np.all(np.abs(got - want) <= tol)
            pad = slice(off, off + -(-n // 128) * 128)
            x = torch.from_numpy(s[0][:n]).to(wt.dtype).float().numpy()
            if bits == 8 and i not in missing and n:
                # the quotient m / d is a product with a reciprocal: 2^-22 of it from the rounded one (a unit in the last
                # place of the reciprocal, half a unit for either side's last operation), then two roundings of either
                # side, of the step and of x
                step = np.abs(before[0] * k["keep"] - s[0])
                tol = 1.5 * 2.0 ** -22 * (step + 2.0 ** -23 * np.abs(s[0])) + 2.0 ** -23 * np.abs(s[0])
                if master:
                    got = opt.master[pad].cpu().numpy()
                    x = torch.from_numpy(got[:n]).to(wt.dtype).float().numpy()
                    assert np.all(got[n:] == 0)
                else:
                    got = _pad(_np(wt))
                    tol = tol + np.abs(s[0]) * HALF[wt.dtype] * (1 + 2.0 ** -7) + TINY[wt.dtype]
                    x = got[:n]
                assert np.all(np.abs(got - s[0]) <= tol), (i, n, t)
                s[0] = got
            elif master:
                assert _same(opt.master[pad].cpu().numpy(), s[0]), (i, n, t)
            assert _same(_np(wt), x), (i, n, t)
            if not master:
                s[0][:n] = x                               # the weight itself is what the next step reads
            if bits == 8:
                rows = slice(pad.start // 128, pad.stop // 128)
                if i not in missing:
                    assert _same(opt.m_scale[rows].cpu().numpy(), s[2]) and _same(opt.r_scale[rows].cpu().numpy(), s[4]), (i, n, t)
                assert np.array_equal(opt.m[pad].cpu().numpy(), s[1]) and np.array_equal(opt.r[pad].cpu().numpy(), s[3]), (i, n, t)
            else:
                assert _same(opt.m[pad].cpu().numpy(), s[1]) and _same(opt.v[pad].cpu().numpy(), s[2]), (i, n, t)
    _untouched(wroom, lens, shift)
    _untouched(groom, lens, shift)
    assert opt.poll_status() == 0
    return opt, state


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w,g,master", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", True), ("bf16", "f32", True),
                                        ("f16", "f16", True), ("f32", "f32", True), ("bf16", "bf16", False), ("f16", "f32", False), ("f32", "f16", True)])
def test_step_is_the_plain_statement(bits, w, g, master):
    _run(RAGGED, DTYPES[w], DTYPES[g], bits, master)


@pytest.mark.parametrize("large,master", [(2_700_001, False), (5_300_000, True), (10_600_130, False)])
def test_several_pairs_of_rows_to_a_warp(large, master):
    # from 2.56, 5.12 and 10.24 x 10^6 elements on a warp takes 2, 4 and 8 pairs; compared: small tensors around a large one,
    # and parts of that one (a tensor's random bits go by its offset: a part that begins at a multiple of 256 is one of its own)
    lens = [700, large, 129, 4000]
    gen = torch.Generator(device="cuda").manual_seed(large)
    wtype = torch.bfloat16 if master else torch.float32
    w = [(torch.randn(n, device="cuda", generator=gen) * 0.05).to(wtype) for n in lens]
    g = [(torch.randn(n, device="cuda", generator=gen) * 0.01).to(wtype) for n in lens]
    opt = qb.AdamW(w, g, state_bits=8, master=master, seed=77, **HYPER)
    x0 = [(opt.view(opt.master, i) if master else t).clone() for i, t in enumerate(w)]
    opt.step(1)
    k = adamw_constants(HYPER["beta1"], HYPER["beta2"], HYPER["lr"], 0.0, 1)
    last = (large // 4096 - 1) * 4096
    parts = [(0, 0, 700), (1, 0, 8192), (1, 1 << 20, (1 << 20) + 9000), (1, last, large), (2, 0, 129), (3, 0, 4000)]
    for i, lo, hi in parts:
        off, gp = opt.off[i] + lo, _pad(_np(g[i][lo:hi]))
        z, s = np.zeros(gp.size, np.uint8), np.zeros(gp.size // 128, np.float32)
        x, cm, sm, cr, sr = adamw8(_pad(_np(x0[i][lo:hi])), z, s, z, s, gp, k, HYPER["eps"], off, 1, 77)
        # whole rows of the part: a row that goes on behind it has another largest value
        n = hi - lo if hi == lens[i] else (hi - lo) // 128 * 128
        live = slice(off, off + n)
        rows = slice(off // 128, off // 128 + n // 128)
        assert np.array_equal(opt.m[live].cpu().numpy(), cm[:n]) and np.array_equal(opt.r[live].cpu().numpy(), cr[:n]), (i, lo)
        assert _same(_np(opt.m_scale[rows]), sm[:n // 128]) and _same(_np(opt.r_scale[rows]), sr[:n // 128])
        got = _np((opt.view(opt.master, i) if master else w[i])[lo:lo + n])
        # the step is at most lr (1 + 2^-10) at t = 1; its quotient is off by 1.5 x 2^-22, x by a rounding on either side
        assert np.all(np.abs(got - x[:n]) <= 1.1e-3 * 1.5 * 2.0 ** -22 + 2.0 ** -23 * np.abs(x[:n]))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 2, 3, 4])
def test_tensors_off_alignment(bits, shift):
    _run(RAGGED, DTYPES["f32"], DTYPES["bf16"], bits, False, shift=shift)
    _run(RAGGED, DTYPES["bf16"], DTYPES["f32"], bits, True, shift=shift, steps=1)


@pytest.mark.parametrize("bits", [32, 8])
def test_types_mixed_in_one_list(bits):
    w = [DTYPES[("f32", "bf16", "f16")[i % 3]] for i in range(len(RAGGED))]
    g = [DTYPES[("bf16", "f32")[i % 2]] for i in range(len(RAGGED))]
    opt, _ = _run(RAGGED, w, g, bits, False)
    # one launch a step, or one for each pair of widths: weights f32, bf16, f16 and gradients bf16, f32 in turn make all four
    assert opt.launches == 3 * (1 if bits == 32 else 4)


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_factor_and_missing_gradients(bits):
    _run(RAGGED, DTYPES["f32"], DTYPES["f32"], bits, False, scale=0.37, missing=(3, 8, 13))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [447, 449, 4000])
def test_many_tensors(bits, count):
    lens = [(7 * i) % 300 for i in range(count)]
    opt, _ = _run(lens, DTYPES["f32"], DTYPES["bf16"], bits, False, steps=1)
    assert opt.launches == (2 if count > 3584 else 1)


def test_seeds_differ_and_repeat():
    def codes(seed):
        opt, _ = _run([5000], DTYPES["f32"], DTYPES["f32"], 8, False, seed=seed)
        return opt.m.cpu(), opt.r.cpu()
    a, b, c = codes(1), codes(1), codes(1 + (1 << 40))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert not torch.equal(a[0], c[0]) and not torch.equal(a[1], c[1])


def test_moments_are_decoded():
    opt, state = _run(RAGGED, DTYPES["f32"], DTYPES["f32"], 8, False)
    m, v = opt.moments()
    want_m = np.concatenate([decode_m(s[1].reshape(-1, 128), s[2]).reshape(-1) for s in state])
    want_r = np.concatenate([decode_r(s[3].reshape(-1, 128), s[4]).reshape(-1) for s in state])
    assert _same(m.cpu().numpy(), want_m) and _same(v.cpu().numpy(), want_r * want_r)
    out = (torch.empty(opt.D, device="cuda"), torch.empty(opt.D, device="cuda"))
    assert opt.moments(out=out)[0] is out[0] and torch.equal(out[0], m) and torch.equal(out[1], v)


def test_rounding_at_random_has_the_right_mean():
    # one value y between two codes in every place but a row's first (which sets the scale): the mean of what is held
    # must be y.  n places, steps of width s: the mean's deviation is at most s / 2 / sqrt(n), five of those are allowed,
    # beside the resolution of the random bits (half of s / 64 for m)
    n, rows = 128 * 400, 400
    w = torch.zeros(n, device="cuda")
    g = torch.full((n,), 0.43, device="cuda")
    g[::128] = 1.0
    opt = qb.AdamW([w], [g], state_bits=8, beta1=0.5, beta2=0.5, eps=1e-8, lr=0.0, seed=3)
    opt.step(1)
    m, v = (a.cpu().numpy().astype(np.float64).reshape(rows, 128) for a in opt.moments())
    assert np.all(m[:, 0] == 0.5)
    for got, want, mantissa, res in ((m, 0.215, 3, 64), (np.sqrt(v), 0.43 * np.sqrt(0.5), 4, 1024)):
        scale = got[0, 0]
        values = code_values(mantissa) * scale
        at = np.searchsorted(values, want)
        step = values[at] - values[at - 1]
        assert set(np.unique(np.round(got[:, 1:] / step, 3))) <= set(np.round(values[at - 1:at + 1] / step, 3))
        assert abs(got[:, 1:].mean() - want) <= 5 * step / 2 / np.sqrt(n - rows) + step / (2 * res)


def test_second_moment_follows_a_change_that_nearest_rounding_would_not():
    # r halfway between two codes of its row's scale, gradients of twice its size: with beta2 = 0.999 one step moves r by
    # 0.15 %, a fortieth of a code's step.  After 1500 steps r is within 20 % of where 32-bit moments are (spread
    # of one place about 17 %; the mean over 1024 places is compared)
    n = 1024
    w = torch.zeros(n, device="cuda")
    g = torch.full((n,), 0.1, device="cuda")
    g[::128] = 1.0
    opt = qb.AdamW([w], [g], state_bits=8, lr=0.0, seed=11)
    opt.step(1)
    g.fill_(0.2)
    g[::128] = 1.0
    ref = qb.AdamW([w], [g], state_bits=32, lr=0.0)
    g.fill_(0.1)
    g[::128] = 1.0
    ref.step(1)
    g.fill_(0.2)
    g[::128] = 1.0
    for t in range(2, 1500):
        opt.step(t)
        ref.step(t)
    live = torch.ones(n, dtype=torch.bool, device="cuda")
    live[::128] = False
    r8, r32 = opt.moments()[1][live].sqrt().mean(), ref.v[live].sqrt().mean()
    assert abs(float(r8 / r32) - 1) < 0.2


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_factor_that_is_not_finite_stops_the_step(bits, bad):
    w, g = torch.randn(3000, device="cuda"), torch.randn(3000, device="cuda")
    opt = qb.AdamW([w], [g], state_bits=bits)
    opt.step(1)
    before = [t.clone() for t in (w, opt.m, opt.v if bits == 32 else opt.r)]
    assert opt.poll_status() == 0
    opt.step(2, grad_scale=torch.tensor([bad], device="cuda"))
    after = (w, opt.m, opt.v if bits == 32 else opt.r)
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    assert opt.poll_status() == qb.ST_NONFINITE
    opt.step_counted(grad_scale=torch.tensor([bad], device="cuda"))
    assert int(opt.count) == 0 and all(torch.equal(a, b) for a, b in zip(before, after))


@pytest.mark.parametrize("bits", [32, 8])
def test_nonfinite_gradients_without_a_factor(bits):
    g = torch.full((1024,), 0.5, device="cuda")
    g[300], g[700] = float("nan"), float("inf")
    w = torch.zeros(1024, device="cuda")
    opt = qb.AdamW([w], [g], state_bits=bits)
    opt.step(1)
    m, v = opt.moments()
    if bits == 32:
        assert bool(torch.isnan(m[300])) and bool(torch.isinf(m[700])) and int(torch.isfinite(m).sum()) == 1022
    else:
        # the rows that hold them, and no other
        rows = torch.isfinite(m).reshape(8, 128)
        assert not rows[2].any() and rows[[0, 1, 3, 4, 6, 7]].all() and not rows[5].any()
        assert opt.poll_status() == qb.ST_NONFINITE
    assert int(torch.isfinite(w).sum()) >= 1022


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_tiny_and_huge_gradients(bits):
    g = torch.zeros(640, device="cuda")
    g[128:256] = 1e-42                          # subnormal moments
    g[256:384] = 1e18
    g[384:512] = torch.tensor([1e-30, 1e10] * 64, device="cuda")
    w = torch.full((640,), 0.25, device="cuda")
    opt = qb.AdamW([w], [g], state_bits=bits, **HYPER)
    k = adamw_constants(HYPER["beta1"], HYPER["beta2"], HYPER["lr"], 0.0, 1)
    opt.step(1)
    if bits == 32:
        x, m, v = adamw32(np.full(640, 0.25, np.float32), np.zeros(640, np.float32), np.zeros(640, np.float32), _np(g), k, HYPER["eps"])
        assert _same(_np(opt.m), m) and _same(_np(opt.v), v)
    else:
        z, s = np.zeros(640, np.uint8), np.zeros(5, np.float32)
        x, cm, sm, cr, sr = adamw8(np.full(640, 0.25, np.float32), z, s, z, s, _np(g), k, HYPER["eps"], 0, 1, 0)
        assert np.array_equal(opt.m.cpu().numpy(), cm) and np.array_equal(opt.r.cpu().numpy(), cr)
        assert _same(_np(opt.m_scale), sm) and _same(_np(opt.r_scale), sr)
    # (8 bits: a step of lr, off by 1.5 x 2^-22 of itself, and a rounding of x on either side)
    assert np.all(np.abs(_np(w) - x) <= (0 if bits == 32 else 0.25 * 2.0 ** -23 + 1e-3 * 1.5 * 2.0 ** -22))
    assert bool((w[:128] == 0.25).all()) and bool((w[512:] == 0.25).all())


# ---------------------------------------------------------------- norm

@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("lens", [[1], [0, 5], RAGGED, [100003], [8191, 8192, 8193], [13] * 450, [3] * 7200])
def test_norm(dtype, shift, lens):
    gen = torch.Generator(device="cuda").manual_seed(len(lens))
    ts, room = _tensors(lens, DTYPES[dtype], gen, 0.3, shift)
    norm = qb.GradNorm(ts)
    want = np.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))
    for limit in (float("inf"), 0.25):
        n, f = norm(limit)
        # at most 7 roundings of binary32 in a sum of squares (a half of that in its root), the rest in binary64, one
        # rounding to binary32
        assert abs(float(n) - want) <= want * (3.5 * 2.0 ** -24 + 2.0 ** -24 + 1e-11)
        assert float(f) == float(np.float32(min(1.0, np.float32(limit) / np.float32(float(n)))))
    first = norm(0.25)[0].clone()
    for _ in range(5):
        assert torch.equal(norm(0.25)[0], first)
    _untouched(room, lens, shift)


@pytest.mark.parametrize("value", [1e-30, 1e30, 1e-42])
def test_norm_of_squares_beyond_binary32(value):
    x = torch.full((70001,), value, device="cuda")
    n, f = qb.GradNorm([x])()
    want = float(x[0].double()) * np.sqrt(70001.0)
    assert abs(float(n) - want) <= want * 2.0 ** -24 + 2.0 ** -149 and float(f) == 1.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_that_is_not_finite(bad):
    x = torch.ones(20000, device="cuda")
    x[15000] = bad
    norm = qb.GradNorm([x, torch.ones(5, device="cuda")])
    n, f = norm(1.0)
    assert not np.isfinite(float(n)) and np.isnan(float(f))
    x[15000] = 1.0
    assert np.isfinite(float(norm(1.0)[0]))


def test_norm_of_nothing_and_of_missing_tensors():
    n, f = qb.GradNorm([torch.empty(0, device="cuda")])(2.0)
    assert float(n) == 0.0 and float(f) == 1.0
    a, b = torch.full((9000,), 2.0, device="cuda"), torch.ones(7, device="cuda")
    norm = qb.GradNorm([a, b])
    norm.bind([None, b])
    out = torch.zeros(2, device="cuda")
    n, f = norm(1.0, out=out)
    assert float(out[0]) == float(np.sqrt(np.float32(7))) and float(f) == float(np.float32(1) / np.sqrt(np.float32(7)))


def test_step_clipped_by_the_norm():
    w, g = [torch.randn(n, device="cuda") for n in (1000, 50)], [torch.randn(n, device="cuda") for n in (1000, 50)]
    opt = qb.AdamW([t.clone() for t in w], g)
    n, f = opt.grad_norm(0.5)
    opt.step(1, grad_scale=f)
    ref = qb.AdamW([t.clone() for t in w], [t * f for t in g])
    ref.step(1)
    assert all(torch.equal(a, b) for a, b in zip(opt.weights, ref.weights)) and torch.equal(opt.v, ref.v)
    opt.bind([None, g[1]])
    assert abs(float(opt.grad_norm()[0]) - float(g[1].double().norm())) <= 1e-6 * float(g[1].norm())


# ---------------------------------------------------------------- streams and graphs

@pytest.mark.parametrize("bits", [32, 8])
def test_captured_step_counts_on_and_reads_lr(bits):
    def make():
        gen = torch.Generator(device="cuda").manual_seed(9)
        w = [torch.randn(n, device="cuda", generator=gen) for n in (3000, 17)]
        g = [torch.randn(n, device="cuda", generator=gen) for n in (3000, 17)]
        return qb.AdamW(w, g, state_bits=bits, seed=4)
    lrs = [1e-3, 5e-4, 2e-3, 0.0]
    a, b = make(), make()
    lr = torch.tensor([lrs[0]], device="cuda")
    a.grad_norm(1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, f = a.grad_norm(1.0)
        a.step_counted(lr=lr, grad_scale=f)
    for t, value in enumerate(lrs, 1):
        lr.fill_(value)
        graph.replay()
        _, f = b.grad_norm(1.0)
        b.step(t, lr=value, grad_scale=f)
        for x, y in zip(a.weights, b.weights):
            # the bias corrections come from the device's pow: two roundings of the step (at most lr * 8) may differ
            assert float((x - y).abs().max()) <= 8 * 2e-3 * 2.0 ** -22 + float(x.abs().max()) * 2.0 ** -23
        for name in ("m", "v") if bits == 32 else ("m", "r", "m_scale", "r_scale"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        for x, y in zip(a.weights, b.weights):
            y.copy_(x)
    assert int(a.count) == len(lrs)


def test_step_runs_on_the_current_stream():
    w, g = torch.zeros(1 << 22, device="cuda"), torch.zeros(1 << 22, device="cuda")
    opt = qb.AdamW([w], [g])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(20):
            g.add_(0.05)
        opt.step(1)
        got = w.clone()
    s.synchronize()
    assert bool((got != 0).all()) and abs(float(opt.m[0]) - 0.1) < 1e-6      # g = 20 * 0.05, m = 0.1 g


def test_refusals_of_the_holders():
    w, g = torch.zeros(100, device="cuda"), torch.zeros(100, device="cuda")
    for bad in (lambda: qb.AdamW([w], []), lambda: qb.AdamW([], []), lambda: qb.AdamW([w, w[50:]], [g, g[50:]]), lambda: qb.AdamW([w, w], [g, g]),
                lambda: qb.AdamW([w.double()], [g]), lambda: qb.AdamW([w], [g.int()]), lambda: qb.AdamW([w], [g[:99]]),
                lambda: qb.AdamW([w.view(10, 10).t()], [g]), lambda: qb.AdamW([w], [g], weight_decay=[0.1, 0.1]),
                lambda: qb.AdamW([w], [g.cpu()]), lambda: qb.GradNorm([]), lambda: qb.GradNorm([g.view(10, 10)[:, :3]]),
                lambda: qb.GradNorm([g])(1.0, out=torch.zeros(3, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qb.AdamW([w], [g], state_bits=16), lambda: qb.AdamW([w], [g], beta1=1.0), lambda: qb.AdamW([w], [g], eps=0.0),
                lambda: qb.GradNorm([g])(0.0), lambda: qb.GradNorm([g])(float("nan"))):
        with pytest.raises(qb.QAdamError):
            bad()
    opt = qb.AdamW([w], [g])
    for bad in (lambda: opt.bind([g.bfloat16()]), lambda: opt.bind([]), lambda: opt.step(1, lr=-1.0), lambda: opt.step(1, lr=float("nan")),
                lambda: opt.step(1, grad_scale=torch.zeros(2, device="cuda")), lambda: opt.step(1, grad_scale=torch.zeros(1)),
                lambda: opt.moments(out=(w, g))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(qb.QAdamError):
        opt.step(0)
    opt.close()
    with pytest.raises(qb.QAdamError):
        opt.step(1)


def test_resume_from_saved_buffers():
    def make():
        gen = torch.Generator(device="cuda").manual_seed(2)
        return (qb.AdamW([torch.randn(700, device="cuda", generator=gen).bfloat16()], [torch.zeros(700, device="cuda")], state_bits=8,
                         master=True, seed=8, weight_decay=0.1))
    gs = [torch.randn(700, device="cuda") for _ in range(4)]
    a, b = make(), make()
    for t, g in enumerate(gs, 1):
        a.grads[0].copy_(g)
        a.step(t)
        if t == 2:
            saved = {k: getattr(a, k).clone() for k in ("master", "m", "r", "m_scale", "r_scale")}
    for k, v in saved.items():
        getattr(b, k).copy_(v)
    for t in (3, 4):
        b.grads[0].copy_(gs[t - 1])
        b.step(t)
    assert torch.equal(a.weights[0], b.weights[0]) and torch.equal(a.master, b.master) and torch.equal(a.r, b.r)


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_beyond_32_bits(bits):
    """A tensor of more than 2^32 elements, and one behind it: their last elements are stepped, and count in the norm.
    (8.6 GB for each of weight and gradient, 17 GB a moment.)"""
    large, tail = (1 << 32) + 4105, 1300
    first = large - tail - (large - tail) % 1024
    gen = torch.Generator(device="cuda").manual_seed(bits)
    w = [torch.zeros(large, device="cuda", dtype=torch.bfloat16), torch.randn(700, device="cuda", generator=gen)]
    g = [torch.zeros(large, device="cuda", dtype=torch.bfloat16), torch.randn(700, device="cuda", generator=gen)]
    w[0][first:] = torch.randn(large - first, device="cuda", generator=gen)
    g[0][first:] = torch.randn(large - first, device="cuda", generator=gen)
    ends = [w[0][first:].clone(), w[1].clone()]
    opt = qb.AdamW(w, g, state_bits=bits, seed=5, **HYPER)
    # the same elements as tensors of their own; a step's weights do not depend on the random bits
    small = qb.AdamW(ends, [g[0][first:].clone(), g[1]], state_bits=bits, seed=5, **HYPER)
    opt.step(1)
    small.step(1)
    assert torch.equal(w[0][first:], ends[0]) and torch.equal(w[1], ends[1])
    assert not bool(w[0][first - 4096:first].any()) and not bool(w[0][:4096].any())
    scale, m = (1, lambda o: o.m) if bits == 32 else (128, lambda o: o.m_scale)
    end = opt.off[1] + 700 if bits == 32 else opt.off[1] + 768
    ours, its = m(opt)[first // scale:end // scale], m(small)[:(end - first) // scale]
    assert torch.equal(ours, its) and bool(ours.any())
    norm, _ = opt.grad_norm()
    want = float(torch.sqrt(g[0][first:].double().square().sum() + g[1].double().square().sum()))
    # eight squares at a time are off by at most 7 x 2^-24, the norm by half of that and its own rounding
    assert abs(float(norm) - want) <= want * 5 * 2.0 ** -24
