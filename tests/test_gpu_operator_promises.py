"""What the operators around the quantized step promise beside their values: how each operation of the 8-bit step is
rounded, first calls on a stream of their own, what is allocated, what a step without gradients tells, what autograd is told
of writes."""
import numpy as np
import pytest
import torch

from _training import adamw_constants

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

F = np.float32
HYPER = dict(beta1=0.9, beta2=0.999, eps=1e-8, lr=1e-3)


@pytest.mark.parametrize("eps", [1e-8, 0.05])
@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_eight_bit_weights_round_every_operation_but_the_quotient(shift, master, eps):
    # Weights that a step nearly cancels show each rounding of x k - a q: the result has fewer bits than a q, so that
    # it is one of those that the quotients within 3 units in the last place give (the reciprocal is off by at most one of its own,
    # which is less than two of the quotient's; the product and the rounded quotient by half a unit each), or it is not.
    n, decay = 5000, 0.3
    rng = np.random.default_rng(7)
    g = (rng.standard_normal(n) * 0.01).astype(F)
    k = adamw_constants(HYPER["beta1"], HYPER["beta2"], HYPER["lr"], decay, 1)
    m, v = k["c1"] * g, k["c2"] * (g * g)
    q = m / (np.sqrt(v) * k["b"] + F(eps))
    x = (k["a"] * q / k["keep"] * (1 + rng.standard_normal(n).astype(F) * F(2.0 ** -9))).astype(F)
    room = torch.zeros(n + 8, device="cuda", dtype=torch.bfloat16 if master else torch.float32)
    gt = torch.zeros(n + 8, device="cuda")
    w, gt = room[shift:shift + n], gt[shift:shift + n]
    gt.copy_(torch.from_numpy(g))
    if not master:
        w.copy_(torch.from_numpy(x))
    opt = qb.AdamW([w], [gt], state_bits=8, master=master, weight_decay=decay, seed=1, **dict(HYPER, eps=eps))
    if master:
        opt.master[:n] = torch.from_numpy(x).cuda()
    opt.step(1)
    got = (opt.master[:n] if master else w).cpu().numpy()
    near = [(q.view(np.int32) + j).view(F) for j in range(-3, 4)]
    may = np.stack([x * k["keep"] - k["a"] * near_q for near_q in near])
    assert np.all((may == got).any(axis=0))


def test_first_norm_on_another_stream(monkeypatch):
    # nothing that a new holder has queued on the stream of its creation may reach its result after a call elsewhere
    lib = qb.binding.load_library()
    create, big = lib.qadam_norm_create, torch.ones(8192, 8192, device="cuda")

    def create_then_be_busy(*args):
        rc = create(*args)
        for _ in range(20):
            torch.mm(big, big)
        return rc

    x, s = torch.full((1000,), 2.0, device="cuda"), torch.cuda.Stream()
    with torch.cuda.stream(s):
        qb.GradNorm([x])(1.0)                                    # (kernels are loaded by their first call)
    torch.mm(big, big)
    torch.cuda.synchronize()
    monkeypatch.setattr(lib, "qadam_norm_create", create_then_be_busy)
    norm = qb.GradNorm([x])
    with torch.cuda.stream(s):
        n, f = norm(1.0)
    torch.cuda.synchronize()
    assert abs(float(n) - 2 * np.sqrt(1000)) < 1e-3 and float(f) < 0.1


def test_norm_of_missing_gradients_takes_no_memory_for_them():
    w = [torch.zeros(1 << 24, device="cuda"), torch.zeros(5, device="cuda", dtype=torch.bfloat16), torch.zeros(7, device="cuda")]
    g = torch.full((7,), 2.0, device="cuda")
    opt = qb.AdamW(w, [None, None, g])
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    n, _ = opt.grad_norm()
    assert torch.cuda.max_memory_allocated() - before < 1 << 20
    assert abs(float(n) - 2 * np.sqrt(7)) < 1e-5
    g1 = torch.full((5,), 1.0, device="cuda", dtype=torch.bfloat16)
    opt.bind([None, g1, None])
    assert abs(float(opt.grad_norm()[0]) - np.sqrt(5)) < 1e-5


@pytest.mark.parametrize("bits", [32, 8])
def test_a_factor_that_is_not_finite_is_told_without_gradients_too(bits):
    opt = qb.AdamW([torch.ones(2000, device="cuda"), torch.ones(0, device="cuda")], [None, None], state_bits=bits)
    opt.step(1, grad_scale=torch.ones(1, device="cuda"))
    assert opt.poll_status() == 0
    opt.step(1, grad_scale=torch.full((1,), float("nan"), device="cuda"))
    assert opt.poll_status() == qb.ST_NONFINITE and bool((opt.weights[0] == 1).all())


# ---------------------------------------------------------------- what autograd is told

@pytest.mark.parametrize("counted", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_a_backward_pass_through_stepped_weights_is_refused(packed, counted):
    base = torch.ones(300, device="cuda")
    w = [base[:100], base[100:300]] if packed else [torch.nn.Parameter(torch.ones(n, device="cuda")) for n in (100, 200)]
    s = torch.ones(1, device="cuda", requires_grad=True)
    opt = qb.AdamW(w, [torch.ones(n, device="cuda") for n in (100, 200)])
    for used in w:
        y = (s * used).sum()
        opt.step_counted() if counted else opt.step(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
        (s * used).sum().backward()


def test_weights_made_in_inference_mode_are_stepped():
    with torch.inference_mode():
        w, g = torch.ones(100, device="cuda"), torch.ones(100, device="cuda")
        opt = qb.AdamW([w], [g])
        opt.step(1)
        out = torch.empty(2, device="cuda")
        opt.grad_norm()
        qb.GradNorm([g])(1.0, out=out)
        rows = qb.embedding_lookup(w.view(10, 10), torch.tensor([3, 0], device="cuda"), out=torch.empty(2, 10, device="cuda"))
    assert bool((w < 1).all()) and float(out[0]) == 10.0 and torch.equal(rows, w.view(10, 10)[[3, 0]])


@pytest.mark.parametrize("call", ["lookup", "held", "grad", "norm", "own norm", "moments"])
def test_a_backward_pass_through_an_overwritten_result_is_refused(call):
    ids = torch.tensor([1, 0, 3], device="cuda")
    table, codes = torch.ones(4, 8, device="cuda"), torch.zeros(32, dtype=torch.uint8, device="cuda")
    s = torch.ones(1, device="cuda", requires_grad=True)
    out = torch.empty((3, 8) if call in ("lookup", "held") else (4, 8) if call == "grad" else 2, device="cuda")
    norm = qb.GradNorm([table])
    opt = qb.AdamW([table], [table.clone()], state_bits=8)
    pair = (torch.empty(128, device="cuda"), torch.empty(128, device="cuda"))
    run = {"lookup": lambda: qb.embedding_lookup(table, ids, out=out), "held": lambda: qb.held_lookup(codes, 6, ids, 4, 8, out=out),
           "grad": lambda: qb.embedding_grad(ids, table[:3], 4, out=out), "norm": lambda: norm(1.0, out=out)[1],
           "own norm": lambda: norm(1.0)[1], "moments": lambda: opt.moments(out=pair)[1]}[call]
    y = (s * run()).sum()
    run()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
