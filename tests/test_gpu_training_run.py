"""The operators as a training step uses them: rows of the embedding, a layer, the gradients, their norm, the step; and the
gradient that goes into a worker's part of the quantized step.  The layer between is torch's, the gradients are compared
with autograd's in binary64."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

ROWS, WIDTH, CLASSES, TOKENS = 300, 64, 17, 1000


class _Model:
    """Embedding rows, one matrix, cross entropy."""

    def __init__(self, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.table = torch.randn(ROWS, WIDTH, generator=gen, device="cuda") * 0.1
        self.matrix = torch.randn(WIDTH, CLASSES, generator=gen, device="cuda") * 0.1
        self.g_table, self.g_matrix = torch.zeros_like(self.table), torch.zeros_like(self.matrix)
        self.ids = torch.zeros(TOKENS, dtype=torch.int64, device="cuda")
        self.target = torch.zeros(TOKENS, dtype=torch.int64, device="cuda")
        self.gen = gen

    def batch(self):
        self.ids.copy_(torch.randint(0, ROWS, (TOKENS,), generator=self.gen, device="cuda"))
        self.ids[::7] = 3                                        # one frequent token
        self.ids[5::50] = -1                                     # padding
        self.target.copy_(torch.randint(0, CLASSES, (TOKENS,), generator=self.gen, device="cuda"))

    def gradients(self, scale=8.0):
        x = qb.embedding_lookup(self.table, self.ids, scale=scale)
        logits = x @ self.matrix
        d = (torch.softmax(logits, 1) - torch.nn.functional.one_hot(self.target, CLASSES)) / TOKENS
        self.g_matrix.copy_(x.t() @ d)
        qb.embedding_grad(self.ids, d @ self.matrix.t(), ROWS, scale=scale, out=self.g_table)


def test_gradients_of_the_step():
    m = _Model()
    m.batch()
    m.gradients()
    table, matrix = m.table.double().requires_grad_(), m.matrix.double().requires_grad_()
    live = (m.ids >= 0).double()[:, None]
    x = table[m.ids.clamp_min(0)] * 8.0 * live
    torch.nn.functional.cross_entropy(x @ matrix, m.target).backward()
    # binary32 products of up to 1000 terms (TF32 is off): relative to the largest gradient, 2^-24 for each of the few
    # hundred operations behind an element
    for got, want in ((m.g_table, table.grad), (m.g_matrix, matrix.grad)):
        assert float((got.double() - want).abs().max()) <= 1000 * 2.0 ** -24 * float(want.abs().max())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_run_is_the_eager_run(bits):
    def run(captured):
        m = _Model(5)
        opt = qb.AdamW([m.table, m.matrix], [m.g_table, m.g_matrix], state_bits=bits, lr=1e-2, weight_decay=[0.0, 0.1], seed=9)
        lr = torch.tensor([1e-2], device="cuda")

        def step():
            m.gradients()
            norm, factor = opt.grad_norm(0.5)
            opt.step_counted(lr=lr, grad_scale=factor)
            return norm

        m.batch()
        opt.grad_norm(0.5)                                       # (its context is made outside the capture)
        if captured:
            keep = [t.clone() for t in (m.table, m.matrix, opt.m, opt.v if bits == 32 else opt.r)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()                                           # warms cuBLAS up
            torch.cuda.current_stream().wait_stream(side)
            for t, k in zip((m.table, m.matrix, opt.m, opt.v if bits == 32 else opt.r), keep):
                t.copy_(k)
            opt.count.zero_()
            if bits == 8:
                opt.m_scale.zero_()
                opt.r_scale.zero_()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for t in range(4):
            if t:
                m.batch()
            lr.fill_(1e-2 / (t + 1))
            graph.replay() if captured else step()
        torch.cuda.synchronize()
        assert int(opt.count) == 4 and opt.poll_status() == 0
        return [m.table, m.matrix, *opt.moments()]

    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b) and bool(torch.isfinite(a).all())


def test_a_workers_gradient_and_held_rows():
    # two workers read rows of the 8-bit weights that they hold, and put the table's gradient into their part of the
    # gradient buffer, in the padded layout; the quantized step runs on it
    seg, n = [ROWS * WIDTH, WIDTH * CLASSES], 2
    x1 = torch.randn(sum(seg)) * 0.1
    q = qb.QAdam(seg, n, kx=6, x1=x1)
    g = torch.zeros(n, q.D, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    for i in range(n):
        ids = torch.randint(0, ROWS, (200,), generator=gen, device="cuda")
        rows = q.lookup(0, WIDTH, ids, scale=2.0, out_dtype=torch.float32)
        # Q_x: nearest multiple of 2^-7 in [-1/2, 1/2], ties toward zero
        x = x1[:seg[0]].view(ROWS, WIDTH).double()
        y = (x.abs() * 128).clamp_max(64)
        held = torch.sign(x) * torch.ceil(y - 0.5) / 128
        assert torch.equal(rows.double().cpu(), 2.0 * held[ids.cpu()])
        part = g[i, q.seg_off[0]:q.seg_off[0] + seg[0]].view(ROWS, WIDTH)
        got = qb.embedding_grad(ids, rows, ROWS, scale=2.0, out=part)
        want = torch.zeros(ROWS, WIDTH, dtype=torch.float64, device="cuda").index_add_(0, ids, rows.double()) * 2.0
        assert got.data_ptr() == part.data_ptr()
        assert float((got.double() - want).abs().max()) <= 200 * 2.0 ** -24 * float(want.abs().max())
    before = q.x.clone()
    q.step(1, g)
    torch.cuda.synchronize()
    assert q.poll_status() == 0 and not torch.equal(q.x, before)
    norm, _ = qb.GradNorm([g[0], g[1]])()
    assert abs(float(norm) - float(g.double().norm())) <= 5 * 2.0 ** -24 * float(norm)
    q.close()


def test_calls_on_two_streams_with_scratch_of_their_own():
    gen = torch.Generator(device="cuda").manual_seed(3)
    jobs = []
    for k in range(2):
        ids = torch.randint(0, 50, (30000,), generator=gen, device="cuda")
        dy = torch.randn(30000, 40, generator=gen, device="cuda")
        jobs.append((ids, dy, torch.cuda.Stream(), qb.embedding_grad(ids, dy, 50)))
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for ids, dy, s, _ in jobs:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(qb.embedding_grad(ids, dy, 50))
        torch.cuda.synchronize()
        for (_, _, _, want), out in zip(jobs, got):
            assert torch.equal(out, want)


def test_contexts_do_not_share_anything():
    def make(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        return qb.AdamW([torch.randn(5000, generator=gen, device="cuda")], [torch.randn(5000, generator=gen, device="cuda")], state_bits=8,
                        seed=seed)
    alone = make(1)
    alone.step(1)
    a, b = make(1), make(2)
    b.step(1)
    a.step(1)
    b.close()
    assert torch.equal(a.weights[0], alone.weights[0]) and torch.equal(a.m, alone.m) and np.isfinite(float(a.grad_norm()[0]))
