"""Norms and products of all kinds on several streams at once: each gives what it gives alone."""
import pytest
import torch

from _layer import gen_of, randn
from test_gpu_int8 import int8_rows

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


def test_calls_on_several_streams_at_once():
    gen = gen_of(81)
    calls = []
    # few tokens that share a sum, that do not (one block: beside a pair's CTA there is room for one), pairs with short and long sums, a held table
    for m, k, n in ((1, 4096, 512), (9, 100, 20000), (60, 2048, 4096), (100, 4096, 640), (300, 768, 4096), (3000, 4096, 1024)):
        a, b = int8_rows(gen, m, k), int8_rows(gen, n, k)
        calls.append(lambda a=a, b=b: qb.int8_matmul(a, b))
    codes, c = torch.randint(0, 129, (3000 * 768,), generator=gen, device="cuda").to(torch.uint8), int8_rows(gen, 700, 768)
    calls.append(lambda: qb.held_matmul(c, codes, 6, 3000, 768))
    x, dy = randn(gen, 5000, 1032).bfloat16(), randn(gen, 5000, 1032).bfloat16()
    calls.append(lambda: qb.layer_norm(x, residual=dy, int8=True).rows.values())
    ran = qb.layer_norm(x)
    calls.append(lambda: torch.cat([t.flatten().float() for t in qb.layer_norm_grad(dy, x, ran.mean, ran.rstd)]))
    want = [f() for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    got = []
    for turn in range(30):
        for i, s in enumerate(streams):
            j = (turn * 5 + i * 2 + turn // 9) % len(calls)
            with torch.cuda.stream(s):
                got.append((j, calls[j]()))
    torch.cuda.synchronize()
    assert {j for j, _ in got} == set(range(len(calls)))
    for j, y in got:
        assert torch.equal(y, want[j])
