"""Waits inside the products that run out, made to happen without a fault: a CTA leaves the last block of its sum out (test_missing_blocks), what
waits for it gives up after few polls, the status word says so, and the GPU goes on working."""
import pytest
import torch

from _layer import gen_of
from test_gpu_int8 import check, int8_rows

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402
from paper_2004_14180_b200.adamw import stream_of  # noqa: E402
from paper_2004_14180_b200.binding import PRODUCT_ARGS  # noqa: E402

NOTHING = -12345.0


def product(a, b, out, status, missing, transposed=0, accumulate=0):
    n = out.shape[1]
    args = dict(a=a.q_at, a_stride=a.stride, a_scale=a.scale_at, rows=a.rows, depth=a.width, b=b.q_at, b_stride=b.stride,
                b_scale=0 if transposed else b.scale_at, channels=n, out=out.data_ptr(), out_stride=out.stride(0), status=status.data_ptr(),
                transposed=transposed, out_type={torch.float32: 0, torch.bfloat16: 1}[out.dtype], accumulate=accumulate, wait_polls=1 << 14,
                test_missing_blocks=missing, b_worth=1.0)
    assert qb.load_library().qadam_row_product(PRODUCT_ARGS.pack(*[args.get(f) or 0 for f in PRODUCT_ARGS.fields]), stream_of(out.device)) == 0


# few tokens: a CTA to a tile, eight of them that share a sum; pairs: a tile each, several each, sums longer than the ring
@pytest.mark.parametrize("m,k,n,masks", [(16, 128, 300, [1]), (9, 300, 128, [1]), (1, 4096, 512, [1, 128, 255, 4]), (70, 2048, 256, [1, 9, 255]),
                                         (300, 100, 70, [1, 2, 3]), (300, 768, 512, [1, 2, 3]), (513, 4096, 512, [1, 2, 3]), (6000, 512, 4098, [1, 2, 3])])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_a_wait_that_runs_out_is_told_and_the_device_stays_usable(m, k, n, masks, kind):
    gen = gen_of(m, k, n)
    a, b = int8_rows(gen, m, k), int8_rows(gen, n, k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = qb.int8_matmul(a, b, out_dtype=kind, status=status)
    check(want, a, b.q, b.scale, None, "f32" if kind is torch.float32 else "bf16")
    assert int(status) == 0
    for missing in masks:
        for transposed in (0, 1):
            c = int8_rows(gen, k, n) if transposed else b
            out = torch.full((m, n), NOTHING, dtype=kind, device="cuda")
            product(a, c, out, status, missing, transposed)       # returns: every wait is bounded
            torch.cuda.synchronize()
            assert int(status) == qb.ST_TIMEOUT
            whole = want if not transposed else qb.int8_matmul(a, c, out_dtype=kind, transpose=True)
            left = out == torch.tensor(NOTHING, dtype=kind)
            assert bool(left.any()) and bool((left | (out == whole)).all())          # written rightly, or not at all
            status.zero_()
            again = qb.int8_matmul(a, b, out_dtype=kind, status=status)
            assert torch.equal(again, want) and int(status) == 0
    many = [torch.full((m, n), NOTHING, dtype=kind, device="cuda") for _ in range(4)]
    for i, out in enumerate(many):                                # one behind the other, whole ones between them
        product(a, b, out, status, 0 if i % 2 else masks[-1])
    torch.cuda.synchronize()
    assert int(status) == qb.ST_TIMEOUT and torch.equal(many[1], want) and torch.equal(many[3], want)


def test_a_contexts_status_word_goes_with_its_products(monkeypatch):
    from paper_2004_14180_b200 import int8
    q = qb.QAdam([32 * 64], 1, kg=0, kx=6)
    given = []
    held = int8.held_matmul
    monkeypatch.setattr(int8, "held_matmul", lambda *args, **kw: given.append(kw["status"]) or held(*args, **kw))
    a, own = int8_rows(gen_of(3), 5, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    q.matmul(0, 64, a)
    q.matmul(0, 64, a, status=own)
    assert given[0].data_ptr() == q.bufs.status and given[1] is own and q.poll_status() == 0
    given[0].fill_(qb.ST_TIMEOUT)
    torch.cuda.synchronize()
    assert q.poll_status() == qb.ST_TIMEOUT
    q.close()
