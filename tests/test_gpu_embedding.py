"""Embedding rows (dense and packed) and their gradient against plain numpy in binary64."""
import numpy as np
import pytest
import torch

from _training import embedding_grad64, held_rows

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # half a step, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}   # smallest step


def _ids(gen, count, rows, hot=0.3, dtype=torch.int64):
    ids = torch.randint(0, rows, (count,), generator=gen, device="cuda")
    frequent = torch.rand(count, generator=gen, device="cuda") < hot
    return torch.where(frequent, rows // 2, ids).to(dtype)


def _gen(*parts):
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * p for i, p in enumerate(parts)))


@pytest.mark.parametrize("table,out", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("count,rows,width", [(0, 3, 8), (1, 1, 1), (1, 5, 768), (7, 100, 3), (33, 40, 129), (500, 30522, 768), (64, 9, 5001)])
def test_lookup(table, out, count, rows, width):
    gen = _gen(count, rows, width)
    w = (torch.randn(rows, width, generator=gen, device="cuda") * 0.05).to(DTYPES[table])
    for dtype in (torch.int64, torch.int32):
        ids = _ids(gen, count, rows, dtype=dtype)
        got = qb.embedding_lookup(w, ids, scale=27.7, out_dtype=DTYPES[out])
        assert got.shape == (count, width) and got.dtype == DTYPES[out]
        want = w.double().cpu().numpy()[ids.cpu().numpy()] * float(np.float32(27.7))
        err = np.abs(got.double().cpu().numpy() - want)
        # one binary32 product, one rounding to the output's type
        assert np.all(err <= np.abs(want) * (2.0 ** -24 + HALF[out] * (1 + 2.0 ** -24)) + TINY[out])


def test_lookup_strides_offsets_shapes_and_bounds():
    gen = _gen(1)
    big = torch.randn(50, 103, generator=gen, device="cuda")
    w = big[:, 2:2 + 96]                                        # rows 103 apart, off alignment
    ids = torch.tensor([[0, 49, -1], [7, 50, 1 << 40]], device="cuda")
    room = torch.full((2, 3, 101), 7.0, device="cuda", dtype=torch.bfloat16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = qb.embedding_lookup(w, ids, out=room[..., 1:97], status=status)
    assert int(status) == qb.ST_INDEX
    want = torch.zeros(2, 3, 96, device="cuda")
    want[0, 0], want[0, 1], want[1, 0] = w[0], w[49], w[7]
    assert torch.equal(got.float(), want.bfloat16().float())
    assert bool((room[..., 0] == 7).all()) and bool((room[..., 97:] == 7).all())
    status.zero_()
    qb.embedding_lookup(w, ids[:1], status=status)
    assert int(status) == 0                                     # a negative id is a padded position
    row = qb.embedding_lookup(w, torch.tensor(3, device="cuda"))
    assert row.shape == (96,) and torch.equal(row, w[3])
    empty = qb.embedding_lookup(w, torch.empty(2, 0, dtype=torch.int64, device="cuda"))
    assert empty.shape == (2, 0, 96)


@pytest.mark.parametrize("kx", range(15))
@pytest.mark.parametrize("rows,width,first", [(1, 1, 0), (9, 7, 0), (40, 129, 256), (200, 64, 128), (3, 1000, 131)])
def test_held_lookup(kx, rows, width, first):
    gen = _gen(kx, rows, width)
    b = kx + 2
    total = -(-(first + rows * width) // 128) * 128
    q = torch.randint(-(1 << kx), (1 << kx) + 1, (total,), generator=gen, device="cuda").cpu().numpy()
    bits = ((q[:, None] + (1 << kx)) >> np.arange(b)) & 1
    codes = torch.from_numpy(np.packbits(bits.reshape(-1).astype(np.uint8), bitorder="little")).cuda()
    assert codes.numel() == total * b // 8
    table = held_rows(codes.cpu().numpy(), kx, first, rows, width)
    ids = torch.cat([torch.arange(rows, device="cuda"), torch.tensor([-1, rows], device="cuda")])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = qb.held_lookup(codes, kx, ids, rows, width, scale=3.0, out_dtype=torch.float32, first=first, status=status)
    assert np.array_equal(got[:rows].cpu().numpy(), (table * 3).astype(np.float32))    # exact: at most 17 bits
    assert bool((got[rows:] == 0).all()) and int(status) == qb.ST_INDEX


def test_rows_of_what_a_worker_holds():
    seg, n = [40 * 64, 130, 33 * 24], 2
    x1 = torch.randn(sum(seg)) * 0.2
    for kx in (0, 6):
        q = qb.QAdam(seg, n, kx=kx, x1=x1)
        g = q.to_padded(torch.randn(n, sum(seg), device="cuda") * 0.01)
        q.step(1, g)
        codes = q.wcodes[:q.wcode_bytes].cpu().numpy()
        for s, width in ((0, 64), (2, 24)):
            table = held_rows(codes, kx, q.seg_off[s], seg[s] // width, width)
            ids = torch.tensor([0, seg[s] // width - 1, 5, 5], device="cuda")
            got = q.lookup(s, width, ids, out_dtype=torch.float32)
            assert np.array_equal(got.cpu().numpy(), table[ids.cpu().numpy()].astype(np.float32))
        with pytest.raises(ValueError):
            q.lookup(1, 64, ids)
        q.close()


# ---------------------------------------------------------------- gradient

def _check_grad(got, ids, dy, rows, scale, out, old=None, padding=-1):
    total, size, n = embedding_grad64(ids.cpu().numpy(), dy.double().cpu().numpy(), rows, padding)
    scale = float(np.float32(scale))
    want = total * scale
    u = 2.0 ** -24
    # n tokens: at most n additions in binary32, the product, then (accumulated) one more, then the type's rounding
    tol = abs(scale) * size * ((n + 1) * u * 1.01)[:, None] + np.abs(want) * 2 * u
    if old is not None:
        old = old.double().cpu().numpy()
        want = want + old
        tol = tol + (np.abs(old) + np.abs(want)) * u
    tol = tol + np.abs(want) * HALF[out] * (1 + 2.0 ** -8) + tol * HALF[out] + TINY[out]
    got = got.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol)
    if old is not None:
        assert np.array_equal(got[n == 0], old[n == 0])         # not touched
    else:
        assert np.all(got[n == 0] == 0)


SIZES = [(1, 1, 1), (1, 5, 768), (2, 2, 3), (31, 7, 127), (32, 7, 128), (33, 7, 129), (64, 1, 64), (65, 40, 4), (300, 513, 100),
         (1025, 512, 257), (4096, 30522, 64), (4097, 2, 260), (8192, 1, 9), (8193, 600000, 5), (100, 2000000, 2), (1500, 5000000, 1), (9001, 300000, 12),
         (20000, 50, 40), (40001, 700, 300), (90000, 30, 20), (1100000, 1000, 3)]


@pytest.mark.parametrize("dy,dw", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("count,rows,width", SIZES)
def test_gradient(dy, dw, count, rows, width):
    gen = _gen(count, rows, width)
    g = (torch.randn(count, width, generator=gen, device="cuda") * 0.1).to(DTYPES[dy])
    for dtype, hot in ((torch.int64, 0.3), (torch.int32, 0.0)):
        ids = _ids(gen, count, rows, hot, dtype)
        got = qb.embedding_grad(ids, g, rows, scale=1.7, dtype=DTYPES[dw])
        assert got.shape == (rows, width) and got.dtype == DTYPES[dw]
        _check_grad(got, ids, g, rows, 1.7, dw)
        assert torch.equal(qb.embedding_grad(ids, g, rows, scale=1.7, dtype=DTYPES[dw]), got)      # the same bits


@pytest.mark.parametrize("dw", ["f32", "bf16"])
@pytest.mark.parametrize("count,rows,width", SIZES)
def test_gradient_added(dw, count, rows, width):
    gen = _gen(count, rows, width, 3)
    g = torch.randn(count, width, generator=gen, device="cuda").bfloat16()
    ids = _ids(gen, count, rows, 0.5)
    ids[::5] = -1
    old = torch.randn(rows, width, generator=gen, device="cuda").to(DTYPES[dw])
    out = old.clone()
    got = qb.embedding_grad(ids, g, rows, scale=0.5, out=out, accumulate=True)
    assert got is out
    _check_grad(got, ids, g, rows, 0.5, dw, old=old)


@pytest.mark.parametrize("count", [5, 100, 5000])
def test_padding_bad_ids_and_a_batch_of_padding(count):
    gen = _gen(count, 77)
    g = torch.randn(count, 72, generator=gen, device="cuda")
    ids = _ids(gen, count, 30)
    ids[1::4] = -100
    ids[2::4] = 3
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = qb.embedding_grad(ids, g, 30, padding=3, status=status)
    _check_grad(got, ids, g, 30, 1.0, "f32", padding=3)
    assert int(status) == 0 and bool((got[3] == 0).all())
    ids[0], ids[-1] = 30, (1 << 40)
    got = qb.embedding_grad(ids, g, 30, padding=3, status=status)
    _check_grad(got, ids, g, 30, 1.0, "f32", padding=3)
    assert int(status) == qb.ST_INDEX
    for ids in (torch.full((count,), -1, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")):
        out = torch.full((30, 72), 7.0, device="cuda")
        assert bool((qb.embedding_grad(ids, g[:ids.numel()], 30, out=out) == 0).all())
        out.fill_(7.0)
        assert bool((qb.embedding_grad(ids, g[:ids.numel()], 30, out=out, accumulate=True) == 7).all())


def test_strided_gradients_leave_the_rest_alone():
    gen = _gen(5)
    ids = _ids(gen, 3 * 41, 17).reshape(3, 41)
    wide = torch.randn(3, 41, 70, generator=gen, device="cuda")
    dy = wide[..., 3:36]
    room = torch.full((17, 50), 7.0, device="cuda")
    got = qb.embedding_grad(ids, dy, 17, out=room[:, 5:38])
    _check_grad(got, ids.reshape(-1), dy.reshape(-1, 33), 17, 1.0, "f32")
    assert bool((room[:, :5] == 7).all()) and bool((room[:, 38:] == 7).all())


@pytest.mark.parametrize("count,rows", [(50, 20), (3000, 20), (20000, 9)])
def test_gradient_against_differences(count, rows):
    # the loss sum(dy * lookup(table)) is linear in the table: its difference along a direction is the gradient's
    # product with it, in binary64 from the operator's own outputs
    gen = _gen(count, rows, 9)
    ids = _ids(gen, count, rows)
    dy = torch.randn(count, 24, generator=gen, device="cuda")
    table = torch.randn(rows, 24, generator=gen, device="cuda")
    step = torch.randn(rows, 24, generator=gen, device="cuda")
    scale = 2.0                                                   # (lookups of float32 by a power of two are exact)
    loss = lambda w: float((dy.double() * qb.embedding_lookup(w, ids, scale=scale).double()).sum())  # noqa: E731
    h = 2.0 ** -10
    up, down = table + h * step, table - h * step
    slope = (loss(up) - loss(down))
    want = float((qb.embedding_grad(ids, dy, rows, scale=scale).double() * (up.double() - down.double())).sum())
    size = float((dy.double().abs() * (up.double() - down.double()).abs()[ids] * scale).sum())
    assert abs(slope - want) <= size * (count + 2) * 2.0 ** -24 + 1e-9


def test_refusals():
    t, ids, dy = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, 8, device="cuda")
    codes = torch.zeros(160, dtype=torch.uint8, device="cuda")
    for bad in (lambda: qb.embedding_lookup(t, ids.float()), lambda: qb.embedding_lookup(t, ids.cpu()), lambda: qb.embedding_lookup(t.t(), ids),
                lambda: qb.embedding_lookup(t.double(), ids), lambda: qb.embedding_lookup(t[0], ids),
                lambda: qb.embedding_lookup(t, ids, out=torch.zeros(4, 7, device="cuda")),
                lambda: qb.embedding_lookup(t, ids, out=torch.zeros(4, 8, device="cuda"), out_dtype=torch.bfloat16),
                lambda: qb.embedding_lookup(t, ids, out=torch.zeros(8, 4, device="cuda").t()),
                lambda: qb.embedding_lookup(t, ids, status=torch.zeros(1, device="cuda")),
                lambda: qb.held_lookup(codes.int(), 6, ids, 10, 16), lambda: qb.held_lookup(codes[::2], 6, ids, 5, 16),
                lambda: qb.embedding_grad(ids, dy[:3], 10), lambda: qb.embedding_grad(ids, dy, 10, accumulate=True),
                lambda: qb.embedding_grad(ids, dy, 10, out=torch.zeros(9, 8, device="cuda")), lambda: qb.embedding_grad(ids, dy.double(), 10),
                lambda: qb.embedding_grad(ids, dy[:1].expand(4, 8), 10), lambda: qb.embedding_grad(ids, dy, 10, dtype=torch.float64)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: qb.held_lookup(codes, 15, ids, 10, 16), lambda: qb.held_lookup(codes, 6, ids, 11, 16),
                lambda: qb.held_lookup(codes[:150], 6, ids, 9, 16), lambda: qb.embedding_lookup(t, ids, scale=float("nan")),
                lambda: qb.embedding_grad(ids, dy, 10, scale=float("inf"))):
        with pytest.raises(qb.QAdamError):
            bad()


@pytest.mark.parametrize("count", [2000, 5000, 40000])
def test_captured_and_replayed_with_new_tokens(count):
    gen = _gen(6)
    ids, dy = _ids(gen, count, 300), torch.randn(count, 96, generator=gen, device="cuda")
    table, out = torch.randn(300, 96, generator=gen, device="cuda"), torch.empty(300, 96, device="cuda")
    qb.embedding_grad(ids, dy, 300, out=out)
    qb.embedding_lookup(table, ids)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rows = qb.embedding_lookup(table, ids, scale=2.0)
        qb.embedding_grad(ids, rows, 300, out=out)
    for _ in range(3):
        ids.copy_(_ids(gen, count, 300))
        graph.replay()
        fresh = qb.embedding_lookup(table, ids, scale=2.0)
        assert torch.equal(rows, fresh) and torch.equal(out, qb.embedding_grad(ids, fresh, 300))


def test_offsets_beyond_32_bits():
    """Rows, tokens and packed codes whose elements lie 2^32 and more behind the first: 8.6 GB at a time."""
    gen = _gen(8)
    rows, width = 4_300_007, 1000
    assert (rows - 100) * width > 2 ** 32
    table = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
    table[-100:] = torch.randn(100, width, generator=gen, device="cuda")
    ids = torch.tensor([rows - 1, 3, rows - 100, rows - 57, rows - 1], device="cuda")
    got = qb.embedding_lookup(table, ids)
    assert torch.equal(got, table[ids])
    # its gradient: the whole table is cleared, from the last row to the first
    table.fill_(7.0)
    dy = torch.randn(5, width, generator=gen, device="cuda").bfloat16()
    qb.embedding_grad(ids, dy, rows, out=table)
    assert torch.equal(table[3], dy[1]) and torch.equal(table[rows - 100], dy[2]) and torch.equal(table[rows - 57], dy[3])
    assert torch.equal(table[-1], (dy[0].float() + dy[4].float()).bfloat16())
    for i in (3, rows - 100, rows - 57, rows - 1):
        table[i] = 0
    assert not any(bool(part.any()) for part in table.split(1 << 19))
    # as many tokens: all but the last few have no gradient
    many = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    many[-4:] = torch.tensor([2, 0, 2, 1], dtype=torch.int32, device="cuda")
    table[-4:] = dy[:4]
    got = qb.embedding_grad(many, table, 5, dtype=torch.float32)
    assert torch.equal(got[0], dy[1].float()) and torch.equal(got[1], dy[3].float()) and not bool(got[3:].any())
    assert torch.equal(got[2], dy[0].float() + dy[2].float())
    # and a row for each of them: the last tokens' rows of the result
    source = torch.randn(3, width, generator=gen, device="cuda").bfloat16()
    qb.embedding_lookup(source, many, out=table)
    assert torch.equal(table[-4], source[2]) and torch.equal(table[-3], source[0]) and not bool(table[0].any())
    # packed codes, 8 bits each
    codes = table.view(-1).view(torch.uint8)
    codes[-8000:] = torch.randint(0, 129, (8000,), generator=gen, device="cuda").to(torch.uint8)
    codes = codes[:codes.numel() // 16 * 16]
    first = codes.numel() - 5000
    assert first > 2 ** 32
    got = qb.held_lookup(codes, 6, torch.tensor([4, 0], device="cuda"), 5, 1000, out_dtype=torch.float32, first=first)
    want = ((codes[first:].double() - 64) / 128).view(5, 1000)
    assert torch.equal(got.double(), want[[4, 0]])


def test_a_batch_without_tokens_waits_for_what_is_before_it():
    gen = _gen(9)
    big = torch.randn(4096, 4096, generator=gen, device="cuda")
    for _ in range(20):
        out = torch.mm(big, big)                               # a long kernel that writes `out` to its end
        got = qb.embedding_grad(torch.empty(0, dtype=torch.int64, device="cuda"), big[:0], 4096, out=out)
        assert not bool(got.any())


def test_an_expanded_gradient_is_refused():
    ids = torch.tensor([0, 1, 2], device="cuda")
    for dy in (torch.ones(1, 8, device="cuda").expand(3, 8), torch.ones(3, 1, device="cuda").expand(3, 8)):
        with pytest.raises(ValueError, match="dy"):
            qb.embedding_grad(ids, dy, 4)
        assert bool((qb.embedding_grad(ids, dy.contiguous(), 4)[:3] == 1).all())


@pytest.mark.parametrize("each", range(1, 9))
def test_batches_around_what_a_cluster_sorts(each):
    """Whole and nearly whole clusters of 8 x 512 threads with 1 to 8 tokens each, over one, two and three digits."""
    for rows in (300, 30522, 300000):
        for count in (4096 * each - 1, 4096 * each, 4096 * each + 1):
            ids = torch.randint(0, rows, (count,), generator=_gen(count, rows), device="cuda")
            ids[::3] = rows - 1
            dy = torch.arange(count, device="cuda").remainder(2048).float().view(-1, 1)
            got = qb.embedding_grad(ids, dy, rows)
            # sums of whole numbers: exact in binary32 while below 2^24
            want = torch.zeros(rows, dtype=torch.float64, device="cuda").index_add_(0, ids, dy[:, 0].double())
            exact = want < 2 ** 24
            assert torch.equal(got[exact, 0].double(), want[exact])
            assert bool(((got[:, 0].double() - want).abs() <= want * (count + 1) * 2.0 ** -24).all())
