"""Kernels of the operators around the quantized step that differ by type and alignment alone, each against its plain
statement: pairs of types, rows on 8 bytes, packed codes into 16 bits, unaligned tensors with several pairs of rows to a warp."""
import numpy as np
import pytest
import torch

from _training import held_rows
from test_gpu_embedding import DTYPES, HALF, TINY, _check_grad, _gen, _ids

pytestmark = pytest.mark.gpu

import paper_2004_14180_b200 as qb  # noqa: E402


# ---------------------------------------------------------------- gradient

@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dy,dw", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("f16", "f32"), ("f16", "bf16"), ("f16", "f16"), ("bf16", "f16")])
@pytest.mark.parametrize("count,rows,width", [(1, 5, 768), (33, 7, 129), (65, 40, 4), (300, 513, 100), (1025, 512, 264), (8193, 6000, 5),
                                              (20000, 50, 40), (40001, 700, 300)])
def test_gradient_of_every_pair_of_types(dy, dw, add, count, rows, width):
    gen = _gen(count, rows, width, 11)
    g = (torch.randn(count, width, generator=gen, device="cuda") * 0.1).to(DTYPES[dy])
    ids = _ids(gen, count, rows)
    ids[::9] = -1
    if not add:
        _check_grad(qb.embedding_grad(ids, g, rows, scale=1.7, dtype=DTYPES[dw]), ids, g, rows, 1.7, dw)
        return
    old = torch.randn(rows, width, generator=gen, device="cuda").to(DTYPES[dw])
    out = old.clone()
    qb.embedding_grad(ids, g, rows, scale=0.5, out=out, accumulate=True)
    _check_grad(out, ids, g, rows, 0.5, dw, old=old)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("dy", list(DTYPES))
@pytest.mark.parametrize("dw", list(DTYPES))
@pytest.mark.parametrize("first,stride", [(4, 80), (8, 76), (4, 77)])
def test_gradient_rows_on_eight_bytes(dy, dw, add, first, stride):
    # 16-bit rows that begin on 8 bytes and not on 16 (their first one, all but every second, or only every fourth), rows of dy on 16
    count, rows, width = 700, 60, 64
    gen = _gen(first, stride, 5)
    g = torch.randn(count, width, generator=gen, device="cuda").to(DTYPES[dy])
    ids = _ids(gen, count, rows)
    room = torch.full((rows * stride + 16,), 7.0, device="cuda", dtype=DTYPES[dw])
    out = room[first:first + (rows - 1) * stride + width].as_strided((rows, width), (stride, 1))
    if add:
        out.copy_(torch.randn(rows, width, generator=gen, device="cuda"))
    old = out.clone() if add else None
    qb.embedding_grad(ids, g, rows, scale=0.5, out=out, accumulate=add)
    _check_grad(out, ids, g, rows, 0.5, dw, old=old)
    out.fill_(7.0)
    assert bool((room == 7).all())


# ---------------------------------------------------------------- lookup

@pytest.mark.parametrize("table,out", [("f16", "f32"), ("f32", "f16"), ("f16", "bf16"), ("bf16", "f16")])
@pytest.mark.parametrize("count,rows,width", [(1, 5, 768), (33, 40, 129), (500, 3000, 768), (64, 9, 5001)])
def test_lookup_of_every_pair_of_types(table, out, count, rows, width):
    gen = _gen(count, rows, width, 13)
    w = (torch.randn(rows, width, generator=gen, device="cuda") * 0.05).to(DTYPES[table])
    ids = _ids(gen, count, rows)
    got = qb.embedding_lookup(w, ids, scale=27.7, out_dtype=DTYPES[out])
    want = w.double()[ids].cpu().numpy() * float(np.float32(27.7))
    # one binary32 product, one rounding to the output's type
    err = np.abs(got.double().cpu().numpy() - want)
    assert got.dtype == DTYPES[out] and np.all(err <= np.abs(want) * (2.0 ** -24 + HALF[out] * (1 + 2.0 ** -24)) + TINY[out])


@pytest.mark.parametrize("out", ["bf16", "f16"])
@pytest.mark.parametrize("kx", range(15))
@pytest.mark.parametrize("rows,width,first", [(9, 7, 0), (40, 129, 256), (200, 64, 128), (3, 1000, 131)])
def test_packed_rows_into_16_bits(out, kx, rows, width, first):
    gen = _gen(kx, rows, width, 17)
    b = kx + 2
    total = -(-(first + rows * width) // 128) * 128
    q = torch.randint(-(1 << kx), (1 << kx) + 1, (total,), generator=gen, device="cuda").cpu().numpy()
    bits = ((q[:, None] + (1 << kx)) >> np.arange(b)) & 1
    codes = torch.from_numpy(np.packbits(bits.reshape(-1).astype(np.uint8), bitorder="little")).cuda()
    table = held_rows(codes.cpu().numpy(), kx, first, rows, width)
    ids = torch.arange(rows, device="cuda").flip(0)
    got = qb.held_lookup(codes, kx, ids, rows, width, scale=3.0, out_dtype=DTYPES[out], first=first)
    # three times a code of at most 15 bits is exact in binary32: one rounding
    want = torch.from_numpy((table * 3).astype(np.float32)).to(DTYPES[out]).flip(0)
    assert torch.equal(got.cpu(), want)


# ---------------------------------------------------------------- AdamW

@pytest.mark.parametrize("shift", [1, 2])
@pytest.mark.parametrize("large", [2_700_001, 5_300_000, 10_600_130])
@pytest.mark.parametrize("master", [False, True])
def test_several_pairs_of_rows_of_unaligned_tensors(large, master, shift):
    # from 2.56, 5.12 and 10.24 x 10^6 elements on a warp takes 2, 4 and 8 pairs; the same bits as where all is aligned
    wtype = torch.bfloat16 if master else torch.float32
    lens = [700, large, 129, 4000]

    def make(off):
        gen = torch.Generator(device="cuda").manual_seed(large)
        out = []
        for s in (0.05, 0.01):
            rooms = [torch.full((n + 16,), 7.0, device="cuda", dtype=wtype) for n in lens]
            out.append([r[off:off + n] for r, n in zip(rooms, lens)])
            for t in out[-1]:
                t.copy_(torch.randn(t.numel(), device="cuda", generator=gen) * s)
        return qb.AdamW(out[0], out[1], state_bits=8, master=master, seed=77, lr=1e-3, weight_decay=0.1)

    a, b = make(0), make(shift)
    for t in (1, 2):
        a.step(t)
        b.step(t)
    for name in ("m", "r", "m_scale", "r_scale") + (("master",) if master else ()):
        assert torch.equal(getattr(a, name), getattr(b, name)), name
    for x, y in zip(a.weights, b.weights):
        assert torch.equal(x, y)
        around = y.as_strided((16 - shift,), (1,), y.storage_offset() + y.numel())
        assert bool((around == 7).all())
