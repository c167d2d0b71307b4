"""The token embedding and its gradient on the GPU against the fp64 oracle.

Sums of whole numbers are exact in fp32 and compared bit for bit.  Otherwise a sum of c rows is off by at most
(c + 8) 2^-24 times the sum of magnitudes in any order, its product with the scale by 2^-24 of itself, and an output by
2^-8 (bf16) or 2^-24 (fp32) of itself."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from oracle import decoder_oracle as do

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f64(t):
    return t.detach().cpu().double().numpy()


def strided(rows, cols, dtype, pad=0, shift=0):
    buf = torch.full((rows * (cols + pad) + shift + 16,), float("nan"), dtype=DT[dtype], device=DEV)
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def untouched(v):
    if v.shape[0] < 2 or v.stride(0) == v.shape[1]:
        return True
    whole = torch.as_strided(v, (v.shape[0] - 1, v.stride(0)), v.stride(), v.storage_offset())
    return bool(torch.isnan(whole[:, v.shape[1]:]).all())


def rounding(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


@pytest.mark.parametrize("tdtype,dtype", [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("m,rows,d,pad", [(1, 1, 1, 0), (4, 100, 768, 0), (37, 11, 7, 3), (300, 50, 33, 1), (129, 1000, 1025, 0)])
def test_lookup(tdtype, dtype, m, rows, d, pad):
    gen = torch.Generator(DEV).manual_seed(m)
    table = strided(rows, d, tdtype, pad, 1)
    table.copy_(torch.randn(rows, d, generator=gen, device=DEV))
    ids = torch.randint(0, rows, (m,), generator=gen, device=DEV)
    if m > 2:
        ids[1], ids[m - 1] = -1, rows       # rows of NaN
    for scale in (1.0, 8.0, 0.3):
        out = strided(m, d, dtype, pad + 1, 3)
        smat.smat_embed(table, ids, out, scale=scale)
        want = do.embed(f64(table), ids.cpu().numpy(), float(np.float32(scale)))
        got = f64(out)
        assert np.array_equal(np.isnan(got), np.isnan(want)) and untouched(out)
        ok = ~np.isnan(want)
        if scale != 0.3 and (dtype == "f32" or tdtype == dtype):
            assert np.array_equal(got[ok], want[ok])
        assert np.all(np.abs(got - want)[ok] <= np.abs(want)[ok] * (rounding(dtype) + 2.0 ** -23))


def ids_of(kind, m, rows, gen):
    if kind == "one":
        return torch.full((m,), rows // 2, device=DEV, dtype=torch.int64)
    if kind == "all":                                    # every row once, in a mixed order
        return torch.randperm(rows, generator=gen, device=DEV)[:m]
    ids = torch.randint(0, rows, (m,), generator=gen, device=DEV)
    if kind == "skew":                                   # a few rows hold most tokens
        hot = torch.rand(m, generator=gen, device=DEV)
        ids = torch.where(hot < 0.5, ids % 3, ids)
    if kind == "outside":
        out = torch.rand(m, generator=gen, device=DEV)
        ids = torch.where(out < 0.3, ids - rows, torch.where(out > 0.8, ids + rows, ids))
    return ids


# from one token to several tiles of the sort, chunk ends inside and between runs, vocabularies of one to four digits
GRADS = [(255, 40, 600, "skew"), (256, 300, 9, "outside"), (60, 64, 1300, "all"), (64, 9, 40, "any"), (65, 9, 3, "one"), (1, 1, 1, "one"), (1, 50, 40, "any"), (31, 7, 9, "any"), (32, 5, 8, "one"), (33, 5, 8, "one"), (64, 2, 65, "any"),
         (100, 100, 513, "all"), (1000, 37, 1025, "skew"), (257, 300, 2048, "any"), (4096, 1000, 64, "skew"),
         (4097, 255, 31, "any"), (4097, 256, 31, "any"), (5000, 257, 17, "outside"), (8192, 70000, 8, "skew"),
         (20000, 3, 24, "any"), (40000, 65535, 5, "any"), (40000, 65536, 5, "skew"), (70001, 131072, 3, "skew"),
         (33000, 20000000, 2, "any"), (130000, 11, 12, "one"), (300000, 70000, 2, "any")]


@pytest.mark.parametrize("dtype,tdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("m,rows,d,kind", GRADS)
def test_gradient_of_whole_numbers_is_exact(dtype, tdtype, m, rows, d, kind):
    """A token left out, taken twice or put into another row shows.  (A row's sum stays under 2^24, its bf16 rounding is
    compared with torch's.)"""
    gen = torch.Generator(DEV).manual_seed(m + rows)
    ids = ids_of(kind, m, rows, gen)
    dy = strided(m, d, dtype, 3, 1)
    dy.copy_(torch.randint(-50, 51, (m, d), generator=gen, device=DEV))
    inside = (ids >= 0) & (ids < rows)
    want = torch.zeros(rows, d, dtype=torch.float64, device=DEV)
    want.index_add_(0, ids[inside], dy.double()[inside])
    out = strided(rows, d, tdtype, 2, 1)
    smat.smat_embed_grad(dy, ids, out)
    assert torch.equal(out, want.to(DT[tdtype])) and untouched(out)
    # accumulated: rows with tokens gain their sum, the others keep their bits, a NaN's too
    base = torch.randint(-50, 51, (rows, d), generator=gen, device=DEV).to(DT[tdtype])
    hit = torch.zeros(rows, dtype=torch.bool, device=DEV)
    hit[ids[inside]] = True
    base[~hit] = float("nan")
    out.copy_(base)
    smat.smat_embed_grad(dy, ids, out, scale=2.0, accumulate=True)
    assert torch.equal(out[hit], (base.double() + 2 * want)[hit].to(DT[tdtype])) and out[~hit].isnan().all() and untouched(out)
    # the padding id's row stays without a gradient
    pad = int(ids[inside][0]) if bool(inside.any()) else 0
    want[pad] = 0
    smat.smat_embed_grad(dy, ids, out, padding_idx=pad)
    assert torch.equal(out, want.to(DT[tdtype]))


@pytest.mark.parametrize("dtype,tdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("m,rows,d,kind", [(777, 50, 100, "skew"), (9000, 500, 40, "skew"), (3000, 10, 700, "any")])
def test_gradient(dtype, tdtype, m, rows, d, kind):
    gen = torch.Generator(DEV).manual_seed(m)
    ids = ids_of(kind, m, rows, gen)
    dy = torch.randn(m, d, generator=gen, device=DEV).to(DT[dtype])
    out = torch.empty(rows, d, dtype=DT[tdtype], device=DEV)
    scale = float(np.float32(0.3))
    smat.smat_embed_grad(dy, ids, out, scale=0.3)
    at = ids.cpu().numpy()
    want = do.embed_grad(f64(dy), at, rows, scale)
    size = do.embed_grad(np.abs(f64(dy)), at, rows, scale)
    err = (np.bincount(at, minlength=rows)[:, None] + 8) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want)
    assert np.all(np.abs(f64(out) - want) <= err + (np.abs(want) + err) * rounding(tdtype))
    again = torch.empty_like(out)
    smat.smat_embed_grad(dy, ids, again, scale=0.3)
    assert torch.equal(out, again)


def test_rows_without_a_number():
    """NaN and infinities stay in their tokens' rows; those of a padding token and of one outside the table go nowhere."""
    dy = torch.ones(200, 9, device=DEV)
    ids = torch.arange(200, device=DEV) % 5
    dy[5] = float("nan")        # id 0
    dy[1] = float("inf")        # id 1
    dy[3::5] = float("nan")     # id 3, the padding
    ids[4] = 77
    dy[4] = float("nan")
    out = torch.empty(6, 9, device=DEV)
    smat.smat_embed_grad(dy, ids, out, padding_idx=3)
    assert out[0].isnan().all() and out[1].isinf().all() and not out[3].any() and not out[5].any()
    assert torch.equal(out[2], torch.full((9,), 40.0, device=DEV)) and torch.equal(out[4], torch.full((9,), 39.0, device=DEV))


def test_empty():
    ids = torch.empty(0, dtype=torch.int64, device=DEV)
    smat.smat_embed(torch.ones(3, 4, device=DEV), ids, torch.empty(0, 4, device=DEV))
    out = torch.full((3, 4), 5.0, device=DEV)
    smat.smat_embed_grad(torch.empty(0, 4, device=DEV), ids, out, accumulate=True)
    assert out.eq(5).all()
    smat.smat_embed_grad(torch.empty(0, 4, device=DEV), ids, out)
    assert not out.any()
    one = torch.zeros(2, dtype=torch.int64, device=DEV)
    smat.smat_embed(torch.empty(0, 4, device=DEV), one, wide := torch.zeros(2, 4, device=DEV))
    assert wide.isnan().all()
    smat.smat_embed_grad(torch.ones(2, 4, device=DEV), one, torch.empty(0, 4, device=DEV))
    smat.smat_embed(torch.empty(3, 0, device=DEV), one, torch.empty(2, 0, device=DEV))
    smat.smat_embed_grad(torch.empty(2, 0, device=DEV), one, torch.empty(3, 0, device=DEV))
    torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """A table and gradients of more than 2^32 bytes, the last rows of which are read and written."""
    rows, d = (1 << 21) + 3, 1100
    table = torch.zeros(rows, d, dtype=torch.bfloat16, device=DEV)
    table[-1] = 3.0
    table[-2] = 2.0
    ids = torch.tensor([rows - 1, 0, rows - 2, rows - 1], device=DEV)
    out = torch.empty(4, d, dtype=torch.bfloat16, device=DEV)
    smat.smat_embed(table, ids, out)
    assert out[0].eq(3).all() and out[1].eq(0).all() and out[2].eq(2).all()
    table.fill_(9.0)
    smat.smat_embed_grad(out, ids, table)
    assert table[-1].eq(6).all() and table[-2].eq(2).all() and not table[:-2].any()


def test_workspace_stream_and_graph():
    m, rows, d = 5000, 333, 40
    gen = torch.Generator(DEV).manual_seed(1)
    dy, ids = torch.randn(m, d, generator=gen, device=DEV), ids_of("skew", m, rows, gen)
    eager, other, held = (torch.empty(rows, d, device=DEV) for _ in range(3))
    smat.smat_embed_grad(dy, ids, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    smat.smat_embed_grad(dy, ids, other, stream=side, workspace=torch.empty(1 << 23, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(eager, other)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        smat.smat_embed_grad(dy, ids, held)
    for turn in range(3):
        ids.copy_(ids_of("any", m, rows, gen))
        dy.copy_(torch.randn(m, d, generator=gen, device=DEV))
        smat.smat_embed_grad(dy, ids, eager)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, held), turn


def test_binding_refuses():
    table, ids, out = torch.zeros(5, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, 8, device=DEV)
    for fn in (lambda: smat.smat_embed(table, ids.int(), out), lambda: smat.smat_embed(table, ids[:3], out),
               lambda: smat.smat_embed(table, ids.cpu(), out), lambda: smat.smat_embed(table, ids, out[:, :7]),
               lambda: smat.smat_embed(table, ids, table[:4]), lambda: smat.smat_embed(table.half(), ids, out),
               lambda: smat.smat_embed(table.t(), ids, out), lambda: smat.smat_embed(table, ids.view(2, 2), out),
               lambda: smat.smat_embed_grad(out, ids, table[:, :7]), lambda: smat.smat_embed_grad(out, ids, out),
               lambda: smat.smat_embed_grad(out, ids, table.cpu()), lambda: smat.smat_embed(table, ids, out, scale=float("inf")),
               lambda: smat.smat_embed_grad(out, torch.zeros(8, dtype=torch.int64, device=DEV)[::2], table)):
        with pytest.raises(smat.SmatError):
            fn()
