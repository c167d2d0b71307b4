"""Products whose operands lie off 16-byte rows, with NaN between the rows and after them: at these sizes they are copied to
16-byte rows first, or go through registers.  And few rows at sizes on both sides of the choice between the vector units and
the small tiles.  Against float64 products on the GPU; bounds as in test_gpu_linear.py: (R + 8) 2^-23 of the sums'
magnitudes, 2^-8 (bf16) or 2^-22 of the result."""
import pytest
import torch

import paper_2609_33437_amd as smat

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}


def view(gen, rows, cols, dtype, pad, shift, std=1.0):
    buf = torch.full((rows * (cols + pad) + shift + 64,), float("nan"), dtype=DT[dtype], device=DEV)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * std)
    return v


def check(got, want, mag, r, dtype, what):
    err = (r + 8) * 2.0 ** -23 * mag
    bad = ~((got.double() - want).abs() <= err + (want.abs() + err) * U[dtype])
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("m,n,k", [(513, 2049, 2049), (1001, 2001, 1999), (130, 258, 8193), (2055, 1023, 517), (33, 65, 131)])
@pytest.mark.parametrize("pad,shift", [(3, 1), (0, 0), (1, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_off_16_bytes(m, n, k, pad, shift, dtype):
    gen = torch.Generator(DEV).manual_seed(m + n + k + pad)
    x, w, out = (view(gen, *s, dtype, pad, shift) for s in ((m, k), (n, k), (m, n)))
    smat.smat_linear(x, w, out)
    check(out, x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t(), k, dtype, "linear")
    dy, w2 = view(gen, m, n, dtype, pad, shift), view(gen, n, k, dtype, pad, shift)
    dx = view(gen, m, k, dtype, pad, shift)
    smat.smat_linear_dgrad(dy, w2, dx)
    check(dx, dy.double() @ w2.double(), dy.double().abs() @ w2.double().abs(), n, dtype, "dgrad")
    dw, db = view(gen, n, k, dtype, pad, shift), torch.empty(n, dtype=DT[dtype], device=DEV)
    smat.smat_linear_wgrad(dy, x, dw, db=db)
    check(dw, dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs(), m, dtype, "wgrad")
    check(db, dy.double().sum(0), dy.double().abs().sum(0), m, dtype, "db")
    for v in (x, w, dy, w2, out, dx, dw):
        if pad:
            between = torch.as_strided(v, (v.shape[0] - 1, v.stride(0)), v.stride(), v.storage_offset())[:, v.shape[1]:]
            assert bool(torch.isnan(between).all())


@pytest.mark.parametrize("n,k", [(14336, 1024), (8960, 1536), (2048, 2048), (960, 4096), (1536, 8960), (257, 769)])
@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_few_rows(m, n, k, dtype):
    gen = torch.Generator(DEV).manual_seed(m + n + k)
    x, w, res = view(gen, m, k, dtype, 0, 0), view(gen, n, k, dtype, 0, 0, 0.1), view(gen, m, n, dtype, 0, 0)
    out = torch.empty(m, n, dtype=DT[dtype], device=DEV)
    smat.smat_linear(x, w, out, residual=res)
    want, mag = x.double() @ w.double().t() + res.double(), x.double().abs() @ w.double().abs().t() + res.double().abs()
    check(out, want, mag, k, dtype, "few rows")


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (257, 33), (1025, 8191), (300, 8192), (1030, 8223)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_column_sums(rows, cols, dtype):
    """Few rows, a last batch of rows that is not whole, the last columns, and both widths of block."""
    gen = torch.Generator(DEV).manual_seed(rows + cols)
    dy, x = view(gen, rows, cols, dtype, 5, 3), view(gen, rows, 8, dtype, 0, 0)
    dw, db = torch.empty(cols, 8, dtype=DT[dtype], device=DEV), torch.empty(cols, dtype=DT[dtype], device=DEV)
    smat.smat_linear_wgrad(dy, x, dw, db=db)
    check(db, dy.double().sum(0), dy.double().abs().sum(0), rows, dtype, "db")
    again = torch.empty_like(db)
    smat.smat_linear_wgrad(dy, x, dw, db=again)
    assert torch.equal(db, again)
