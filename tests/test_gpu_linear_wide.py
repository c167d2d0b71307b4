"""Products with operands on both sides of the widest rows that are copied to LDS directly (2^22 elements along r, 2^24 across
it).  Operands are -1, 0 or 1, so every sum, in any order, is exact in fp32 and the result is its one rounding."""
import pytest
import torch

import paper_2609_33437_amd as smat

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
PIECE = 1 << 20


def ternary(gen, rows, cols, dtype):
    return torch.randint(-1, 2, (rows, cols), generator=gen, device=DEV, dtype=torch.int8).to(DT[dtype])


@pytest.mark.parametrize("dtype,k", [("bf16", (1 << 22) - 8), ("bf16", 4_300_800), ("bf16", (1 << 22) + 1), ("f32", (1 << 22) - 4),
                                     ("f32", 1 << 22)])
def test_long_rows(dtype, k):
    """r along the rows: both operands of a layer, the first of a data gradient."""
    gen = torch.Generator(DEV).manual_seed(k)
    m, n = 300, 264
    x, w = ternary(gen, m, k, dtype), ternary(gen, n, k, dtype)
    out = torch.full((m, n), float("nan"), dtype=DT[dtype], device=DEV)
    smat.smat_linear(x, w, out)
    want = torch.zeros(m, n, dtype=torch.float64, device=DEV)
    for at in range(0, k, PIECE):
        want += x[:, at:at + PIECE].double() @ w[:, at:at + PIECE].double().t()
    assert torch.equal(out, want.to(DT[dtype]))
    del w
    w = ternary(gen, k, 40, dtype)
    out = torch.full((m, 40), float("nan"), dtype=DT[dtype], device=DEV)
    smat.smat_linear_dgrad(x, w, out)
    want = torch.zeros(m, 40, dtype=torch.float64, device=DEV)
    for at in range(0, k, PIECE):
        want += x[:, at:at + PIECE].double() @ w[at:at + PIECE].double()
    assert torch.equal(out, want.to(DT[dtype]))


def test_long_rows_of_the_largest_tile():
    """2048 x 2048 takes 256 x 256 tiles: their last rows' offsets are the largest that direct copies have."""
    gen = torch.Generator(DEV).manual_seed(1)
    k, size = (1 << 22) - 8, 2048
    x, w = ternary(gen, size, k, "bf16"), ternary(gen, size, k, "bf16")
    out = torch.full((size, size), float("nan"), dtype=torch.bfloat16, device=DEV)
    smat.smat_linear(x, w, out)
    want = torch.zeros(size, size, dtype=torch.float64, device=DEV)
    for at in range(0, k, PIECE):
        want += x[:, at:at + PIECE].double() @ w[:, at:at + PIECE].double().t()
    assert torch.equal(out, want.bfloat16())


@pytest.mark.parametrize("dtype,n", [("bf16", (1 << 24) - 8), ("bf16", 17_000_000), ("bf16", 1 << 25), ("bf16", (1 << 24) + 3),
                                     ("f32", (1 << 24) - 4), ("f32", 1 << 24)])
def test_rows_across(dtype, n):
    """r across the rows: the weight of a data gradient, both operands of a weight gradient."""
    gen = torch.Generator(DEV).manual_seed(n)
    m, k = 64, 64
    wide = ternary(gen, m, n, dtype)
    dy = ternary(gen, 512, m, dtype)
    out = torch.full((512, n), float("nan"), dtype=DT[dtype], device=DEV)
    smat.smat_linear_dgrad(dy, wide, out)
    for at in range(0, n, PIECE):
        assert torch.equal(out[:, at:at + PIECE].float(), dy.float() @ wide[:, at:at + PIECE].float()), at
    del out
    x = ternary(gen, m, k, dtype)
    dw, db = torch.full((n, k), float("nan"), dtype=DT[dtype], device=DEV), torch.empty(n, dtype=DT[dtype], device=DEV)
    smat.smat_linear_wgrad(wide, x, dw, db=db)
    for at in range(0, n, PIECE):
        assert torch.equal(dw[at:at + PIECE].float(), wide[:, at:at + PIECE].float().t() @ x.float()), at
    assert torch.equal(db.float(), wide.sum(0, dtype=torch.float32))
    del dw
    dw = torch.full((k, n), float("nan"), dtype=DT[dtype], device=DEV)
    smat.smat_linear_wgrad(x, wide, dw)
    for at in range(0, n, PIECE):
        assert torch.equal(dw[:, at:at + PIECE].float(), x.float().t() @ wide[:, at:at + PIECE].float()), at
