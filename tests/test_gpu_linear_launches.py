"""Calls whose launches would have 2^32 threads or more in a row of blocks: every output is written, the last ones too.
Products of -1, 0 and 1 over 8 terms are exact in bf16."""
import pytest
import torch

import paper_2609_33437_amd as smat

pytestmark = pytest.mark.gpu
DEV = "cuda"
PIECE = 1 << 22


def ternary(gen, rows, cols):
    return torch.randint(-1, 2, (rows, cols), generator=gen, device=DEV, dtype=torch.int8).bfloat16()


def exact(got, want_of):
    """got [rows, n] equals want_of(columns) piece by piece."""
    for at in range(0, got.shape[1], PIECE):
        assert torch.equal(got[:, at:at + PIECE], want_of(slice(at, at + PIECE))), at


def test_checkpoint_of_more_than_2_to_the_35_values():
    rows, cols = (1 << 20) + 100, 32768
    gen = torch.Generator(DEV).manual_seed(1)
    piece = torch.randn(4096, cols, generator=gen, device=DEV).bfloat16()
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)      # 69 GB, and half of it for the checkpoint
    for at in range(0, rows, 4096):
        x[at:at + 4096] = piece[:min(4096, rows - at)]
    c = smat.ActCheckpoint.empty(rows, cols)
    c.exps.fill_(7)
    smat.smat_ckpt_write(x, c)
    one = smat.ActCheckpoint.empty(4096, cols)
    smat.smat_ckpt_write(piece, one)
    back = torch.empty_like(piece)
    smat.smat_ckpt_read(one, back)
    x.fill_(float("nan"))
    smat.smat_ckpt_read(c, x)
    for at in range(0, rows, 4096):
        n = min(4096, rows - at)
        assert torch.equal(c.codes[at:at + n], one.codes[:n]) and torch.equal(c.exps[at:at + n], one.exps[:n]), at
        assert torch.equal(x[at:at + n], back[:n]), at


@pytest.mark.parametrize("m", [1, 4])
def test_few_rows_of_a_layer(m):
    n, k = (1 << 28) + 40, 8
    gen = torch.Generator(DEV).manual_seed(2)
    x, w = ternary(gen, m, k), ternary(gen, n, k)
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=DEV)
    smat.smat_linear(x, w, out)
    exact(out, lambda s: (x.float() @ w[s].float().t()).bfloat16())


@pytest.mark.parametrize("n", [(1 << 29) + 40, (1 << 29) + 43])
def test_small_tiles_of_a_data_gradient(n):
    """On and off 16-byte rows."""
    m, k = 9, 8
    gen = torch.Generator(DEV).manual_seed(3)
    dy, w = ternary(gen, m, k), ternary(gen, k, n)
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device=DEV)
    smat.smat_linear_dgrad(dy, w, out)
    exact(out, lambda s: (dy.float() @ w[:, s].float()).bfloat16())


def test_column_sums_and_their_weight_gradient():
    m, n, k = 8, (1 << 28) + 72, 1
    gen = torch.Generator(DEV).manual_seed(4)
    dy, x = ternary(gen, m, n), ternary(gen, m, k)
    dw, db = torch.full((n, k), float("nan"), dtype=torch.bfloat16, device=DEV), torch.empty(n, dtype=torch.bfloat16, device=DEV)
    smat.smat_linear_wgrad(dy, x, dw, db=db)
    exact(db.view(1, n), lambda s: dy[:, s].float().sum(0, keepdim=True).bfloat16())
    exact(dw.view(1, n), lambda s: (x.float().t() @ dy[:, s].float()).bfloat16())
