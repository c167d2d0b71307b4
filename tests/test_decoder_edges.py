"""Further argument checks of the output layer's calls, and sizes of their workspaces: no GPU is needed (see
test_decoder_refusals.py)."""
import pytest

from test_decoder_refusals import BF16, CALLS, F32, at, make, refused, size_of


@pytest.mark.parametrize("fn,kw", [("smat_linear_xent", kw) for kw in (
    dict(lse_low=at(9, 2)), dict(lse_low=at(4)), dict(lse_low=at(3, 28)), dict(lse_low=at(5, 8)), dict(lse_low=at(0)),
    dict(lse_low=at(2, 4)))] + [("smat_linear_xent_grad", kw) for kw in (
        dict(lse_low=at(9, 1)), dict(lse_low=at(7)), dict(lse_low=at(8, 8)))], ids=str)
def test_refuses_the_low_part(fn, kw):
    """Alignment and overlaps of lse_low, an output of the losses and an input of the gradients."""
    assert refused(fn, kw)


@pytest.mark.parametrize("fn", ["smat_linear_xent", "smat_linear_xent_grad"])
def test_accepts_the_low_part(fn):
    status, need = size_of(fn, make(*CALLS[fn], dict(lse_low=at(9, 4))))
    assert status == 0 and need == size_of(fn, make(*CALLS[fn], {}))[1]
    assert size_of(fn, make(*CALLS[fn], dict(m=0, x=None, targets=None, loss=None, lse=None, lse_low=None)
                            if fn == "smat_linear_xent" else dict(lse_low=None)))[0] == 0


@pytest.mark.parametrize("n,k", [(40, 16), (50304, 1024), (151936, 4096), (1 << 20, 8192)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("wanted", ["dx", "dw", "both"])
def test_an_empty_batch_needs_no_workspace(n, k, dtype, wanted):
    """No row is looked for, so no number of them is read from memory that nothing wrote, however large the products are."""
    outputs = dict(dx=at(2000) if wanted != "dw" else None, lddx=k, dw=at(4000) if wanted != "dx" else None, lddw=k)
    status, need = size_of("smat_linear_xent_grad", make(*CALLS["smat_linear_xent_grad"], dict(
        dtype=dtype, m=0, n=n, k=k, x=None, ldx=k, w=at(200), ldw=k, targets=None, lse=None, row_scale=None, **outputs)))
    assert status == 0 and need == 0
