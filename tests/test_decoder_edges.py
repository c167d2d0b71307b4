"""Further argument checks of the output layer's calls, and sizes of their workspaces: no GPU is needed (see
test_decoder_refusals.py)."""
import pytest

from test_decoder_refusals import CALLS, at, make, refused, size_of


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
