"""Row strides whose byte counts pass 64 bits, and negative ones, are refused: a product of the stride and the element size
that wraps must not look like a small stride.  No GPU is needed."""
import pytest

import paper_2609_33437_amd as smat
from paper_2609_33437_amd import _lib
from test_linear_refusals import at, dgrad, linear, refused, wgrad

# strides that come out as a multiple of the matrix's bytes modulo 2^64, or below zero
STRIDES = [(0, (1 << 62) + 128), (0, (1 << 61) + 128), (1, (1 << 62) + 128), (1, -(1 << 63) + 128), (0, -(1 << 62) + 128), (0, -1),
           (1, -128), (0, (1 << 63) - 1), (1, (1 << 63) - 1), (1, (1 << 60) + 1)]


@pytest.mark.parametrize("dtype,ld", STRIDES)
@pytest.mark.parametrize("name", ["ldx", "ldw", "ldout", "ldmul", "ldres"])
def test_linear(dtype, ld, name):
    sides = dict(mul=at(3), ldmul=128, residual=at(4), ldres=128, ldx=128, ldw=128, ldout=128, dtype=dtype, n=128)
    assert refused("smat_linear", linear(**{**sides, name: ld}))


@pytest.mark.parametrize("dtype,ld", STRIDES)
@pytest.mark.parametrize("name", ["lddy", "ldw", "lddy2", "ldw2", "ldout", "ldup"])
def test_dgrad(dtype, ld, name):
    args = dict(dtype=dtype, n=128, k=128, k2=128, lddy=128, ldw=128, dy2=at(3), lddy2=128, w2=at(4), ldw2=128, ldout=128,
                z_codes=at(5), z_exps=at(6), up_codes=at(7), up_exps=at(8), out_up=at(9), ldup=128)
    assert refused("smat_linear_dgrad", dgrad(**{**args, name: ld}))


@pytest.mark.parametrize("dtype,ld", STRIDES)
@pytest.mark.parametrize("name", ["lddy", "ldx", "lddw"])
def test_wgrad(dtype, ld, name):
    assert refused("smat_linear_wgrad", wgrad(**{**dict(dtype=dtype, n=128, lddy=128, ldx=128, lddw=128), name: ld}))


@pytest.mark.parametrize("dtype,ld", STRIDES)
def test_checkpoints(dtype, ld):
    L = _lib.lib()
    assert L.smat_ckpt_write(at(0), ld, dtype, 4, 128, at(1), at(2), None) == smat._lib.SMAT_ERR_INVALID
    assert L.smat_ckpt_read(at(1), at(2), None, None, 0, dtype, 4, 128, at(0), ld, None) == smat._lib.SMAT_ERR_INVALID
