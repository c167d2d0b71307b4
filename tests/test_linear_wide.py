"""Operands so wide that a tile's 32-bit offsets would pass 2^31 bytes are not copied to LDS directly, and not packed first
either: packed, their rows are as wide.  The size call tells, since it reports the copies; no GPU is needed."""
import pytest

import paper_2609_33437_amd as smat
from test_linear_refusals import at, dgrad, linear, size_of, wgrad

# call, arguments, elements of the (smaller) wide operand
CASES = [
    ("smat_linear_wgrad", wgrad(m=64, n=1 << 25, k=64, lddy=1 << 25, x=at(40), ldx=64, dw=at(80), lddw=64), 64 << 25),
    ("smat_linear_wgrad", wgrad(m=64, n=(1 << 25) + 3, k=64, lddy=(1 << 25) + 3, x=at(40), ldx=64, dw=at(80), lddw=64), 64 << 25),
    ("smat_linear_wgrad", wgrad(m=64, n=64, k=1 << 24, lddy=64, x=at(40), ldx=1 << 24, dw=at(80), lddw=1 << 24), 64 << 24),
    ("smat_linear", linear(m=2048, n=2048, k=5 << 20, ldx=5 << 20, w=at(200), ldw=5 << 20, out=at(400), ldout=2048), 2048 * (5 << 20)),
    ("smat_linear", linear(m=300, n=264, k=(1 << 22) + 1, ldx=(1 << 22) + 1, w=at(200), ldw=(1 << 22) + 1, out=at(400), ldout=264),
     264 << 22),
    ("smat_linear", linear(dtype=0, m=300, n=264, k=1 << 22, ldx=1 << 22, w=at(200), ldw=1 << 22, out=at(400), ldout=264), 264 << 22),
    ("smat_linear_dgrad", dgrad(m=512, n=17_000_000, k=64, lddy=64, w=at(200), ldw=17_000_000, out=at(400), ldout=17_000_000),
     64 * 17_000_000),
    # as wide as direct copies take: nothing to cure
    ("smat_linear", linear(m=300, n=264, k=(1 << 22) - 8, ldx=(1 << 22) - 8, w=at(200), ldw=(1 << 22) - 8, out=at(400), ldout=264),
     264 << 22),
    ("smat_linear_wgrad", wgrad(m=64, n=(1 << 24) - 8, k=64, lddy=(1 << 24) - 8, x=at(40), ldx=64, dw=at(80), lddw=64), 64 << 24),
]


@pytest.mark.parametrize("fn,args,copied", CASES, ids=lambda v: v if isinstance(v, str) else None)
def test_wide_operands_are_not_packed(fn, args, copied):
    status, need = size_of(fn + "_workspace_bytes", args)
    assert status == smat._lib.SMAT_OK
    assert need < copied // 2       # bytes: a copy takes four times as many or more, partial sums far fewer


def test_narrow_operands_of_wide_strides_are_packed():
    """Where the rows that are read are narrow, a copy cures the stride, and pays where the product is large enough."""
    ld = 1 << 25
    args = dgrad(m=8192, n=4096, k=4096, lddy=4096, w=at(200), ldw=ld, out=at(900), ldout=4096)
    status, need = size_of("smat_linear_dgrad_workspace_bytes", args)
    assert status == smat._lib.SMAT_OK and need >= 4096 * 4096 * 2
