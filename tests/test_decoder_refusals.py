"""Argument checks of the norms, the token embedding and the output layer with its loss: they return before any HIP call, so
no GPU is needed.  Pointers are made-up addresses that nothing dereferences."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_33437_amd as smat
from paper_2609_33437_amd import _lib, layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GIB = 1 << 30
BF16, F32 = _lib.SMAT_BF16, _lib.SMAT_F32
INVALID, DTYPE = _lib.SMAT_ERR_INVALID, _lib.SMAT_ERR_DTYPE


def at(slot, offset=0):
    """Address `slot` GiB away from every other slot."""
    return (slot + 16) * GIB + offset


def make(kind, base, kw):
    a = kind(**base)
    for key, v in kw.items():
        setattr(a, key, v)
    return a


NORM = dict(dtype=BF16, wdtype=F32, kind=0, eps=1e-5, m=8, n=96, x=at(0), ldx=96, weight=at(1), bias=at(2), y=at(3), ldy=96,
            mean=at(4), rstd=at(5))
NORM_GRAD = dict(dtype=BF16, wdtype=F32, kind=0, m=300, n=96, dy=at(0), lddy=96, x=at(1), ldx=96, weight=at(2), mean=at(3),
                 rstd=at(4), dx=at(5), lddx=96, dweight=at(6), dbias=at(7))
EMBED = dict(dtype=BF16, table_dtype=F32, scale=1.0, m=8, rows=50, d=96, table=at(0), ldtable=96, ids=at(1), out=at(2), ldout=96)
EMBED_GRAD = dict(dtype=BF16, table_dtype=F32, scale=1.0, m=300, rows=50, d=96, padding=-1, dy=at(0), lddy=96, ids=at(1),
                  dtable=at(2), ldtable=96)
XENT = dict(dtype=BF16, m=8, n=50, k=96, x=at(0), ldx=96, w=at(1), ldw=96, targets=at(2), ignore_index=-100, loss=at(3),
            lse=at(4), totals=at(5))
XENT_GRAD = dict(dtype=BF16, m=8, n=50, k=96, x=at(0), ldx=96, w=at(1), ldw=96, targets=at(2), ignore_index=-100, lse=at(3),
                 row_scale=at(4), scale=at(5), totals=at(6), dx=at(7), lddx=96, dw=at(8), lddw=96)
CALLS = {"smat_norm": (_lib.smat_norm_args, NORM), "smat_norm_grad": (_lib.smat_norm_grad_args, NORM_GRAD),
         "smat_embed": (_lib.smat_embed_args, EMBED), "smat_embed_grad": (_lib.smat_embed_grad_args, EMBED_GRAD),
         "smat_linear_xent": (_lib.smat_linear_xent_args, XENT),
         "smat_linear_xent_grad": (_lib.smat_linear_xent_grad_args, XENT_GRAD)}
SIZED = [f for f in CALLS if f not in ("smat_norm", "smat_embed")]


def size_of(fn, a):
    need = ctypes.c_size_t(1 << 62)
    return getattr(_lib.lib(), fn + "_workspace_bytes")(ctypes.byref(a), ctypes.byref(need)), need.value


def call(fn, a, workspace=None, size=0):
    f = getattr(_lib.lib(), fn)
    return f(ctypes.byref(a), workspace, size, None) if fn in SIZED else f(ctypes.byref(a), None)


def refused(fn, kw, status=INVALID):
    """The size call and the call refuse the arguments, with a message that names the call."""
    a = make(*CALLS[fn], kw)
    if fn in SIZED and size_of(fn, a)[0] != status:
        return False
    st = call(fn, a, at(40), 1 << 40)
    message = _lib.lib().smat_last_error().decode()
    return st == status and message.startswith(fn) and len(message) > len(fn) + 3


BAD = [("smat_norm", kw) for kw in (
    dict(m=-1), dict(n=-1), dict(m=1 << 31), dict(kind=2), dict(kind=-1), dict(eps=-1e-6), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(x=None), dict(y=None), dict(ldx=95), dict(ldy=95), dict(ldx=-96), dict(x=at(0, 1)),
    dict(y=at(3, 1)), dict(weight=at(1, 2)), dict(bias=at(2, 2)), dict(mean=at(4, 2)), dict(rstd=at(5, 1)), dict(y=at(0)),
    dict(y=at(0, 8 * 96 * 2 - 2)), dict(mean=at(0, 4)), dict(rstd=at(4, 4)), dict(y=at(1)), dict(mean=at(2, 380)),
    dict(ldx=1 << 60))]
BAD += [("smat_norm_grad", kw) for kw in (
    dict(m=-1), dict(n=1 << 31), dict(kind=2), dict(reserved=1), dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None),
    dict(lddy=95), dict(ldx=95), dict(lddx=95), dict(dx=at(0)), dict(dx=at(1, 2)), dict(dweight=at(2)), dict(dbias=at(6, 4)),
    dict(dweight=at(6, 2)), dict(dbias=at(3)), dict(dy=at(0, 1)))]
BAD += [("smat_embed", kw) for kw in (
    dict(m=-1), dict(rows=-1), dict(d=-1), dict(rows=1 << 31), dict(scale=float("inf")), dict(scale=float("nan")), dict(reserved=1),
    dict(table=None), dict(ids=None), dict(out=None), dict(ldtable=95), dict(ldout=95), dict(out=at(0)), dict(out=at(1)),
    dict(ids=at(1, 4)), dict(out=at(2, 1)), dict(table=at(0, 2)))]
BAD += [("smat_embed_grad", kw) for kw in (
    dict(m=-1), dict(rows=-1), dict(d=1 << 31), dict(scale=float("inf")), dict(accumulate=2), dict(accumulate=-1), dict(dy=None),
    dict(ids=None), dict(dtable=None), dict(lddy=95), dict(ldtable=95), dict(dtable=at(0)), dict(dtable=at(1, 32)),
    dict(ids=at(1, 2)), dict(dtable=at(2, 2)))]
BAD += [("smat_linear_xent", kw) for kw in (
    dict(m=-1), dict(n=0), dict(n=-1), dict(k=-1), dict(n=1 << 31), dict(reserved=1), dict(x=None), dict(w=None),
    dict(targets=None), dict(loss=None), dict(lse=None), dict(ldx=95), dict(ldw=95), dict(targets=at(2, 4)), dict(loss=at(3, 2)),
    dict(lse=at(3, 28)), dict(loss=at(0)), dict(totals=at(1, 4)), dict(totals=at(5, 1)), dict(lse=at(2)))]
BAD += [("smat_linear_xent_grad", kw) for kw in (
    dict(m=-1), dict(n=0), dict(k=-1), dict(reserved=1), dict(x=None), dict(w=None), dict(targets=None), dict(lse=None),
    dict(ldx=95), dict(ldw=95), dict(lddx=95), dict(lddw=95), dict(dx=at(0)), dict(dw=at(1)), dict(dw=at(7, 96)), dict(dx=at(3)),
    dict(row_scale=at(4, 2)), dict(scale=at(5, 1)), dict(totals=at(6, 2)), dict(dx=at(6)), dict(dw=at(5)))]


@pytest.mark.parametrize("fn,kw", BAD, ids=str)
def test_refuses(fn, kw):
    assert refused(fn, kw)


@pytest.mark.parametrize("fn", CALLS)
def test_refuses_dtypes_and_no_arguments(fn):
    assert refused(fn, dict(dtype=2), DTYPE) and refused(fn, dict(dtype=-1), DTYPE)
    for other in ("wdtype", "table_dtype"):
        if other in CALLS[fn][1]:
            assert refused(fn, {other: 2}, DTYPE)
    f = getattr(_lib.lib(), fn)
    assert (f(None, None, 0, None) if fn in SIZED else f(None, None)) == INVALID
    if fn in SIZED:
        a = make(*CALLS[fn], {})
        assert getattr(_lib.lib(), fn + "_workspace_bytes")(ctypes.byref(a), None) == INVALID


@pytest.mark.parametrize("fn", SIZED)
def test_refuses_workspaces(fn):
    a = make(*CALLS[fn], {})
    st, need = size_of(fn, a)
    assert st == 0 and need > 0 and need % 4 == 0
    assert call(fn, a, None, need) == INVALID and call(fn, a, at(40), need - 1) == INVALID
    assert call(fn, a, at(40, 8), need) == INVALID
    inside = {"smat_norm_grad": at(5), "smat_embed_grad": at(2), "smat_linear_xent": at(1), "smat_linear_xent_grad": at(8)}[fn]
    assert call(fn, a, inside, need) == INVALID
    assert "overlaps" in _lib.lib().smat_last_error().decode()


ACCEPTED = [("smat_norm_grad", dict(dx=None)), ("smat_norm_grad", dict(dweight=None, dbias=None)),
            ("smat_norm_grad", dict(kind=1, mean=None)), ("smat_norm_grad", dict(weight=None, dy=at(0, 2))),
            ("smat_norm_grad", dict(m=0, dy=None, x=None, mean=None, rstd=None, dx=None)),
            ("smat_embed_grad", dict(m=0, dy=None, ids=None)), ("smat_embed_grad", dict(rows=0, dtable=None)),
            ("smat_embed_grad", dict(accumulate=1, lddy=200, ldtable=97, dtable=at(2, 4))),
            ("smat_linear_xent", dict(totals=None)), ("smat_linear_xent", dict(m=0, x=None, targets=None, loss=None, lse=None)),
            ("smat_linear_xent", dict(k=0, x=None, w=None)), ("smat_linear_xent_grad", dict(dx=None)),
            ("smat_linear_xent_grad", dict(dw=None, row_scale=None, scale=None, totals=None)),
            ("smat_linear_xent_grad", dict(dx=at(0, 192), lddx=192, ldx=192))]


@pytest.mark.parametrize("fn,kw", ACCEPTED, ids=str)
def test_accepts(fn, kw):
    """What the size call takes; columns of one buffer are apart, and empty dimensions need no pointers."""
    st, need = size_of(fn, make(*CALLS[fn], kw))
    assert st == 0 and need < 1 << 40


@pytest.mark.parametrize("fn,kw", [("smat_norm", dict(m=0, x=None, y=None, mean=None, rstd=None)),
                                   ("smat_norm", dict(n=0, x=None, y=None, weight=None, bias=None)),
                                   ("smat_embed", dict(m=0, ids=None, out=None)), ("smat_embed", dict(d=0, table=None, out=None)),
                                   ("smat_norm_grad", dict(n=0, dweight=None, dbias=None)),
                                   ("smat_embed_grad", dict(rows=0, dtable=None))], ids=str)
def test_nothing_to_do(fn, kw):
    assert call(fn, make(*CALLS[fn], kw), at(40), 1 << 40) == 0


def test_workspaces_do_not_grow_with_the_vocabulary():
    """The logits are not kept: a gradient's workspace is a piece of the vocabulary and the fp32 sums of dx."""
    sizes = []
    for n in (32768, 131072, 524288):
        st, need = size_of("smat_linear_xent_grad", make(*CALLS["smat_linear_xent_grad"], dict(
            m=4096, n=n, k=2048, ldx=2048, ldw=2048, lddx=2048, lddw=2048, w=at(64), dw=at(96))))
        assert st == 0
        sizes.append(need)
    assert max(sizes) < 4096 * 32768 * 2 + 3 * 4096 * 2048 * 4 and max(sizes) - min(sizes) < 0.1 * max(sizes)


def test_struct_layout_matches_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("gcc or HIP headers missing")
    names = ["smat_norm_args", "smat_norm_grad_args", "smat_embed_args", "smat_embed_grad_args", "smat_linear_xent_args",
             "smat_linear_xent_grad_args"]
    lines = []
    for name in names:
        for field, _ in getattr(_lib, name)._fields_:
            lines.append(f'  printf("%zu ", offsetof({name}, {field}));')
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "smat.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([gcc, "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src),
                    "-o", str(exe)], check=True, capture_output=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines()
    for name, line in zip(names, out):
        s = getattr(_lib, name)
        assert [int(v) for v in line.split()] == [getattr(s, f).offset for f, _ in s._fields_] + [ctypes.sizeof(s)], name


def test_binding_refuses_host_tensors():
    x, w, t, v = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for fn in (lambda: smat.smat_norm(x, x.clone()), lambda: smat.smat_norm_grad(x, x, v),
               lambda: smat.smat_embed(w, t, x), lambda: smat.smat_embed_grad(x, t, w),
               lambda: smat.smat_linear_xent(x, w, t, v, v.clone()), lambda: smat.smat_linear_xent_grad(x, w, t, v),
               lambda: layers.layer_norm(x), lambda: layers.rms_norm(x), lambda: layers.embedding(t, w),
               lambda: layers.linear_cross_entropy(x, w, t)):
        with pytest.raises(smat.SmatError):
            fn()
