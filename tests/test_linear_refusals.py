"""Argument checks of the linear-layer products and the activation checkpoints: they return before any HIP
call, so no GPU is needed.  Pointers are made-up addresses that nothing dereferences."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2609_33437_amd as smat
from paper_2609_33437_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GIB = 1 << 30


def at(slot, offset=0):
    """Address `slot` GiB away from every other slot."""
    return (slot + 16) * GIB + offset


def linear(**kw):
    a = _lib.smat_linear_args(dtype=_lib.SMAT_BF16, act=0, m=64, n=96, k=128, x=at(0), ldx=128, w=at(1), ldw=128,
                              out=at(2), ldout=96)
    for key, v in kw.items():
        setattr(a, key, v)
    return a


def dgrad(**kw):
    a = _lib.smat_linear_dgrad_args(dtype=_lib.SMAT_BF16, act=0, m=64, n=96, k=128, k2=0, dy=at(0), lddy=128, w=at(1),
                                    ldw=96, out=at(2), ldout=96)
    for key, v in kw.items():
        setattr(a, key, v)
    return a


def wgrad(**kw):
    a = _lib.smat_linear_wgrad_args(dtype=_lib.SMAT_BF16, m=64, n=96, k=128, dy=at(0), lddy=96, x=at(1), ldx=128,
                                    dw=at(2), lddw=128)
    for key, v in kw.items():
        setattr(a, key, v)
    return a


def size_of(fn, args):
    need = ctypes.c_size_t(1 << 62)
    return getattr(_lib.lib(), fn)(ctypes.byref(args), ctypes.byref(need)), need.value


def refused(fn, args, status=smat._lib.SMAT_ERR_INVALID):
    """Both the size call and the call itself refuse the arguments, with a message."""
    st, _ = size_of(fn + "_workspace_bytes", args)
    assert st == status
    st = getattr(_lib.lib(), fn)(ctypes.byref(args), None, 0, None)
    message = _lib.lib().smat_last_error().decode()
    return st == status and message.startswith(fn) and len(message) > len(fn) + 3


LINEAR = [dict(m=-1), dict(n=-1), dict(k=-1), dict(m=1 << 31), dict(x=None), dict(w=None), dict(out=None), dict(ldx=127),
          dict(ldw=127), dict(ldout=95), dict(act=4), dict(act=-1), dict(x=at(0, 1)), dict(w=at(1, 1)), dict(out=at(2, 1)),
          dict(bias=at(3, 1)), dict(mul=at(3), ldmul=95), dict(residual=at(3), ldres=95), dict(z_codes=at(3)),
          dict(z_exps=at(3)), dict(z_codes=at(3, 8), z_exps=at(4)), dict(out=at(0)), dict(out=at(1, 2)),
          dict(out=at(0, 64 * 128 * 2 - 2)), dict(bias=at(2, 4)), dict(mul=at(2, 2), ldmul=96),
          dict(residual=at(2), ldres=97), dict(z_codes=at(2), z_exps=at(4)), dict(z_codes=at(3), z_exps=at(3, 100)),
          dict(z_codes=at(3), z_exps=at(0)), dict(z_codes=at(0), z_exps=at(4)), dict(ldx=1 << 60)]


@pytest.mark.parametrize("kw", LINEAR, ids=str)
def test_linear_refuses(kw):
    assert refused("smat_linear", linear(**kw))


@pytest.mark.parametrize("kw", [dict(out=None, m=0), dict(x=None, w=None, out=None, n=0), dict(x=None, w=None, k=0),
                                dict(mul=at(2), ldmul=96), dict(residual=at(2), ldres=96),
                                dict(ldx=256, out=at(0, 256), ldout=256), dict(x=at(0, 2)), dict(z_codes=at(3), z_exps=at(4, 1))],
                         ids=str)
def test_linear_accepts(kw):
    """Empty dimensions need no pointers; out may be mul or residual; columns of one buffer are apart."""
    st, need = size_of("smat_linear_workspace_bytes", linear(**kw))
    assert st == smat._lib.SMAT_OK and need < 1 << 40


@pytest.mark.parametrize("kw", [dict(m=-1), dict(k2=-1), dict(dy=None), dict(w=None), dict(out=None), dict(lddy=127),
                                dict(ldw=95), dict(k2=5), dict(k2=5, dy2=at(3), lddy2=5), dict(k2=5, dy2=at(3), lddy2=4, w2=at(4), ldw2=96),
                                dict(act=1), dict(act=5), dict(z_codes=at(3)), dict(z_exps=at(3)),
                                dict(up_codes=at(3), up_exps=at(4), out_up=at(5), ldup=96),
                                dict(z_codes=at(3), z_exps=at(4), up_codes=at(5), up_exps=at(6)),
                                dict(z_codes=at(3), z_exps=at(4), out_up=at(5), ldup=96),
                                dict(z_codes=at(3), z_exps=at(4), up_codes=at(5), up_exps=at(6), out_up=at(2, 8), ldup=96),
                                dict(z_codes=at(3), z_exps=at(4), up_codes=at(5), up_exps=at(6), out_up=at(5), ldup=96),
                                dict(z_codes=at(2), z_exps=at(4)), dict(out=at(0)), dict(out=at(1))], ids=str)
def test_dgrad_refuses(kw):
    assert refused("smat_linear_dgrad", dgrad(**kw))


def test_dgrad_accepts_one_checkpoint_for_both():
    st, _ = size_of("smat_linear_dgrad_workspace_bytes", dgrad(z_codes=at(3), z_exps=at(4), up_codes=at(3), up_exps=at(4),
                                                               out_up=at(5), ldup=96))
    assert st == smat._lib.SMAT_OK


@pytest.mark.parametrize("kw", [dict(m=-1), dict(n=-1), dict(k=1 << 31), dict(dy=None), dict(x=None), dict(dw=None),
                                dict(lddy=95), dict(ldx=127), dict(lddw=127), dict(reserved=1), dict(x_codes=at(3)),
                                dict(x_codes=at(3), x_exps=at(4)), dict(x=None, x_codes=at(3)), dict(x=None, x_exps=at(3)),
                                dict(db=at(2)), dict(db=at(0)), dict(db=at(3, 1)), dict(dw=at(0)), dict(dw=at(1)),
                                dict(x=None, x_codes=at(3, 4), x_exps=at(4))], ids=str)
def test_wgrad_refuses(kw):
    assert refused("smat_linear_wgrad", wgrad(**kw))


def test_unknown_dtypes_are_refused():
    for fn, a in (("smat_linear", linear(dtype=2)), ("smat_linear_dgrad", dgrad(dtype=-1)), ("smat_linear_wgrad", wgrad(dtype=7))):
        assert refused(fn, a, smat._lib.SMAT_ERR_DTYPE)
    L = _lib.lib()
    assert L.smat_ckpt_write(at(0), 4, 2, 4, 4, at(1), at(2), None) == smat._lib.SMAT_ERR_DTYPE
    assert L.smat_ckpt_read(at(0), at(1), None, None, 0, 3, 4, 4, at(2), 4, None) == smat._lib.SMAT_ERR_DTYPE


def test_missing_arguments_and_workspaces_are_refused():
    L, invalid = _lib.lib(), smat._lib.SMAT_ERR_INVALID
    for name in ("smat_linear", "smat_linear_dgrad", "smat_linear_wgrad"):
        assert getattr(L, name)(None, None, 0, None) == invalid
        assert getattr(L, name + "_workspace_bytes")(None, ctypes.byref(ctypes.c_size_t())) == invalid
    assert L.smat_linear_workspace_bytes(ctypes.byref(linear()), None) == invalid
    # a sum of 100,000 terms into few outputs is split: it needs memory, all of it, aligned
    a = wgrad(m=100000, n=32, k=32, lddy=32, ldx=32, lddw=32)
    st, need = size_of("smat_linear_wgrad_workspace_bytes", a)
    assert st == smat._lib.SMAT_OK and need > 0
    for ptr, size in ((None, need), (at(9), need - 1), (at(9, 8), need)):
        assert L.smat_linear_wgrad(ctypes.byref(a), ptr, size, None) == invalid
        assert b"workspace" in L.smat_last_error()


@pytest.mark.parametrize("args", [(None, 8, 1, 4, 8, at(1), at(2)), (at(0), 7, 1, 4, 8, at(1), at(2)), (at(0), 8, 1, -1, 8, at(1), at(2)),
                                  (at(0), 8, 1, 4, 8, None, at(2)), (at(0), 8, 1, 4, 8, at(1), None), (at(0), 8, 1, 4, 8, at(1, 8), at(2)),
                                  (at(0), 8, 1, 4, 8, at(0), at(2)), (at(0), 8, 1, 4, 8, at(1), at(1)), (at(0, 1), 8, 1, 4, 8, at(1), at(2))],
                         ids=str)
def test_ckpt_write_refuses(args):
    assert _lib.lib().smat_ckpt_write(*args, None) == smat._lib.SMAT_ERR_INVALID


@pytest.mark.parametrize("args", [(None, at(1), None, None, 0, 1, 4, 8, at(2), 8), (at(0), None, None, None, 0, 1, 4, 8, at(2), 8),
                                  (at(0), at(1), at(3), None, 0, 1, 4, 8, at(2), 8), (at(0), at(1), None, at(3), 0, 1, 4, 8, at(2), 8),
                                  (at(0), at(1), None, None, 4, 1, 4, 8, at(2), 8), (at(0), at(1), None, None, 0, 1, 4, 8, None, 8),
                                  (at(0), at(1), None, None, 0, 1, 4, 8, at(2), 7), (at(0), at(1), None, None, 0, 1, 4, 8, at(0), 8),
                                  (at(0), at(1), None, None, 0, 1, 1 << 32, 8, at(2), 8)], ids=str)
def test_ckpt_read_refuses(args):
    assert _lib.lib().smat_ckpt_read(*args, None) == smat._lib.SMAT_ERR_INVALID


def test_empty_checkpoints_are_no_ops():
    L = _lib.lib()
    assert L.smat_ckpt_write(None, 8, 1, 0, 8, None, None, None) == smat._lib.SMAT_OK
    assert L.smat_ckpt_read(None, None, None, None, 0, 0, 4, 0, None, 0, None) == smat._lib.SMAT_OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, w, out = torch.ones(4, 8), torch.ones(6, 8), torch.ones(4, 6)
    with pytest.raises(smat.SmatError):
        smat.smat_linear(x, w, out)
    with pytest.raises(smat.SmatError):
        smat.smat_ckpt_write(x, None)
    with pytest.raises(smat.SmatError):
        smat.smat_linear_wgrad(x, x, out)
    with pytest.raises(smat.SmatError):
        smat.smat_linear_dgrad(x, x, out)
    with pytest.raises(smat.SmatError):
        smat.ActCheckpoint.empty(4, 8, device="cpu")
    with pytest.raises(smat.SmatError):
        smat.ActCheckpoint(torch.zeros(4, 32), torch.zeros(4, 1), 8)


def test_struct_layouts_match_c(tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("gcc or HIP headers missing")
    structs = {"smat_linear_args": _lib.smat_linear_args, "smat_linear_dgrad_args": _lib.smat_linear_dgrad_args,
               "smat_linear_wgrad_args": _lib.smat_linear_wgrad_args}
    lines = [f'printf("%zu\\n", sizeof({name}));' for name in structs]
    lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for name, s in structs.items() for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "smat.h"\nint main(void) {\n' + "\n".join(lines)
                   + "\nreturn 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run([gcc, "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", str(src),
                    "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [ctypes.sizeof(s) for s in structs.values()]
    want += [getattr(s, f).offset for s in structs.values() for f, _ in s._fields_]
    assert got == want
