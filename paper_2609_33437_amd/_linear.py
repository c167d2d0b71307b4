"""ctypes binding of the linear-layer products and the 8-bit activation checkpoints (argument
marshalling only; see include/smat.h for what each call computes).

Matrices are 2-D GPU tensors with contiguous rows (any row stride); outputs are the caller's.  A call that
needs device memory for partial sums takes it from `workspace` (a contiguous uint8 GPU tensor) or,
without one, from torch's allocator on the call's stream.  Tensors, stream and the current device are of one
GPU; a call refuses others.
"""
from __future__ import annotations

import ctypes
from ctypes import byref, c_size_t
from typing import Optional

from . import _lib
from ._lib import (SMAT_ACT_GELU, SMAT_ACT_GELU_TANH, SMAT_ACT_NONE, SMAT_ACT_SILU, SMAT_ERR_DTYPE, SMAT_ERR_INVALID,
                   SmatError, _check, _torch, dtype_code, lib, smat_linear_args, smat_linear_dgrad_args,
                   smat_linear_wgrad_args)

CKPT_BLOCK = 32     # elements along a row that share a power of two


class ActCheckpoint:
    """A matrix [rows, cols] held in 8 bits: int8 codes [rows, 32 * blocks] and one uint8 exponent per
    block of 32, [rows, blocks] (the format is in include/smat.h).  8.25 bits a value, against 16 or 32."""

    __slots__ = ("codes", "exps", "rows", "cols")

    def __init__(self, codes, exps, cols: int):
        torch = _torch()
        blocks = -(-int(cols) // CKPT_BLOCK)
        if codes.dtype != torch.int8 or exps.dtype != torch.uint8:
            raise SmatError(SMAT_ERR_DTYPE, "a checkpoint has int8 codes and uint8 exps")
        if codes.dim() != 2 or tuple(exps.shape) != (codes.shape[0], blocks) or codes.shape[1] != blocks * CKPT_BLOCK:
            raise SmatError(SMAT_ERR_INVALID, f"a checkpoint of {cols} columns has codes [rows, {blocks * CKPT_BLOCK}] "
                                              f"and exps [rows, {blocks}]")
        if not (codes.is_cuda and exps.is_cuda and codes.is_contiguous() and exps.is_contiguous()
                and codes.get_device() == exps.get_device()):
            raise SmatError(SMAT_ERR_INVALID, "codes and exps must be contiguous tensors on one GPU")
        self.codes, self.exps, self.rows, self.cols = codes, exps, codes.shape[0], int(cols)

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda") -> "ActCheckpoint":
        """An unwritten checkpoint in new GPU memory."""
        torch = _torch()
        blocks = -(-int(cols) // CKPT_BLOCK)
        return cls(torch.empty(rows, blocks * CKPT_BLOCK, dtype=torch.int8, device=device),
                   torch.empty(rows, blocks, dtype=torch.uint8, device=device), cols)

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()


# ------------------------------------------------------------------ marshalling helpers
def _matrix(t, rows: int, cols: int, like, what: str):
    """(pointer, row stride) of a matrix [rows, cols] of like's dtype on like's GPU."""
    if t.shape != (rows, cols):
        raise SmatError(SMAT_ERR_INVALID, f"{what} has shape {tuple(t.shape)}, expected ({rows}, {cols})")
    if t.dtype is not like.dtype:
        raise SmatError(SMAT_ERR_DTYPE, f"{what} has dtype {t.dtype}, expected {like.dtype}")
    if t.get_device() != like.get_device():     # -1 on the host; like is a GPU tensor
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be on the same GPU as the call's first matrix")
    ld, step = t.stride()
    if step != 1 or ld < cols:
        if cols > 1 and rows > 0 and step != 1:
            raise SmatError(SMAT_ERR_INVALID, f"{what} must have contiguous rows")
        if rows <= 1 or cols == 0:
            ld = cols           # the stride of a single row (or of empty rows) addresses nothing
        elif ld < cols:
            raise SmatError(SMAT_ERR_INVALID, f"rows of {what} overlap (row stride {ld}, {cols} columns)")
    return t.data_ptr(), ld


def _first(t, what: str):
    """dtype code of the matrix that the other arguments are checked against."""
    if t.dim() != 2:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be a matrix")
    if not t.is_cuda:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be a GPU tensor")
    return dtype_code(t)


def _vector(t, n: int, like, what: str) -> int:
    if t.shape != (n,):
        raise SmatError(SMAT_ERR_INVALID, f"{what} has shape {tuple(t.shape)}, expected ({n},)")
    if t.dtype is not like.dtype:
        raise SmatError(SMAT_ERR_DTYPE, f"{what} has dtype {t.dtype}, expected {like.dtype}")
    if t.get_device() != like.get_device():
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be on the same GPU as the call's first matrix")
    if n > 1 and t.stride(0) != 1:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be contiguous")
    return t.data_ptr()


def _ckpt(c, rows: int, cols: int, device: int, what: str):
    if not isinstance(c, ActCheckpoint):
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be an ActCheckpoint")
    if c.rows != rows or c.cols != cols:
        raise SmatError(SMAT_ERR_INVALID, f"{what} holds [{c.rows}, {c.cols}], expected [{rows}, {cols}]")
    if c.codes.get_device() != device:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be on the same GPU as the call's first matrix")
    return c.codes.data_ptr(), c.exps.data_ptr()


def _stream_on(device: int, stream) -> int:
    """Handle of the given stream, or of the current one, where work on that GPU's tensors can be launched."""
    C = _torch()._C
    current = C._cuda_getDevice()
    if current != device:
        raise SmatError(SMAT_ERR_INVALID, f"the tensors are on GPU {device} and the current device is {current}: "
                                          "call under torch.cuda.device(tensor.device)")
    if stream is None:
        return C._cuda_getCurrentRawStream(device)
    if getattr(stream, "device_index", device) != device:
        raise SmatError(SMAT_ERR_INVALID, f"the stream is of GPU {stream.device_index}, the tensors are on GPU {device}")
    return stream.cuda_stream


def _call(fn, size_fn, args, workspace, device: int, stream) -> None:
    need = c_size_t()
    _check(size_fn(byref(args), byref(need)))
    ptr, have, handle = None, 0, _stream_on(device, stream)
    if need.value:
        if workspace is None:
            torch = _torch()
            if stream is None:
                workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
            else:       # memory that torch hands out for work on that stream
                with torch.cuda.stream(stream):
                    workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
        elif not (workspace.is_cuda and workspace.is_contiguous() and workspace.get_device() == device):
            raise SmatError(SMAT_ERR_INVALID, "workspace must be a contiguous tensor on the same GPU")
        ptr, have = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(fn(byref(args), ptr, have, handle))


# ------------------------------------------------------------------ checkpoints
def smat_ckpt_write(x, ckpt: ActCheckpoint, stream=None) -> None:
    """ckpt <- x, a matrix of fp32 or bf16 (see include/smat.h)."""
    code = _first(x, "x")
    rows, cols = x.shape
    px, ldx = _matrix(x, rows, cols, x, "x")
    device = x.get_device()
    codes, exps = _ckpt(ckpt, rows, cols, device, "ckpt")
    _check(lib().smat_ckpt_write(px, ldx, code, rows, cols, codes, exps, _stream_on(device, stream)))


def smat_ckpt_read(ckpt: ActCheckpoint, out, act: int = SMAT_ACT_NONE, up: Optional[ActCheckpoint] = None,
                   stream=None) -> None:
    """out = act(values of ckpt), times the values of `up` where given (see include/smat.h)."""
    code = _first(out, "out")
    rows, cols = out.shape
    pout, ldout = _matrix(out, rows, cols, out, "out")
    device = out.get_device()
    codes, exps = _ckpt(ckpt, rows, cols, device, "ckpt")
    up_codes, up_exps = _ckpt(up, rows, cols, device, "up") if up is not None else (None, None)
    _check(lib().smat_ckpt_read(codes, exps, up_codes, up_exps, int(act), code, rows, cols, pout, ldout,
                                _stream_on(device, stream)))


# ------------------------------------------------------------------ products
def smat_linear(x, w, out, bias=None, act: int = SMAT_ACT_NONE, mul=None, residual=None,
                z_ckpt: Optional[ActCheckpoint] = None, workspace=None, stream=None) -> None:
    """out = act(x w^T + bias) (.) mul + residual; z_ckpt receives the checkpoint of x w^T + bias."""
    code = _first(x, "x")
    m, k = x.shape
    n = w.shape[0] if w.dim() == 2 else -1
    a = smat_linear_args(dtype=code, act=int(act), m=m, n=n, k=k)
    a.x, a.ldx = _matrix(x, m, k, x, "x")
    a.w, a.ldw = _matrix(w, n, k, x, "w")
    a.out, a.ldout = _matrix(out, m, n, x, "out")
    if bias is not None:
        a.bias = _vector(bias, n, x, "bias")
    if mul is not None:
        a.mul, a.ldmul = _matrix(mul, m, n, x, "mul")
    if residual is not None:
        a.residual, a.ldres = _matrix(residual, m, n, x, "residual")
    device = x.get_device()
    if z_ckpt is not None:
        a.z_codes, a.z_exps = _ckpt(z_ckpt, m, n, device, "z_ckpt")
    L = lib()
    _call(L.smat_linear, L.smat_linear_workspace_bytes, a, workspace, device, stream)


def smat_linear_dgrad(dy, w, out, act: int = SMAT_ACT_NONE, z_ckpt: Optional[ActCheckpoint] = None,
                      up_ckpt: Optional[ActCheckpoint] = None, out_up=None, dy2=None, w2=None, workspace=None,
                      stream=None) -> None:
    """v = dy w (+ dy2 w2).  out = v; with z_ckpt v (.) act'(z); with z_ckpt and up_ckpt v (.) u (.) act'(z),
    and out_up = v (.) act(z).  w is the layer's weight [k, n]: dy's columns by its input's."""
    code = _first(dy, "dy")
    m, k = dy.shape
    n = out.shape[1] if out.dim() == 2 else -1
    a = smat_linear_dgrad_args(dtype=code, act=int(act), m=m, n=n, k=k)
    a.dy, a.lddy = _matrix(dy, m, k, dy, "dy")
    a.w, a.ldw = _matrix(w, k, n, dy, "w")
    a.out, a.ldout = _matrix(out, m, n, dy, "out")
    if (dy2 is None) != (w2 is None) or (up_ckpt is None) != (out_up is None):
        raise SmatError(SMAT_ERR_INVALID, "dy2 goes with w2, and up_ckpt with out_up")
    if dy2 is not None:
        if dy2.dim() != 2:
            raise SmatError(SMAT_ERR_INVALID, "dy2 must be a matrix")
        a.k2 = k2 = dy2.shape[1]
        a.dy2, a.lddy2 = _matrix(dy2, m, k2, dy, "dy2")
        a.w2, a.ldw2 = _matrix(w2, k2, n, dy, "w2")
    device = dy.get_device()
    if z_ckpt is not None:
        a.z_codes, a.z_exps = _ckpt(z_ckpt, m, n, device, "z_ckpt")
    if up_ckpt is not None:
        a.up_codes, a.up_exps = _ckpt(up_ckpt, m, n, device, "up_ckpt")
        a.out_up, a.ldup = _matrix(out_up, m, n, dy, "out_up")
    L = lib()
    _call(L.smat_linear_dgrad, L.smat_linear_dgrad_workspace_bytes, a, workspace, device, stream)


def smat_linear_wgrad(dy, x, dw, db=None, workspace=None, stream=None) -> None:
    """dw = dy^T x, with x a matrix or an ActCheckpoint; db = the column sums of dy."""
    code = _first(dy, "dy")
    m, n = dy.shape
    device = dy.get_device()
    ckpt = isinstance(x, ActCheckpoint)
    k = x.cols if ckpt else (x.shape[1] if x.dim() == 2 else -1)
    a = smat_linear_wgrad_args(dtype=code, m=m, n=n, k=k)
    a.dy, a.lddy = _matrix(dy, m, n, dy, "dy")
    if ckpt:
        a.x_codes, a.x_exps = _ckpt(x, m, k, device, "x")
    else:
        a.x, a.ldx = _matrix(x, m, k, dy, "x")
    a.dw, a.lddw = _matrix(dw, n, k, dy, "dw")
    if db is not None:
        a.db = _vector(db, n, dy, "db")
    L = lib()
    _call(L.smat_linear_wgrad, L.smat_linear_wgrad_workspace_bytes, a, workspace, device, stream)
