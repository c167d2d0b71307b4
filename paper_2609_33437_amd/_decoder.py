"""ctypes binding of the norms, the token embedding and the output layer with its loss (argument marshalling only;
see include/smat.h for what each call computes).

Matrices, workspaces, streams and devices are as in the linear-layer calls: 2-D GPU tensors with contiguous rows (any row
stride), outputs the caller's, device memory that a call needs from `workspace` or torch's allocator, everything on the
current GPU.  Weights may have another dtype than the matrices.
"""
from __future__ import annotations

from ctypes import byref

from ._lib import (SMAT_ERR_DTYPE, SMAT_ERR_INVALID, SMAT_NORM_LAYER, SMAT_NORM_RMS, SmatError, _check, _torch, dtype_code, lib,
                   smat_embed_args, smat_embed_grad_args, smat_linear_xent_args, smat_linear_xent_grad_args, smat_norm_args,
                   smat_norm_grad_args)
from ._linear import _call, _first, _matrix, _stream_on


def _refuse_vector(t, n: int, device: int, what: str) -> None:
    """Raises for what makes t no contiguous vector [n] on that GPU."""
    if t.shape != (n,):
        raise SmatError(SMAT_ERR_INVALID, f"{what} has shape {tuple(t.shape)}, expected ({n},)")
    if t.get_device() != device:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be on the same GPU as the call's first matrix")
    raise SmatError(SMAT_ERR_INVALID, f"{what} must be contiguous")


def _typed(t, n: int, dtype, device: int, what: str) -> int:
    """Pointer of a contiguous vector [n] of that dtype on that GPU."""
    if t.dtype is not dtype:
        raise SmatError(SMAT_ERR_DTYPE, f"{what} has dtype {t.dtype}, expected {dtype}")
    if t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
        _refuse_vector(t, n, device, what)
    return t.data_ptr()


def _weights(code: int, n: int, device: int, *named):
    """(their dtype code, pointers) of the vectors [n] that are given, which share a dtype; `code` where there are none."""
    dtype, ptrs = None, []
    for t, what in named:
        if t is None:
            ptrs.append(None)
            continue
        if t.shape != (n,) or t.get_device() != device or not t.is_contiguous():
            _refuse_vector(t, n, device, what)
        if t.dtype is not dtype:
            if dtype is not None:
                raise SmatError(SMAT_ERR_DTYPE, f"{what} has dtype {t.dtype}, another one than the weights before it")
            code, dtype = dtype_code(t), t.dtype
        ptrs.append(t.data_ptr())
    return code, ptrs


# ------------------------------------------------------------------ norms
def smat_norm(x, y, weight=None, bias=None, kind: int = SMAT_NORM_LAYER, eps: float = 1e-5, mean=None, rstd=None,
              stream=None) -> None:
    """y = the rows of x normalised, times weight, plus bias; mean and rstd (fp32 [m]) are what smat_norm_grad takes."""
    code = _first(x, "x")
    m, n = x.shape
    a = smat_norm_args(dtype=code, kind=int(kind), eps=float(eps), m=m, n=n)
    a.x, a.ldx = _matrix(x, m, n, x, "x")
    a.y, a.ldy = _matrix(y, m, n, x, "y")
    device, f32 = x.get_device(), _torch().float32
    a.wdtype, (a.weight, a.bias) = _weights(code, n, device, (weight, "weight"), (bias, "bias"))
    if mean is not None:
        a.mean = _typed(mean, m, f32, device, "mean")
    if rstd is not None:
        a.rstd = _typed(rstd, m, f32, device, "rstd")
    _check(lib().smat_norm(byref(a), _stream_on(device, stream)))


def smat_norm_grad(dy, x, rstd, weight=None, mean=None, kind: int = SMAT_NORM_LAYER, dx=None, dw=None, db=None,
                   workspace=None, stream=None) -> None:
    """The gradients that are given of a norm of x, whose smat_norm wrote rstd (and mean, for a layer norm)."""
    code = _first(dy, "dy")
    m, n = dy.shape
    a = smat_norm_grad_args(dtype=code, kind=int(kind), m=m, n=n)
    a.dy, a.lddy = _matrix(dy, m, n, dy, "dy")
    a.x, a.ldx = _matrix(x, m, n, dy, "x")
    device, f32 = dy.get_device(), _torch().float32
    a.rstd = _typed(rstd, m, f32, device, "rstd")
    if kind == SMAT_NORM_LAYER:
        if mean is None:
            raise SmatError(SMAT_ERR_INVALID, "a layer norm's gradients need mean")
        a.mean = _typed(mean, m, f32, device, "mean")
    a.wdtype, (a.weight, a.dweight, a.dbias) = _weights(code, n, device, (weight, "weight"), (dw, "dw"), (db, "db"))
    if dx is not None:
        a.dx, a.lddx = _matrix(dx, m, n, dy, "dx")
    L = lib()
    _call(L.smat_norm_grad, L.smat_norm_grad_workspace_bytes, a, workspace, device, stream)


# ------------------------------------------------------------------ embedding
def smat_embed(table, ids, out, scale: float = 1.0, stream=None) -> None:
    """out[i] = scale * table[ids[i]]; ids are int64 [m], and one outside the table gives a row of NaN."""
    a = smat_embed_args(table_dtype=_first(table, "table"), dtype=_first(out, "out"), scale=float(scale))
    a.rows, a.d = rows, d = table.shape
    a.m = m = out.shape[0]
    a.table, a.ldtable = _matrix(table, rows, d, table, "table")
    device = table.get_device()
    if out.get_device() != device:
        raise SmatError(SMAT_ERR_INVALID, "out must be on the same GPU as the call's first matrix")
    a.out, a.ldout = _matrix(out, m, d, out, "out")
    a.ids = _typed(ids, m, _torch().int64, device, "ids")
    _check(lib().smat_embed(byref(a), _stream_on(device, stream)))


def smat_embed_grad(dy, ids, dtable, scale: float = 1.0, padding_idx=None, accumulate: bool = False, workspace=None,
                    stream=None) -> None:
    """dtable[v] = scale * the sum of the dy[i] with ids[i] = v, added to dtable with `accumulate`; none for padding_idx."""
    a = smat_embed_grad_args(dtype=_first(dy, "dy"), table_dtype=_first(dtable, "dtable"), scale=float(scale),
                             accumulate=1 if accumulate else 0, padding=-1 if padding_idx is None else int(padding_idx))
    a.m, a.d = m, d = dy.shape
    a.rows = rows = dtable.shape[0]
    a.dy, a.lddy = _matrix(dy, m, d, dy, "dy")
    device = dy.get_device()
    if dtable.get_device() != device:
        raise SmatError(SMAT_ERR_INVALID, "dtable must be on the same GPU as the call's first matrix")
    a.dtable, a.ldtable = _matrix(dtable, rows, d, dtable, "dtable")
    a.ids = _typed(ids, m, _torch().int64, device, "ids")
    L = lib()
    _call(L.smat_embed_grad, L.smat_embed_grad_workspace_bytes, a, workspace, device, stream)


# ------------------------------------------------------------------ output layer
def _xent(a, x, w, targets, lse, totals, lse_low):
    torch = _torch()
    m, k = x.shape
    n = w.shape[0] if w.dim() == 2 else -1
    a.m, a.n, a.k = m, n, k
    a.x, a.ldx = _matrix(x, m, k, x, "x")
    a.w, a.ldw = _matrix(w, n, k, x, "w")
    device = x.get_device()
    a.targets = _typed(targets, m, torch.int64, device, "targets")
    a.lse = _typed(lse, m, torch.float32, device, "lse")
    if totals is not None:
        a.totals = _typed(totals, 3, torch.float32, device, "totals")
    if lse_low is not None:
        a.lse_low = _typed(lse_low, m, torch.float32, device, "lse_low")
    return m, n, k, device


def smat_linear_xent(x, w, targets, loss, lse, totals=None, ignore_index: int = -100, workspace=None, stream=None,
                     lse_low=None) -> None:
    """loss[i] = lse[i] - z[i, targets[i]] with z = x w^T and lse[i] = log sum_j exp z[i, j], without storing z whole; totals (fp32
    [3]) = the losses' sum, the number of rows with a target, and their mean.  lse_low (fp32 [m]) = what rounding lse left."""
    a = smat_linear_xent_args(dtype=_first(x, "x"), ignore_index=int(ignore_index))
    m, _, _, device = _xent(a, x, w, targets, lse, totals, lse_low)
    a.loss = _typed(loss, m, _torch().float32, device, "loss")
    L = lib()
    _call(L.smat_linear_xent, L.smat_linear_xent_workspace_bytes, a, workspace, device, stream)


def smat_linear_xent_grad(x, w, targets, lse, dx=None, dw=None, row_scale=None, scale=None, totals=None,
                          ignore_index: int = -100, workspace=None, stream=None, lse_low=None) -> None:
    """The gradients of scale / totals[1] * sum_i row_scale[i] loss[i] (row_scale fp32 [m], scale fp32 [1] on the GPU; without
    them and totals 1), from the lse and lse_low that smat_linear_xent wrote.  Without lse_low rows whose target has nearly the
    whole probability have gradients of lse's rounding."""
    a = smat_linear_xent_grad_args(dtype=_first(x, "x"), ignore_index=int(ignore_index))
    m, n, k, device = _xent(a, x, w, targets, lse, totals, lse_low)
    f32 = _torch().float32
    if row_scale is not None:
        a.row_scale = _typed(row_scale, m, f32, device, "row_scale")
    if scale is not None:
        a.scale = _typed(scale.view(1) if scale.dim() == 0 else scale, 1, f32, device, "scale")
    if dx is not None:
        a.dx, a.lddx = _matrix(dx, m, k, x, "dx")
    if dw is not None:
        a.dw, a.lddw = _matrix(dw, n, k, x, "dw")
    L = lib()
    _call(L.smat_linear_xent_grad, L.smat_linear_xent_grad_workspace_bytes, a, workspace, device, stream)
