"""Linear layers and MLP blocks whose saved activations are held in 8 bits, as differentiable torch functions.

The forward passes run as products with their bias, activation, gate and residual in the epilogue
(smat_linear).  What a training step must keep for the backward pass is saved as checkpoints of 8.25 bits
a value (ActCheckpoint): a layer's input, and the pre-activations, written by the product's own
epilogue.  The hidden activation of an MLP is not saved at all; the backward recomputes it from the
pre-activations (smat_ckpt_read), takes the data gradient through the activation in the product's
epilogue (smat_linear_dgrad) and takes the weight gradient from the input's checkpoint, which the call reads
back into its workspace (smat_linear_wgrad; once for each weight, the gate's and the up projection's).  A token's MLP of width d and ffn f keeps d + f (act) or d + 2 f (gated) values of about a
byte, against d + 2 f or d + 3 f of two bytes.

Gradients are those of the checkpointed values: they differ from exact ones by what 8 bits lose of the
saved activations (about one per cent of a weight gradient's norm), never in the forward pass.  They have no
derivatives of their own, and there are none in forward mode: asking for either raises.  Without gradients (a merged
model answering) nothing is saved, and a few tokens take the product's form for few rows.

Tensors are fp32 or bf16 on the GPU; under torch.autocast floating inputs are cast to its dtype first, as
torch's own linear layers do, except a residual: one of another dtype is added to the result in torch's
promoted dtype.  Otherwise a call's tensors share one dtype.  A residual has the output's
shape, or is the output's matrix of rows.  Row strides are kept where the last dimension
is contiguous; other layouts, those of weights and biases too, are copied in every call.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from ._lib import SMAT_ERR_INVALID, SmatError
from ._linear import (SMAT_ACT_NONE, SMAT_ACT_SILU, ActCheckpoint, smat_ckpt_read, smat_ckpt_write, smat_linear,
                      smat_linear_dgrad, smat_linear_wgrad)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """x [.., k] as a matrix of contiguous rows."""
    if x.dim() == 2 and x.is_contiguous():
        return x
    if x.dim() == 0:
        raise SmatError(SMAT_ERR_INVALID, "the layers take tensors with a last dimension")
    m = x if x.dim() == 2 else x.reshape(x.shape[:-1].numel(), x.shape[-1])
    if m.shape[1] > 1 and m.stride(1) != 1 or m.shape[0] > 1 and m.stride(0) < m.shape[1]:
        m = m.contiguous()
    return m


def _weight(w: torch.Tensor) -> torch.Tensor:
    if w.dim() != 2:
        raise SmatError(SMAT_ERR_INVALID, f"a weight is a matrix, got shape {tuple(w.shape)}")
    return _rows(w)


def _bias(b: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    return None if b is None else b.contiguous()


def _cast(*tensors):
    """The tensors as autocast would hand them to a linear layer (the casts are differentiable)."""
    first = next(t for t in tensors if t is not None)
    if not first.is_cuda:
        raise SmatError(SMAT_ERR_INVALID, "the layers run on GPU tensors")
    if not torch.is_autocast_enabled("cuda"):
        return tensors
    dtype = torch.get_autocast_dtype("cuda")
    return tuple(t if t is None or t.dtype == dtype else t.to(dtype) for t in tensors)


def _residual(residual: Optional[torch.Tensor], x: torch.Tensor, shape):
    """(the residual as the product's epilogue adds it, or as torch adds it to the product's result).  Under autocast one of
    another dtype, an fp32 residual stream beside bf16 products, is not cast: torch adds it in its own dtype, as it does
    to the result of its own layers."""
    if residual is None:
        return None, None
    if residual.shape != shape and residual.shape != (x.shape[0], shape[-1]):
        raise SmatError(SMAT_ERR_INVALID, f"residual has shape {tuple(residual.shape)}, the output {tuple(shape)}")
    if residual.dtype != x.dtype and torch.is_autocast_enabled("cuda"):
        return None, residual.reshape(shape)
    return _rows(residual), None


def _sum(y: torch.Tensor, after: Optional[torch.Tensor]) -> torch.Tensor:
    return y if after is None else after + y


def _elsewhere(x: torch.Tensor) -> bool:
    """Whether x's GPU is not the current one, which a model split over GPUs does not set.  The public functions enter it
    then; autograd does for the backward."""
    return x.is_cuda and x.get_device() != torch._C._cuda_getDevice()


def _saves(*tensors) -> bool:
    """Whether autograd records the call.  Where it does not, tangents, which torch carries through frozen
    weights and no_grad too, are refused (the recorded functions raise on them themselves)."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return True
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(      # -1: no tangents are about
            t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise SmatError(SMAT_ERR_INVALID, "the layers have no forward-mode derivatives")
    return False


def _checkpoint(x: torch.Tensor) -> ActCheckpoint:
    c = ActCheckpoint.empty(x.shape[0], x.shape[1], x.device)
    smat_ckpt_write(x, c)
    return c


def _keep(ctx, *checkpoints) -> None:
    """Saves checkpoints' tensors, so that they live and die as autograd's saved tensors do."""
    ctx.cols = [c.cols for c in checkpoints]
    ctx.tensors = [t for c in checkpoints for t in (c.codes, c.exps)]


def _kept(ctx, saved):
    return [ActCheckpoint(saved[2 * i], saved[2 * i + 1], cols) for i, cols in enumerate(ctx.cols)]


def _wgrad(dy, x, weight, bias_wanted: bool):
    """(dw, db) of a layer whose weight gradient is wanted."""
    dw = torch.empty(weight.shape, dtype=weight.dtype, device=weight.device)
    db = torch.empty(weight.shape[0], dtype=weight.dtype, device=weight.device) if bias_wanted else None
    smat_linear_wgrad(dy, x, dw, db=db)
    return dw, db


def _column_sums(dy):
    """The bias gradient where the weight's is not wanted."""
    empty = dict(dtype=dy.dtype, device=dy.device)
    db = torch.empty(dy.shape[1], **empty)
    smat_linear_wgrad(dy, torch.empty(dy.shape[0], 0, **empty), torch.empty(dy.shape[1], 0, **empty), db=db)
    return db


class _Linear(torch.autograd.Function):
    """x w^T + b + r on matrices."""

    @staticmethod
    def forward(ctx, x, w, b, r):
        out = torch.empty(x.shape[0], w.shape[0], dtype=x.dtype, device=x.device)
        smat_linear(x, w, out, bias=b, residual=r)
        _keep(ctx, *([_checkpoint(x)] if ctx.needs_input_grad[1] else []))
        ctx.save_for_backward(w, *ctx.tensors)
        del ctx.tensors
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        w, *saved = ctx.saved_tensors
        need_x, need_w, need_b, need_r = ctx.needs_input_grad
        dy = _rows(dy)
        dx = dw = db = None
        if need_x:
            dx = torch.empty(dy.shape[0], w.shape[1], dtype=dy.dtype, device=dy.device)
            smat_linear_dgrad(dy, w, dx)
        if need_w:
            dw, db = _wgrad(dy, _kept(ctx, saved)[0], w, need_b)
        elif need_b:
            db = _column_sums(dy)
        return dx, dw, db, dy if need_r else None


class _Mlp(torch.autograd.Function):
    """act(x w1^T + b1) w2^T + b2 + r on matrices."""

    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, r, act):
        m = x.shape[0]
        z = ActCheckpoint.empty(m, w1.shape[0], x.device)
        h = torch.empty(m, w1.shape[0], dtype=x.dtype, device=x.device)
        smat_linear(x, w1, h, bias=b1, act=act, z_ckpt=z)
        out = torch.empty(m, w2.shape[0], dtype=x.dtype, device=x.device)
        smat_linear(h, w2, out, bias=b2, residual=r)
        _keep(ctx, z, *([_checkpoint(x)] if ctx.needs_input_grad[1] else []))
        ctx.act = act
        ctx.save_for_backward(w1, w2, *ctx.tensors)
        del ctx.tensors
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        w1, w2, *saved = ctx.saved_tensors
        kept = _kept(ctx, saved)
        z = kept[0]
        need_x, need_w1, need_b1, need_w2, need_b2, need_r, _ = ctx.needs_input_grad
        dy = _rows(dy)
        m = dy.shape[0]
        dx = dw1 = db1 = dw2 = db2 = None
        if need_w2:
            h = torch.empty(m, w2.shape[1], dtype=dy.dtype, device=dy.device)
            smat_ckpt_read(z, h, act=ctx.act)
            dw2, db2 = _wgrad(dy, h, w2, need_b2)
            del h
        elif need_b2:
            db2 = _column_sums(dy)
        if need_x or need_w1 or need_b1:
            dz = torch.empty(m, w1.shape[0], dtype=dy.dtype, device=dy.device)
            smat_linear_dgrad(dy, w2, dz, act=ctx.act, z_ckpt=z)
            if need_w1:
                dw1, db1 = _wgrad(dz, kept[1], w1, need_b1)
            elif need_b1:
                db1 = _column_sums(dz)
            if need_x:
                dx = torch.empty(m, w1.shape[1], dtype=dy.dtype, device=dy.device)
                smat_linear_dgrad(dz, w1, dx)
        return dx, dw1, db1, dw2, db2, dy if need_r else None, None


class _GatedMlp(torch.autograd.Function):
    """(act(x wg^T) (.) (x wu^T)) wd^T + r on matrices."""

    @staticmethod
    def forward(ctx, x, wg, wu, wd, r, act):
        m, f = x.shape[0], wg.shape[0]
        g, u = ActCheckpoint.empty(m, f, x.device), ActCheckpoint.empty(m, f, x.device)
        h = torch.empty(m, f, dtype=x.dtype, device=x.device)
        smat_linear(x, wu, h, z_ckpt=u)
        smat_linear(x, wg, h, act=act, mul=h, z_ckpt=g)     # in place over the up projection
        out = torch.empty(m, wd.shape[0], dtype=x.dtype, device=x.device)
        smat_linear(h, wd, out, residual=r)
        _keep(ctx, g, u, *([_checkpoint(x)] if ctx.needs_input_grad[1] or ctx.needs_input_grad[2] else []))
        ctx.act = act
        ctx.save_for_backward(wg, wu, wd, *ctx.tensors)
        del ctx.tensors
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        wg, wu, wd, *saved = ctx.saved_tensors
        kept = _kept(ctx, saved)
        g, u = kept[:2]
        need_x, need_g, need_u, need_d, need_r, _ = ctx.needs_input_grad
        dy = _rows(dy)
        m, f = dy.shape[0], wg.shape[0]
        dx = dwg = dwu = dwd = None
        if need_d:
            h = torch.empty(m, f, dtype=dy.dtype, device=dy.device)
            smat_ckpt_read(g, h, act=ctx.act, up=u)
            dwd, _ = _wgrad(dy, h, wd, False)
            del h
        if need_x or need_g or need_u:
            dg, du = torch.empty(m, f, dtype=dy.dtype, device=dy.device), torch.empty(m, f, dtype=dy.dtype, device=dy.device)
            smat_linear_dgrad(dy, wd, dg, act=ctx.act, z_ckpt=g, up_ckpt=u, out_up=du)
            if need_g:
                dwg, _ = _wgrad(dg, kept[2], wg, False)
            if need_u:
                dwu, _ = _wgrad(du, kept[2], wu, False)
            if need_x:
                dx = torch.empty(m, wg.shape[1], dtype=dy.dtype, device=dy.device)
                smat_linear_dgrad(dg, wg, dx, dy2=du, w2=wu)
        return dx, dwg, dwu, dwd, dy if need_r else None, None


# ------------------------------------------------------------------ public functions
def linear(x, weight, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x weight^T + bias + residual for x [.., k]; the weight gradient reads x from an 8-bit checkpoint."""
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return linear(x, weight, bias, residual)
    x, weight, bias = _cast(x, weight, bias)
    weight, bias = _weight(weight), _bias(bias)
    shape, x = x.shape[:-1] + weight.shape[:1], _rows(x)
    r, after = _residual(residual, x, shape)
    if _saves(x, weight, bias, r):
        return _sum(_Linear.apply(x, weight, bias, r).view(shape), after)
    out = torch.empty(x.shape[0], weight.shape[0], dtype=x.dtype, device=x.device)
    smat_linear(x, weight, out, bias=bias, residual=r)
    return _sum(out.view(shape), after)


def mlp(x, w1, b1, w2, b2, act: int, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(x w1^T + b1) w2^T + b2 + residual for x [.., d] (biases and residual may be None)."""
    if act == SMAT_ACT_NONE:
        raise SmatError(SMAT_ERR_INVALID, "an MLP needs an activation")
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return mlp(x, w1, b1, w2, b2, act, residual)
    x, w1, b1, w2, b2 = _cast(x, w1, b1, w2, b2)
    w1, b1, w2, b2 = _weight(w1), _bias(b1), _weight(w2), _bias(b2)
    shape, x = x.shape[:-1] + w2.shape[:1], _rows(x)
    r, after = _residual(residual, x, shape)
    if _saves(x, w1, b1, w2, b2, r):
        return _sum(_Mlp.apply(x, w1, b1, w2, b2, r, int(act)).view(shape), after)
    h = torch.empty(x.shape[0], w1.shape[0], dtype=x.dtype, device=x.device)
    smat_linear(x, w1, h, bias=b1, act=act)
    out = torch.empty(x.shape[0], w2.shape[0], dtype=x.dtype, device=x.device)
    smat_linear(h, w2, out, bias=b2, residual=r)
    return _sum(out.view(shape), after)


def gated_mlp(x, w_gate, w_up, w_down, act: int = SMAT_ACT_SILU,
              residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """(act(x w_gate^T) (.) (x w_up^T)) w_down^T + residual for x [.., d] (SwiGLU with the default act)."""
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return gated_mlp(x, w_gate, w_up, w_down, act, residual)
    x, w_gate, w_up, w_down = _cast(x, w_gate, w_up, w_down)
    w_gate, w_up, w_down = _weight(w_gate), _weight(w_up), _weight(w_down)
    shape, x = x.shape[:-1] + w_down.shape[:1], _rows(x)
    r, after = _residual(residual, x, shape)
    if _saves(x, w_gate, w_up, w_down, r):
        return _sum(_GatedMlp.apply(x, w_gate, w_up, w_down, r, int(act)).view(shape), after)
    h = torch.empty(x.shape[0], w_gate.shape[0], dtype=x.dtype, device=x.device)
    smat_linear(x, w_up, h)
    smat_linear(x, w_gate, h, act=act, mul=h)
    out = torch.empty(x.shape[0], w_down.shape[0], dtype=x.dtype, device=x.device)
    smat_linear(h, w_down, out, residual=r)
    return _sum(out.view(shape), after)
