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
model answering) nothing is saved, and a few tokens take the product's form for few rows.  torch.jit.trace keeps a call as
one node; make_fx and torch.export, which would lose it, are refused.

What stands between a decoder's linear layers is here too: the token embedding, layer and RMS norms, and the output layer
with its cross entropy, whose logits are not kept (smat_embed, smat_norm, smat_linear_xent).  Norms compute in fp32
and return their input's dtype, whatever autocast says, and their weights may be fp32 beside bf16 activations; an
embedding under autocast returns its dtype.  The loss is fp32.

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

from ._decoder import smat_embed, smat_embed_grad, smat_linear_xent, smat_linear_xent_grad, smat_norm, smat_norm_grad
from ._lib import SMAT_ERR_INVALID, SMAT_NORM_LAYER, SMAT_NORM_RMS, SmatError
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


_modes, _included = torch._C._len_torch_dispatch_stack, torch._C._dispatch_tls_is_dispatch_key_included
_pre_dispatch, _jit_trace = torch._C.DispatchKey.PreDispatch, torch._C._get_tracing_state


def _refuse_graph_tracers() -> None:
    """Raises while make_fx or torch.export records the operators that torch dispatches: it would see an output's allocation and
    not the call that writes it, inside an autograd function too."""
    if _modes() or _included(_pre_dispatch):
        from torch.fx.experimental.proxy_tensor import get_proxy_mode

        if get_proxy_mode() is not None:
            raise SmatError(SMAT_ERR_INVALID, "the layers cannot be recorded by make_fx or torch.export")


def _derivative(backward):
    """A backward pass that has no derivatives of its own and is not recorded by graph tracers."""

    @once_differentiable
    def checked(ctx, *grads):
        _refuse_graph_tracers()
        return backward(ctx, *grads)

    return checked


def _saves(*tensors) -> bool:
    """Whether the call goes through its autograd function: autograd records it, or torch.jit.trace does, which keeps the
    function as one node.  Where it does not, tangents, which torch carries through frozen weights and no_grad too, are
    refused (the recorded functions raise on them themselves)."""
    _refuse_graph_tracers()
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return True
    if _jit_trace() is not None:
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
    @_derivative
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
    @_derivative
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
    @_derivative
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


class _Norm(torch.autograd.Function):
    """Rows of a matrix normalised."""

    @staticmethod
    def forward(ctx, x, w, b, kind, eps):
        m = x.shape[0]
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(m, dtype=torch.float32, device=x.device)
        mean = torch.empty_like(rstd) if kind == SMAT_NORM_LAYER else None
        smat_norm(x, y, weight=w, bias=b, kind=kind, eps=eps, mean=mean, rstd=rstd)
        ctx.kind = kind
        ctx.bias = None if b is None else b.dtype
        ctx.save_for_backward(x, w, mean, rstd)
        return y

    @staticmethod
    @_derivative
    def backward(ctx, dy):
        x, w, mean, rstd = ctx.saved_tensors
        need_x, need_w, need_b, _, _ = ctx.needs_input_grad
        dy = _rows(dy)
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
        dw = torch.empty(x.shape[1], dtype=w.dtype, device=x.device) if need_w else None
        db = torch.empty(x.shape[1], dtype=ctx.bias, device=x.device) if need_b else None
        if need_x or need_w or need_b:
            smat_norm_grad(dy, x, rstd, weight=w, mean=mean, kind=ctx.kind, dx=dx, dw=dw, db=db)
        return dx, dw, db, None, None


class _Embedding(torch.autograd.Function):
    """Rows of a table by a vector of ids."""

    @staticmethod
    def forward(ctx, table, ids, scale, padding_idx, dtype):
        out = torch.empty(ids.shape[0], table.shape[1], dtype=dtype, device=table.device)
        smat_embed(table, ids, out, scale=scale)
        ctx.scale, ctx.padding_idx, ctx.shape, ctx.dtype = scale, padding_idx, table.shape, table.dtype
        ctx.save_for_backward(ids)
        return out

    @staticmethod
    @_derivative
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        dtable = torch.empty(ctx.shape, dtype=ctx.dtype, device=dy.device)
        smat_embed_grad(_rows(dy), ids, dtable, scale=ctx.scale, padding_idx=ctx.padding_idx)
        return dtable, None, None, None, None


class _LinearXent(torch.autograd.Function):
    """Per-row losses, or their sum (1) or mean (2), of x w^T against targets."""

    @staticmethod
    def forward(ctx, x, w, targets, ignore_index, reduction):
        loss, lse, totals = _losses(x, w, targets, ignore_index, reduction, True)
        ctx.ignore_index, ctx.reduction = ignore_index, reduction
        ctx.save_for_backward(x, w, targets, lse, totals)
        return loss if reduction == 0 else totals[2 * reduction - 2].clone()

    @staticmethod
    @_derivative
    def backward(ctx, grad):
        x, w, targets, lse, totals = ctx.saved_tensors
        need_x, need_w = ctx.needs_input_grad[:2]
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
        dw = torch.empty(w.shape, dtype=w.dtype, device=w.device) if need_w else None
        grad = grad.contiguous()
        rows = ctx.reduction == 0
        smat_linear_xent_grad(x, w, targets, lse[0], dx=dx, dw=dw, row_scale=grad if rows else None, scale=None if rows else grad,
                              totals=totals if ctx.reduction == 2 else None, ignore_index=ctx.ignore_index, lse_low=lse[1])
        return dx, dw, None, None, None


def _losses(x, w, targets, ignore_index: int, reduction: int, saved: bool):
    """(loss of each row, lse and for gradients what its rounding left, totals or None)."""
    empty = dict(dtype=torch.float32, device=x.device)
    loss, lse = torch.empty(x.shape[0], **empty), torch.empty(2 if saved else 1, x.shape[0], **empty)
    totals = torch.empty(3, **empty) if reduction else None
    smat_linear_xent(x, w, targets, loss, lse[0], totals=totals, ignore_index=ignore_index, lse_low=lse[1] if saved else None)
    return loss, lse, totals


def _ids(ids: torch.Tensor, like: torch.Tensor, what: str) -> torch.Tensor:
    if ids.dtype != torch.int64:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be int64, got {ids.dtype}")
    if ids.device != like.device:
        raise SmatError(SMAT_ERR_INVALID, f"{what} must be on the GPU of the other tensors")
    return ids.reshape(-1).contiguous()      # a column of a batch stays strided


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


def _norm(x, weight, bias, kind: int, eps: float) -> torch.Tensor:
    if not x.is_cuda:
        raise SmatError(SMAT_ERR_INVALID, "the layers run on GPU tensors")
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return _norm(x, weight, bias, kind, eps)
    for t, what in ((weight, "weight"), (bias, "bias")):
        if t is not None and (t.dim() != 1 or t.shape[0] != x.shape[-1:].numel()):
            raise SmatError(SMAT_ERR_INVALID, f"{what} has shape {tuple(t.shape)}, the rows of x {tuple(x.shape[-1:])}")
    shape, x = x.shape, _rows(x)
    weight, bias = _bias(weight), _bias(bias)
    if _saves(x, weight, bias):
        return _Norm.apply(x, weight, bias, kind, float(eps)).view(shape)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    smat_norm(x, y, weight=weight, bias=bias, kind=kind, eps=eps)
    return y.view(shape)


def layer_norm(x, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
               eps: float = 1e-5) -> torch.Tensor:
    """(x - mean) / sqrt(var + eps) weight + bias over the last dimension of x."""
    return _norm(x, weight, bias, SMAT_NORM_LAYER, eps)


def rms_norm(x, weight: Optional[torch.Tensor] = None, eps: float = 1e-6) -> torch.Tensor:
    """x / sqrt(mean x^2 + eps) weight over the last dimension of x."""
    return _norm(x, weight, None, SMAT_NORM_RMS, eps)


def embedding(ids, weight, scale: float = 1.0, padding_idx: Optional[int] = None) -> torch.Tensor:
    """scale * weight[ids] for int64 ids of any shape; the row of padding_idx has no gradient.  An id outside the table gives a
    row of NaN.  Under autocast the result has its dtype."""
    if not weight.is_cuda:
        raise SmatError(SMAT_ERR_INVALID, "the layers run on GPU tensors")
    if _elsewhere(weight):
        with torch.cuda.device(weight.get_device()):
            return embedding(ids, weight, scale, padding_idx)
    if padding_idx is not None and not 0 <= padding_idx < weight.shape[0]:
        raise SmatError(SMAT_ERR_INVALID, f"padding_idx {padding_idx} is outside the table")
    dtype = torch.get_autocast_dtype("cuda") if torch.is_autocast_enabled("cuda") else weight.dtype
    weight = _weight(weight)
    saved, shape, flat = _saves(weight), ids.shape, _ids(ids, weight, "ids")
    if saved:
        out = _Embedding.apply(weight, flat, float(scale), padding_idx, dtype)
    else:
        out = torch.empty(flat.shape[0], weight.shape[1], dtype=dtype, device=weight.device)
        smat_embed(weight, flat, out, scale=scale)
    return out.view(shape + weight.shape[1:])


def linear_cross_entropy(x, weight, targets, ignore_index: int = -100, reduction: str = "mean") -> torch.Tensor:
    """The cross entropy of the logits x weight^T for x [.., k] against int64 targets [..], in fp32, without keeping the logits.
    Rows whose target is ignore_index have no loss and no gradient; another target outside the vocabulary gives NaN.
    reduction: "mean" over the rows with a target (NaN where there is none, with gradients of 0), "sum", or "none" for each
    row's loss in targets' shape."""
    if reduction not in ("none", "sum", "mean"):
        raise SmatError(SMAT_ERR_INVALID, f"unknown reduction {reduction!r}")
    if _elsewhere(x):
        with torch.cuda.device(x.get_device()):
            return linear_cross_entropy(x, weight, targets, ignore_index, reduction)
    x, weight = _cast(x, weight)
    if x.shape[:-1] != targets.shape:
        raise SmatError(SMAT_ERR_INVALID, f"targets have shape {tuple(targets.shape)}, the rows of x {tuple(x.shape[:-1])}")
    x, weight, how = _rows(x), _weight(weight), ("none", "sum", "mean").index(reduction)
    saved, flat = _saves(x, weight), _ids(targets, x, "targets")
    if saved:
        loss = _LinearXent.apply(x, weight, flat, int(ignore_index), how)
    else:
        loss, _, totals = _losses(x, weight, flat, int(ignore_index), how, False)
        if how:
            loss = totals[2 * how - 2]
    return loss.view(targets.shape) if how == 0 else loss
