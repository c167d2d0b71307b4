"""Plain fp64 definition of the linear-layer products and the 8-bit activation checkpoints.

Everything is computed in float64 from float64 arrays, without the library's code: products as sums,
activations and their derivatives from their formulas, checkpoints by frexp and rint.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
NONE, GELU, GELU_TANH, SILU = 0, 1, 2, 3

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _logistic(t):
    e = np.exp(-np.abs(t))
    return np.where(t >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def act(z, kind):
    """act(z)."""
    if kind == GELU:
        return 0.5 * z * _erfc(-z / math.sqrt(2.0))
    if kind == GELU_TANH:
        return z * _logistic(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3))
    if kind == SILU:
        return z * _logistic(z)
    return z


def act_grad(z, kind):
    """act'(z)."""
    if kind == GELU:
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    if kind == GELU_TANH:
        a = math.sqrt(2.0 / math.pi)
        g = _logistic(2.0 * a * (z + 0.044715 * z ** 3))
        return g + z * g * (1.0 - g) * 2.0 * a * (1.0 + 3.0 * 0.044715 * z * z)
    if kind == SILU:
        g = _logistic(z)
        return g + z * g * (1.0 - g)
    return np.ones_like(z)


def _blocked(x):
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = np.zeros((rows, blocks * BLOCK))
    v[:, :cols] = x
    return v.reshape(rows, blocks, BLOCK)


def ckpt_exponent(top):
    """E of blocks whose largest magnitude is `top`: max(floor(log2 top) - 6, -126)."""
    top = np.asarray(top, dtype=np.float64)
    finite = np.where(np.isfinite(top) & (top > 0), top, 1.0)
    e = np.frexp(finite)[1] - 7
    return np.where(top > 0, np.maximum(e, -126), -126)


def ckpt_write(x):
    """(codes int8 [rows, 32 blocks], exps uint8 [rows, blocks]) of x [rows, cols]."""
    v = _blocked(np.asarray(x, dtype=np.float64))
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v)
    e = ckpt_exponent(np.abs(v).max(axis=2) if v.size else np.zeros(v.shape[:2]))
    q = np.clip(np.rint(np.ldexp(v, -e[:, :, None])), -127, 127)
    exps = np.where(bad, 255, e + 127)
    return q.astype(np.int8).reshape(v.shape[0], -1), exps.astype(np.uint8)


def ckpt_read(codes, exps, cols):
    """The float64 values [rows, cols] of a checkpoint."""
    rows, blocks = exps.shape
    e = exps.astype(np.int64)
    v = np.ldexp(codes.astype(np.float64).reshape(rows, blocks, BLOCK), (e - 127)[:, :, None])
    v = np.where((e == 255)[:, :, None], np.nan, v)
    return v.reshape(rows, blocks * BLOCK)[:, :cols]


def linear(x, w, bias=None, kind=NONE, mul=None, residual=None):
    """(out, z): z = x w^T + bias, out = act(z) * mul + residual."""
    z = x @ w.T
    if bias is not None:
        z = z + bias
    out = act(z, kind)
    if mul is not None:
        out = out * mul
    if residual is not None:
        out = out + residual
    return out, z


def dgrad(dy, w, kind=NONE, z=None, up=None, dy2=None, w2=None):
    """(out, out_up): v = dy w + dy2 w2 through act'(z) (and up)."""
    v = dy @ w
    if dy2 is not None:
        v = v + dy2 @ w2
    if z is None:
        return v, None
    if up is None:
        return v * act_grad(z, kind), None
    return v * up * act_grad(z, kind), v * act(z, kind)


def wgrad(dy, x):
    """(dw, db)."""
    return dy.T @ x, dy.sum(axis=0)
