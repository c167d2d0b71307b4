"""Plain fp64 definition of the norms, the token embedding and the output layer with its cross entropy.

Everything is computed in float64 NumPy from float64 arrays, without the library's code, from the formulas.
"""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------- norms
def norm_stats(x, eps, layer):
    """(mean, rstd) of the rows of x; mean is 0 for an RMS norm."""
    mean = x.mean(axis=1) if layer else np.zeros(x.shape[0])
    d = x - mean[:, None]
    return mean, 1.0 / np.sqrt((d * d).mean(axis=1) + eps)


def norm(x, w, b, eps, layer):
    mean, rstd = norm_stats(x, eps, layer)
    return (x - mean[:, None]) * rstd[:, None] * w + b


def norm_grad(dy, x, w, mean, rstd, layer):
    """(dx, dw, db) for given statistics."""
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = g - xh * (g * xh).mean(axis=1)[:, None]
    if layer:
        dx = dx - g.mean(axis=1)[:, None]
    return dx * rstd[:, None], (dy * xh).sum(axis=0), dy.sum(axis=0)


# ---------------------------------------------------------------- embedding
def embed(table, ids, scale):
    out = np.full((len(ids), table.shape[1]), np.nan)
    ok = (ids >= 0) & (ids < table.shape[0])
    out[ok] = scale * table[ids[ok]]
    return out


def embed_grad(dy, ids, rows, scale, padding=None):
    out = np.zeros((rows, dy.shape[1]))
    ok = (ids >= 0) & (ids < rows)
    if padding is not None:
        ok &= ids != padding
    np.add.at(out, ids[ok], dy[ok])
    return scale * out


# ---------------------------------------------------------------- output layer
def logits_lse(z):
    top = z.max(axis=1)
    return np.log(np.exp(z - top[:, None]).sum(axis=1)) + top


def xent(z, targets, ignore):
    """(loss, lse) of logits z."""
    lse = logits_lse(z)
    loss = np.full(z.shape[0], np.nan)
    ok = (targets >= 0) & (targets < z.shape[1]) & (targets != ignore)
    loss[ok] = lse[ok] - z[np.nonzero(ok)[0], targets[ok]]
    loss[targets == ignore] = 0.0
    return loss, lse


def xent_dz(z, targets, ignore, lse, row_scale):
    """Gradient of sum_i row_scale[i] loss[i] at z, for given lse."""
    p = np.exp(z - lse[:, None])
    for i, t in enumerate(targets):
        if t == ignore:
            p[i] = 0.0
        elif 0 <= t < z.shape[1]:
            p[i, t] -= 1.0
        else:
            p[i] = np.nan
    keep = targets != ignore
    p[keep] *= row_scale[keep][:, None]
    return p
