"""Slopes and values of the activations over all magnitudes that a checkpoint can hold, against the fp64 oracle: z where the
exponentials overflow, vanish and cross zero.  dy is 1 and r is 1, so what comes out is the activation times u.

Bounds: values within 2^-21 |z| and slopes within 2^-20 (as in test_gpu_linear.py), times u; slopes' larger terms are |z| times
what is left of an exponential, below 1.2 for every z; one rounding of the output, and 1e-37 for what underflows."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from oracle import linear_oracle as lo

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = [smat.SMAT_ACT_GELU, smat.SMAT_ACT_GELU_TANH, smat.SMAT_ACT_SILU]


def f64(t):
    return t.detach().cpu().double().numpy()


def magnitudes():
    """[rows, 64]: each row's block of one magnitude of both signs, from subnormals' neighbours to the largest number."""
    tops = [3.4e38, 3e38, 1e30, 1e20, 1e13, 1e10, 1e6, 1e4, 400.0, 128.0, 105.0, 100.0, 90.0, 88.5, 87.5, 64.0, 32.0, 17.0, 16.0, 12.0,
            9.0, 6.0, 4.0, 2.0, 1.0, 0.25, 1e-3, 1e-10, 1e-30, 1e-37]
    z = torch.tensor(tops, dtype=torch.float64)[:, None] * torch.linspace(1.0, 0.3, 32, dtype=torch.float64)[None]
    return torch.cat([-z, z], dim=1).float().to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_every_magnitude(dtype, act, gated):
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    zs = magnitudes()
    m, n = zs.shape
    c, u = smat.ActCheckpoint.empty(m, n), smat.ActCheckpoint.empty(m, n)
    smat.smat_ckpt_write(zs, c)
    smat.smat_ckpt_write(torch.full((m, n), 0.5, device=DEV), u)
    dy, w = torch.ones(m, 1, dtype=dt, device=DEV), torch.ones(1, n, dtype=dt, device=DEV)
    out, up, hidden = (torch.full((m, n), float("nan"), dtype=dt, device=DEV) for _ in range(3))
    smat.smat_linear_dgrad(dy, w, out, act=act, z_ckpt=c, **(dict(up_ckpt=u, out_up=up) if gated else {}))
    z = lo.ckpt_read(*lo.ckpt_write(f64(zs)), n)
    half = 0.5 if gated else 1.0
    rounding = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    slope = lo.act_grad(z, act) * half
    err = half * 2.0 ** -20
    assert np.all(np.abs(f64(out) - slope) <= err + (np.abs(slope) + err) * rounding)
    # far below zero both are zero, not what is left of a capped exponential times z
    far = z < -200
    assert not f64(out)[far].any()
    if gated:
        value = lo.act(z, act)
        err = 2.0 ** -21 * np.minimum(np.abs(z), 1e37) + 1e-37
        assert np.all(np.abs(f64(up) - value) <= err + (np.abs(value) + err) * rounding)
        assert not f64(up)[far].any()
        # the recomputed hidden activation of the weight gradient is the same function
        smat.smat_ckpt_read(c, hidden, act=act)
        assert np.all(np.abs(f64(hidden) - f64(up)) <= 2 * (err + (np.abs(value) + err) * rounding))
        assert not f64(hidden)[far].any()
