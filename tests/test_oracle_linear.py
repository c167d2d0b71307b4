"""The fp64 oracle of the linear layers and the activation checkpoints: derivatives against differences,
checkpoint properties, and the gradients of a small gated MLP against differences of its loss."""
import numpy as np
import pytest

from oracle import linear_oracle as lo

ACTS = [lo.NONE, lo.GELU, lo.GELU_TANH, lo.SILU]


@pytest.mark.parametrize("kind", ACTS)
def test_activation_derivatives(kind):
    z = np.linspace(-9.0, 9.0, 1801)
    h = 1e-5
    diff = (lo.act(z + h, kind) - lo.act(z - h, kind)) / (2 * h)
    # central differences: third derivatives below 2 give h^2/3, rounding 2^-53 * 9 / h
    assert np.max(np.abs(diff - lo.act_grad(z, kind))) < 2 * h * h + 1e-9


def test_activation_values():
    assert lo.act(np.array([1.0]), lo.GELU)[0] == pytest.approx(0.8413447460685429, abs=1e-15)
    assert lo.act(np.array([1.0]), lo.SILU)[0] == pytest.approx(0.7310585786300049, abs=1e-15)
    assert lo.act(np.array([1.0]), lo.GELU_TANH)[0] == pytest.approx(0.8411919906082768, abs=1e-12)


@pytest.mark.parametrize("cols", [1, 31, 32, 33, 200])
def test_checkpoint_error_bound(cols):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((50, cols)) * np.exp(rng.uniform(-20, 20, (50, 1)))
    codes, exps = lo.ckpt_write(x)
    step = np.ldexp(1.0, exps.astype(int) - 127).repeat(32, axis=1)[:, :cols]
    err = np.abs(lo.ckpt_read(codes, exps, cols) - x)
    held = np.abs(x) > 127.5 * step
    assert np.all(err[~held] <= step[~held] / 2)
    assert np.all(err[held] < step[held])
    assert codes.shape == (50, -(-cols // 32) * 32) and not codes[:, cols:].any()
    top = np.abs(x).max(axis=1)
    assert np.all(exps.max(axis=1) == np.floor(np.log2(top)) - 6 + 127)


def test_checkpoint_is_idempotent_and_exact_on_its_own_values():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((20, 96))
    codes, exps = lo.ckpt_write(x)
    again = lo.ckpt_write(lo.ckpt_read(codes, exps, 96))
    # a block whose largest value was held to 127 may shrink its exponent only if that value fell below 64 steps: never
    assert np.array_equal(codes, again[0]) and np.array_equal(exps, again[1])


def test_checkpoint_of_zeros_subnormals_and_nonfinite():
    x = np.zeros((4, 64))
    x[1, 3] = 2.0 ** -140
    x[2, 40] = np.nan
    x[3, 0] = -np.inf
    codes, exps = lo.ckpt_write(x)
    assert exps.tolist() == [[1, 1], [1, 1], [1, 255], [255, 1]]
    back = lo.ckpt_read(codes, exps, 64)
    assert not back[0].any() and not back[1].any()
    assert np.isnan(back[2, 32:]).all() and not back[2, :32].any()
    assert np.isnan(back[3, :32]).all() and not back[3, 32:].any()


@pytest.mark.parametrize("kind", [lo.GELU, lo.GELU_TANH, lo.SILU])
@pytest.mark.parametrize("gated", [False, True])
def test_gradients_against_differences(kind, gated):
    """L = sum(c * mlp(x)) with mlp = (act(x wg^T + b) * (x wu^T)) wd^T: dgrad and wgrad against differences."""
    rng = np.random.default_rng(3)
    m, d, f = 3, 5, 4
    p = dict(x=rng.standard_normal((m, d)), wg=rng.standard_normal((f, d)), b=rng.standard_normal(f),
             wu=rng.standard_normal((f, d)), wd=rng.standard_normal((d, f)))
    c = rng.standard_normal((m, d))

    def parts(p):
        u = p["x"] @ p["wu"].T if gated else np.ones((m, f))
        h, z = lo.linear(p["x"], p["wg"], p["b"], kind, mul=u)
        return u, h, z

    def loss(p):
        return float((c * lo.linear(parts(p)[1], p["wd"])[0]).sum())

    u, h, z = parts(p)
    dz, du = lo.dgrad(c, p["wd"], kind, z=z, up=u)
    assert np.allclose(lo.dgrad(c, p["wd"], kind, z=z)[0] * u, dz)
    got = dict(wd=lo.wgrad(c, h)[0], wg=lo.wgrad(dz, p["x"])[0], b=lo.wgrad(dz, p["x"])[1])
    if gated:
        got["wu"] = lo.wgrad(du, p["x"])[0]
        got["x"] = lo.dgrad(dz, p["wg"], dy2=du, w2=p["wu"])[0]
    else:
        got["x"] = lo.dgrad(dz, p["wg"])[0]
    step = 1e-5
    for name, g in got.items():
        num = np.zeros_like(g)
        for i in np.ndindex(g.shape):
            lo_, hi = {k: v.copy() for k, v in p.items()}, {k: v.copy() for k, v in p.items()}
            hi[name][i] += step
            lo_[name][i] -= step
            num[i] = (loss(hi) - loss(lo_)) / (2 * step)
        # |L'''| stays below 1e4 here: h^2/6 * 1e4 = 2e-7, plus rounding of L (about 1e2 * 2^-53 / h = 1e-9)
        assert np.max(np.abs(num - g)) < 1e-6, name
