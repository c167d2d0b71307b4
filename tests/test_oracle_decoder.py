"""The fp64 definitions of norms, embedding and output layer against torch's own operators in double precision."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import decoder_oracle as do


def double(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("m,n", [(1, 1), (3, 7), (17, 64)])
def test_norm(layer, m, n):
    x, w, b, dy = double(m, n, seed=1).requires_grad_(), double(n, seed=2).requires_grad_(), double(n, seed=3).requires_grad_(), double(m, n, seed=4)
    if layer:
        y = F.layer_norm(x, (n,), w, b, 1e-3)
    else:
        y = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + 1e-3) * w + b
    y.backward(dy)
    xn, wn, bn = x.detach().numpy(), w.detach().numpy(), b.detach().numpy()
    np.testing.assert_allclose(do.norm(xn, wn, bn, 1e-3, layer), y.detach().numpy(), rtol=1e-11, atol=1e-11)
    mean, rstd = do.norm_stats(xn, 1e-3, layer)
    for got, want in zip(do.norm_grad(dy.numpy(), xn, wn, mean, rstd, layer), (x.grad, w.grad, b.grad)):
        np.testing.assert_allclose(got, want.numpy(), rtol=1e-9, atol=1e-9)


def test_embedding():
    table, dy = double(11, 5, seed=1).requires_grad_(), double(9, 5, seed=2)
    ids = torch.tensor([3, 3, 0, 10, 3, 7, 0, 1, 10])
    y = F.embedding(ids, table, padding_idx=7) * 1.5
    y.backward(dy)
    np.testing.assert_array_equal(do.embed(table.detach().numpy(), ids.numpy(), 1.5), y.detach().numpy())
    np.testing.assert_allclose(do.embed_grad(dy.numpy(), ids.numpy(), 11, 1.5, padding=7), table.grad.numpy(), rtol=1e-13)
    assert np.isnan(do.embed(np.ones((2, 3)), np.array([0, 2, -1]), 1.0)).sum() == 6
    assert not do.embed_grad(np.ones((2, 3)), np.array([5, -1]), 4, 1.0).any()


def test_cross_entropy():
    z = (double(7, 13, seed=1) * 4).requires_grad_()
    t = torch.tensor([0, 12, -100, 5, 5, -100, 3])
    g = double(7, seed=2)
    loss = F.cross_entropy(z, t, reduction="none")
    loss.backward(g)
    zn, tn = z.detach().numpy(), t.numpy()
    got, lse = do.xent(zn, tn, -100)
    np.testing.assert_allclose(got, loss.detach().numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(lse, torch.logsumexp(z, 1).detach().numpy(), rtol=1e-13)
    np.testing.assert_allclose(do.xent_dz(zn, tn, -100, lse, g.numpy()), z.grad.numpy(), rtol=1e-11, atol=1e-14)
    assert np.isnan(do.xent(zn, np.full(7, 13), -100)[0]).all()
