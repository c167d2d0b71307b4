"""The layers whose activations are saved in 8 bits: forward and gradients against fp64 on the checkpointed values,
against differences and against torch's autograd on exact ones, inside a simulated step, and what they keep.

Exact gradients differ by what 8 bits lose: values of a block of 32 normals are rounded to steps of at
most max / 64, so by at most max / 64 / sqrt(12) in the mean square, about 1.2 % of their own mean square for
max = 2.6 standard deviations.  A weight gradient reads one or two checkpoints, an input gradient the
pre-activations: 3 % of the norm holds each."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from oracle import linear_oracle as lo
from paper_2609_33437_amd import layers
from paper_2609_33437_amd.training import SimulatedMergeTraining
from workloads.model import TINY, make_decoder, token_batches

pytestmark = pytest.mark.gpu
DEV = "cuda"
LOSS_8BIT = 0.03


def leaf(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device=DEV) * std).to(dtype).requires_grad_(True)


def rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def torch_mlp(x, w1, b1, w2, b2, act, r):
    f = {smat.SMAT_ACT_GELU: torch.nn.functional.gelu, smat.SMAT_ACT_SILU: torch.nn.functional.silu,
         smat.SMAT_ACT_GELU_TANH: lambda z: torch.nn.functional.gelu(z, approximate="tanh")}[act]
    return torch.nn.functional.linear(f(torch.nn.functional.linear(x, w1, b1)), w2, b2) + r


@pytest.mark.parametrize("act", [smat.SMAT_ACT_GELU, smat.SMAT_ACT_GELU_TANH, smat.SMAT_ACT_SILU])
@pytest.mark.parametrize("shape", [(2, 37), (300,), (1,)])
def test_mlp_gradients_close_to_exact_ones(act, shape):
    gen = torch.Generator(DEV).manual_seed(1)
    d, f = 96, 200
    args = [leaf(gen, *shape, d), leaf(gen, f, d, std=0.1), leaf(gen, f), leaf(gen, d, f, std=0.1), leaf(gen, d)]
    r = leaf(gen, *shape, d)
    y = layers.mlp(*args, act, residual=r)
    want = torch_mlp(*[t.double() for t in args], act, r.double())
    assert rel(y, want) < 1e-6
    c = torch.randn(y.shape, generator=gen, device=DEV)
    got = torch.autograd.grad(y, args + [r], c)
    exact = torch.autograd.grad(want, args + [r], c.double())
    for g, e in zip(got, exact):
        assert g.shape == e.shape and rel(g, e) < LOSS_8BIT
    assert torch.equal(got[-1], c) and rel(got[4], exact[4]) < 1e-6     # nothing saved stands between


def test_mlp_gradients_are_those_of_the_checkpoints():
    """Every gradient against fp64 on the saved values: the oracle's checkpoints of x and of the pre-activation."""
    gen = torch.Generator(DEV).manual_seed(2)
    m, d, f, act = 70, 64, 130, smat.SMAT_ACT_GELU
    x, w1, b1, w2, b2 = leaf(gen, m, d), leaf(gen, f, d, std=0.1), leaf(gen, f), leaf(gen, d, f, std=0.1), leaf(gen, d)
    y = layers.mlp(x, w1, b1, w2, b2, act)
    c = torch.randn(m, d, generator=gen, device=DEV)
    dx, dw1, db1, dw2, db2 = torch.autograd.grad(y, (x, w1, b1, w2, b2), c)
    n = lambda t: t.detach().cpu().double().numpy()     # noqa: E731
    z = smat.ActCheckpoint.empty(m, f)
    smat.smat_linear(x.detach(), w1.detach(), torch.empty(m, f, device=DEV), bias=b1.detach(), act=act, z_ckpt=z)
    zh = lo.ckpt_read(z.codes.cpu().numpy(), z.exps.cpu().numpy(), f)
    xh = lo.ckpt_read(*lo.ckpt_write(n(x)), d)
    dz = lo.dgrad(n(c), n(w2), act, z=zh)[0]
    want = dict(dx=lo.dgrad(dz, n(w1))[0], dw1=lo.wgrad(dz, xh)[0], db1=dz.sum(axis=0), dw2=lo.wgrad(n(c), lo.act(zh, act))[0],
                db2=n(c).sum(axis=0))
    for name, g in dict(dx=dx, dw1=dw1, db1=db1, dw2=dw2, db2=db2).items():
        # fp32 sums of up to 130 terms of mixed sign: 200 * 2^-23 of their absolute sum, at most 20 times the norm here
        assert np.linalg.norm(n(g) - want[name]) <= 1e-4 * np.linalg.norm(want[name]), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [1, 65, 600])
def test_gated_mlp_gradients_close_to_exact_ones(dtype, m):
    gen = torch.Generator(DEV).manual_seed(3)
    d, f = 128, 160
    args = [leaf(gen, m, d, dtype=dtype), leaf(gen, f, d, std=0.1, dtype=dtype), leaf(gen, f, d, std=0.1, dtype=dtype),
            leaf(gen, d, f, std=0.1, dtype=dtype)]
    r = leaf(gen, m, d, dtype=dtype)
    y = layers.gated_mlp(*args, residual=r)
    x, wg, wu, wd = [t.double() for t in args]
    lin = torch.nn.functional.linear
    want = lin(torch.nn.functional.silu(lin(x, wg)) * lin(x, wu), wd) + r.double()
    # bf16 rounds u, h and the result: three roundings of 2^-8 / sqrt(3) each, h and u inside the last product
    assert rel(y, want) < (1e-6 if dtype == torch.float32 else 8e-3)
    c = torch.randn(m, d, generator=gen, device=DEV).to(dtype)
    got = torch.autograd.grad(y, args + [r], c)
    exact = torch.autograd.grad(want, args + [r], c.double())
    for g, e in zip(got, exact):
        assert g.dtype == dtype and rel(g, e) < LOSS_8BIT


def test_gradient_against_differences():
    """dL/dt along random directions against central differences of the layer's own forward pass (fp32)."""
    gen = torch.Generator(DEV).manual_seed(4)
    args = [leaf(gen, 50, 64), leaf(gen, 96, 64, std=0.1), leaf(gen, 96, 64, std=0.1), leaf(gen, 64, 96, std=0.1)]
    c = torch.randn(50, 64, generator=gen, device=DEV)
    grads = torch.autograd.grad(layers.gated_mlp(*args), args, c)
    with torch.no_grad():
        for i, (t, g) in enumerate(zip(args, grads)):
            v = g / g.norm()        # along the gradient itself: the derivative is its norm
            h = 1e-3 * float(t.norm())
            shifted = lambda s: [a + s * v if j == i else a for j, a in enumerate(args)]    # noqa: E731
            num = float(((layers.gated_mlp(*shifted(h)) - layers.gated_mlp(*shifted(-h))).double() * c.double()).sum()) / (2 * h)
            # 8 bits turn the direction by up to LOSS_8BIT and change the length by as much; differences add h^2 and 1e-4
            assert abs(num - float(g.norm())) < (LOSS_8BIT + 0.005) * float(g.norm()), i


def test_linear_layer_and_frozen_parts():
    gen = torch.Generator(DEV).manual_seed(5)
    x, w, b = leaf(gen, 4, 33, 64), leaf(gen, 100, 64, std=0.1), leaf(gen, 100)
    c = torch.randn(4, 33, 100, generator=gen, device=DEV)
    want = torch.nn.functional.linear(x, w, b)
    exact = torch.autograd.grad(want, (x, w, b), c)
    y = layers.linear(x, w, b)
    assert rel(y, want) < 1e-6
    for g, e in zip(torch.autograd.grad(y, (x, w, b), c), exact):
        assert rel(g, e) < LOSS_8BIT
    # only the bias, only the input
    assert rel(torch.autograd.grad(layers.linear(x.detach(), w.detach(), b), b, c)[0], exact[2]) < 1e-6
    assert rel(torch.autograd.grad(layers.linear(x, w.detach(), b.detach()), x, c)[0], exact[0]) < 1e-6
    y = layers.mlp(x.detach(), w, b, leaf(gen, 64, 100).detach(), None, smat.SMAT_ACT_GELU)
    assert y.requires_grad and all(g is not None for g in torch.autograd.grad(y.sum(), (w, b)))
    # non-contiguous input and gradient
    xt = x.detach().transpose(0, 1).requires_grad_(True)
    y = layers.linear(xt, w, b)
    g = torch.autograd.grad(y.transpose(0, 1), (xt, w), c)
    assert rel(g[0].transpose(0, 1), exact[0]) < 1e-6 and rel(g[1], exact[1]) < LOSS_8BIT


def test_saved_bytes():
    """A gated MLP keeps about d + 2 f bytes a token (and its parameters), where bf16 activations take 2 (d + 3 f) or more."""
    gen = torch.Generator(DEV).manual_seed(6)
    m, d, f = 256, 128, 352
    args = [leaf(gen, m, d, dtype=torch.bfloat16)] + [leaf(gen, f, d, dtype=torch.bfloat16) for _ in range(2)] + \
        [leaf(gen, d, f, dtype=torch.bfloat16)]
    kept = {}
    weights = {t.untyped_storage().data_ptr() for t in args[1:]}

    def pack(t):
        if t.untyped_storage().data_ptr() not in weights:
            kept[t.data_ptr()] = t.numel() * t.element_size()
        return t

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        y = layers.gated_mlp(*args)
    assert sum(kept.values()) == m * (d + 2 * f) * 33 // 32
    y.sum().backward()
    assert all(t.grad is not None for t in args)


def test_no_grad_saves_nothing_and_single_tokens_agree():
    gen = torch.Generator(DEV).manual_seed(7)
    x = leaf(gen, 40, 128, dtype=torch.bfloat16)
    ws = [leaf(gen, 352, 128, std=0.1, dtype=torch.bfloat16), leaf(gen, 352, 128, std=0.1, dtype=torch.bfloat16),
          leaf(gen, 128, 352, std=0.1, dtype=torch.bfloat16)]
    with torch.no_grad():
        whole = layers.gated_mlp(x, *ws, residual=x)
        assert not whole.requires_grad
        for i in (0, 17, 39):       # another order of the same sums: a rounding of u, h and y apart
            one = layers.gated_mlp(x[i:i + 1], *ws, residual=x[i:i + 1])
            assert rel(one, whole[i:i + 1]) < 8e-3
    assert torch.equal(layers.gated_mlp(x, *ws, residual=x).detach(), whole)


def test_empty_batch():
    gen = torch.Generator(DEV).manual_seed(8)
    x, ws = leaf(gen, 0, 64), [leaf(gen, 96, 64), leaf(gen, 96, 64), leaf(gen, 64, 96)]
    y = layers.gated_mlp(x, *ws)
    assert y.shape == (0, 64)
    y.sum().backward()
    assert x.grad.shape == (0, 64) and all(not w.grad.any() for w in ws)


def test_refusals():
    cpu = torch.ones(4, 8)
    with pytest.raises(smat.SmatError):
        layers.linear(cpu, cpu)
    x = torch.ones(4, 8, device=DEV)
    with pytest.raises(smat.SmatError):
        layers.mlp(x, x, None, x.t().contiguous(), None, smat.SMAT_ACT_NONE)
    with pytest.raises(smat.SmatError):
        layers.linear(x, x.bfloat16())
    with pytest.raises(smat.SmatError):
        layers.linear(x.double(), x.double())


@pytest.mark.parametrize("buffer_dtype", [torch.bfloat16, torch.float32])
def test_decoder_in_simulated_steps(buffer_dtype):
    """Two decoders with the same weights, one through the operators: ordinary and simulated steps give the same
    losses up to bf16 and gradients of the MLPs within what 8 bits and bf16 lose."""
    grads, losses = {}, {}
    for checkpointed in (False, True):
        model = make_decoder(TINY, 0, DEV, checkpointed=checkpointed)
        batches = token_batches(TINY, 2, 16, 4, 1, DEV)
        base = {n: p.detach().clone() for n, p in model.named_parameters()}
        w = SimulatedMergeTraining.from_module(model, keep=0.5, period=2, seed=3, buffer_dtype=buffer_dtype, theta0=base)
        out, gs = [], []
        for k in range(2):
            for p in model.parameters():
                p.grad = None
            sim = w.begin(k)
            with torch.autocast("cuda", dtype=torch.bfloat16, enabled=buffer_dtype == torch.bfloat16):
                loss = model.loss(batches[k])
            loss.backward()
            if sim:
                w.end()
            out.append(loss.item())
            gs.append([p.grad.clone() for n, p in model.named_parameters() if ".mlp." in n])
        losses[checkpointed], grads[checkpointed] = out, gs
        w.close()
    assert np.allclose(losses[False], losses[True], rtol=1e-2 if buffer_dtype == torch.bfloat16 else 1e-5)
    for a, b in zip(grads[False], grads[True]):
        for x, y in zip(a, b):
            # bf16 rounds every activation and gradient on both sides: a few 2^-8 each on top of the 8 bits
            assert rel(y, x) < (0.1 if buffer_dtype == torch.bfloat16 else 2 * LOSS_8BIT)
