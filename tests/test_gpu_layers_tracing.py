"""The layers under torch's tracers: torch.jit.trace keeps each call, with and without gradients, and make_fx, which would record
the output's allocation and not the kernel that writes it, is refused in both passes."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

import paper_2609_33437_amd as smat
from paper_2609_33437_amd import layers

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * 0.3


W, V, B, G = (rand(*s, seed=1) for s in ((96, 64), (64, 96), (96,), (64,))) if torch.cuda.is_available() else [None] * 4
IDS = torch.arange(6, device=DEV) % 5 if torch.cuda.is_available() else None
FORMS = {
    "linear": lambda x: layers.linear(x, W, B),
    "mlp": lambda x: layers.mlp(x, W, B, V, None, smat.SMAT_ACT_GELU, x),
    "gated_mlp": lambda x: layers.gated_mlp(x, W, W, V),
    "layer_norm": lambda x: layers.layer_norm(x, G, G),
    "rms_norm": lambda x: layers.rms_norm(x, G),
    "cross_entropy": lambda x: layers.linear_cross_entropy(x, W, IDS),
    "cross_entropy_rows": lambda x: layers.linear_cross_entropy(x, W, IDS, reduction="none"),
    "embedding": lambda x: layers.embedding(IDS, x),
}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("grads", [False, True])
def test_jit_trace_keeps_the_call(form, grads):
    x = rand(6, 64, seed=5).requires_grad_(grads)
    with torch.set_grad_enabled(grads):
        traced = torch.jit.trace(FORMS[form], (x,))
        for seed in (6, 7):
            other = rand(6, 64, seed=seed)
            torch.full((1 << 20,), float("nan"), device=DEV)      # what an allocation finds
            assert torch.equal(traced(other), FORMS[form](other))
            mine, want = other.clone().requires_grad_(grads), other.clone().requires_grad_(grads)
            if grads:
                traced(mine).sum().backward()
                FORMS[form](want).sum().backward()
                assert torch.equal(mine.grad, want.grad)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("mode", ["real", "fake", "symbolic"])
@pytest.mark.parametrize("early", [False, True])
def test_graph_tracers_are_refused(form, mode, early):
    for x in (rand(6, 64, seed=5), rand(6, 64, seed=5).requires_grad_()):
        with pytest.raises(smat.SmatError, match="make_fx"):
            make_fx(FORMS[form], tracing_mode=mode, pre_dispatch=early)(x)
    assert torch.isfinite(FORMS[form](rand(6, 64, seed=5))).all()


@pytest.mark.parametrize("form", FORMS)
def test_graph_tracers_of_a_backward_pass_are_refused(form):
    x = rand(6, 64, seed=5).requires_grad_()
    loss = FORMS[form](x).square().sum()
    with pytest.raises(smat.SmatError, match="make_fx"):
        make_fx(lambda g: torch.autograd.grad(loss, x, g, retain_graph=True))(torch.ones((), device=DEV))
    assert torch.isfinite(torch.autograd.grad(loss, x)[0]).all()


def test_other_dispatch_modes_are_not():
    from torch.utils.flop_counter import FlopCounterMode

    x = rand(6, 64, seed=5).requires_grad_()
    want = layers.rms_norm(x, G)
    with FlopCounterMode(display=False):
        got = layers.rms_norm(x, G)
        got.sum().backward()
    assert torch.equal(got, want)
