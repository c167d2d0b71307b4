"""Gradients of the output layer's loss where a row's target has nearly the whole probability, against the definition: the
term p - 1 of the target is then far smaller than the rounding of the row's log sum or of its logits.

The first test's logits are exact: 1016 for 255 classes and 1016 + margin for the target, so q = 1 - p = 255 exp(-margin) /
(1 + 255 exp(-margin)).  With U = 2^-24, the row's sum of exponentials is 1 and at most 0.09 beside it, joined by at most 48
additions, each within U, of exponentials within 2^-20 of themselves: within 50 U + 2^-20 q, and its logarithm likewise, which is the
loss.  The log sum reaches the gradient as two numbers, within U of the smaller one, itself below 2^-14; so dz of the target, -q by
expm1, and the other classes' together, q, are each off by at most e = 56 U + 2^-18 q.  In bf16 with more than 128 rows each
dz is rounded, by at most 2^-8 of itself, and by 2^-16 with fewer; the products are fp32 sums of N terms, within (N + 16) 2^-23 of their
magnitudes, and the outputs are rounded once."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from paper_2609_33437_amd import layers
from test_gpu_xent import check_gradients, logits

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def confident(m, margin, dtype):
    """x [m, 32], W [256, 32], target 3: its logit stands `margin` above 255 equal ones of 1016."""
    x, w = torch.zeros(m, 32, device=DEV, dtype=DT[dtype]), torch.zeros(256, 32, device=DEV, dtype=DT[dtype])
    x[:, 0], x[:, 1] = 8.0, 1.0
    w[:, 0] = 127.0
    w[3, 1] = margin
    return x, w, torch.full((m,), 3, device=DEV)


def check_confident(m, margin, dtype, dx, dw):
    beside = 255 * np.exp(-float(margin))
    q = beside / (1 + beside)
    each = 0.0 if dtype == "f32" else 2.0 ** -16 if m <= 128 else 2.0 ** -8
    out = U if dtype == "f32" else 2.0 ** -8
    e = 56 * U + 2.0 ** -18 * q + each * q
    dx, dw = dx.double(), dw.double()
    # column 0 of dx: 127 times the sum of dz, which is 0
    sums = (256 + 16) * 2.0 ** -23
    assert float(dx[:, 0].abs().max()) <= (127 * (2 * e) + sums * 127 * 2 * (q + e)) * (1 + out)
    # column 1: margin times dz of the target
    err = margin * (e + sums * (q + e))
    assert float((dx[:, 1] + margin * q).abs().max()) <= err + (margin * q + err) * out
    assert not dx[:, 2:].any()
    sums = (m + 16) * 2.0 ** -23
    for column, by in ((0, 8.0), (1, 1.0)):
        err = by * m * (e + sums * (q + e))
        assert abs(float(dw[3, column]) + by * m * q) <= err + (by * m * q + err) * out
        others = torch.cat([dw[:3, column], dw[4:, column]])
        err /= 255
        assert float((others - by * m * q / 255).abs().max()) <= err + (by * m * q / 255 + err) * out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 2, 64, 200, 600])
@pytest.mark.parametrize("margin", [8, 12, 16])
def test_confident_rows(dtype, m, margin):
    x, w, t = confident(m, margin, dtype)
    own = x.requires_grad_(), w.requires_grad_()
    layers.linear_cross_entropy(*own, t, reduction="sum").backward()
    check_confident(m, margin, dtype, own[0].grad, own[1].grad)
    summed = own[0].grad, own[1].grad
    own[0].grad = own[1].grad = None
    layers.linear_cross_entropy(*own, t, reduction="none").sum().backward()
    assert torch.equal(own[0].grad, summed[0]) and torch.equal(own[1].grad, summed[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 5, 200])
def test_equal_logits_of_any_size(dtype, m):
    """Two classes with the same logit, whatever its size, have half of the probability each: exp(-log 2) and expm1(-log 2) in
    fp32 are within 2^-20 of that, and the products below have one term or, in columns of W, m equal ones."""
    for power in (0, 12, 24, 31, 60):
        x, w = torch.zeros(m, 16, device=DEV, dtype=DT[dtype]), torch.zeros(40, 16, device=DEV, dtype=DT[dtype])
        x[:, 0], x[:, 1] = 2.0 ** power, 1.0
        w[:, 0] = -1.0 if power > 8 else -256.0
        w[5, 0] = w[9, 0] = 1.0
        w[5, 1], w[9, 1] = 0.0, 0.0
        w[5, 2], w[9, 3] = 1.0, 1.0
        x.requires_grad_()
        w.requires_grad_()
        layers.linear_cross_entropy(x, w, torch.full((m,), 5, device=DEV), reduction="sum").backward()
        tol = 2.0 ** -20 + (2.0 ** -8 * 2 if dtype == "bf16" else 0.0)
        assert float((x.grad[:, 2].double() + 0.5).abs().max()) <= 0.5 * tol, power
        assert float((x.grad[:, 3].double() - 0.5).abs().max()) <= 0.5 * tol, power
        err = 0.5 * m * (tol + (m + 16) * 2.0 ** -23)
        assert abs(float(w.grad[5, 1]) + 0.5 * m) <= err and abs(float(w.grad[9, 1]) - 0.5 * m) <= err, power


# tiles alone, with rows left over for other tiles or for the kernel for few rows, ranges of k
SAME = [("bf16", 1, 900, 1001), ("bf16", 5, 2000, 1001), ("bf16", 8, 40000, 512), ("bf16", 40, 700, 2048), ("bf16", 129, 9000, 130),
        ("bf16", 157, 43584, 2829), ("bf16", 300, 50, 4001), ("bf16", 515, 32003, 769), ("bf16", 515, 32003, 2048),
        ("bf16", 1283, 128256, 1024), ("bf16", 2100, 60000, 2048), ("bf16", 3001, 50257, 768), ("bf16", 700, 1000, 4096),
        ("f32", 515, 32003, 769), ("f32", 157, 43584, 2829), ("f32", 1030, 20001, 770), ("f32", 259, 30000, 1024)]


def check_same_logits(dtype, m, n, k, ignored=0.0):
    """Where a target has the whole probability a gradient is exactly zero, if its logit is computed again to the same bits."""
    gen = torch.Generator(DEV).manual_seed(3)
    w = torch.randn(n, k, generator=gen, device=DEV).to(DT[dtype])
    t = torch.randint(0, n, (m,), generator=gen, device=DEV)
    x = (w[t].float() * (600.0 / k)).to(DT[dtype])          # logits of about 600, others within 600 / sqrt(k) times 6
    t[torch.rand(m, generator=gen, device=DEV) < ignored] = -100
    loss, lse, low = (torch.empty(m, device=DEV) for _ in range(3))
    smat.smat_linear_xent(x, w, t, loss, lse, lse_low=low)
    assert not loss.any() and not low.any()
    dx, dw = torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, lse_low=low)
    rows = dx.any(1)
    assert not rows.any() and not dw.any(), f"{int(rows.sum())} rows, dx up to {float(dx.abs().max())} beside W of {float(w.abs().max())}"


@pytest.mark.parametrize("dtype,m,n,k", SAME)
def test_logits_are_the_same_in_both_calls(dtype, m, n, k):
    check_same_logits(dtype, m, n, k)


@pytest.mark.parametrize("dtype,m,n,k", [s for s in SAME if s[1] > 128] + [("f32", 771, 32003, 769), ("f32", 1027, 50304, 300)])
@pytest.mark.parametrize("ignored", [0.1, 0.5, 0.99])
def test_logits_are_the_same_without_some_rows(dtype, m, n, k, ignored):
    """Rows without a target are left out of large products; the others stay with those that sum in their order."""
    check_same_logits(dtype, m, n, k, ignored)


@pytest.mark.parametrize("where", ["first", "last", "all_but_last", "one"])
def test_a_part_without_rows(where):
    """512 rows by tiles and 3 by the kernel for few rows, of which one part has no target."""
    m, n, k = 515, 32003, 769
    gen = torch.Generator(DEV).manual_seed(9)
    x, w = torch.randn(m, k, generator=gen, device=DEV), torch.randn(n, k, generator=gen, device=DEV) * 0.1
    t = torch.randint(0, n, (m,), generator=gen, device=DEV)
    keep = torch.zeros(m, dtype=torch.bool, device=DEV)
    keep[{"first": slice(0, 512), "last": slice(512, 515), "all_but_last": slice(0, 514), "one": slice(513, 514)}[where]] = True
    t[~keep] = -100
    weights = torch.rand(m, generator=gen, device=DEV) + 0.5
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    check_gradients(x, w, t, "f32", *logits(x, w), lse, row_scale=weights)


@pytest.mark.parametrize("dtype,n,k", [("f32", 151936, 4096), ("bf16", 40000, 1024)])
def test_an_empty_batch_before_a_large_head(dtype, n, k):
    """No rows, and a head whose products would be long: a gradient of zeros."""
    x, w, t = torch.empty(0, k, device=DEV, dtype=DT[dtype]), torch.ones(n, k, device=DEV, dtype=DT[dtype]), torch.empty(0, dtype=torch.int64, device=DEV)
    lse, dw = torch.empty(0, device=DEV), torch.full_like(w, 7.0)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=torch.empty_like(x), dw=dw)
    assert not dw.any()
    dw.fill_(7.0)
    smat.smat_linear_xent_grad(x, w, t, lse, dw=dw, workspace=torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV))
    assert not dw.any()


def test_captured_with_rows_left_out():
    """One graph of losses and gradients, replayed for batches that leave out other rows, whole parts of them too."""
    m, n, k = 515, 32003, 769
    gen = torch.Generator(DEV).manual_seed(4)
    x, w = torch.randn(m, k, generator=gen, device=DEV), torch.randn(n, k, generator=gen, device=DEV) * 0.1
    t = torch.randint(0, n, (m,), generator=gen, device=DEV)

    def step():
        loss, lse, low, tot = (torch.empty(s, device=DEV) for s in (m, m, m, 3))
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        smat.smat_linear_xent(x, w, t, loss, lse, totals=tot, lse_low=low)
        smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, totals=tot, lse_low=low)
        return loss, lse, low, tot, dx, dw

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = step()
    for left_out in (slice(0, 0), slice(0, 512), slice(512, 515), slice(100, 514), slice(0, 515), slice(3, 4)):
        t.copy_(torch.randint(0, n, (m,), generator=gen, device=DEV))
        t[left_out] = -100
        g.replay()
        torch.cuda.synchronize()
        got = [h.clone() for h in held]
        for a, b in zip(got, step()):
            assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num()), left_out
