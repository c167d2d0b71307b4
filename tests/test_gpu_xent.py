"""The output layer with its cross entropy on the GPU, losses and gradients, against its definition in float64.

Bounds, with u = 2^-24.  A logit of k products is off by at most e_z = (k + 8) 2^-23 sum |x w| (fp32 sums in any order; bf16
products are exact there).  Its row's sum of exponentials joins at most 35 parts a thread (32 columns each, 151,936 columns
over 256 threads, then a tree), each with three roundings and two exponentials of 2^-22 relative error, beside the
exponentials' own: within 2^-16 of itself; so lse is off by max e_z + 2^-15 + 2 u |lse|, and the loss by that, the target's
e_z and 2 u of both.

p = exp(z - lse), for an lse that is an input, is off by p (e_z + 2^-20 + |z - lse| 2^-22) to first order (1.1 covers the
rest); dz = (p - 1) g by two more roundings.  A gradient sums N products of dz: its bound is the sum of |dz's error| times the
other factor's magnitude, (N + 16) 2^-23 of the sum of magnitudes, what dz's rounding to the call's dtype adds, 2^-21 of
itself for s, and the output's rounding.  In fp32 a dz rounds by u.  In bf16 each dz rounds by at most 2^-8 of itself, up or
down, and their sum is held to Hoeffding's bound for such sums, 2^-8 sqrt(2 ln(2 / q)) times the root of the sum of squares
of the products, with q = 1e-15 an element: sqrt(2 ln(2 / q)) = 8.4."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from oracle import decoder_oracle as do

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24
IGNORE = -100


def strided(rows, cols, dtype, pad=0, shift=0):
    buf = torch.full((rows * (cols + pad) + shift + 16,), float("nan"), dtype=DT[dtype], device=DEV)
    return buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def untouched(v):
    if v.shape[0] < 2 or v.stride(0) == v.shape[1]:
        return True
    whole = torch.as_strided(v, (v.shape[0] - 1, v.stride(0)), v.stride(), v.storage_offset())
    return bool(torch.isnan(whole[:, v.shape[1]:]).all())


def rounding(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U


def make(m, n, k, dtype, pad=0, shift=0, ignored=0.2):
    """x, W and targets whose probabilities range from 1 / n to nearly 1, some rows without a target."""
    gen = torch.Generator(DEV).manual_seed(m * 7 + n * 3 + k)
    w = strided(n, k, dtype, pad, shift)
    w.copy_(torch.randn(n, k, generator=gen, device=DEV) * 0.3)
    t = torch.randint(0, n, (m,), generator=gen, device=DEV)
    x = strided(m, k, dtype, pad, shift)
    lean = torch.rand(m, 1, generator=gen, device=DEV) * (15.0 / max(1.0, 0.09 * k))
    x.copy_(torch.randn(m, k, generator=gen, device=DEV) * (3.0 / max(k, 1) ** 0.5) + lean * w[t].float())
    t[torch.rand(m, generator=gen, device=DEV) < ignored] = IGNORE
    if m > 2:
        t[m - 1] = n - 1
        t[0] = 0
    return x, w, t


def logits(x, w):
    """(z, bound of its error)"""
    xd, wd = x.double(), w.double()
    return xd @ wd.t().contiguous(), (x.shape[1] + 8) * 2.0 ** -23 * (xd.abs() @ wd.abs().t().contiguous())


def close(got, want, err, what):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan()), what
    bad = (got - want).abs() > err
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()}, worst {float(((got - want).abs() / err).nan_to_num().max())}"


def check_forward(x, w, t, totals=True):
    m, n = x.shape[0], w.shape[0]
    loss, lse = torch.full((m,), 7.0, device=DEV), torch.full((m,), 7.0, device=DEV)
    tot = torch.full((3,), 7.0, device=DEV) if totals else None
    smat.smat_linear_xent(x, w, t, loss, lse, totals=tot, ignore_index=IGNORE)
    z, e_z = logits(x, w)
    want_lse = torch.logsumexp(z, 1)
    e_lse = e_z.amax(1) + 2.0 ** -15 + 2 * U * want_lse.abs()
    close(lse, want_lse, e_lse, "lse")
    has = t != IGNORE
    at = torch.where(has, t, 0)[:, None]
    zt, e_zt = z.gather(1, at)[:, 0], e_z.gather(1, at)[:, 0]
    want = torch.where(has, want_lse - zt, 0.0)
    err = torch.where(has, e_lse + e_zt + 2 * U * (want_lse.abs() + zt.abs()), 0.0)
    close(loss, want, err, "loss")
    if totals:
        count = int(has.sum())
        total = loss.double()[has].sum()
        assert float(tot[1]) == count and abs(float(tot[0] - total)) <= 2 * U * abs(float(total))
        assert tot[2].isnan() if count == 0 else abs(float(tot[2]) - float(total) / count) <= 2 * U * abs(float(total) / count)
    return z, e_z, loss, lse, tot


def check_gradients(x, w, t, dtype, z, e_z, lse, row_scale=None, scale=None, totals=None, pad=0, shift=0):
    m, k = x.shape
    n = w.shape[0]
    dx, dw = strided(m, k, dtype, pad, shift), strided(n, k, dtype, pad, shift)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, row_scale=row_scale, scale=scale, totals=totals, ignore_index=IGNORE)
    has = t != IGNORE
    g = (row_scale.double() if row_scale is not None else torch.ones(m, dtype=torch.float64, device=DEV)) * has
    rel = z - lse.double()[:, None]
    p = torch.exp(rel)
    e_dz = 1.1 * p * (e_z + 2.0 ** -20 + rel.abs() * 2.0 ** -22)
    rows = torch.nonzero(has)[:, 0]
    p[rows, t[rows]] -= 1.0
    e_dz = (e_dz + 2 * U * p.abs()) * g.abs()[:, None]
    dz = p * g[:, None]
    s = (float(scale) if scale is not None else 1.0) / (float(totals[1]) if totals is not None else 1.0)
    xd, wd = x.double(), w.double()

    def bound(a, e_a, b):       # of a @ b
        err = e_a @ b.abs() + (a.shape[1] + 16) * 2.0 ** -23 * (a.abs() @ b.abs())
        if dtype == "f32":
            return err + U * (a.abs() @ b.abs())
        return err + 2.0 ** -8 * 8.4 * torch.sqrt(((a.abs() + e_a) ** 2) @ (b * b))

    for got, want, err, what in ((dx, dz @ wd, bound(dz, e_dz, wd), "dx"),
                                 (dw, dz.t().contiguous() @ xd, bound(dz.t().contiguous(), e_dz.t().contiguous(), xd), "dw")):
        want, err = s * want, abs(s) * err
        err = err + (want.abs() + err) * (rounding(dtype) + 2.0 ** -21)
        close(got, want, err, f"{what} {m} x {n} x {k}")
        assert untouched(got)
    assert not dx[~has].any()
    return dx, dw


# single tokens and few rows, one class, odd and ragged sizes, no width at all, every tile, splits of k
SIZES = [(1, 1, 1), (1, 2, 8), (1, 50304, 768), (2, 1000, 64), (3, 31, 5), (5, 32, 40), (8, 33, 200), (8, 5000, 512), (9, 257, 100),
         (17, 4097, 24), (33, 64, 512), (64, 4096, 256), (100, 96, 2048), (130, 1000, 1024), (300, 1024, 1024), (257, 2003, 130),
         (512, 8192, 64), (1000, 2048, 96), (1024, 16384, 64), (2049, 4096, 128), (4, 7, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_loss_and_gradients(dtype, m, n, k):
    x, w, t = make(m, n, k, dtype)
    z, e_z, _, lse, tot = check_forward(x, w, t)
    if float(tot[1]) > 0:
        check_gradients(x, w, t, dtype, z, e_z, lse, totals=tot)
    gen = torch.Generator(DEV).manual_seed(5)
    weights = torch.randn(m, generator=gen, device=DEV)
    check_gradients(x, w, t, dtype, z, e_z, lse, row_scale=weights, scale=torch.full((1,), 0.37, device=DEV))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k,pad,shift", [(1, 300, 77, 3, 1), (7, 1001, 33, 1, 3), (40, 999, 129, 0, 1), (130, 517, 513, 2, 0),
                                             (515, 2003, 769, 0, 0), (600, 1500, 200, 4, 5), (1024, 5000, 131, 1, 1)])
def test_rows_off_16_bytes(dtype, m, n, k, pad, shift):
    """Operands and outputs at any element's address, with NaN between their rows."""
    x, w, t = make(m, n, k, dtype, pad, shift)
    z, e_z, _, lse, _ = check_forward(x, w, t, totals=False)
    check_gradients(x, w, t, dtype, z, e_z, lse, pad=pad + 1, shift=shift)


@pytest.mark.parametrize("dtype,m,n,k", [("bf16", 8192, 20000, 64), ("bf16", 9000, 17000, 33), ("f32", 8192, 9000, 40),
                                         ("bf16", 70000, 2500, 32), ("f32", 40000, 2049, 16)])
def test_vocabulary_in_pieces(dtype, m, n, k):
    """Batches whose gradients take several pieces of the vocabulary, the last one narrower."""
    x, w, t = make(m, n, k, dtype)
    z, e_z, _, lse, tot = check_forward(x, w, t)
    check_gradients(x, w, t, dtype, z, e_z, lse, totals=tot)


@pytest.mark.parametrize("dtype,m,n,k,pad,shift", [("bf16", 4096, 40000, 1024, 0, 0), ("bf16", 3001, 50257, 768, 8, 0),
                                                   ("bf16", 2500, 40001, 1025, 1, 3), ("f32", 1500, 16000, 768, 0, 0),
                                                   ("f32", 1030, 20001, 770, 1, 1)])
@pytest.mark.parametrize("ignored", [0.0, 0.6, 0.999, 1.0])
def test_large_batches_take_their_rows_with_a_target(dtype, m, n, k, pad, shift, ignored):
    """Where the products are long the gradient's take the rows with a target alone: none left out, a part, a handful, none."""
    x, w, t = make(m, n, k, dtype, pad, shift, ignored)
    if ignored == 1.0:
        t.fill_(IGNORE)
    elif ignored:
        t[:300] = IGNORE        # whole tiles of them
        t[-300:] = IGNORE
        t[301] = 5
    z, e_z, _, lse, tot = check_forward(x, w, t)
    check_gradients(x, w, t, dtype, z, e_z, lse, totals=tot if ignored < 1.0 else None, pad=pad, shift=shift)
    weights = torch.randn(m, generator=torch.Generator(DEV).manual_seed(5), device=DEV)
    dx, dw = check_gradients(x, w, t, dtype, z, e_z, lse, row_scale=weights)
    if ignored == 1.0:
        assert not dw.any()
    # one gradient at a time
    only = torch.full_like(dx, float("nan"))
    smat.smat_linear_xent_grad(x, w, t, lse, dx=only, row_scale=weights, ignore_index=IGNORE)
    assert torch.equal(only, dx)
    only = torch.full_like(dw, float("nan"))
    smat.smat_linear_xent_grad(x, w, t, lse, dw=only, row_scale=weights, ignore_index=IGNORE)
    assert torch.equal(only, dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_gradient_alone_and_repeated(dtype):
    x, w, t = make(1200, 3000, 96, dtype)
    loss, lse = torch.empty(1200, device=DEV), torch.empty(1200, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw)
    for names in (("dx",), ("dw",), ("dx", "dw"), ()):
        got = {k: torch.full_like(v, float("nan")) for k, v in (("dx", dx), ("dw", dw)) if k in names}
        smat.smat_linear_xent_grad(x, w, t, lse, **got)
        for k, v in got.items():
            assert torch.equal(v, dx if k == "dx" else dw), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [4, 40, 700])
def test_rows_without_a_target(dtype, m):
    """All rows without one: no loss, a mean of nothing, gradients of zero; and targets that are no class: NaN."""
    x, w, t = make(m, 500, 64, dtype)
    t.fill_(IGNORE)
    loss, lse, tot = torch.empty(m, device=DEV), torch.empty(m, device=DEV), torch.empty(3, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse, totals=tot, ignore_index=IGNORE)
    assert not loss.any() and float(tot[0]) == 0 and float(tot[1]) == 0 and tot[2].isnan() and torch.isfinite(lse).all()
    dx, dw = torch.full_like(x, 5.0), torch.full_like(w, 5.0)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, totals=tot, ignore_index=IGNORE)
    assert not dx.any() and not dw.any()
    for outside in (500, -1, -101, 1 << 40):
        t.fill_(IGNORE)
        t[1] = outside
        smat.smat_linear_xent(x, w, t, loss, lse, totals=tot, ignore_index=IGNORE)
        assert loss[1].isnan() and not loss[0].any() and tot[0].isnan() and float(tot[1]) == 1
        smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, totals=tot, ignore_index=IGNORE)
        assert dx[1].isnan().all() and not dx[0].any() and dw.isnan().all()
    # a class as the one to ignore
    t.copy_(torch.arange(m, device=DEV) % 3)
    smat.smat_linear_xent(x, w, t, loss, lse, totals=tot, ignore_index=2)
    assert not loss[2::3].any() and float(tot[1]) == m - len(range(2, m, 3)) and loss[0] > 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(3, 40, 16), (100, 500, 64), (600, 3000, 130), (4096, 40000, 1024)])
def test_padded_rows_without_a_number(dtype, m, n, k):
    """What lies in the rows without a target, NaN and infinities, reaches no loss and no gradient."""
    if dtype == "f32" and n > 3000:
        m, n, k = 1500, 16000, 768
    x, w, t = make(m, n, k, dtype, ignored=0.3)
    t[1] = IGNORE
    t[0] = 0
    none = t == IGNORE
    weights = torch.rand(m, generator=torch.Generator(DEV).manual_seed(5), device=DEV) + 0.5
    clean = x.clone()
    clean[none] = 0
    want = []
    for rows in (clean, x):
        if rows is x:
            x[none] = float("nan")
            x[1] = float("inf")
            weights[none] = float("nan")
        loss, lse, tot = torch.empty(m, device=DEV), torch.empty(m, device=DEV), torch.empty(3, device=DEV)
        smat.smat_linear_xent(rows, w, t, loss, lse, totals=tot, ignore_index=IGNORE)
        dx, dw = torch.full_like(rows, 3.0), torch.full_like(w, 3.0)
        smat.smat_linear_xent_grad(rows, w, t, lse, dx=dx, dw=dw, row_scale=weights, totals=tot, ignore_index=IGNORE)
        want.append((loss, lse[~none], tot, dx, dw))
    assert all(torch.equal(a, b) for a, b in zip(*want)) and not want[1][3][none].any() and torch.isfinite(want[1][4]).all()
    # and a W that spoils everything else leaves those rows of dx alone
    w[3] = float("nan")
    smat.smat_linear_xent(x, w, t, loss, lse, ignore_index=IGNORE)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, ignore_index=IGNORE)
    assert not loss[none].any() and not dx[none].any() and dx[~none].isnan().all()


@pytest.mark.parametrize("m,n,k", [(1, 900, 1001), (5, 2000, 1001), (8, 40000, 515), (40, 700, 515), (129, 9000, 130), (157, 43584, 2829),
                                   (300, 50, 4001), (515, 3001, 769), (600, 20000, 1024), (2100, 1000, 333)])
@pytest.mark.parametrize("pad", [0, 1])
def test_fp32_logits_are_the_same_in_both_calls(m, n, k, pad):
    """Where a target has the whole probability an fp32 gradient is exactly zero: its logit is computed again to the same bits."""
    gen = torch.Generator(DEV).manual_seed(3)
    x, w = strided(m, k, "f32", pad), strided(n, k, "f32", pad, pad)
    w.copy_(torch.randn(n, k, generator=gen, device=DEV))
    t = torch.randint(0, n, (m,), generator=gen, device=DEV)
    x.copy_(w[t] * (600.0 / k))          # logits of about 600, others within 600 / sqrt(k) times 6
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    assert not loss.any()
    dx, dw = torch.full((m, k), float("nan"), device=DEV), torch.full((n, k), float("nan"), device=DEV)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw)
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [2, 200])
def test_small_losses_beside_large_logits(dtype, m):
    """A target 8 above 255 equal logits of 1016 has a loss of log(1 + 255 exp(-8)), which the row's log sum, rounded by up to
    2^-14, would hide."""
    n, k = 256, 32
    x, w = torch.zeros(m, k, device=DEV, dtype=DT[dtype]), torch.zeros(n, k, device=DEV, dtype=DT[dtype])
    x[:, 0] = 8.0
    w[:, 0] = 127.0
    w[3, 0] = 128.0
    t = torch.full((m,), 3, device=DEV)
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    want = float(np.log1p(255 * np.exp(-8.0)))
    # the terms beside the 1 sum to 0.09, each within 16 U; a thread adds up to 32 values to the 1, then at most 16 sums of others,
    # each within U of 1.09; and the logarithm: below 52 U = 3.1e-6
    assert float((loss.double() - want).abs().max()) < 4e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 3, 64, 600])
@pytest.mark.parametrize("power", [0, 20, 31, 33, 60, 110])
def test_logits_of_any_size(dtype, m, power):
    """Logits of multiples of 2^(power - 8) up to 2^power, whose differences no exponential can tell from infinite ones from
    power 20 on: losses and gradients are then exact."""
    n, k = 300, 32
    x, w = torch.zeros(m, k, device=DEV, dtype=DT[dtype]), torch.zeros(n, k, device=DEV, dtype=DT[dtype])
    x[:, 3] = 2.0 ** power
    w[:, 3] = (torch.arange(n, device=DEV) % 255 + 1) / 256
    t = torch.arange(m, device=DEV) * 7 % 255
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    z = x.double() @ w.double().t().contiguous()
    want = torch.logsumexp(z, 1)
    if power < 20:
        assert float((lse - want).abs().max()) < 1e-4
        return
    assert torch.equal(lse.double(), want) and torch.equal(loss.double(), want - z.gather(1, t[:, None])[:, 0])
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw)
    dz = torch.zeros(m, n, device=DEV, dtype=torch.float64)
    dz[:, 254] = 1.0
    dz[torch.arange(m), t] -= 1.0
    assert torch.equal(dx.double(), dz @ w.double())
    want = dz.t().contiguous() @ x.double()      # multiples of 2^power, up to 600 of them
    assert torch.equal(dw.double(), want.to(dw.dtype).double())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [3, 64, 600])
def test_logits_without_a_number(dtype, m):
    """Logits of -inf have no probability; +inf and NaN spoil their rows and no others; huge logits do not overflow."""
    n, k = 300, 32
    x, w, t = make(m, n, k, dtype, ignored=0.0)
    t.fill_(7)
    x[:, 0] = 0.0
    w[:, 0] = 0.0
    w[5, 0] = -float("inf")
    x[0, 0] = 1.0                    # row 0: z_5 = -inf; the other rows: 0 * -inf = NaN
    loss, lse = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse)
    z = x[:1].double() @ w.double().t().contiguous()
    assert abs(float(lse[0]) - float(torch.logsumexp(z, 1))) < 1e-4 and loss[1:].isnan().all() and lse[1:].isnan().all()
    dx = torch.empty_like(x)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx)
    assert dx[1:].isnan().all()
    w[5, 0] = float("inf")           # row 0: +inf
    smat.smat_linear_xent(x, w, t, loss, lse)
    assert loss.isnan().all()
    # all logits -inf: no distribution
    w[:, 0] = -float("inf")
    smat.smat_linear_xent(x[:1], w, t[:1], loss[:1], lse[:1])
    assert loss[0].isnan()
    # far apart: a row's probability is all on one class
    w[:, 0] = 0.0
    w[9, 0] = 1.0
    x[:, 0] = 30000.0
    t.fill_(9)
    t[1] = 8
    smat.smat_linear_xent(x, w, t, loss, lse)
    assert float(loss[0].abs()) < 0.01 and abs(float(loss[1]) / 30000.0 - 1.0) < 0.01
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx)
    assert torch.isfinite(dx).all() and float(dx[0].abs().max()) < 0.02


def test_empty_batch():
    x, w, t = torch.empty(0, 16, device=DEV), torch.ones(40, 16, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    loss, tot = torch.empty(0, device=DEV), torch.full((3,), 7.0, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, loss.clone(), totals=tot)
    assert float(tot[0]) == 0 and float(tot[1]) == 0 and tot[2].isnan()
    dw = torch.full_like(w, 7.0)
    smat.smat_linear_xent_grad(x, w, t, loss, dx=torch.empty_like(x), dw=dw, totals=tot)
    assert not dw.any()


def test_small_definition():
    """The same against the NumPy definition."""
    x, w, t = make(20, 50, 16, "f32")
    loss, lse = torch.empty(20, device=DEV), torch.empty(20, device=DEV)
    smat.smat_linear_xent(x, w, t, loss, lse, ignore_index=IGNORE)
    z = x.cpu().double().numpy() @ w.cpu().double().numpy().T
    tn = t.cpu().numpy()
    want, want_lse = do.xent(z, tn, IGNORE)
    np.testing.assert_allclose(loss.cpu().numpy(), want, rtol=1e-4, atol=1e-4)
    dx = torch.empty_like(x)
    smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, ignore_index=IGNORE)
    np.testing.assert_allclose(dx.cpu().numpy(), do.xent_dz(z, tn, IGNORE, want_lse, np.ones(20)) @ w.cpu().double().numpy(),
                               rtol=1e-3, atol=1e-4)


def test_workspace_stream_and_graph():
    m, n, k = 700, 5000, 64
    x, w, t = make(m, n, k, "bf16")
    gen = torch.Generator(DEV).manual_seed(2)
    scale = torch.full((1,), 3.0, device=DEV)

    def step(stream=None, workspace=None, out=None):
        loss, lse, tot, dx, dw = out or outputs()
        kw = dict(totals=tot, ignore_index=IGNORE, stream=stream, workspace=workspace)
        smat.smat_linear_xent(x, w, t, loss, lse, **kw)
        smat.smat_linear_xent_grad(x, w, t, lse, dx=dx, dw=dw, scale=scale, **kw)
        return loss, lse, tot, dx, dw

    def outputs():
        return (torch.empty(m, device=DEV), torch.empty(m, device=DEV), torch.empty(3, device=DEV), torch.empty_like(x),
                torch.empty_like(w))

    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other, ready = outputs(), torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    step(side, ready, other)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    g, held = torch.cuda.CUDAGraph(), outputs()
    with torch.cuda.graph(g):
        step(out=held)
    for turn in range(3):
        x.copy_(torch.randn(m, k, generator=gen, device=DEV))
        t.copy_(torch.randint(0, n, (m,), generator=gen, device=DEV))
        scale.fill_(turn + 0.5)
        want = step()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held)), turn


def test_binding_refuses():
    x, w, t, v = torch.zeros(4, 8, device=DEV), torch.zeros(6, 8, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), torch.zeros(4, device=DEV)
    o = torch.zeros(4, device=DEV)
    for fn in (lambda: smat.smat_linear_xent(x, w.bfloat16(), t, v, o), lambda: smat.smat_linear_xent(x, w, t.int(), v, o),
               lambda: smat.smat_linear_xent(x, w, t[:3], v, o), lambda: smat.smat_linear_xent(x, w[:, :7], t, v, o),
               lambda: smat.smat_linear_xent(x, w, t, v.double(), o), lambda: smat.smat_linear_xent(x, w, t, v, v),
               lambda: smat.smat_linear_xent(x, w, t, v, o, totals=v), lambda: smat.smat_linear_xent(x, w[:0], t, v, o),
               lambda: smat.smat_linear_xent(x, w.cpu(), t, v, o), lambda: smat.smat_linear_xent(x.half(), w.half(), t, v, o),
               lambda: smat.smat_linear_xent(x, w, t, v, o, workspace=torch.empty(8, device=DEV)),
               lambda: smat.smat_linear_xent_grad(x, w, t, v, dx=x), lambda: smat.smat_linear_xent_grad(x, w, t, v, dw=x),
               lambda: smat.smat_linear_xent_grad(x, w, t, v, scale=2.0), lambda: smat.smat_linear_xent_grad(x, w, t, v, scale=v),
               lambda: smat.smat_linear_xent_grad(x, w, t, v, row_scale=v[:3])):
        with pytest.raises((smat.SmatError, AttributeError)):
            fn()
