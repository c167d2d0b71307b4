"""The linear-layer products and the activation checkpoints on the GPU against the fp64 oracle.

Bounds.  bf16 products are exact in fp32 and an fp32 sum of R terms, in any order, is off by at most
(R + 8) 2^-23 times the sum of their magnitudes (S; one rounding is 2^-24, the factor 2 covers adders
that do not round to nearest).  Activations change by at most 1.13 times their argument's error and are
evaluated within 2^-21 |z| (slopes within 2^-20).  Each later fp32 operation rounds by 2^-24 of what it
forms (2^-21 covers the handful), and a bf16 output by 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paper_2609_33437_amd as smat
from oracle import linear_oracle as lo

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = [smat.SMAT_ACT_NONE, smat.SMAT_ACT_GELU, smat.SMAT_ACT_GELU_TANH, smat.SMAT_ACT_SILU]
SLOPE = 1.13


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(gen, rows, cols, dtype, std=1.0, pad=0, shift=0):
    """A [rows, cols] view: row stride cols + pad, first element `shift` into its buffer, NaN around it."""
    buf = torch.full((rows * (cols + pad) + shift + 16,), float("nan"), dtype=DT[dtype], device=DEV)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * std)
    return v


def untouched(v, pad):
    """The NaNs between the rows of a view made by rand() are still there."""
    if pad == 0 or v.shape[0] < 2:
        return True
    whole = torch.as_strided(v, (v.shape[0] - 1, v.stride(0)), v.stride(), v.storage_offset())
    return bool(torch.isnan(whole[:, v.shape[1]:]).all())


def final(want, err, dtype):
    return err + (np.abs(want) + err) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)


def check(got, want, err, dtype, what):
    got = f64(got)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    ok = np.isfinite(want)
    bad = np.abs(got - want)[ok] > final(want, err, dtype)[ok]
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.max((np.abs(got - want) / final(want, err, dtype))[ok])}"


def sum_error(a, b):
    """(R + 8) 2^-23 S of a @ b."""
    return (a.shape[1] + 8) * 2.0 ** -23 * (np.abs(a) @ np.abs(b))


def check_ckpt(c, want, err, what):
    """A checkpoint of values within `err` of `want` [rows, cols]: exponents of a value in that range, codes
    rounded within half a step (or held to 127), padding zero."""
    rows, cols = want.shape
    codes, exps = c.codes.cpu().numpy().astype(np.float64), c.exps.cpu().numpy().astype(np.int64)
    pad = (-cols) % 32
    z = np.pad(want, ((0, 0), (0, pad))).reshape(rows, -1, 32)
    d = np.pad(np.broadcast_to(err, want.shape), ((0, 0), (0, pad))).reshape(rows, -1, 32)
    lo_e = lo.ckpt_exponent(np.maximum(np.abs(z) - d, 0).max(axis=2)) + 127
    hi_e = lo.ckpt_exponent((np.abs(z) + d).max(axis=2)) + 127
    assert np.all((exps >= lo_e) & (exps <= hi_e)), what
    step = np.ldexp(1.0, exps - 127)[:, :, None]
    q = codes.reshape(z.shape)
    off = np.abs(q * step - z)
    held = (np.abs(q) == 127) & (np.abs(z) + d >= 127.5 * step)
    assert np.all(off <= np.where(held, step, step / 2) + d), what
    assert not codes[:, cols:].any(), what


# ---------------------------------------------------------------- checkpoints
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 0), (7, 33, 5, 1),
                                                 (130, 257, 1, 3), (64, 1536, 0, 0), (9, 4095, 0, 0), (1, 14336, 0, 1)])
def test_ckpt_write_and_read(dtype, rows, cols, pad, shift):
    gen = torch.Generator(DEV).manual_seed(rows * 1000 + cols)
    x = rand(gen, rows, cols, dtype, 1.0, pad, shift)
    x.mul_(torch.exp2(torch.randint(-30, 30, (rows, 1), generator=gen, device=DEV).float()).to(x.dtype))
    c = smat.ActCheckpoint.empty(rows, cols)
    c.codes.fill_(77)
    smat.smat_ckpt_write(x, c)
    codes, exps = lo.ckpt_write(f64(x))
    assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.exps.cpu().numpy(), exps)
    for out_dtype in ("bf16", "f32"):       # exact in both
        out = rand(gen, rows, cols, out_dtype, 1.0, pad, shift)
        smat.smat_ckpt_read(c, out)
        assert np.array_equal(f64(out), lo.ckpt_read(codes, exps, cols))
        assert untouched(out, pad)


def test_ckpt_edge_values():
    """Zeros, subnormals, the largest and smallest numbers, values held to 127, infinities and NaN."""
    x = torch.zeros(10, 70, device=DEV)
    x[1, 5] = 2.0 ** -140
    x[2, 5] = 2.0 ** -126
    x[3, 5], x[3, 6] = 3.4028234663852886e38, -1.0
    x[4, 40] = float("nan")
    x[5, 0] = float("inf")
    x[6, 69] = -float("inf")
    x[7, 0], x[7, 1] = 1.0 - 2.0 ** -24, 0.5
    x[8, :] = torch.arange(70, device=DEV) - 35.5
    x[9, 3] = 2.0 ** -120
    for dtype in ("f32", "bf16"):
        xs = x.to(DT[dtype])
        c = smat.ActCheckpoint.empty(10, 70)
        smat.smat_ckpt_write(xs, c)
        codes, exps = lo.ckpt_write(f64(xs))
        assert np.array_equal(c.codes.cpu().numpy(), codes) and np.array_equal(c.exps.cpu().numpy(), exps)
        out = torch.empty_like(xs)
        smat.smat_ckpt_read(c, out)
        want = lo.ckpt_read(codes, exps, 70)
        assert np.array_equal(f64(out), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("gated", [False, True])
def test_ckpt_read_recomputes(dtype, act, gated):
    gen = torch.Generator(DEV).manual_seed(5)
    rows, cols = 65, 161
    z, u = rand(gen, rows, cols, "f32", 3.0), rand(gen, rows, cols, "f32")
    z[3, 7], z[4, 8], z[5, 9] = float("nan"), 3e38, -3e38
    cz, cu = smat.ActCheckpoint.empty(rows, cols), smat.ActCheckpoint.empty(rows, cols)
    smat.smat_ckpt_write(z, cz)
    smat.smat_ckpt_write(u, cu)
    out = torch.empty(rows, cols, dtype=DT[dtype], device=DEV)
    smat.smat_ckpt_read(cz, out, act=act, up=cu if gated else None)
    zh = lo.ckpt_read(*lo.ckpt_write(f64(z)), cols)
    uh = lo.ckpt_read(*lo.ckpt_write(f64(u)), cols) if gated else np.ones((rows, cols))
    with np.errstate(over="ignore", invalid="ignore"):
        want = lo.act(zh, act) * uh
    huge = np.abs(zh) > 1e30        # z^3 overflows: only the sign of the limit is asked for
    got = f64(out)
    ok = ~huge & np.isfinite(zh)
    err = (2.0 ** -21 * np.abs(zh * uh))[ok]
    assert np.all(np.abs(got - want)[ok] <= final(want[ok], err, dtype))
    assert np.isnan(got[np.isnan(zh)]).all()
    assert (got[5, 9] == 0 or act == smat.SMAT_ACT_NONE) and not np.isnan(got[huge]).any()


# ---------------------------------------------------------------- the layer
SHAPES = [(1, 1, 1), (1, 32, 64), (1, 768, 768), (2, 40, 257), (3, 1000, 64), (5, 33, 7), (7, 64, 4096), (15, 31, 100),
          (16, 256, 512), (17, 129, 257), (31, 96, 128), (33, 128, 65), (64, 96, 64), (100, 70, 1000), (128, 128, 128),
          (130, 160, 200), (257, 384, 72), (300, 257, 129), (256, 512, 512), (511, 520, 320)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_linear_sizes(dtype, m, n, k):
    gen = torch.Generator(DEV).manual_seed(m * 7919 + n * 31 + k)
    x, w = rand(gen, m, k, dtype), rand(gen, n, k, dtype, 0.1)
    bias, mul, res = rand(gen, 1, n, dtype).view(-1), rand(gen, m, n, dtype), rand(gen, m, n, dtype)
    act = ACTS[(m + n + k) % 4]
    err_z = sum_error(f64(x), f64(w).T) + 2.0 ** -23 * (np.abs(f64(bias)) + np.abs(f64(x)) @ np.abs(f64(w)).T)
    # with everything
    out, c = torch.empty(m, n, dtype=DT[dtype], device=DEV), smat.ActCheckpoint.empty(m, n)
    c.codes.fill_(77)
    smat.smat_linear(x, w, out, bias=bias, act=act, mul=mul, residual=res, z_ckpt=c)
    want, z = lo.linear(f64(x), f64(w), f64(bias), act, f64(mul), f64(res))
    err = (SLOPE * err_z + 2.0 ** -21 * np.abs(z)) * np.abs(f64(mul)) + 2.0 ** -21 * (np.abs(want) + np.abs(f64(res)))
    check(out, want, err, dtype, "all")
    check_ckpt(c, z, err_z, "z")
    # the bare product
    smat.smat_linear(x, w, out)
    check(out, f64(x) @ f64(w).T, err_z, dtype, "bare")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 96, 200), (4, 70, 129), (40, 130, 264), (200, 264, 136), (300, 513, 130)])
@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 1), (5, 2)])
def test_linear_strides_and_alignment(dtype, m, n, k, pad, shift):
    """Row strides and starts on and off a vector's boundary; the NaNs around every matrix stay outside."""
    gen = torch.Generator(DEV).manual_seed(m + n + k + pad + shift)
    x, w = rand(gen, m, k, dtype, 1.0, pad, shift), rand(gen, n, k, dtype, 0.1, pad, shift)
    mul, res = rand(gen, m, n, dtype, 1.0, pad, shift), rand(gen, m, n, dtype, 1.0, pad, shift)
    out = rand(gen, m, n, dtype, 1.0, pad, shift)
    bias = rand(gen, 1, n, dtype, 1.0, 0, shift).view(-1)
    smat.smat_linear(x, w, out, bias=bias, act=smat.SMAT_ACT_SILU, mul=mul, residual=res)
    want, z = lo.linear(f64(x), f64(w), f64(bias), lo.SILU, f64(mul), f64(res))
    err_z = sum_error(f64(x), f64(w).T) + 2.0 ** -22 * (np.abs(f64(bias)) + np.abs(z))
    err = (SLOPE * err_z + 2.0 ** -21 * np.abs(z)) * np.abs(f64(mul)) + 2.0 ** -21 * (np.abs(want) + np.abs(f64(res)))
    check(out, want, err, dtype, "out")
    assert untouched(out, pad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(3, 64, 96), (200, 300, 64)])
def test_linear_in_place_over_residual_and_mul(dtype, m, n, k):
    gen = torch.Generator(DEV).manual_seed(1)
    x, w, res = rand(gen, m, k, dtype), rand(gen, n, k, dtype, 0.1), rand(gen, m, n, dtype)
    apart = torch.empty_like(res)
    smat.smat_linear(x, w, apart, residual=res)
    same = res.clone()
    smat.smat_linear(x, w, same, residual=same)
    assert torch.equal(apart, same)
    smat.smat_linear(x, w, apart, mul=res, act=smat.SMAT_ACT_GELU)
    same = res.clone()
    smat.smat_linear(x, w, same, mul=same, act=smat.SMAT_ACT_GELU)
    assert torch.equal(apart, same)


def test_linear_empty_dimensions():
    x0, w0 = torch.empty(0, 64, device=DEV), torch.ones(32, 64, device=DEV)
    smat.smat_linear(x0, w0, torch.empty(0, 32, device=DEV), z_ckpt=smat.ActCheckpoint.empty(0, 32))
    # an empty sum: out = act(bias) * mul + residual, z = bias
    out, c = torch.empty(5, 33, device=DEV), smat.ActCheckpoint.empty(5, 33)
    bias, res = torch.randn(33, device=DEV), torch.randn(5, 33, device=DEV)
    smat.smat_linear(torch.empty(5, 0, device=DEV), torch.empty(33, 0, device=DEV), out, bias=bias,
                     act=smat.SMAT_ACT_SILU, residual=res, z_ckpt=c)
    z = np.broadcast_to(f64(bias), (5, 33))
    assert np.max(np.abs(f64(out) - lo.act(z, lo.SILU) - f64(res))) < 1e-5
    check_ckpt(c, z, 0.0, "z")
    out = torch.ones(5, 33, device=DEV)
    smat.smat_linear_dgrad(torch.empty(5, 0, device=DEV), torch.empty(0, 33, device=DEV), out)
    assert not out.any()
    dw, db = torch.ones(4, 33, device=DEV), torch.ones(4, device=DEV)
    smat.smat_linear_wgrad(torch.empty(0, 4, device=DEV), torch.empty(0, 33, device=DEV), dw, db=db)
    assert not dw.any() and not db.any()
    smat.smat_linear_wgrad(torch.empty(0, 4, device=DEV), smat.ActCheckpoint.empty(0, 33), dw.fill_(1), db=db.fill_(1))
    assert not dw.any() and not db.any()
    db.fill_(1)
    smat.smat_linear_wgrad(torch.ones(7, 4, device=DEV), torch.empty(7, 0, device=DEV), torch.empty(4, 0, device=DEV), db=db)
    assert (db == 7).all()


@pytest.mark.parametrize("m", [1, 3, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_linear_nonfinite_values_stay_in_their_row_and_column(dtype, m):
    gen = torch.Generator(DEV).manual_seed(2)
    x, w = rand(gen, m, 200, dtype), rand(gen, 150, 200, dtype, 0.1)
    clean = torch.empty(m, 150, dtype=DT[dtype], device=DEV)
    smat.smat_linear(x, w, clean)
    r = m // 2
    x[r, 13] = float("inf")
    w[77, 199] = float("nan")
    out, c = torch.empty_like(clean), smat.ActCheckpoint.empty(m, 150)
    smat.smat_linear(x, w, out, z_ckpt=c)
    assert torch.isnan(out[:, 77]).all()
    keep = torch.ones(m, 150, dtype=torch.bool, device=DEV)
    keep[r], keep[:, 77] = False, False
    assert torch.equal(out[keep], clean[keep])
    assert not torch.isfinite(out[r]).any()
    bad = c.exps == 255
    assert bad[r].all() and bad[:, 77 // 32].all() and bad.sum() == m + 5 - 1


# ---------------------------------------------------------------- the data gradient
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 64, 128), (5, 33, 7), (17, 130, 100), (64, 96, 64), (130, 161, 257),
                                   (257, 384, 72), (300, 520, 130), (256, 256, 512)])
@pytest.mark.parametrize("form", ["plain", "act", "gated", "pair"])
def test_dgrad(dtype, m, n, k, form):
    gen = torch.Generator(DEV).manual_seed(m + n + k)
    pad, shift = (3, 1) if (m + k) % 2 else (0, 0)
    dy, w = rand(gen, m, k, dtype, 1e-2, pad, shift), rand(gen, k, n, dtype, 0.1, pad, shift)
    out, out_up = rand(gen, m, n, dtype, 1.0, pad, shift), rand(gen, m, n, dtype, 1.0, pad, shift)
    kw, args = {}, {}
    err_v = sum_error(f64(dy), f64(w))
    if form == "pair":
        k2 = k + 9
        dy2, w2 = rand(gen, m, k2, dtype, 1e-2), rand(gen, k2, n, dtype, 0.1)
        kw, args = dict(dy2=dy2, w2=w2), dict(dy2=f64(dy2), w2=f64(w2))
        err_v = (k + k2 + 16) * 2.0 ** -23 * (np.abs(f64(dy)) @ np.abs(f64(w)) + np.abs(f64(dy2)) @ np.abs(f64(w2)))
    if form in ("act", "gated"):
        act = ACTS[1 + (m + n + k) % 3]
        cz, zs = smat.ActCheckpoint.empty(m, n), rand(gen, m, n, "f32", 3.0)
        smat.smat_ckpt_write(zs, cz)
        z = lo.ckpt_read(*lo.ckpt_write(f64(zs)), n)
        kw, args = dict(act=act, z_ckpt=cz), dict(kind=act, z=z)
        if form == "gated":
            cu, us = smat.ActCheckpoint.empty(m, n), rand(gen, m, n, "f32")
            smat.smat_ckpt_write(us, cu)
            u = lo.ckpt_read(*lo.ckpt_write(f64(us)), n)
            kw.update(up_ckpt=cu, out_up=out_up)
            args["up"] = u
    smat.smat_linear_dgrad(dy, w, out, **kw)
    want, want_up = lo.dgrad(f64(dy), f64(w), **args)
    v = lo.dgrad(f64(dy), f64(w))[0]
    if form in ("plain", "pair"):
        err = err_v
    else:
        u = args.get("up", 1.0)
        err = np.abs(u) * (SLOPE * err_v + 2.0 ** -20 * np.abs(v)) + 2.0 ** -21 * np.abs(want)
    check(out, want, err, dtype, form)
    assert untouched(out, pad)
    if form == "gated":
        check(out_up, want_up, np.abs(z) * (err_v + 2.0 ** -20 * np.abs(v)), dtype, "up")
        assert untouched(out_up, pad)


def test_dgrad_without_activation_through_a_gate():
    """A bilinear gate: act none with both checkpoints."""
    gen = torch.Generator(DEV).manual_seed(4)
    m, n, k = 33, 70, 40
    dy, w = rand(gen, m, k, "f32"), rand(gen, k, n, "f32")
    cz, cu = smat.ActCheckpoint.empty(m, n), smat.ActCheckpoint.empty(m, n)
    smat.smat_ckpt_write(rand(gen, m, n, "f32"), cz)
    smat.smat_ckpt_write(rand(gen, m, n, "f32"), cu)
    zf, uf = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    smat.smat_ckpt_read(cz, zf)
    smat.smat_ckpt_read(cu, uf)
    out, out_up = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    smat.smat_linear_dgrad(dy, w, out, z_ckpt=cz, up_ckpt=cu, out_up=out_up)
    v = f64(dy) @ f64(w)
    err = sum_error(f64(dy), f64(w))
    check(out, v * f64(uf), err * np.abs(f64(uf)), "f32", "out")
    check(out_up, v * f64(zf), err * np.abs(f64(zf)), "f32", "up")


def test_dgrad_nan_checkpoint_blocks_give_nan_gradients():
    gen = torch.Generator(DEV).manual_seed(4)
    dy, w, zs = rand(gen, 40, 64, "bf16"), rand(gen, 64, 96, "bf16"), rand(gen, 40, 96, "f32")
    zs[7, 33] = float("inf")
    for act in ACTS[1:]:
        cz, out = smat.ActCheckpoint.empty(40, 96), torch.empty(40, 96, dtype=torch.bfloat16, device=DEV)
        smat.smat_ckpt_write(zs, cz)
        smat.smat_linear_dgrad(dy, w, out, act=act, z_ckpt=cz)
        bad = torch.isnan(out)
        assert bad[7, 32:64].all() and bad.sum() == 32


# ---------------------------------------------------------------- the weight gradient
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (2, 64, 33), (17, 130, 100), (64, 64, 64), (129, 96, 257), (300, 257, 130),
                                   (1000, 40, 72), (2500, 136, 264), (512, 256, 512)])
@pytest.mark.parametrize("saved", [False, True])
def test_wgrad(dtype, m, n, k, saved):
    gen = torch.Generator(DEV).manual_seed(m + n + k)
    pad, shift = (3, 1) if (m + k) % 2 else (0, 0)
    dy, x = rand(gen, m, n, dtype, 1e-2, pad, shift), rand(gen, m, k, dtype, 1.0, pad, shift)
    dw, db = rand(gen, n, k, dtype, 1.0, pad, shift), torch.empty(n, dtype=DT[dtype], device=DEV)
    xin, xv = x, f64(x)
    if saved:
        xin = smat.ActCheckpoint.empty(m, k)
        smat.smat_ckpt_write(x, xin)
        xv = lo.ckpt_read(*lo.ckpt_write(xv), k)
    smat.smat_linear_wgrad(dy, xin, dw, db=db)
    want, want_b = lo.wgrad(f64(dy), xv)
    check(dw, want, sum_error(f64(dy).T, xv), dtype, "dw")
    check(db, want_b, (m + 8) * 2.0 ** -23 * np.abs(f64(dy)).sum(axis=0), dtype, "db")
    assert untouched(dw, pad)
    again, againb = torch.empty_like(dw), torch.empty_like(db)
    for _ in range(3):      # the order of the sums is fixed
        smat.smat_linear_wgrad(dy, xin, again, db=againb)
        assert torch.equal(again, dw) and torch.equal(againb, db)


# ---------------------------------------------------------------- size, streams, graphs
def test_offsets_past_32_bits():
    """Rows so far apart that element and byte offsets pass 2^32 in every operand and in the output."""
    gen = torch.Generator(DEV).manual_seed(6)
    ld, m, n, k = (1 << 24) + 8, 300, 264, 136
    buf = torch.empty(m * ld, dtype=torch.bfloat16, device=DEV)     # 10 GB, touched only where the views lie

    def view(rows, cols, at):
        return torch.as_strided(buf, (rows, cols), (ld, 1), at)

    x, w, out, res = view(m, k, 0), view(n, k, 1024), view(m, n, 2048), view(m, n, 4096)
    x.copy_(torch.randn(m, k, generator=gen, device=DEV))
    w.copy_(torch.randn(n, k, generator=gen, device=DEV) * 0.1)
    res.copy_(torch.randn(m, n, generator=gen, device=DEV))
    smat.smat_linear(x, w, out, residual=res)
    want = f64(x) @ f64(w).T + f64(res)
    check(out, want, sum_error(f64(x), f64(w).T) + 2.0 ** -22 * np.abs(f64(res)), "bf16", "linear")
    smat.smat_linear(x[299:], w, out[299:], residual=res[299:])     # a single token's row
    check(out[299:], want[299:], (sum_error(f64(x), f64(w).T) + 2.0 ** -22 * np.abs(f64(res)))[299:], "bf16", "row")
    dx = view(m, k, 8192)
    smat.smat_linear_dgrad(res, w, dx)
    check(dx, f64(res) @ f64(w), sum_error(f64(res), f64(w)), "bf16", "dgrad")
    dw = view(n, k, 16384)
    smat.smat_linear_wgrad(res, x, dw)
    check(dw, f64(res).T @ f64(x), sum_error(f64(res).T, f64(x)), "bf16", "wgrad")
    c = smat.ActCheckpoint.empty(m, k)
    smat.smat_ckpt_write(x, c)
    smat.smat_ckpt_read(c, dx)
    assert np.array_equal(f64(dx), lo.ckpt_read(*lo.ckpt_write(f64(x)), k))


def _all_calls(s, stream=None):
    smat.smat_linear(s["x"], s["w"], s["h"], bias=s["b"], act=smat.SMAT_ACT_GELU, z_ckpt=s["z"], stream=stream)
    smat.smat_linear(s["x"][:1], s["w"], s["h1"], stream=stream)
    smat.smat_ckpt_write(s["x"], s["xc"], stream=stream)
    smat.smat_ckpt_read(s["z"], s["hh"], act=smat.SMAT_ACT_GELU, stream=stream)
    smat.smat_linear_dgrad(s["dy"], s["w2"], s["dz"], act=smat.SMAT_ACT_GELU, z_ckpt=s["z"], stream=stream)
    smat.smat_linear_wgrad(s["dz"], s["xc"], s["dw"], db=s["db"], stream=stream)


def _state(seed, m=600, d=128, f=256):
    gen = torch.Generator(DEV).manual_seed(seed)
    r = lambda a, b: torch.randn(a, b, generator=gen, device=DEV).to(torch.bfloat16)    # noqa: E731
    e = lambda a, b: torch.zeros(a, b, device=DEV, dtype=torch.bfloat16)                # noqa: E731
    return dict(x=r(m, d), w=r(f, d), b=r(1, f).view(-1), h=e(m, f), h1=e(1, f), hh=e(m, f), dz=e(m, f), dy=r(m, d),
                w2=r(d, f), dw=e(f, d), db=e(1, f).view(-1), z=smat.ActCheckpoint.empty(m, f),
                xc=smat.ActCheckpoint.empty(m, d))


OUTS = ("h", "h1", "hh", "dz", "dw", "db")


def test_side_stream_orders_after_its_own_work():
    s, want = _state(1), _state(1)
    _all_calls(want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        big = torch.randn(4096, 4096, device=DEV)
        for _ in range(20):
            big = big @ big * 1e-4
        s["x"].copy_(s["x"] * 1.0)
        _all_calls(s)
    _all_calls(s, stream=stream)        # the same calls given the stream
    torch.cuda.current_stream().wait_stream(stream)
    for name in OUTS:
        assert torch.equal(s[name], want[name]), name


def test_graph_replays():
    s = _state(2)
    _all_calls(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _all_calls(s)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _all_calls(s)
    for seed in range(3, 7):
        fresh = _state(seed)
        for name in ("x", "w", "b", "dy", "w2"):
            s[name].copy_(fresh[name])
        g.replay()
        torch.cuda.synchronize()
        _all_calls(fresh)
        for name in OUTS:
            assert torch.equal(s[name], fresh[name]), (seed, name)


def test_given_workspace_is_used_and_checked():
    dy, x = torch.randn(5000, 40, device=DEV), torch.randn(5000, 72, device=DEV)
    want, dw = torch.empty(40, 72, device=DEV), torch.empty(40, 72, device=DEV)
    smat.smat_linear_wgrad(dy, x, want)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    smat.smat_linear_wgrad(dy, x, dw, workspace=ws)
    assert torch.equal(dw, want)
    with pytest.raises(smat.SmatError):
        smat.smat_linear_wgrad(dy, x, dw, workspace=ws[:64])
    with pytest.raises(smat.SmatError):
        smat.smat_linear_wgrad(dy, x, dw, workspace=ws[8:])
