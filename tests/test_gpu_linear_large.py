"""The linear-layer products at sizes that take every tile, ranges of r, copies on 16-byte rows and launches of
left-over rows, against float64 products on the GPU.  Bounds as in test_gpu_linear.py: (R + 8) 2^-23 of the sums'
magnitudes, 2^-8 (bf16) or 2^-22 of the result."""
import pytest
import torch

import paper_2609_33437_amd as smat

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}


def rand(gen, rows, cols, dtype, std=1.0):
    return (torch.randn(rows, cols, generator=gen, device=DEV) * std).to(DT[dtype])


def check(got, want, mag, r, dtype, what):
    err = (r + 8) * 2.0 ** -23 * mag
    bad = (got.double() - want).abs() > err + (want.abs() + err) * U[dtype]
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0].tolist()}"


def silu_bound(v, z_err):
    return 1.13 * z_err + 2.0 ** -20 * v.abs()


SHAPES = [
    # m, n, k: few rows up to the vector units' form and just past it
    (8, 1000, 4096), (9, 1000, 4096), (5, 8200, 520), (7, 33, 14336), (33, 4096, 768),
    # narrow and short tiles, long r
    (64, 960, 960), (96, 96, 8192), (90, 961, 4095), (300, 512, 4096), (17, 17, 20000),
    # middle tiles, ragged ends, left-over rows
    (512, 2048, 2048), (1000, 2000, 2000), (1001, 2001, 2001), (2056, 4096, 1024), (2055, 4095, 1023), (1999, 2048, 257),
    (640, 8960, 1536),
    # large tiles, rounds and left-over rows, ranges of r
    (4096, 4096, 768), (4100, 8960, 1536), (4096, 2048, 8192), (2049, 14336, 520), (3333, 5001, 1111),
]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("op", ["linear", "dgrad", "wgrad"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products(op, m, n, k, dtype):
    if dtype == "f32" and m * n * k > 2e10:
        pytest.skip("fp32 has the same launches at the smaller sizes")
    gen = torch.Generator(DEV).manual_seed(m + 3 * n + 7 * k)
    if op == "linear":
        x, w = rand(gen, m, k, dtype), rand(gen, n, k, dtype, 0.1)
        bias, mul, res = rand(gen, 1, n, dtype).view(-1), rand(gen, m, n, dtype), rand(gen, m, n, dtype)
        out, c = torch.empty(m, n, dtype=DT[dtype], device=DEV), smat.ActCheckpoint.empty(m, n)
        smat.smat_linear(x, w, out, bias=bias, act=smat.SMAT_ACT_SILU, mul=mul, residual=res, z_ckpt=c)
        z = x.double() @ w.double().t() + bias.double()
        mag = x.double().abs() @ w.double().abs().t() + bias.double().abs()
        z_err = (k + 9) * 2.0 ** -23 * mag
        want = z * torch.sigmoid(z) * mul.double() + res.double()
        err = silu_bound(z, z_err) * mul.double().abs() + 2.0 ** -21 * (want.abs() + res.double().abs())
        bad = (out.double() - want).abs() > err + (want.abs() + err) * U[dtype]
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0].tolist()}"
        # the checkpoint reads back within half a step (a whole one where a code is held to 127) of z
        zh = torch.empty(m, n, device=DEV)
        smat.smat_ckpt_read(c, zh)
        step = torch.exp2(c.exps.double() - 127).repeat_interleave(32, dim=1)[:, :n]
        held = c.codes[:, :n].abs() == 127
        assert bool(((zh.double() - z).abs() <= torch.where(held, step, step / 2) + z_err).all())
        top = torch.nn.functional.pad(z.abs(), (0, -n % 32)).view(m, -1, 32).amax(2)
        want_e = torch.floor(torch.log2(top)) - 6 + 127
        near = (torch.log2(top) - torch.round(torch.log2(top))).abs() < 1e-3        # a maximum near a power of two
        assert bool(((c.exps.double() == want_e) | near).all())
    elif op == "dgrad":
        dy, w = rand(gen, m, k, dtype), rand(gen, k, n, dtype, 0.1)
        out = torch.empty(m, n, dtype=DT[dtype], device=DEV)
        smat.smat_linear_dgrad(dy, w, out)
        check(out, dy.double() @ w.double(), dy.double().abs() @ w.double().abs(), k, dtype, op)
    else:
        dy, x = rand(gen, k, m, dtype), rand(gen, k, n, dtype)
        c = smat.ActCheckpoint.empty(k, n)
        smat.smat_ckpt_write(x, c)
        dw, db = torch.empty(m, n, dtype=DT[dtype], device=DEV), torch.empty(m, dtype=DT[dtype], device=DEV)
        smat.smat_linear_wgrad(dy, x, dw, db=db)
        check(dw, dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs(), k, dtype, op)
        check(db, dy.double().sum(0), dy.double().abs().sum(0), k, dtype, "db")
        smat.smat_linear_wgrad(dy, c, dw)
        xh = torch.empty(k, n, device=DEV)
        smat.smat_ckpt_read(c, xh)
        check(dw, dy.double().t() @ xh.double(), dy.double().abs().t() @ xh.double().abs(), k, dtype, "from the checkpoint")


@pytest.mark.parametrize("m,n,k,k2", [(300, 512, 64, 640), (4096, 2048, 1000, 1048), (512, 520, 4096, 72), (1024, 256, 8192, 8192),
                                      (257, 300, 130, 67), (2048, 1024, 3000, 77)])
@pytest.mark.parametrize("gated", [False, True])
def test_two_products_of_different_lengths(m, n, k, k2, gated):
    """The second product begins at any stage of a range; the gated epilogue after left-over rows."""
    gen = torch.Generator(DEV).manual_seed(m + n + k)
    dy, w, dy2, w2 = rand(gen, m, k, "bf16"), rand(gen, k, n, "bf16", 0.1), rand(gen, m, k2, "bf16"), rand(gen, k2, n, "bf16", 0.1)
    out, up = torch.empty(m, n, dtype=torch.bfloat16, device=DEV), torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    v = dy.double() @ w.double() + dy2.double() @ w2.double()
    mag = dy.double().abs() @ w.double().abs() + dy2.double().abs() @ w2.double().abs()
    err = (k + k2 + 16) * 2.0 ** -23 * mag
    if not gated:
        smat.smat_linear_dgrad(dy, w, out, dy2=dy2, w2=w2)
        check(out, v, mag, k + k2, "bf16", "sum")
        return
    cz, cu = smat.ActCheckpoint.empty(m, n), smat.ActCheckpoint.empty(m, n)
    smat.smat_ckpt_write(rand(gen, m, n, "f32", 2.0), cz)
    smat.smat_ckpt_write(rand(gen, m, n, "f32"), cu)
    z, u = torch.empty(m, n, device=DEV), torch.empty(m, n, device=DEV)
    smat.smat_ckpt_read(cz, z)
    smat.smat_ckpt_read(cu, u)
    smat.smat_linear_dgrad(dy, w, out, act=smat.SMAT_ACT_SILU, z_ckpt=cz, up_ckpt=cu, out_up=up, dy2=dy2, w2=w2)
    z, u = z.double(), u.double()
    g = torch.sigmoid(z)
    for got, factor in ((out, u * (g + z * g * (1 - g))), (up, z * g)):
        want = v * factor
        e = (err + v.abs() * 2.0 ** -20) * 1.13 * torch.maximum(u.abs(), z.abs()).clamp(min=1.0)
        bad = (got.double() - want).abs() > e + (want.abs() + e) * U["bf16"]
        assert not bad.any()


def test_row_strides_that_pass_32_bits_with_direct_copies():
    """Rows a million elements apart, still copied to LDS directly: tiles' bases pass 2^32 bytes, their offsets do not."""
    gen = torch.Generator(DEV).manual_seed(9)
    ld, m, n, k = (1 << 20) - 8, 2600, 512, 520
    buf = torch.empty(m * ld, dtype=torch.bfloat16, device=DEV)      # 5.4 GB, touched where the views lie

    def view(rows, cols, at):
        v = torch.as_strided(buf, (rows, cols), (ld, 1), at)
        v.copy_(torch.randn(rows, cols, generator=gen, device=DEV))
        return v

    x, w, dy = view(m, k, 0), view(n, k, 1024), view(m, n, 2048)
    out = torch.as_strided(buf, (m, n), (ld, 1), 4096)
    smat.smat_linear(x, w, out)
    check(out, x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t(), k, "bf16", "linear")
    dx = torch.as_strided(buf, (m, k), (ld, 1), 8192)
    smat.smat_linear_dgrad(dy, w, dx)
    check(dx, dy.double() @ w.double(), dy.double().abs() @ w.double().abs(), n, "bf16", "dgrad")
    dw = torch.empty(n, k, dtype=torch.bfloat16, device=DEV)
    smat.smat_linear_wgrad(dy, x, dw)
    check(dw, dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs(), m, "bf16", "wgrad")


@pytest.mark.parametrize("op", ["linear", "dgrad", "wgrad"])
@pytest.mark.parametrize("m,n,k", [(600, 1000, 2000), (4096, 2048, 8192), (257, 300, 4001), (4100, 8960, 1536)])
def test_same_bits_every_time(op, m, n, k):
    gen = torch.Generator(DEV).manual_seed(10)
    a = rand(gen, *((k, m) if op == "wgrad" else (m, k)), "bf16")
    b = rand(gen, *((n, k) if op == "linear" else (k, n)), "bf16")
    first, again = torch.empty(m, n, dtype=torch.bfloat16, device=DEV), torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    fn = {"linear": smat.smat_linear, "dgrad": smat.smat_linear_dgrad, "wgrad": smat.smat_linear_wgrad}[op]
    fn(a, b, first)
    for _ in range(3):
        fn(a, b, again)
        assert torch.equal(first, again)


def test_nan_outside_the_operands_stays_outside():
    """Direct copies and packed copies read 16 bytes at a time: NaNs between rows and after the last one never show."""
    gen = torch.Generator(DEV).manual_seed(11)
    for m, n, k, pad in ((600, 520, 1032, 8), (600, 520, 1032, 24), (601, 519, 1031, 3), (2100, 1100, 1029, 11)):
        def operand(rows, cols):
            buf = torch.full((rows * (cols + pad) + 64,), float("nan"), dtype=torch.bfloat16, device=DEV)
            v = buf[8:8 + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
            v.copy_(torch.randn(rows, cols, generator=gen, device=DEV))
            return v

        x, w, dy = operand(m, k), operand(n, k), operand(m, n)
        for fn, a, b, shape in ((smat.smat_linear, x, w, (m, n)), (smat.smat_linear_dgrad, dy, w, (m, k)),
                                (smat.smat_linear_wgrad, dy, x, (n, k))):
            out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
            fn(a, b, out)
            assert torch.isfinite(out).all(), (fn.__name__, m, n, k, pad)
