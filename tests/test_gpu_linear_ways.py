"""Every way in which a product is computed: each tile, with r whole and in ranges, operands copied to LDS directly, packed
first or by way of registers, alone, before left-over rows and as left-over rows.  The sizes are the smallest, of 400,000 drawn
ones, that the choice of tiles sends there.  NaN lies before, between and after the rows of every operand and output, and must
neither come in nor be written over.

Against float64 products on the GPU; bounds as in test_gpu_linear.py: (R + 8) 2^-23 of the sums' magnitudes; SiLU changes by
1.1 times its argument's error and is evaluated within 2^-21 of z (slopes within 2^-20); 2^-8 (bf16) or 2^-22 of the result."""
import pytest
import torch

import paper_2609_33437_amd as smat
from test_gpu_linear_large import SHAPES

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}
SILU = smat.SMAT_ACT_SILU

# m, n, k, whether there is a second product, whether rows lie off 16 bytes, epilogue (linear: all of it; dgrad: 1 through an
# activation, 2 gated)
SIZES = {
    ("dgrad", "f32"): [
        (1, 18, 16, 0, 1, 0), (1, 20, 20, 0, 0, 0), (1, 22, 384, 1, 1, 1), (1, 20, 1060, 0, 0, 1), (1, 16, 12110, 1, 0, 2),
        (24, 10176, 16, 0, 0, 2), (22, 12320, 16, 0, 1, 0), (51, 14262, 16, 0, 0, 2), (2096, 480, 16, 0, 0, 1), (68, 10376,
        16, 1, 0, 2), (6964, 35, 192, 0, 0, 0), (67, 11488, 128, 0, 0, 1), (6062, 36, 576, 0, 0, 0), (6656, 37, 256, 1, 0,
        0), (4960, 1690, 16, 0, 1, 0), (4352, 1952, 16, 0, 0, 1), (6816, 18, 1184, 0, 0, 1), (49, 7488, 416, 0, 1, 1),
        (2005, 4352, 18, 0, 0, 2), (33, 8507, 322, 1, 0, 1), (1247, 7928, 20, 0, 0, 0), (800, 1600, 386, 0, 0, 0), (6127,
        1632, 37, 1, 0, 1), (1824, 160, 2588, 0, 0, 2), (7392, 131, 864, 0, 0, 0), (2752, 69, 5216, 0, 0, 0), (4343, 288,
        864, 0, 0, 1), (2144, 13632, 19, 1, 0, 2), (4352, 4128, 34, 1, 1, 2), (6240, 12489, 16, 0, 1, 2), (928, 329, 5472,
        0, 0, 0), (768, 11680, 192, 0, 0, 0)],
    ("dgrad", "bf16"): [
        (1, 17, 17, 0, 1, 0), (1, 64, 24, 0, 0, 2), (1, 17, 1568, 0, 0, 0), (1, 32, 576, 1, 0, 0), (1, 24, 3392, 0, 0, 0),
        (2, 32, 1472, 0, 0, 1), (17, 12320, 18, 0, 1, 2), (20, 12333, 16, 0, 1, 0), (4810, 71, 18, 0, 1, 1), (53, 8896, 16,
        0, 0, 2), (160, 6176, 24, 0, 0, 1), (21, 12948, 138, 1, 0, 0), (544, 13274, 16, 0, 0, 0), (149, 6112, 71, 1, 0, 0),
        (1472, 5600, 16, 0, 1, 2), (3160, 2593, 18, 0, 1, 1), (6636, 1344, 17, 0, 1, 1), (86, 11520, 96, 1, 0, 1), (1850,
        8832, 16, 0, 0, 2), (1724, 6624, 24, 0, 0, 1), (4157, 16, 2144, 1, 0, 2), (4064, 4463, 17, 0, 0, 0), (5285, 1600,
        21, 1, 1, 1), (2240, 33, 4864, 0, 0, 1), (3968, 35, 2656, 0, 0, 0), (743, 10912, 24, 1, 0, 1), (83, 10720, 250, 1,
        0, 0), (544, 13760, 64, 0, 0, 2), (1600, 37, 8256, 0, 0, 1), (96, 14176, 437, 0, 0, 1), (1696, 744, 480, 0, 0, 0),
        (1568, 5152, 96, 0, 0, 1), (150, 6016, 960, 0, 0, 0), (67, 2080, 3587, 1, 0, 2), (983, 10752, 72, 1, 0, 2), (592,
        13792, 219, 0, 0, 2), (1120, 9372, 480, 0, 0, 2), (134, 11424, 4835, 0, 0, 2), (142, 11264, 4768, 0, 0, 0), (4126,
        957, 2013, 0, 0, 0), (3344, 5376, 224, 1, 0, 0), (1664, 2543, 2112, 0, 1, 1), (6556, 1433, 1187, 0, 0, 1), (545,
        14309, 738, 1, 0, 1), (5472, 768, 3008, 0, 0, 0), (1186, 8160, 1600, 0, 0, 1), (2976, 6784, 2089, 0, 1, 1), (2456,
        3264, 6388, 0, 0, 2), (864, 11264, 2880, 1, 0, 2)],
    ("linear", "f32"): [
        (1, 18, 17, 0, 0, 0), (9, 18, 17, 0, 0, 0), (10, 22, 16, 0, 0, 1), (9, 17, 713, 0, 0, 0), (10, 26, 800, 0, 0, 0),
        (5218, 38, 16, 0, 0, 1), (22, 13333, 18, 0, 1, 0), (146, 5152, 18, 0, 0, 1), (86, 9021, 20, 0, 0, 1), (5824, 145,
        36, 0, 0, 1), (37, 9440, 165, 0, 1, 1), (79, 9129, 128, 0, 0, 1), (6208, 38, 512, 0, 0, 0), (566, 14058, 19, 0, 1,
        1), (1427, 5984, 18, 0, 1, 0), (1824, 6362, 16, 0, 0, 0), (801, 9787, 24, 0, 0, 0), (57, 7430, 448, 0, 1, 1), (6688,
        35, 885, 0, 1, 0), (849, 541, 512, 0, 1, 1), (263, 734, 1574, 0, 1, 0), (1856, 153, 2880, 0, 0, 1), (7014, 192, 608,
        0, 0, 0), (3616, 288, 819, 0, 1, 0), (878, 10193, 102, 0, 0, 0), (2752, 12768, 33, 0, 0, 0), (5440, 12675, 17, 0, 1,
        0), (763, 11622, 140, 0, 0, 1), (7751, 295, 960, 0, 1, 0), (5536, 3168, 133, 0, 0, 1), (646, 416, 11904, 0, 1, 0),
        (2985, 1031, 1408, 0, 1, 1)],
    ("linear", "bf16"): [
        (1, 18, 17, 0, 0, 0), (9, 17, 16, 0, 1, 1), (11, 22, 16, 0, 0, 0), (9, 17, 1557, 0, 0, 1), (9, 17, 2656, 0, 0, 0),
        (22, 10016, 16, 0, 0, 0), (18, 13216, 17, 0, 0, 1), (4768, 67, 16, 0, 0, 1), (21, 12384, 20, 0, 0, 0), (4128, 70,
        19, 0, 0, 1), (96, 8238, 16, 0, 0, 0), (19, 12928, 257, 0, 0, 1), (832, 9536, 16, 0, 1, 0), (576, 13632, 18, 0, 0,
        1), (6240, 1440, 16, 0, 0, 0), (5096, 1568, 18, 0, 1, 1), (3305, 2474, 18, 0, 0, 1), (832, 39, 4576, 0, 0, 1), (544,
        13805, 20, 0, 1, 1), (2304, 4224, 16, 0, 0, 1), (5632, 146, 224, 0, 0, 1), (928, 12352, 17, 0, 0, 1), (2625, 6752,
        16, 0, 1, 1), (936, 8704, 40, 0, 0, 1), (85, 9076, 480, 0, 0, 0), (2944, 7936, 16, 0, 0, 1), (2816, 38, 3584, 0, 0,
        1), (2368, 3392, 64, 0, 0, 1), (790, 10272, 64, 0, 0, 1), (150, 5822, 928, 0, 0, 1), (1568, 928, 583, 0, 0, 0),
        (1061, 8787, 209, 0, 0, 1), (3840, 2592, 232, 0, 0, 1), (832, 12736, 448, 0, 1, 1), (1056, 9887, 507, 0, 0, 1),
        (142, 13013, 3744, 0, 0, 1), (1344, 3016, 1812, 0, 0, 0), (4611, 2400, 736, 0, 0, 1), (2440, 1664, 2176, 0, 0, 1),
        (7200, 1131, 1120, 0, 1, 1), (832, 4631, 2468, 0, 0, 1), (1216, 7480, 1235, 0, 0, 1), (3155, 3168, 1168, 0, 0, 1),
        (2048, 2097, 3904, 0, 0, 0), (4160, 4744, 2135, 0, 0, 1), (4463, 2557, 5216, 0, 0, 1)],
    ("wgrad", "f32"): [
        (20, 17, 20, 0, 0, 0), (47, 16, 16, 0, 0, 0), (672, 18, 16, 0, 1, 0), (1120, 16, 24, 0, 0, 0), (19, 9440, 16, 0, 0,
        0), (19, 18, 12704, 0, 0, 0), (22, 9436, 76, 0, 0, 0), (65, 7936, 33, 0, 0, 0), (176, 7584, 33, 0, 0, 0), (136, 96,
        8512, 0, 0, 0), (114, 2400, 416, 0, 0, 0), (403, 7020, 41, 0, 0, 0), (17, 672, 11015, 0, 1, 0), (576, 36, 6912, 0,
        0, 0), (16, 6036, 1568, 0, 0, 0), (17, 8192, 1089, 0, 1, 0), (18, 6912, 1280, 0, 0, 0), (595, 7904, 35, 0, 0, 0),
        (33, 576, 13120, 0, 1, 0), (672, 2793, 160, 0, 0, 0), (369, 147, 6172, 0, 0, 0), (7490, 832, 89, 0, 0, 0), (2008,
        160, 1888, 0, 0, 0), (512, 1152, 1216, 0, 0, 0), (418, 13984, 142, 0, 0, 0), (768, 3296, 390, 0, 0, 0), (105, 9735,
        992, 0, 0, 0), (1376, 11232, 71, 0, 0, 0), (33, 4160, 8316, 0, 1, 0), (4704, 141, 1956, 0, 0, 0), (187, 3720, 2372,
        0, 0, 0), (148, 1760, 9664, 0, 1, 0)],
    ("wgrad", "bf16"): [
        (16, 16, 20, 0, 0, 0), (18, 24, 16, 0, 0, 0), (992, 18, 17, 0, 0, 0), (992, 16, 64, 0, 0, 0), (16, 12512, 16, 0, 1,
        0), (26, 8992, 16, 0, 0, 0), (22, 4576, 48, 0, 0, 0), (5120, 16, 96, 0, 0, 0), (65, 6221, 34, 0, 0, 0), (17, 8768,
        96, 0, 0, 0), (76, 13952, 17, 0, 0, 0), (348, 17, 12972, 0, 0, 0), (192, 8896, 71, 0, 0, 0), (1041, 17, 7136, 0, 0,
        0), (17, 13888, 537, 0, 0, 0), (17, 1600, 5016, 0, 0, 0), (4189, 1280, 34, 0, 0, 0), (3104, 4512, 16, 0, 0, 0),
        (2516, 2720, 34, 0, 0, 0), (347, 66, 10816, 0, 0, 0), (17, 13287, 1161, 0, 0, 0), (16, 5120, 3216, 0, 1, 0), (16,
        4116, 4064, 0, 1, 0), (16, 2193, 7694, 0, 1, 0), (17, 4864, 3344, 0, 0, 0), (16, 10816, 1696, 0, 0, 0), (358, 3328,
        288, 0, 0, 0), (7472, 3488, 17, 0, 0, 0), (2944, 8224, 19, 0, 0, 0), (31, 5024, 3264, 0, 0, 0), (1152, 66, 8320, 0,
        0, 0), (39, 5952, 2784, 0, 0, 0), (800, 96, 8624, 0, 0, 0), (970, 96, 9248, 0, 0, 0), (432, 7392, 1026, 0, 1, 0),
        (480, 4896, 1792, 0, 0, 0), (326, 11136, 1593, 0, 0, 0), (325, 9440, 1888, 0, 0, 0), (5212, 139, 8512, 0, 0, 0),
        (1730, 4669, 896, 0, 0, 0), (2432, 448, 8608, 0, 0, 0), (2677, 3008, 1376, 0, 0, 0), (3050, 1464, 2720, 0, 1, 0),
        (2912, 4672, 928, 0, 1, 0), (832, 8224, 1952, 0, 0, 0), (3125, 1632, 2688, 0, 0, 0), (802, 1615, 10624, 0, 1, 0),
        (2016, 1024, 9088, 0, 0, 0), (5408, 2612, 1553, 0, 1, 0), (2560, 4145, 4672, 0, 0, 0), (2688, 3264, 6048, 0, 0, 0)],
}
CASES = [(op, dtype, *size) for (op, dtype), sizes in SIZES.items() for size in sizes]


def view(gen, rows, cols, dtype, off, std=1.0):
    pad, shift = (3, 1) if off else (8, 8)
    buf = torch.full((rows * (cols + pad) + shift + 64,), float("nan"), dtype=DT[dtype], device=DEV)
    v = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    if std:
        v.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * std)
    return v, buf


def check(got, want, err, dtype, what):
    bad = ~((got.double() - want).abs() <= err + (want.abs() + err) * U[dtype])       # true for a NaN
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()}, first {bad.nonzero()[0].tolist()}"


def outside_untouched(v, buf):
    mask = torch.zeros(buf.numel(), dtype=torch.bool, device=DEV)
    torch.as_strided(mask, v.shape, v.stride(), v.storage_offset()).fill_(True)
    assert torch.isnan(buf[~mask]).all()


def silu(z):
    g = torch.sigmoid(z)
    return z * g, g + z * g * (1 - g)


def checkpoint(gen, rows, cols, std):
    c, values = smat.ActCheckpoint.empty(rows, cols), torch.empty(rows, cols, device=DEV)
    smat.smat_ckpt_write(torch.randn(rows, cols, generator=gen, device=DEV) * std, c)
    smat.smat_ckpt_read(c, values)
    return c, values.double()


@pytest.mark.parametrize("op,dtype,m,n,k,pair,off,epilogue", CASES)
def test_every_way(op, dtype, m, n, k, pair, off, epilogue):
    gen = torch.Generator(DEV).manual_seed(m + 3 * n + 7 * k)
    a = lambda rows, cols, std=1.0: view(gen, rows, cols, dtype, off, std)        # noqa: E731
    if op == "linear":
        x, w, (out, buf) = a(m, k)[0], a(n, k, 0.1)[0], a(m, n, 0)
        z, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
        if not epilogue:
            smat.smat_linear(x, w, out)
            check(out, z, (k + 8) * 2.0 ** -23 * mag, dtype, "out")
        else:
            bias, mul, res = a(1, n)[0].view(-1), a(m, n)[0], a(m, n)[0]
            c = smat.ActCheckpoint.empty(m, n)
            c.codes.fill_(77)
            smat.smat_linear(x, w, out, bias=bias, act=SILU, mul=mul, residual=res, z_ckpt=c)
            z, mag = z + bias.double(), mag + bias.double().abs()
            z_err = (k + 9) * 2.0 ** -23 * mag
            want = silu(z)[0] * mul.double() + res.double()
            err = (1.1 * z_err + 2.0 ** -21 * z.abs()) * mul.double().abs() + 2.0 ** -21 * (want.abs() + res.double().abs())
            check(out, want, err, dtype, "out")
            back = torch.empty(m, n, device=DEV)
            smat.smat_ckpt_read(c, back)
            step = torch.exp2(c.exps.double() - 127).repeat_interleave(32, dim=1)[:, :n]
            held = c.codes[:, :n].abs() == 127
            assert bool(((back.double() - z).abs() <= torch.where(held, step, step / 2) + z_err).all())
            top = torch.nn.functional.pad(z.abs(), (0, -n % 32)).view(m, -1, 32).amax(2)
            off_by = torch.nn.functional.pad(z_err, (0, -n % 32)).view(m, -1, 32).amax(2)
            for edge, sign in ((top - off_by).clamp(min=0), 1), (top + off_by, -1):       # the exponent of a maximum in that range
                e = (torch.frexp(edge)[1].double() - 7).clamp(min=-126) + 127
                assert bool((sign * (c.exps.double() - e) >= 0).all())
            assert not c.codes[:, n:].any()
    elif op == "dgrad":
        dy, w, (out, buf) = a(m, k)[0], a(k, n, 0.1)[0], a(m, n, 0)
        v, mag, kw = dy.double() @ w.double(), dy.double().abs() @ w.double().abs(), {}
        if pair:
            dy2, w2 = a(m, k)[0], a(k, n, 0.1)[0]
            v, mag, kw = v + dy2.double() @ w2.double(), mag + dy2.double().abs() @ w2.double().abs(), dict(dy2=dy2, w2=w2)
        err = ((1 + pair) * k + 8) * 2.0 ** -23 * mag
        want = v
        if epilogue:
            cz, z = checkpoint(gen, m, n, 2.0)
            kw.update(act=SILU, z_ckpt=cz)
            value, slope = silu(z)
            u = torch.ones_like(z)
        if epilogue == 2:
            cu, u = checkpoint(gen, m, n, 1.0)
            up, up_buf = a(m, n, 0)
            kw.update(up_ckpt=cu, out_up=up)
        smat.smat_linear_dgrad(dy, w, out, **kw)
        if epilogue:
            want = v * slope * u
            err_out = u.abs() * (1.1 * err + 2.0 ** -20 * v.abs()) + 2.0 ** -21 * want.abs()
            if epilogue == 2:
                check(up, v * value, z.abs() * (err + 2.0 ** -20 * v.abs()), dtype, "up")
                outside_untouched(up, up_buf)
        check(out, want, err_out if epilogue else err, dtype, "out")
    else:
        dy, x, (out, buf) = a(m, n)[0], a(m, k)[0], a(n, k, 0)
        db = torch.full((n,), float("nan"), dtype=DT[dtype], device=DEV)
        smat.smat_linear_wgrad(dy, x, out, db=db)
        check(out, dy.double().t() @ x.double(), (m + 8) * 2.0 ** -23 * (dy.double().abs().t() @ x.double().abs()), dtype, "dw")
        check(db, dy.double().sum(0), (m + 8) * 2.0 ** -23 * dy.double().abs().sum(0), dtype, "db")
    outside_untouched(out, buf)


# the output layer of a decoder with 128,256 words, at a single token, a few and a batch, with its gradients
@pytest.mark.parametrize("m", [1, 5, 64, 515])
def test_vocabulary_wide(m):
    gen = torch.Generator(DEV).manual_seed(m)
    n, k = 128256, 256
    x, w, (out, buf) = view(gen, m, k, "bf16", 0)[0], view(gen, n, k, "bf16", 0, 0.1)[0], view(gen, m, n, "bf16", 0, 0)
    smat.smat_linear(x, w, out)
    check(out, x.double() @ w.double().t(), (k + 8) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t()), "bf16", "logits")
    outside_untouched(out, buf)
    dy = view(gen, m, n, "bf16", 0, 1e-3)[0]
    dx, dw = torch.empty(m, k, dtype=torch.bfloat16, device=DEV), torch.empty(n, k, dtype=torch.bfloat16, device=DEV)
    smat.smat_linear_dgrad(dy, w, dx)
    check(dx, dy.double() @ w.double(), (n + 8) * 2.0 ** -23 * (dy.double().abs() @ w.double().abs()), "bf16", "dx")
    smat.smat_linear_wgrad(dy, x, dw)
    check(dw, dy.double().t() @ x.double(), (m + 8) * 2.0 ** -23 * (dy.double().abs().t() @ x.double().abs()), "bf16", "dw")


@pytest.mark.parametrize("m,n,k", [(32, 4096, 14336), (32, 14336, 4096), (40, 2048, 2048)])
def test_narrow_tiles_of_a_data_gradient(m, n, k):
    """W read along its rows by few rows of dy: the tile that the choice takes for whole cache lines."""
    test_every_way("dgrad", "bf16", m, n, k, 0, 0, 0)
    test_every_way("dgrad", "bf16", m, n, k, 0, 0, 2)


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("op", ["linear", "dgrad", "wgrad"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_ones(op, m, n, k, dtype):
    """The sizes of test_gpu_linear_large.py, whose comparison lets a NaN pass."""
    if dtype == "f32" and m * n * k > 2e10:
        pytest.skip("fp32 has the same launches at the smaller sizes")
    if op == "wgrad":
        m, n, k = k, m, n
    test_every_way(op, dtype, m, n, k, 0, 0, {"linear": 1, "dgrad": 2, "wgrad": 0}[op])


def test_the_check_sees_nan():
    want = torch.zeros(3, 4, dtype=torch.float64, device=DEV)
    got = torch.zeros(3, 4, device=DEV)
    got[1, 2] = float("nan")
    with pytest.raises(AssertionError, match="1 of 12"):
        check(got, want, 1.0 + want, "f32", "planted")
