"""The masked layers' products in 8-bit floating point against the oracle: copies code for code, products on
data whose sums are exact in fp32, and on normal data within what rounding allows."""
import numpy as np
import pytest

from oracle import fp8_oracle as O
from test_checkpoint_gpu import on_gpu, roi  # noqa: F401  (roi: the fixture)

pytestmark = pytest.mark.gpu

EPS = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": 2.0 ** -24}
TINY = {"bfloat16": 2.0 ** -134, "float16": 2.0 ** -25, "float32": 2.0 ** -150}  # half of the least number


def values(rows, cols, dtype, seed):
    """Values of that type (as float64) of a spread of magnitudes, with rows and columns that stand out."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))
    x[:, ::17] *= 30
    x[::5] *= 2.0 ** -9
    if rows > 6:
        x[6] = 0
    return x.to(getattr(torch, dtype))


def copy_of(roi, x, fmt):  # noqa: F811
    c = [t.fill_(0xA5) for t in roi.new_fp8(*x.shape)]
    roi.roi_fp8_save(x, fmt, *c)
    return c


def weight_of(roi, W):  # noqa: F811
    c = [t.fill_(0xA5) for t in roi.new_fp8_weight(*W.shape)]
    roi.roi_fp8_save_weight(W, *c)
    return c


SHAPES = [(1, 1), (1, 128), (3, 130), (37, 896), (129, 2049), (64, 2048), (200, 333), (7, 4864), (65, 8)]


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_save(roi, rows, cols, dtype, fmt):  # noqa: F811
    x = values(rows, cols, dtype, rows + cols)
    codes, scales, _ = O.save(x.double().numpy(), fmt)
    for gap in (0, 8, 3):
        got = copy_of(roi, on_gpu(x, dtype, gap), fmt)
        assert np.array_equal(got[1].cpu().numpy(), scales), gap
        assert np.array_equal(got[0].cpu().numpy(), codes), gap


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_save_borders(roi, fmt):  # noqa: F811
    """Largest magnitudes at and next to a power of two's border, ties, subnormals, infinities and NaN."""
    import torch
    top = O.FORMATS[fmt][0]
    x = torch.zeros(40, 256)
    for i in range(24):
        e = 2.0 ** (5 * i - 60)
        border = torch.tensor(top * e)
        x[i, 0] = border if i % 3 == 0 else torch.nextafter(border, torch.tensor(float("inf") if i % 3 == 1 else 0.0))
        # halves between neighbours, and what lies under the least code
        x[i, 1:128] = torch.arange(1, 128) * (e * 2.0 ** (-10 if fmt == "e4m3" else -17))
        x[i, 128:256] = -torch.linspace(0.5, 33, 128) * e
    x[24, 3], x[25, 200], x[26, 7], x[27, 9] = float("inf"), float("-inf"), float("nan"), 3.4e38
    x[28] = 2.0 ** -149
    x[29, :5] = torch.tensor([2.0 ** -126, -(2.0 ** -127), 2.0 ** -130, 0.0, -0.0])
    x[30] = -0.0
    codes, scales, _ = O.save(x.double().numpy(), fmt)
    got = copy_of(roi, x.cuda(), fmt)
    assert np.array_equal(got[1].cpu().numpy(), scales)
    assert np.array_equal(got[0].cpu().numpy(), codes)
    x16 = torch.zeros(4, 130, dtype=torch.float16)
    x16[0], x16[1, 129], x16[2, 0] = 65504, float("inf"), 6e-8
    codes, scales, _ = O.save(x16.double().numpy(), fmt)
    got = copy_of(roi, x16.cuda(), fmt)
    assert np.array_equal(got[1].cpu().numpy(), scales) and np.array_equal(got[0].cpu().numpy(), codes)


@pytest.mark.parametrize("rows,cols", [(1, 1), (128, 128), (129, 130), (300, 896), (127, 2049), (260, 333), (5, 4104)])
def test_save_weight(roi, rows, cols):  # noqa: F811
    W = values(rows, cols, "bfloat16", 9)
    if rows > 200:
        W[201, 129] = float("nan")
        W[10, 5] = float("inf")
    codes, scales, _ = O.save(W.double().numpy(), "e4m3", 128)
    got = weight_of(roi, W.cuda())
    assert np.array_equal(got[1].cpu().numpy(), scales)
    assert np.array_equal(got[0].cpu().numpy(), codes)


def product(roi, way, x, fmt, W, dtype, gap=0):  # noqa: F811
    """(the kernel's output in float64, the same product of the copies' values, the sums of the magnitudes)."""
    import torch
    x8, w8 = copy_of(roi, x, fmt), weight_of(roi, W)
    xv = torch.from_numpy(O.load(x8[0].cpu().numpy(), x8[1].cpu().numpy(), fmt, x.shape[1]))
    wv = torch.from_numpy(O.load(w8[0].cpu().numpy(), w8[1].cpu().numpy(), "e4m3", W.shape[1], 128))
    wv = wv.T if way == "fwd" else wv
    T, outs = x.shape[0], wv.shape[1]
    whole = torch.full((T, outs + gap), 77.0, dtype=getattr(torch, dtype), device="cuda")
    out = whole[:, :outs]
    getattr(roi, f"roi_fp8_linear_{way}")(x8, fmt, w8, out)
    roi.roi_device_status()
    assert (whole[:, outs:] == 77).all(), "written between the rows"
    return out.double().cpu(), xv @ wv, xv.abs() @ wv.abs()


# (tokens, outputs, width of the sum): one tile and parts of tiles, ranges of the sum in a cluster of every size, several
# tiles of tokens, sums that end inside a block, more blocks than one word of scales
SIZES = [(1, 1, 1), (1, 128, 128), (16, 128, 512), (17, 130, 640), (37, 128, 896), (100, 257, 1000), (256, 384, 1152), (257, 100, 300),
         (300, 640, 130), (1, 2000, 2560), (64, 33, 5000), (600, 1000, 777), (130, 19500, 257), (700, 3000, 900), (2050, 1121, 400),
         (300, 5000, 2500), (10000, 100, 130), (1537, 2001, 4200)]


@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("T,outs,width", SIZES)
def test_exact_sums(roi, way, T, outs, width):  # noqa: F811
    """Small whole numbers times powers of two that change from block to block: every sum is exact in fp32, whatever
    the order (multiples of 2^-8 below 2^16), so that one scale or code out of its place shows."""
    import torch
    g = torch.Generator().manual_seed(T + outs + width)
    x = torch.randint(-3, 4, (T, width), generator=g).float()
    W = torch.randint(-2, 3, (outs, width) if way == "fwd" else (width, outs), generator=g).float()
    # a block's largest code is no multiple of the power of two alone: it holds 7 or 14 of them
    xe = torch.randint(-2, 2, (T, (width + 127) // 128), generator=g).repeat_interleave(128, 1)[:, :width]
    rows, cols = W.shape
    we = torch.randint(-2, 2, ((rows + 127) // 128, (cols + 127) // 128), generator=g)
    we = we.repeat_interleave(128, 0).repeat_interleave(128, 1)[:rows, :cols]
    x, W = x * torch.exp2(xe.float()), W * torch.exp2(we.float())
    got, want, sums = product(roi, way, x.cuda(), "e4m3", W.to(torch.bfloat16).cuda(), "float32")
    assert float(sums.max()) < 2 ** 16
    assert torch.equal(got, want)


@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("dtype,fmt,gap", [("bfloat16", "e4m3", 0), ("float16", "e5m2", 3), ("float32", "e5m2", 0), ("float32", "e4m3", 8)])
@pytest.mark.parametrize("T,outs,width", SIZES)
def test_products(roi, way, dtype, fmt, gap, T, outs, width):  # noqa: F811
    """Sums in fp32 of exact products: a step of 32 products drops less than a unit of 2^-23 of the sum of
    magnitudes at each of its additions (32 and the one to the sum), joined ranges 8 more, and the result is
    rounded once."""
    import torch
    x = values(T, width, dtype, 1)
    W = 0.02 * values(*((outs, width) if way == "fwd" else (width, outs)), "bfloat16", 2)
    got, want, sums = product(roi, way, on_gpu(x, dtype, gap), fmt, W.cuda(), dtype, gap)
    steps = (width + 31) // 32
    tol = sums * (steps + 32 + 8) * 2.0 ** -23
    if dtype == "float16":
        keep = want.abs() < 65000
        assert keep.float().mean() > 0.9
        got, want, tol = got[keep], want[keep], tol[keep]
    tol = tol + (want.abs() + tol) * EPS[dtype] + TINY[dtype]
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("T", [3, 300])
def test_blocks_that_are_not_finite(roi, way, T):  # noqa: F811
    """They make NaN of the sums that they are part of, and of no other."""
    import torch
    rows, cols = 300, 400
    x = values(T, cols if way == "fwd" else rows, "bfloat16", 3).cuda()
    W = values(rows, cols, "bfloat16", 4).cuda()
    x[1, 130], W[140, 260] = float("inf"), float("nan")
    got, _, _ = product(roi, way, x, "e4m3", W, "float32")
    bad = torch.zeros(T, rows if way == "fwd" else cols, dtype=torch.bool)
    bad[1] = True
    bad[:, 128:256 if way == "fwd" else 128] = True
    if way == "dgrad":
        bad[:, 256:384] = True
    assert torch.equal(torch.isnan(got), bad)


def test_empty(roi):  # noqa: F811
    """No tokens, no outputs: nothing; a gradient over no outputs: zeros."""
    import torch
    e = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")  # noqa: E731
    roi.roi_fp8_save(torch.empty(0, 40, device="cuda"), "e4m3", *roi.new_fp8(0, 40))
    roi.roi_fp8_linear_fwd(roi.new_fp8(0, 128), "e4m3", roi.new_fp8_weight(16, 128), torch.empty(0, 16, device="cuda"))
    roi.roi_fp8_linear_fwd(roi.new_fp8(4, 128), "e4m3", (e(0, 128), e(0, 16)), torch.empty(4, 0, device="cuda"))
    dx = torch.full((5, 43), 3.0, device="cuda")
    roi.roi_fp8_linear_dgrad((e(5, 0), e(5, 0)), "e5m2", (e(0, 128), e(0, 16)), dx[:, :40])
    roi.roi_device_status()
    assert not dx[:, :40].any() and (dx[:, 40:] == 3).all()


def test_slices_of_a_copy(roi):  # noqa: F811
    """Rows of an activation's copy and 128s of a weight's rows by themselves give the same bits."""
    import torch
    x, W = values(300, 500, "bfloat16", 5).cuda(), values(384, 500, "bfloat16", 6).cuda()
    x8, w8 = copy_of(roi, x, "e4m3"), weight_of(roi, W)
    part = (w8[0][128:256], w8[1][1:2])
    rows = (x8[0][40:141], x8[1][40:141])
    assert torch.equal(copy_of(roi, x[40:141], "e4m3")[0], rows[0])
    a, b = torch.empty(101, 128, device="cuda"), torch.empty(101, 128, device="cuda")
    roi.roi_fp8_linear_fwd(rows, "e4m3", part, a)
    roi.roi_fp8_linear_fwd(tuple(copy_of(roi, x[40:141], "e4m3")), "e4m3", tuple(weight_of(roi, W[128:256].contiguous())), b)
    roi.roi_device_status()
    assert torch.equal(a, b)


@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("T,outs", [(1, 256), (40, 3000), (250, 2000), (900, 1024)])
def test_long_sums_in_fp32(roi, way, T, outs):  # noqa: F811
    """A sum's error grows with its steps: in pieces of 16 blocks, which are rounded when they are added, it is a fraction
    of the 1.4e-6 of the norm that 148 blocks unbroken come to: (16 / 148) of it for the pieces and ten roundings of 2^-24
    at most, 7.5e-7 in all if they all went one way."""
    import torch
    width = 18944
    g = torch.Generator("cuda").manual_seed(T)
    x = torch.randn(T, width, device="cuda", generator=g)
    W = torch.randn(*((outs, width) if way == "fwd" else (width, outs)), device="cuda", generator=g).bfloat16()
    got, want, _ = product(roi, way, x, "e4m3", W, "float32")
    assert float((got - want).norm()) <= 7.5e-7 * float(want.norm())
