"""The products in 8-bit floating point on every way that the library takes by size: pairs of CTAs with tokens and with outputs in
the lanes, tiles of every width, rows and columns that end inside a tile, and clusters of two to eight CTAs that share a tile's sum."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)
from test_fp8_gpu import EPS, TINY, on_gpu, product, values

pytestmark = pytest.mark.gpu

# (way, tokens, outputs, width, columns between the rows of the result).  With 152 SMs a pair's tiles are, in this order, 224, 192,
# 160, 128, 96 and 64 outputs wide with tokens in the lanes, the last outputs of a row inside a sector; 224, 192, 160, 128, 96 and 64
# tokens with outputs in the lanes.
PAIRS = [("fwd", 1592, 4273, 390, 15), ("fwd", 2000, 4880, 1000, 0), ("fwd", 2479, 2090, 700, 6), ("fwd", 250, 7424, 2622, 0),
         ("fwd", 256, 6520, 2034, 8), ("fwd", 2529, 440, 2681, 8),
         ("dgrad", 2653, 2568, 300, 0), ("dgrad", 2039, 2952, 300, 3), ("fwd", 1601, 3216, 1000, 3), ("fwd", 600, 6784, 386, 1),
         ("dgrad", 256, 4992, 3855, 0), ("dgrad", 300, 3328, 6769, 0)]
# Clusters of two to eight CTAs on such a device, which holds 76, 46, 36, 28, 23, 15 and 15 of them at once (37 tokens are three
# groups of sixteen, which the CTAs of a cluster do not share evenly); then one token, and more groups than CTAs.
CLUSTERS = [(37, 6402, 2451), (37, 4625, 2212), (70, 1538, 1927), (37, 2314, 1803), (37, 2073, 2053), (37, 1567, 2593), (37, 1565, 1941),
            (1, 4800, 1424), (1, 192, 1169), (150, 1200, 2500), (150, 1990, 1300)]
TYPES = ["float32", "bfloat16", "float16"]


def whole_numbers(way, T, outs, width):
    """Small whole numbers times powers of two that change from block to block: products are multiples of 2^-4 and a sum's
    magnitudes stay under 2^16, so that every sum is exact in fp32 whatever its order, and a scale or a code out of
    its place shows.  (Blocks of a weight's rows have scales of their own as well: a tile that lies across two or three of them
    shows whose scale each output has.)"""
    import torch
    g = torch.Generator().manual_seed(T + outs + width)
    x = torch.randint(-3, 4, (T, width), generator=g).float()
    shape = (outs, width) if way == "fwd" else (width, outs)
    W = torch.randint(-2, 3, shape, generator=g).float()
    blocks = lambda n: (n + 127) // 128  # noqa: E731
    xe = torch.randint(-2, 2, (T, blocks(width)), generator=g).repeat_interleave(128, 1)[:, :width]
    we = torch.randint(-2, 2, (blocks(shape[0]), blocks(shape[1])), generator=g)
    we = we.repeat_interleave(128, 0).repeat_interleave(128, 1)[:shape[0], :shape[1]]
    return x * torch.exp2(xe.float()), (W * torch.exp2(we.float())).to(torch.bfloat16)


def check_exact(roi, way, T, outs, width, gap, dtype):  # noqa: F811
    import torch
    x, W = whole_numbers(way, T, outs, width)
    got, want, sums = product(roi, way, x.cuda(), "e4m3", W.cuda(), dtype, gap)
    assert float(sums.max()) < 2 ** 16 and float(want.abs().max()) < 65504
    # one rounding to the type, to the nearest even
    assert torch.equal(got, want.float().to(getattr(torch, dtype)).double())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("way,T,outs,width,gap", PAIRS)
def test_exact_sums_in_pairs(roi, way, T, outs, width, gap, dtype):  # noqa: F811
    check_exact(roi, way, T, outs, width, gap, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("way", ["fwd", "dgrad"])
@pytest.mark.parametrize("T,outs,width", CLUSTERS)
def test_exact_sums_in_clusters(roi, way, T, outs, width, dtype):  # noqa: F811
    check_exact(roi, way, T, outs, width, 0, dtype)


@pytest.mark.parametrize("dtype,fmt", [("bfloat16", "e4m3"), ("float16", "e5m2"), ("float32", "e5m2")])
@pytest.mark.parametrize("way,T,outs,width,gap", PAIRS)
def test_products_in_pairs(roi, way, T, outs, width, gap, dtype, fmt):  # noqa: F811
    """Normal data of a spread of magnitudes.  A step of 32 products drops less than a unit of 2^-23 of the sum of magnitudes at
    each of its additions (32 and the one to the sum), the pieces of a long sum 8 more at most, and the result is rounded once."""
    import torch
    x = values(T, width, dtype, 1)
    W = 0.02 * values(*((outs, width) if way == "fwd" else (width, outs)), "bfloat16", 2)
    got, want, sums = product(roi, way, on_gpu(x, dtype, 0), fmt, W.to(torch.bfloat16).cuda(), dtype, gap)
    tol = sums * ((width + 31) // 32 + 32 + 8) * 2.0 ** -23
    if dtype == "float16":
        keep = want.abs() < 65000
        assert keep.float().mean() > 0.9
        got, want, tol = got[keep], want[keep], tol[keep]
    tol = tol + (want.abs() + tol) * EPS[dtype] + TINY[dtype]
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("way,T,outs,width,gap", [PAIRS[1], PAIRS[2], PAIRS[6], PAIRS[8], ("dgrad", 2000, 4800, 1000, 0)])
def test_blocks_that_are_not_finite_in_pairs(roi, way, T, outs, width, gap, dtype):  # noqa: F811
    """They make NaN of the sums that they are part of, and of no other."""
    import torch
    x = values(T, width, "bfloat16", 3).cuda()
    W = values(*((outs, width) if way == "fwd" else (width, outs)), "bfloat16", 4).cuda()
    x[1, 130], x[T - 1, width - 1] = float("inf"), float("nan")
    # a weight's bad blocks: one in the middle, and the last
    W[140, 260], W[-1, -1] = float("nan"), float("inf")
    got, _, _ = product(roi, way, x, "e4m3", W, dtype, gap)
    bad = torch.zeros(T, outs, dtype=torch.bool)
    bad[1] = bad[T - 1] = True
    first = 128 if way == "fwd" else 256
    bad[:, first:first + 128] = True
    bad[:, (outs - 1) // 128 * 128:] = True
    assert torch.equal(torch.isnan(got), bad)
