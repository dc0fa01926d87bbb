"""Activation checkpoints in 8 bits (roi_checkpoint_save, roi_checkpoint_load) against the CPU
oracle.  Products by a power of two are exact and both sides round ties to even, so codes,
scales and restored values are compared bit for bit: there is no tolerance."""
import numpy as np
import pytest

from oracle import layer_oracle as LO

pytestmark = pytest.mark.gpu
DTYPES = ("bfloat16", "float16", "float32")


@pytest.fixture(scope="module")
def roi():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2608_23048_gb300 import _build
    _build.build()
    import paper_2608_23048_gb300 as roi
    return roi


def values(rows, cols, dtype, seed, kind="plain"):
    """Values of the type, float32 on the CPU."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    x[:, torch.rand(cols, generator=g) < 0.02] *= 30
    if kind == "range":      # every block at its own magnitude, zeros and subnormals among them
        top = {"bfloat16": 127, "float16": 15, "float32": 127}[dtype]
        low = {"bfloat16": -133, "float16": -24, "float32": -149}[dtype]
        x = x * torch.exp2(torch.randint(low, top, (rows, -(-cols // 32)), generator=g).double()
                           ).repeat_interleave(32, 1)[:, :cols]
        big = {"bfloat16": 3.3895314e38, "float16": 65504.0, "float32": 3.4028235e38}[dtype]
        x = x.clamp(-big, big)
        x[torch.rand(rows, cols, generator=g) < 0.1] = 0
        x[::3, :32] = 0
    if kind == "special":
        at = torch.rand(rows, cols, generator=g)
        x[at < 0.003] = float("nan")
        x[(at > 0.003) & (at < 0.006)] = float("inf")
        x[at > 0.997] = -float("inf")
    if kind == "edge":       # halves of a step, and block maxima around 127.5 steps
        x = torch.randint(-255, 256, (rows, cols), generator=g) / 2 * torch.exp2(
            torch.randint(-7, 8, (rows, 1), generator=g).float())
        x[:, ::32] = 127.5 * torch.exp2(torch.randint(-7, 8, (rows, 1), generator=g).float())
    return x.to(getattr(torch, dtype)).float()


def on_gpu(x, dtype, gap=0, offset=0):
    """x as a matrix whose rows are `gap` elements apart, starting `offset` elements into its memory."""
    import torch
    rows, cols = x.shape
    room = torch.full((rows * (cols + gap) + offset,), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    m = room[offset:].view(rows, cols + gap)[:, :cols]
    m.copy_(x.to(getattr(torch, dtype)))
    return m


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


SIZES = [(1, 1), (1, 8), (3, 31), (5, 32), (2, 33), (7, 63), (4, 96), (3, 127), (3, 128), (2, 129), (17, 256), (1, 3584),
         (9, 1000), (33, 1531), (64, 4864), (300, 100)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_save_and_load(roi, rows, cols, dtype):
    import torch
    for n, (kind, gap, offset) in enumerate((("plain", 0, 0), ("range", 0, 0), ("special", 8, 0), ("edge", 3, 0),
                                             ("range", 5, 1), ("special", 16, 8), ("plain", 0, 1))):
        x = values(rows, cols, dtype, 100 * n + rows, kind)
        codes, scales = roi.new_checkpoint(rows, cols)
        codes.fill_(99), scales.fill_(99)
        m = on_gpu(x, dtype, gap, offset)
        roi.roi_checkpoint_save(m, codes, scales)
        want_codes, want_scales = LO.checkpoint_save(x.double().numpy())
        assert same(codes.cpu().numpy(), want_codes) and same(scales.cpu().numpy(), want_scales), (kind, gap, offset)
        back = LO.checkpoint_load(want_codes, want_scales, cols)
        for out in DTYPES:
            got = on_gpu(torch.zeros(rows, cols), out, gap, offset)
            roi.roi_checkpoint_load(codes, scales, got)
            want = torch.from_numpy(back)
            if out == "float16":
                want = want.clamp(-65504, 65504)   # (a NaN stays one)
            assert same(got.float().cpu().numpy(), want.to(got.dtype).float().numpy()), (kind, out)
            if gap and rows > 1:   # nothing between the rows is touched
                between = torch.as_strided(got, (rows - 1, gap), (cols + gap, 1), got.storage_offset() + cols)
                assert torch.isnan(between).all()
    roi.roi_device_status()


def test_every_bfloat16(roi):
    """All finite bfloat16 values, one a block, and as the small member of a block of the next size."""
    import torch
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16).float()
    v = v[torch.isfinite(v)]
    x = torch.zeros(len(v), 64)
    x[:, 5] = v
    x[:, 40], x[:, 41] = v, (v * 8).clamp(-3e38, 3e38).to(torch.bfloat16).float()
    codes, scales = roi.new_checkpoint(len(v), 64)
    roi.roi_checkpoint_save(x.to("cuda", torch.bfloat16), codes, scales)
    want_codes, want_scales = LO.checkpoint_save(x.double().numpy())
    assert same(codes.cpu().numpy(), want_codes) and same(scales.cpu().numpy(), want_scales)
    # the error is at most half a step
    back = torch.empty(len(v), 64, device="cuda")
    roi.roi_checkpoint_load(codes, scales, back)
    step = torch.exp2(torch.from_numpy(want_scales[:, :2].astype(np.float64)) - 133).repeat_interleave(32, 1)
    assert ((back.cpu().double() - x.double()).abs() <= step / 2).all()


def test_slices_of_rows(roi):
    """Rows saved and loaded in slices are those of the whole."""
    import torch
    x = on_gpu(values(100, 200, "bfloat16", 3), "bfloat16")
    whole, parts = roi.new_checkpoint(100, 200), roi.new_checkpoint(100, 200)
    roi.roi_checkpoint_save(x, *whole)
    for a, b in ((0, 1), (1, 37), (37, 100)):
        roi.roi_checkpoint_save(x[a:b], parts[0][a:b], parts[1][a:b])
    assert torch.equal(whole[0], parts[0]) and torch.equal(whole[1], parts[1])
    out, some = torch.empty_like(x), torch.empty_like(x[37:])
    roi.roi_checkpoint_load(*whole, out)
    roi.roi_checkpoint_load(whole[0][37:], whole[1][37:], some)
    assert torch.equal(out[37:], some)


def test_past_32_bits(roi):
    """Element offsets past 2^32 (a long checkpoint of one-byte codes, wide and narrow rows)."""
    import torch
    for rows, cols, gap in ((33_600_000, 128, 0), (2_100_000, 2047, 0)):
        x = torch.zeros(rows, cols + gap, dtype=torch.bfloat16, device="cuda")[:, :cols]
        tail = values(64, cols, "bfloat16", 5).to("cuda", torch.bfloat16)
        x[-64:] = tail
        codes, scales = roi.new_checkpoint(rows, cols)
        roi.roi_checkpoint_save(x, codes, scales)
        want_codes, want_scales = LO.checkpoint_save(tail.double().cpu().numpy())
        assert same(codes[-64:].cpu().numpy(), want_codes) and same(scales[-64:].cpu().numpy(), want_scales)
        assert not codes[:-64].any() and bool((scales[:-64] == 7).all())
        x.zero_()
        roi.roi_checkpoint_load(codes, scales, x)
        back = LO.checkpoint_load(want_codes, want_scales, cols)
        assert same(x[-64:].double().cpu().numpy(), back) and not x[:-64].any()
        del x, codes, scales
        torch.cuda.empty_cache()


def test_empty_and_refusals(roi):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    codes, scales = roi.new_checkpoint(4, 64)
    roi.roi_checkpoint_save(x[:0], codes[:0], scales[:0])
    roi.roi_checkpoint_load(codes[:0], scales[:0], x[:0])
    with pytest.raises(TypeError):
        roi.roi_checkpoint_save(x.double(), codes, scales)
    with pytest.raises(TypeError):
        roi.roi_checkpoint_save(x, codes.view(torch.uint8), scales)
    with pytest.raises(ValueError):
        roi.roi_checkpoint_save(x, codes[:3], scales)
    with pytest.raises(ValueError):
        roi.roi_checkpoint_save(x.T, *roi.new_checkpoint(64, 4))
    with pytest.raises(ValueError):
        roi.roi_checkpoint_save(x.cpu(), codes, scales)
    with pytest.raises(roi.RoiError) as e:    # rows on top of one another
        roi.roi_checkpoint_save(x[:1].expand(4, 64), codes, scales)
    assert e.value.status == 2
    with pytest.raises(roi.RoiError) as e:    # the output lies in the input
        room = torch.zeros(256, dtype=torch.int8, device="cuda")
        roi.roi_checkpoint_load(room[:64].view(2, 32), scales[:2], room[:128].view(torch.bfloat16).view(2, 32))
    assert e.value.status == 6
    torch.cuda.synchronize()
