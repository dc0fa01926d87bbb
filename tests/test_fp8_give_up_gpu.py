"""The products in 8-bit floating point with bounded waits that run out anywhere on the way.  Every copy is valid and
every wait bounded."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# pairs of CTAs with tokens, and with outputs, in the lanes, several tiles a pair and pieces of fp32 sums; single CTAs, and
# clusters of them that join their sums
@pytest.mark.parametrize("way,T,outs,width,dtype,gap", [
    ("fwd", 4096, 4864, 1000, "bfloat16", 0), ("fwd", 3000, 4865, 5000, "float32", 1), ("dgrad", 2048, 3584, 4000, "float32", 0),
    ("fwd", 100, 18944, 1500, "float16", 0), ("dgrad", 37, 128, 896, "bfloat16", 0), ("fwd", 200, 640, 6000, "float32", 3)])
def test_small_limits(roi, way, T, outs, width, dtype, gap):  # noqa: F811
    """Limits from far below to above the time of a wait: every call returns, and either says that it gave up or is
    right.  (Which of the two is the clock's affair.)"""
    import torch
    g = torch.Generator("cuda").manual_seed(T)
    x8 = roi.new_fp8(T, width)
    w8 = roi.new_fp8_weight(*((outs, width) if way == "fwd" else (width, outs)))
    roi.roi_fp8_save(torch.randn(T, width, device="cuda", generator=g), "e4m3", *x8)
    W = torch.randn(*((outs, width) if way == "fwd" else (width, outs)), device="cuda", generator=g).bfloat16()
    roi.roi_fp8_save_weight(W, *w8)
    out = torch.empty(T, outs + gap, dtype=getattr(torch, dtype), device="cuda")[:, :outs]

    def call():
        getattr(roi, f"roi_fp8_linear_{way}")(x8, "e4m3", w8, out)
        return out

    want = call().clone()
    roi.roi_device_status()
    gave_up = 0
    try:
        for ns in (0, 1, 50, 200, 500, 1000, 2000, 3000, 5000, 10000, 30000, 100000):
            roi.roi_set_ring_wait_limit_ns(ns)
            for _ in range(10):
                got = call()
                try:
                    roi.roi_device_status()
                except roi.RoiError as err:
                    assert err.status == 8
                    gave_up += 1
                else:
                    assert ns > 0 and torch.equal(got, want), ns
    finally:
        roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
    assert gave_up >= 10
    assert torch.equal(call(), want)
    roi.roi_device_status()
