"""What the products in 8-bit floating point leave behind when their bounded waits run out on the way: the result is filled
with NaN before every call, so that a tile that was not written, or not whole, shows.  Every copy is valid and every
wait bounded."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

# Pairs with tokens in the lanes, and with outputs, whose sums of 47 and 32 blocks take longer (8 us and more) than a limit of 1 us and
# the time that the hardware suspends a wait for by itself, so that the warps that write give up while copies and MMAs go on; fp32
# pieces in pairs; single CTAs, and clusters, that wait for cold memory; a cluster of few tokens.  `late`: whether some calls
# have to give up at limits above zero.
CASES = [("fwd", 4096, 4864, 6000, "bfloat16", 8, True), ("dgrad", 8192, 3584, 4000, "bfloat16", 0, True), ("fwd", 3000, 4865, 5000, "float32", 1, False),
         ("fwd", 100, 18944, 1500, "float16", 3, True), ("fwd", 100, 1900, 20000, "bfloat16", 5, True), ("dgrad", 37, 1565, 1941, "float32", 0, False)]


@pytest.mark.parametrize("way,T,outs,width,dtype,gap,late", CASES)
def test_written_right_or_not_at_all(roi, way, T, outs, width, dtype, gap, late):  # noqa: F811
    import torch
    g = torch.Generator("cuda").manual_seed(T)
    shape = (outs, width) if way == "fwd" else (width, outs)
    x8, w8 = roi.new_fp8(T, width), roi.new_fp8_weight(*shape)
    roi.roi_fp8_save(torch.randn(T, width, device="cuda", generator=g), "e4m3", *x8)
    roi.roi_fp8_save_weight(torch.randn(*shape, device="cuda", generator=g).bfloat16(), *w8)
    whole = torch.full((T, outs + gap), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    out, flush = whole[:, :outs], torch.empty(256 << 20, dtype=torch.uint8, device="cuda")

    def call():
        whole.fill_(float("nan"))
        flush.zero_()  # (L2)
        getattr(roi, f"roi_fp8_linear_{way}")(x8, "e4m3", w8, out)
        try:
            roi.roi_device_status()
        except roi.RoiError as err:
            assert err.status == 8
            return True
        return False

    assert not call() and not out.isnan().any()
    want, gave_up = out.clone(), 0
    try:
        for ns in (0, 1, 50, 200, 1000, 3000, 5000, 10000, 30000):
            roi.roi_set_ring_wait_limit_ns(ns)
            for _ in range(8):
                up = call()
                assert bool((out.isnan() | (out == want)).all()), ns
                assert gap == 0 or bool(whole[:, outs:].isnan().all()), ns
                if up:
                    gave_up += ns > 0
                else:
                    assert ns > 0 and torch.equal(out, want), ns
    finally:
        roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
    assert gave_up >= 1 or not late
    assert not call() and torch.equal(out, want)
