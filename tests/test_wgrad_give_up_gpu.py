"""The weight gradient with bounded waits that run out anywhere on the way.  Every copy is valid and every wait
bounded."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# fewer and more tiles than pairs of SMs, ranges of tokens that are joined, pieces for acc and for a bfloat16 result
# alone, the three ways out, dY laid out again
@pytest.mark.parametrize("T,rows,cols,acc,gap", [(8192, 512, 3584, False, 0), (4000, 4864, 2560, False, 0), (7000, 1215, 2504, True, 1),
                                                 (40000, 300, 509, False, 0), (500, 257, 510, True, 0), (37, 128, 256, False, 0)])
def test_small_limits(roi, T, rows, cols, acc, gap):  # noqa: F811
    """Limits from far below to above the time of a wait: every call returns, and either says that it gave up or
    is right.  (Which of the two is the clock's affair.)"""
    import torch
    g = torch.Generator("cuda").manual_seed(T)
    dY = torch.randn(T, rows + gap, device="cuda", generator=g).bfloat16()[:, :rows]
    q = roi.new_checkpoint(T, cols)
    roi.roi_checkpoint_save(torch.randn(T, cols, device="cuda", generator=g), *q)
    ws = torch.empty(max(16, roi.roi_masked_linear_wgrad_workspace_size(T, rows, cols, dY.stride(0))), dtype=torch.uint8, device="cuda")
    out, total = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.zeros(rows, cols, device="cuda")

    def call():
        total.zero_()
        roi.roi_masked_linear_wgrad(dY, q, out, total if acc else None, ws)
        return out, total

    want = [t.clone() for t in call()]
    roi.roi_device_status()
    try:
        for ns in (0, 1, 50, 200, 500, 1000, 2000, 3000, 5000, 10000, 30000, 100000):
            roi.roi_set_ring_wait_limit_ns(ns)
            for _ in range(10):
                got = call()
                try:
                    roi.roi_device_status()
                except roi.RoiError as err:
                    assert err.status == 8
                else:
                    assert ns > 0 and all(torch.equal(a, b) for a, b in zip(want, got)), ns
    finally:
        roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
    assert all(torch.equal(a, b) for a, b in zip(want, call()))
    roi.roi_device_status()
