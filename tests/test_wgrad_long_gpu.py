"""Sums of the weight gradient over many tokens, added to acc.

The tensor cores drop what lies below the last bit of their running sum, always towards zero, so an
unbroken sum drifts: on these inputs 4.3e-7 of its norm at 2000 tokens, 1.1e-6 at 4000 and 6.8e-6 at
16000.  A sum for acc is broken off at 2816 tokens at the latest, 6.7e-7 by that growth, and its pieces
are added in float32, whose rounding errors (2^-24 a piece, either way) are small beside it: 1e-6 holds
for any number of tokens."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# (the widths of the three ways out; fewer and more tiles than pairs of SMs, with and without ranges of tokens)
@pytest.mark.parametrize("T,rows,cols", [(2900, 256, 512), (16000, 256, 512), (16000, 257, 510), (8000, 100, 509),
                                         (9000, 1500, 2500), (16000, 4864, 2560)])
@pytest.mark.parametrize("split", [True, False])
def test_long_sums(roi, T, rows, cols, split):  # noqa: F811
    import torch
    g = torch.Generator("cuda").manual_seed(T + cols)
    x = (torch.randn(T, cols, device="cuda", generator=g) + 0.2 * torch.randn(cols, device="cuda", generator=g)).bfloat16()
    dY = torch.randn(T, (rows + 7) // 8 * 8, device="cuda", generator=g).bfloat16()[:, :rows]
    q, back = roi.new_checkpoint(T, cols), torch.empty(T, cols, device="cuda")
    roi.roi_checkpoint_save(x, *q)
    roi.roi_checkpoint_load(*q, back)
    n = roi.roi_masked_linear_wgrad_workspace_size(T, rows, cols, dY.stride(0)) if split else 0
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    acc = torch.randn(rows, cols, device="cuda", generator=g)
    want = dY.double().T @ back.double()
    total = want + acc.double()
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    roi.roi_masked_linear_wgrad(dY, q, out, acc, ws)
    assert float((acc.double() - total).norm() / want.norm()) < 1e-6
    # dWm is the whole sum, rounded
    assert torch.equal(out, acc.bfloat16())
    roi.roi_device_status()
