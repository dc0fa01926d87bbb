"""Sums of the weight gradient over many tokens whose result is bfloat16 alone: broken off at 32768 tokens.

The tensor cores drop what lies below the last bit of their running sum, always towards zero, so that the
error of an unbroken sum grows with the tokens without bound."""
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


# (the widths of the three ways out; one piece, two, more; fewer and more tiles than pairs of SMs)
@pytest.mark.parametrize("T,rows,cols", [(32768, 130, 260), (32769, 130, 260), (70001, 256, 512), (70000, 257, 510), (140000, 100, 509),
                                         (66000, 1500, 2500), (40000, 4864, 2560)])
@pytest.mark.parametrize("split", [True, False])
def test_pieces_are_all_there(roi, T, rows, cols, split):  # noqa: F811
    """Integers whose sums are exact in float32 in any order: the same bits as the sum in one piece."""
    import torch
    g = torch.Generator("cuda").manual_seed(T + cols)
    x = torch.randint(-2, 3, (T, cols), device="cuda", generator=g).bfloat16()
    dY = torch.randint(-2, 3, (T, (rows + 7) // 8 * 8), device="cuda", generator=g).bfloat16()[:, :rows]
    assert 4 * T < 2 ** 24
    q = roi.new_checkpoint(T, cols)
    roi.roi_checkpoint_save(x, *q)
    n = roi.roi_masked_linear_wgrad_workspace_size(T, rows, cols, dY.stride(0)) if split else 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
    out = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
    roi.roi_device_status()
    assert torch.equal(out, (dY.float().T @ x.float()).bfloat16())


@pytest.mark.parametrize("rows,cols,split", [(256, 256, False), (256, 256, True), (100, 129, False)])
def test_error_stays_that_of_the_rounding(roi, rows, cols, split):  # noqa: F811
    """A million tokens.  With r the error of the nearest bfloat16 numbers (1.7e-3 of the norm) and d that of the
    sum before its rounding, the result's is sqrt(r^2 + d^2); pieces of 32768 tokens have d under 3e-5, so it is
    under 1.0002 r.  1.002 r, where an unbroken sum has 1.2 r."""
    import torch
    T = 1 << 20
    g = torch.Generator("cuda").manual_seed(cols)
    x = (torch.randn(T, cols, device="cuda", generator=g) + 0.2 * torch.randn(cols, device="cuda", generator=g)).bfloat16()
    dY = torch.randn(T, (rows + 7) // 8 * 8, device="cuda", generator=g).bfloat16()[:, :rows]
    q, back = roi.new_checkpoint(T, cols), torch.empty(T, cols, device="cuda")
    roi.roi_checkpoint_save(x, *q)
    roi.roi_checkpoint_load(*q, back)
    want = sum(a.double().T @ b.double() for a, b in zip(dY.split(65536), back.split(65536)))
    n = roi.roi_masked_linear_wgrad_workspace_size(T, rows, cols, dY.stride(0)) if split else 0
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
    roi.roi_device_status()
    nearest = float((want.bfloat16().double() - want).norm())
    assert float((out.double() - want).norm()) <= 1.002 * nearest
