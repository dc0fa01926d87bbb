"""Each layer of the example's block with its products in 8-bit floating point, by itself: its output and its input's gradient
are the products of its copies' values with one rounding to bfloat16, its copies those of the oracle, and the gradient of its
logits what the mask's backward gives of the weight gradient."""
import pytest

from oracle import fp8_oracle as O
from test_example_fp8_gpu import example  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,tokens", [(512, 256, 200), (256, 512, 333)])
def test_layer(example, rows, cols, tokens):  # noqa: F811
    import torch
    roi = example.roi
    torch.manual_seed(5)
    layer = example.MaskedLinearFp8(rows, cols, 4, 11, tokens)
    X, dY = (torch.randn(tokens, n, device="cuda").to(torch.bfloat16) for n in (cols, rows))
    checkpoint = roi.new_checkpoint(tokens, cols)
    roi.roi_checkpoint_save(X, *checkpoint)
    workspace = torch.empty(max(16, roi.roi_masked_linear_wgrad_workspace_size(tokens, rows, cols)), dtype=torch.uint8, device="cuda")
    Y = layer.forward(X, 3, 0.5)
    dX = layer.backward(dY, checkpoint, 0.5, None, workspace)
    roi.roi_device_status()
    w = torch.from_numpy(O.save(layer.Wm.double().cpu().numpy(), "e4m3", 128)[2]).cuda()
    x, d = (torch.from_numpy(O.save(t.double().cpu().numpy(), fmt)[2]).cuda() for t, fmt in ((X, "e4m3"), (dY, "e5m2")))
    # a rounding to bfloat16 is off by at most 2^-8 of the value; the sums before it by far less
    for got, want, size in ((Y, x @ w.T, x.abs() @ w.T.abs()), (dX, d @ w, d.abs() @ w.abs())):
        tol = size * (rows + cols) / 32 * 2.0 ** -23
        assert bool(((got.double() - want).abs() <= tol + (want.abs() + tol) * 2.0 ** -8).all())
    # the weight gradient of the checkpoint's values, summed in fp32 and rounded once
    kept = torch.empty(tokens, cols, device="cuda")
    roi.roi_checkpoint_load(*checkpoint, kept)
    want = dY.double().T @ kept.double()
    tol = (dY.double().abs().T @ kept.double().abs()) * (tokens + 40) * 2.0 ** -23
    assert bool(((layer.dWm.double() - want).abs() <= tol + (want.abs() + tol) * 2.0 ** -8).all())
    # the logits' gradient, bit for bit what the call gives by itself
    dlogits = torch.empty_like(layer.logits)
    roi.roi_mask_bwd(layer.logits, layer.W, roi.NoiseState(example.NOISE_SEED, 3, 4, 1.0, 0), example.N, example.M, layer.dWm, 0.5, dlogits)
    assert torch.equal(dlogits, layer.dlogits)
