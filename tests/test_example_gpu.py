"""The example's masked MLP block: its gradients from 8-bit checkpoints against float64 gradients of
the same block, and its loss over some steps.

The norm's input and the layers' inputs are off by at most half a step of their blocks, under 2^-7
of the block's largest magnitude, and bfloat16 activations round by 2^-9 of themselves; each
gradient is a sum of hundreds of such terms with independent errors, so in the 2-norm the gradients
stay within a few times 2^-7: 5 % is allowed."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def example():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    from paper_2608_23048_gb300 import _build
    _build.build()
    import masked_mlp_step
    return masked_mlp_step


def test_gradients(example):
    import torch
    torch.manual_seed(3)
    hidden, inter, tokens = 256, 512, 200
    block = example.MaskedMLP(hidden, inter, tokens)
    x = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    d_out = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    out = block.forward(x, 0, 0.5)
    # the optimizer stands still: the gradients are looked at
    opt = example.roi.AdamW(0.0, 0.9, 0.95, 1e-8, 0.0, 1)
    dx, dgamma = block.backward(d_out, 0.5, opt)
    example.roi.roi_device_status()
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    xd, gamma = leaf(x), leaf(block.gamma)
    Wg, Wu, Wd = leaf(block.gate.Wm), leaf(block.up.Wm), leaf(block.down.Wm)
    y = xd * torch.rsqrt(xd.square().mean(1, keepdim=True) + example.EPS) * gamma
    want = xd + (torch.nn.functional.silu(y @ Wg.T) * (y @ Wu.T)) @ Wd.T
    want.backward(d_out.double())
    for name, got, ref in (("out", out, want.detach()), ("dx", dx, xd.grad), ("dgamma", dgamma, gamma.grad),
                           ("gate", block.gate.dWm, Wg.grad), ("up", block.up.dWm, Wu.grad), ("down", block.down.dWm, Wd.grad)):
        assert (got.double() - ref).norm() <= 0.05 * ref.norm(), name


def test_training_lowers_the_loss(example):
    block, losses = example.train(256, 512, 300, 40)
    assert losses[-1] < 0.8 * losses[0], losses
    kept, plain = block.kept_bytes()
    assert kept < 0.53 * plain
