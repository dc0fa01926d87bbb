"""The example's masked MLP block with its products in 8-bit floating point: it runs, and its gradients are those of float64
within what its roundings allow.

A value of e4m3 is off by at most 2^-4 of itself and one of e5m2 by 2^-3 (half a step of the format; less for most), and those of
a gradient pass two products.  The errors of a sum's hundreds of terms are independent, so in the 2-norm a product is off by
no more than its factors' relative errors added: 2 * 2^-4 = 2^-3 for an output, and for dX 2^-3 + 2^-4; after the three
products in turn that a gradient of the gate goes through, 2^-3 + (2^-3 + 2^-4) + 2^-7 of its checkpoint: 0.33."""
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
    block = example.MaskedMLP(hidden, inter, tokens, fp8=True)
    x = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    d_out = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    before = block.gate.logits.clone()
    out = block.forward(x, 0, 0.5)
    opt = example.roi.AdamW(0.0, 0.9, 0.95, 1e-8, 0.0, 1)
    dx, dgamma = block.backward(d_out, 0.5, opt)
    example.roi.roi_device_status()
    assert torch.equal(before, block.gate.logits)   # lr 0
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    xd, gamma = leaf(x), leaf(block.gamma)
    Wg, Wu, Wd = leaf(block.gate.Wm), leaf(block.up.Wm), leaf(block.down.Wm)
    y = xd * torch.rsqrt(xd.square().mean(1, keepdim=True) + example.EPS) * gamma
    want = xd + (torch.nn.functional.silu(y @ Wg.T) * (y @ Wu.T)) @ Wd.T
    want.backward(d_out.double())
    for name, got, ref in (("out", out, want.detach()), ("dx", dx, xd.grad), ("dgamma", dgamma, gamma.grad),
                           ("gate", block.gate.dWm, Wg.grad), ("up", block.up.dWm, Wu.grad), ("down", block.down.dWm, Wd.grad)):
        assert (got.double() - ref).norm() <= 0.33 * ref.norm(), name


def test_it_runs(example):
    import torch
    block, losses = example.train(256, 512, 300, 5, fp8=True)
    assert all(torch.isfinite(torch.tensor(losses))) and len(losses) == 5
    assert bool(block.gate.moments[0].any()) and bool(block.down.moments[1].any())
