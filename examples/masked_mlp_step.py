"""Mask learning of one MLP block, with its activations kept in 8 bits between the passes.

The block is a transformer's: RMS norm, gate and up projections, SiLU(gate) * up, down projection,
residual.  Its weights are frozen; every weight has a logit, and the loss is the distance of the
masked block's output from the dense block's.  Between forward and backward only 8-bit checkpoints
of the activations are kept: the block's input, the normalised input (written by the norm as it
goes), gate, up and their product.  The backward forms each layer's weight gradient from the
checkpoint of its input, turns it into the logits' AdamW step, and closes with the norm's own
backward.

    python examples/masked_mlp_step.py [--shape qwen2.5-0.5b] [--tokens 2048] [--steps 20]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_23048_gb300 as roi  # noqa: E402
import workloads as WL  # noqa: E402

N, M, EPS = 2, 4, 1e-6


class MaskedLinear:
    """Y = X Wm^T with Wm = W * S(logits); the logits learn, W does not."""

    def __init__(self, rows, cols, tensor_id, seed):
        self.W, self.logits, _ = WL.make_inputs(rows, cols, "logw", seed, device="cuda")
        self.m, self.v = torch.zeros_like(self.logits), torch.zeros_like(self.logits)
        self.Wm, self.dWm = torch.empty_like(self.W), torch.empty_like(self.W)
        self.tensor_id = tensor_id

    def forward(self, X, step, tau):
        self.state = roi.NoiseState(7, step, self.tensor_id, 1.0, 0)
        roi.roi_mask_fwd_ex(self.logits, self.W, N, M, tau, self.state, self.Wm)
        return X @ self.Wm.T

    def backward(self, dY, x_checkpoint, tau, opt, workspace):
        """dX; the weight gradient from the checkpoint of X goes into the logits at once."""
        dX = dY @ self.Wm
        roi.roi_masked_linear_wgrad(dY, x_checkpoint, self.dWm, None, workspace)
        roi.roi_mask_bwd_adamw(self.logits, self.W, self.state, N, M, self.dWm, tau, self.m, self.v, opt)
        return dX


class MaskedMLP:
    def __init__(self, hidden, inter, tokens, seed=1000):
        self.hidden, self.inter, self.tokens = hidden, inter, tokens
        self.gate, self.up = MaskedLinear(inter, hidden, 4, seed + 4), MaskedLinear(inter, hidden, 5, seed + 5)
        self.down = MaskedLinear(hidden, inter, 6, seed + 6)
        self.gamma = (1 + 0.1 * torch.randn(hidden, device="cuda")).to(torch.bfloat16)
        # what lives from the forward to the backward, and the steps' workspace
        self.x8, self.y8 = roi.new_checkpoint(tokens, hidden), roi.new_checkpoint(tokens, hidden)
        self.g8, self.u8, self.h8 = (roi.new_checkpoint(tokens, inter) for _ in range(3))
        self.rstd = torch.empty(tokens, device="cuda")
        need = max([roi.roi_norm_bwd_workspace_size(tokens, hidden)] +
                   [roi.roi_masked_linear_wgrad_workspace_size(tokens, *layer.W.shape) for layer in (self.gate, self.down)])
        self.workspace = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")

    def dense(self, x):
        """The block with its frozen weights whole."""
        y = torch.empty_like(x)
        roi.roi_norm_fwd(x, "rms", self.gamma, None, EPS, y)
        return x + (torch.nn.functional.silu(y @ self.gate.W.T) * (y @ self.up.W.T)) @ self.down.W.T

    def forward(self, x, step, tau):
        y = torch.empty_like(x)
        roi.roi_norm_fwd(x, "rms", self.gamma, None, EPS, y, None, self.rstd, x_checkpoint=self.x8, y_checkpoint=self.y8)
        g, u = self.gate.forward(y, step, tau), self.up.forward(y, step, tau)
        h = torch.nn.functional.silu(g) * u
        for a, q in ((g, self.g8), (u, self.u8), (h, self.h8)):
            roi.roi_checkpoint_save(a, *q)
        return x + self.down.forward(h, step, tau)

    def backward(self, d_out, tau, opt):
        """Gradient of the block's input and of the norm's weight; the layers' logits are updated."""
        dh = self.down.backward(d_out, self.h8, tau, opt, self.workspace)
        g, u = torch.empty_like(dh), torch.empty_like(dh)
        roi.roi_checkpoint_load(*self.g8, g)
        roi.roi_checkpoint_load(*self.u8, u)
        s = torch.sigmoid(g)
        dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
        dy = self.gate.backward(dg, self.y8, tau, opt, self.workspace) + self.up.backward(du, self.y8, tau, opt, self.workspace)
        dx, dgamma = torch.empty_like(dy), torch.empty(self.hidden, device="cuda")
        roi.roi_norm_bwd(dy, self.x8, "rms", self.gamma, None, self.rstd, dx, dgamma, None, self.workspace)
        return dx + d_out, dgamma

    def kept_bytes(self):
        """Of the activations between the passes: as they are kept, and in bfloat16."""
        pairs = (self.x8, self.y8, self.g8, self.u8, self.h8)
        return sum(t.numel() for q in pairs for t in q), 2 * self.tokens * (2 * self.hidden + 3 * self.inter)


def train(hidden, inter, tokens, steps, lr=0.02, tau=0.5):
    """The losses of `steps` steps on one batch."""
    torch.manual_seed(0)
    block = MaskedMLP(hidden, inter, tokens)
    x = torch.randn(tokens, hidden, device="cuda").to(torch.bfloat16)
    target, losses = block.dense(x), []
    for step in range(steps):
        opt = roi.AdamW(lr, 0.9, 0.95, 1e-8, 0.0, step + 1)
        out = block.forward(x, step, tau)
        diff = out - target
        losses.append(diff.float().square().mean())
        block.backward(diff * (2.0 / diff.numel()) * 1e4, tau, opt)
    roi.roi_device_status()
    return block, [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--shape", default="qwen2.5-0.5b", choices=sorted(WL.LAYER_SETS))
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    s = WL.LAYER_SETS[a.shape]
    block, losses = train(s.hidden, s.inter, a.tokens, a.steps)
    kept, plain = block.kept_bytes()
    print(f"{a.shape}-shaped MLP block, {a.tokens} tokens: activations kept {kept / 1e6:.1f} MB (bfloat16: {plain / 1e6:.1f} MB)")
    print("loss " + " ".join(f"{v:.4g}" for v in losses))


if __name__ == "__main__":
    main()
