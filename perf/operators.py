"""The operators around the masked linear layers in training: what is timed of them, and their plain forms.

Every linear layer of a model in mask learning needs its input again in the backward pass, where
dWm = dY^T X is what the mask's backward starts from.  A run keeps those inputs as checkpoints in 8 bits
(blocks of 32 columns that share a power of two), which the norm in front of the layers can write as it goes,
and which the weight gradient and the norm's own backward read.

Kinds of case:
  checkpoint  a tensor of activations saved in 8 bits, and restored.
  norm_fwd    the layer norm or the RMS norm of rows of tokens; `save`: the checkpoint of its output as well (restored,
              for what it stands for).
  norm_bwd    its backward: gradients of the input, the weight and, for the layer norm, the bias; `source`: the
              input as it was ("x") or its checkpoint.
  wgrad       the weight gradient of a masked linear layer from the checkpoint of its input; `acc`: added to a sum
              in 32 bits over the micro-batches of a step, which is updated in place.
"""
import math

import torch

own = False

EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # a handful of tokens of the smallest model, a debugging step: latency counts
        dict(name="checkpoint_small", kind="checkpoint", rows=16, cols=896, dtype="bf16", gap=0),
        # the largest activations of a 7B-shaped block, gate x up of a full micro-batch
        dict(name="checkpoint_7b_inner", kind="checkpoint", rows=8192, cols=18944, dtype="bf16", gap=0),
        # 32-bit activations cut out of a wider tensor, neither a whole number of blocks nor aligned rows
        dict(name="checkpoint_odd", kind="checkpoint", rows=2045, cols=1531, dtype="fp32", gap=6),
        # one token through a 7B-shaped block's norm
        dict(name="norm_fwd_token", kind="norm_fwd", rows=1, cols=3584, dtype="bf16", gap=0, norm="rms", save=False),
        # the norm before the q, k, v (or gate, up) layers of a 7B-shaped block, with the checkpoint of their input
        dict(name="norm_fwd_7b_save", kind="norm_fwd", rows=8192, cols=3584, dtype="bf16", gap=0, norm="rms", save=True),
        # a layer norm of odd width in half precision
        dict(name="norm_fwd_layer_odd", kind="norm_fwd", rows=6000, cols=1001, dtype="fp16", gap=0, norm="layer", save=False),
        # the same block's norm backward, from the input's checkpoint
        dict(name="norm_bwd_7b", kind="norm_bwd", rows=8192, cols=3584, dtype="bf16", gap=0, norm="rms", source="checkpoint"),
        # a layer norm's backward at the 1.5B-shaped width, in 32 bits, a short batch
        dict(name="norm_bwd_layer_1.5b", kind="norm_bwd", rows=1500, cols=1536, dtype="fp32", gap=0, norm="layer", source="x"),
        # one small layer: a unit test, a toy model
        dict(name="wgrad_small", kind="wgrad", T=37, out=128, cols=256, gap=0, acc=False),
        # the key / value layers of a 7B-shaped block: few outputs, a long sum over tokens
        dict(name="wgrad_7b_kv", kind="wgrad", T=8192, out=512, cols=3584, gap=0, acc=False),
        # the gate layer of a 7B-shaped block
        dict(name="wgrad_7b_gate", kind="wgrad", T=8192, out=18944, cols=3584, gap=0, acc=False),
        # ragged in every direction, one micro-batch of several
        dict(name="wgrad_ragged_acc", kind="wgrad", T=1999, out=1215, cols=2504, gap=0, acc=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("checkpoint", "norm_fwd", "norm_bwd", "wgrad", "wgrad"))
    if kind == "wgrad":
        # widths of layers: multiples of a group of 4 or 8 along the inputs, anything along the outputs
        cols = rng.choice((4, 8)) * log_int(16, 2300)
        out, T = log_int(64, 18944), log_int(1, 16384)
        while T * out * cols > 8192 * 18944 * 3584:
            T = max(1, T // 2)
        return dict(kind=kind, T=T, out=out, cols=cols, gap=rng.choice((0, 0, 0, 8, 3)), acc=rng.random() < 0.3)
    cols = log_int(64, 18944 if kind == "checkpoint" else 8192)
    if rng.random() < 0.6:
        cols = max(64, cols // 64 * 64)
    rows = log_int(1, min(32768, (8192 * 18944 if kind == "checkpoint" else 8192 * 3584) // cols))
    c = dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")),
             gap=rng.choice((0, 0, 0, 64, 5)))
    if kind != "checkpoint":
        c["norm"] = rng.choice(("layer", "rms"))
    if kind == "norm_fwd":
        c["save"] = rng.random() < 0.5
    if kind == "norm_bwd":
        c["source"] = rng.choice(("x", "checkpoint"))
    return c


# ---------------------------------------------------------------------------
# the checkpoint's layout
# ---------------------------------------------------------------------------
def _pitches(cols):
    """Bytes of a row's codes, and of its scales."""
    return (cols + 31) // 32 * 32, (cols + 127) // 128 * 4


def _power_of_two(e):
    """2^e in 32 bits, exactly (torch's pow and ldexp may round), for -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _save(x):
    """Codes and scales of x [rows, cols]: blocks of 32 columns share 2^(s - 133), the least power of two with which
    the block's largest magnitude is at most 127.5."""
    x = x.float()
    rows, cols = x.shape
    pitch, scale_pitch = _pitches(cols)
    x = torch.nn.functional.pad(x, (0, 32 * scale_pitch - cols)).view(rows, scale_pitch, 32)
    largest = x.abs().amax(-1)
    s = ((largest.view(torch.int32) + 0xFFFF) >> 23).clamp(7, 254)
    q = (x * _power_of_two(133 - s)[..., None]).round().clamp(-127, 127)
    bad = ~torch.isfinite(largest)
    s = torch.where(bad, 255, s)
    q = torch.where(bad[..., None], 0.0, q)
    return q.view(rows, -1)[:, :pitch].to(torch.int8).contiguous(), s.to(torch.uint8)


def _load(codes, scales, cols):
    """The values that a checkpoint stands for, in 32 bits."""
    s = scales.to(torch.int32)
    step = torch.where(s == 255, math.nan, _power_of_two(s.clamp(max=254) - 133))
    return codes[:, :cols].float() * step.repeat_interleave(32, 1)[:, :cols]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _rows(g, rows, cols, gap, dtype):
    """[rows, cols] with `gap` elements between a row's end and the next one's start."""
    return torch.empty(rows, cols + gap, dtype=dtype, device="cuda").normal_(generator=g)[:, :cols]


def _activations(g, rows, cols, gap, dtype):
    """Activations as a block has them: unit spread around a small offset, one channel in a hundred 20 times as large."""
    x = _rows(g, rows, cols, gap, dtype)
    large = torch.rand(cols, generator=g, device="cuda") < 0.01
    offset = 0.2 * torch.randn(cols, generator=g, device="cuda")
    x.mul_(torch.where(large, 20.0, 1.0).to(dtype)).add_(offset.to(dtype))
    return x


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rand = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    if case["kind"] == "wgrad":
        T, out, cols = case["T"], case["out"], case["cols"]
        d = {"x": _activations(g, T, cols, 0, torch.bfloat16), "dY": _rows(g, T, out, case["gap"], torch.bfloat16)}
        # one token in eight is padding or a prompt's, with no gradient
        d["dY"].mul_(1e-3 * (torch.rand(T, 1, generator=g, device="cuda") >= 0.125))
        if case["acc"]:
            d["acc"] = torch.empty(out, cols, device="cuda").normal_(generator=g).mul_(1e-3 * math.sqrt(T))
        return d
    rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
    d = {"x": _activations(g, rows, cols, case["gap"], dtype)}
    if case["kind"] != "checkpoint":
        d["gamma"] = (1 + 0.2 * rand(cols)).to(dtype)
        d["beta"] = (0.1 * rand(cols)).to(dtype) if case["norm"] == "layer" else None
    if case["kind"] == "norm_bwd":
        d["dy"] = _rows(g, rows, cols, case["gap"], dtype).mul_(0.01)
    return d


def _statistics(x, norm, eps):
    """Mean (None for the RMS norm) and reciprocal deviation of each row, in the type of x."""
    mean = x.mean(1) if norm == "layer" else None
    centred = x - mean[:, None] if norm == "layer" else x
    return mean, 1 / torch.sqrt((centred * centred).mean(1) + eps)


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731

    def checkpoint(rows, cols):
        pitch, scale_pitch = _pitches(cols)
        return empty(rows, pitch, dtype=torch.int8), empty(rows, scale_pitch, dtype=torch.uint8)

    if case["kind"] == "wgrad":
        T, out, cols = case["T"], case["out"], case["cols"]
        s["saved"] = _save(s.pop("x"))
        s["dWm"] = empty(out, cols, dtype=torch.bfloat16)
        s["acc"] = s.get("acc")
        # room for partial sums over tokens, kept from step to step
        s["workspace"] = empty(64 << 20, dtype=torch.uint8)
        if (out + case["gap"]) % 8:  # rows that are not aligned are laid out again
            s["workspace"] = empty((64 << 20) + 2 * T * (out + 16), dtype=torch.uint8)
        return s
    rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
    if case["kind"] == "checkpoint":
        s["saved"], s["out"] = checkpoint(rows, cols), empty(rows, cols, dtype=dtype)
        return s
    s["mean"], s["rstd"] = empty(rows) if case["norm"] == "layer" else None, empty(rows)
    if case["kind"] == "norm_fwd":
        s["out"] = empty(rows, cols, dtype=dtype)
        if case["save"]:
            s["saved"], s["restored"] = checkpoint(rows, cols), empty(rows, cols, dtype=dtype)
        return s
    s["mean"], s["rstd"] = _statistics(s["x"].float(), case["norm"], EPS)
    if case["source"] == "checkpoint":
        s["x"] = _save(s["x"])
    s["dx"], s["dgamma"] = empty(rows, cols, dtype=dtype), empty(cols)
    s["dbeta"] = empty(cols) if case["norm"] == "layer" else None
    s["workspace"] = empty(16 << 20, dtype=torch.uint8)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2608_23048_gb300 as roi
    case = s["case"]
    if case["kind"] == "checkpoint":
        roi.roi_checkpoint_save(s["x"], *s["saved"])
        roi.roi_checkpoint_load(*s["saved"], s["out"])
        return {"restored": s["out"]}
    if case["kind"] == "wgrad":
        roi.roi_masked_linear_wgrad(s["dY"], s["saved"], s["dWm"], s["acc"], s["workspace"])
        return {"dWm": s["dWm"], "acc": s["acc"]}
    if case["kind"] == "norm_fwd":
        roi.roi_norm_fwd(s["x"], case["norm"], s["gamma"], s["beta"], EPS, s["out"], s["mean"], s["rstd"],
                         y_checkpoint=s.get("saved"))
        if case["save"]:
            roi.roi_checkpoint_load(*s["saved"], s["restored"])
        return {"y": s["out"], "mean": s["mean"], "rstd": s["rstd"], "restored": s.get("restored")}
    roi.roi_norm_bwd(s["dy"], s["x"], case["norm"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"],
                     s["workspace"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _run_plain(s):
    case = s["case"]
    cols = case["cols"]
    if case["kind"] == "checkpoint":
        return {"restored": _load(*_save(s["x"]), cols).to(s["out"].dtype)}
    if case["kind"] == "wgrad":
        total = s["dY"].float().T @ _load(*s["saved"], cols)
        if case["acc"]:
            total = s["acc"].add_(total)
        return {"dWm": total.to(torch.bfloat16), "acc": s["acc"]}
    gamma = s["gamma"].float()
    if case["kind"] == "norm_fwd":
        x, dtype = s["x"].float(), s["out"].dtype
        mean, rstd = _statistics(x, case["norm"], EPS)
        y = (x - mean[:, None] if case["norm"] == "layer" else x) * rstd[:, None] * gamma
        y = (y + s["beta"].float() if s["beta"] is not None else y).to(dtype)
        restored = _load(*_save(y), cols).to(dtype) if case["save"] else None
        return {"y": y, "mean": mean, "rstd": rstd, "restored": restored}
    x = _load(*s["x"], cols) if case["source"] == "checkpoint" else s["x"].float()
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = (x - s["mean"][:, None] if case["norm"] == "layer" else x) * rstd
    dxh = dy * gamma
    dx = dxh - xh * (dxh * xh).mean(1, keepdim=True)
    if case["norm"] == "layer":
        dx = dx - dxh.mean(1, keepdim=True)
    return {"dx": (rstd * dx).to(s["dx"].dtype), "dgamma": (dy * xh).sum(0),
            "dbeta": dy.sum(0) if case["norm"] == "layer" else None}


def work(case):
    cols = case["cols"]
    kept = sum(_pitches(cols))  # bytes of a row's checkpoint
    if case["kind"] == "wgrad":
        T, out = case["T"], case["out"]
        return {"bytes": 2 * T * out + T * kept + out * cols * (10 if case["acc"] else 2), "flops": 2 * T * out * cols}
    rows, b = case["rows"], 4 if case["dtype"] == "fp32" else 2
    E, layer = rows * cols, case.get("norm") == "layer"
    if case["kind"] == "checkpoint":
        return {"bytes": 2 * (b * E + rows * kept), "flops": 0}
    if case["kind"] == "norm_fwd":
        bytes_ = 2 * b * E + (2 if layer else 1) * (b * cols + 4 * rows)
        return {"bytes": bytes_ + (2 * rows * kept + b * E if case["save"] else 0), "flops": 8 * E}
    source = rows * kept if case["source"] == "checkpoint" else b * E
    return {"bytes": 2 * b * E + source + b * cols + (2 if layer else 1) * 4 * (rows + cols), "flops": 12 * E}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _nearest(x):
    """What the checkpoint of x (finite values, in 64 bits) stands for: per block the least e with max |x| <= 127.5 2^e,
    no less than -126 and no more than 121, and the nearest multiple of 2^e."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    whole = cols // 32 * 32
    for a, b, n in ((0, whole, 32), (whole, cols, cols - whole)):
        if a == b:
            continue
        part = x[:, a:b].reshape(rows, -1, n)
        fraction, exponent = torch.frexp(part.abs().amax(-1, keepdim=True) / 127.5)  # fraction in [1/2, 1)
        e = torch.where(fraction == 0.5, exponent - 1, exponent).clamp(-126, 121)
        step = ((e.long() + 1023) << 52).view(torch.float64)  # 2^e, exactly
        out[:, a:b] = (torch.round(part / step).clamp(-127, 127) * step).reshape(rows, -1)
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "checkpoint":
        # block by block of rows: the largest case would take ten times its own room at once
        return {"restored": torch.cat([_nearest(x.double()).to(x.dtype).double() for x in d["x"].split(1024)])}
    if case["kind"] == "wgrad":
        total = d["dY"].double().T @ _nearest(d["x"].double())
        if case["acc"]:
            total += d["acc"].double()
        return {"dWm": total, "acc": total if case["acc"] else None}
    x, gamma = d["x"].double(), d["gamma"].double()
    layer = case["norm"] == "layer"
    mean = x.sum(1) / x.shape[1] if layer else None
    if case["kind"] == "norm_fwd":
        c = x - mean[:, None] if layer else x
        rstd = torch.rsqrt(c.square().sum(1) / x.shape[1] + EPS)
        y = c * rstd[:, None] * gamma + (d["beta"].double() if layer else 0)
        restored = _nearest(y.to(d["x"].dtype).double()) if case["save"] else None
        return {"y": y, "mean": mean, "rstd": rstd, "restored": restored}
    # the statistics are inputs, in the 32 bits that the forward left them in
    mean, rstd = _statistics(d["x"].float(), case["norm"], EPS)
    if case["source"] == "checkpoint":
        x = _nearest(x)
    r, dy = rstd.double()[:, None], d["dy"].double()
    xh = (x - mean.double()[:, None] if layer else x) * r
    a, n = dy * gamma, x.shape[1]
    dx = a - (a.sum(1, keepdim=True) / n if layer else 0) - xh * ((a * xh).sum(1, keepdim=True) / n)
    return {"dx": r * dx, "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0) if layer else None}
