"""A step of mask learning in 8 bits around the mask op: what is timed of its operators, and their plain forms.

The masked layers' products with activations, Y = X Wm^T and dX = dY Wm, run on 8-bit floating-point copies whose
blocks of 128 share a power of two (an activation's blocks lie along its rows, a weight's are 128 x 128, so that one
copy serves both products).  The AdamW step that follows a data-parallel reduction of the gradients goes over
all logits and norm weights at once, with its states in 32 bits or in 8.

Kinds of case:
  fwd     Y = X Wm^T: X saved in 8 bits and multiplied with the weight's copy; `fresh`: Wm, which changes with every
          step of mask learning, is copied in the same pass (else the copy is there, as in serving or over the
          micro-batches of a step).
  dgrad   dX = dY Wm, the same way.
  adamw   one step over `layers` blocks of seven matrices and two vectors; `bits` of the states, 32 or 8.  States in
          8 bits are then read back, as what they stand for.  Parameters, gradients and states lie in one buffer each,
          as a reduction in buckets wants them, every tensor from a multiple of 128 elements on.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SEED, STEP = 20240917, 7  # of the states' rounding; steps taken, this one included
OPT = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.05)


def listed():
    return [
        # serving: one token through the gate layer of a 7B-shaped block; the weight's bytes count
        dict(name="fwd_token", kind="fwd", T=1, rows=18944, cols=3584, dtype="bf16", format="e4m3", gap=0, fresh=False),
        # a few tokens through a key / value layer of the smallest model: latency counts
        dict(name="fwd_small", kind="fwd", T=37, rows=128, cols=896, dtype="bf16", format="e4m3", gap=0, fresh=False),
        # a full micro-batch through the gate layer of a 7B-shaped block, the weight masked anew
        dict(name="fwd_7b_gate", kind="fwd", T=8192, rows=18944, cols=3584, dtype="bf16", format="e4m3", gap=0, fresh=True),
        # the down layer with activations and results in 32 bits: a long sum for each output
        dict(name="fwd_7b_down", kind="fwd", T=2048, rows=3584, cols=18944, dtype="fp32", format="e4m3", gap=0, fresh=False),
        # ragged in every direction, half precision, rows cut out of a wider tensor
        dict(name="fwd_ragged", kind="fwd", T=1999, rows=1215, cols=2504, dtype="fp16", format="e4m3", gap=3, fresh=True),
        # the gate layer's gradient of its input, a full micro-batch: the sum runs over 18944 outputs
        dict(name="dgrad_7b_gate", kind="dgrad", T=8192, rows=18944, cols=3584, dtype="bf16", format="e4m3", gap=0, fresh=False),
        # a small ragged layer's, gradients in 32 bits and of a wide range
        dict(name="dgrad_odd", kind="dgrad", T=777, rows=1001, cols=1531, dtype="fp32", format="e5m2", gap=0, fresh=True),
        # a toy model's step: latency counts
        dict(name="adamw_small", kind="adamw", bits=32, layers=1, hidden=64, kv=32, inter=160, grad="fp32", copy="none", scaled=False),
        # a 7B-shaped block's logits
        dict(name="adamw_7b", kind="adamw", bits=32, layers=1, hidden=3584, kv=512, inter=18944, grad="fp32", copy="none", scaled=False),
        # odd sizes, gradients as a reduction in 16 bits leaves them and a clipping factor, weights copied to 16 bits
        dict(name="adamw_odd", kind="adamw", bits=32, layers=3, hidden=333, kv=77, inter=1019, grad="bf16", copy="bf16", scaled=True),
        # the 7B-shaped block with states in 8 bits
        dict(name="adamw8_7b", kind="adamw", bits=8, layers=1, hidden=3584, kv=512, inter=18944, grad="fp32", copy="none", scaled=False),
        # eight blocks of the smallest model in one call: many tensors, half of them small
        dict(name="adamw8_0.5b", kind="adamw", bits=8, layers=8, hidden=896, kv=128, inter=4864, grad="bf16", copy="none", scaled=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("fwd", "fwd", "dgrad", "adamw", "adamw"))
    if kind == "adamw":
        bits = rng.choice((32, 8))
        hidden = log_int(33, 3584)
        if rng.random() < 0.5:
            hidden = max(64, hidden // 64 * 64)
        c = dict(kind=kind, bits=bits, layers=log_int(1, 24), hidden=hidden, kv=max(8, hidden // rng.choice((4, 7))),
                 inter=int(hidden * rng.uniform(2.5, 5.2)), grad=rng.choice(("fp32", "fp32", "bf16", "fp16")),
                 copy=rng.choice(("none", "none", "bf16", "fp16")), scaled=rng.random() < 0.5)
        while c["layers"] > 1 and _elements(c) > 120_000_000:
            c["layers"] -= 1
        return c
    # widths of layers: multiples of a group of 4 or 8 along the inputs, anything along the outputs
    cols = rng.choice((4, 8)) * log_int(16, 2300)
    rows, T = log_int(64, 18944), rng.choice((log_int(1, 64), log_int(1, 16384), log_int(64, 16384)))
    while T * rows * cols > 8192 * 18944 * 3584:
        T = max(1, T // 2)
    return dict(kind=kind, T=T, rows=rows, cols=cols, dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")),
                format=rng.choice(("e4m3", "e4m3", "e5m2")), gap=rng.choice((0, 0, 0, 8, 3)), fresh=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# the copies' layout: blocks of 128 share 2^(s - 127)
# ---------------------------------------------------------------------------
# largest number, bits of the mantissa, least exponent
FORMATS = {"e4m3": (448.0, 3, -6, torch.float8_e4m3fn), "e5m2": (57344.0, 2, -14, torch.float8_e5m2)}


def _pitches(cols):
    """Bytes of a row's codes, and of its scales."""
    return (cols + 127) // 128 * 128, (cols + 2047) // 2048 * 16


def _power_of_two(e):
    """2^e in 32 bits, exactly (torch's pow and ldexp may round), for -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _scale(largest, top, mantissa_above):
    """Scale byte of the least 2^(s - 127) with largest <= top 2^(s - 127); `mantissa_above`: all ones less top's mantissa."""
    s = ((largest.view(torch.int32) + mantissa_above) >> 23) - int(math.floor(math.log2(top)))
    return torch.where(torch.isfinite(largest), s.clamp(1, 254), 255)


def _codes(x, s, format):
    """x in blocks [..., 128] or [..., 128, 128] whose scale bytes are s (of the shape that broadcasts)."""
    bad = s == 255
    q = torch.where(bad, 0.0, x) * _power_of_two(127 - torch.where(bad, 127, s))
    return q.to(FORMATS[format][3])


def _save(x, format):
    """Codes and scales of rows, blocks of 128 columns."""
    x = x.float()
    rows, cols = x.shape
    pitch, scale_pitch = _pitches(cols)
    x = torch.nn.functional.pad(x, (0, pitch - cols)).view(rows, pitch // 128, 128)
    s = _scale(x.abs().amax(-1), FORMATS[format][0], 0x1FFFFF)
    codes = _codes(x, s[..., None], format).view(rows, pitch)
    return codes.view(torch.uint8), torch.nn.functional.pad(s, (0, scale_pitch - pitch // 128), value=1).to(torch.uint8)


def _save_weight(W):
    """Codes (e4m3) and scales of a weight, blocks of 128 x 128."""
    W = W.float()
    rows, cols = W.shape
    pitch, scale_pitch = _pitches(cols)
    high = (rows + 127) // 128 * 128
    W = torch.nn.functional.pad(W, (0, pitch - cols, 0, high - rows)).view(high // 128, 128, pitch // 128, 128)
    s = _scale(W.abs().amax((1, 3)), FORMATS["e4m3"][0], 0x1FFFFF)
    codes = _codes(W, s[:, None, :, None], "e4m3").view(high, pitch)[:rows].contiguous()
    return codes.view(torch.uint8), torch.nn.functional.pad(s, (0, scale_pitch - pitch // 128), value=1).to(torch.uint8)


def _load(codes, scales, format, cols, block_rows=1):
    """The values that a copy stands for, in 32 bits."""
    rows, pitch = codes.shape
    s = scales[:, :pitch // 128].to(torch.int32)
    step = torch.where(s == 255, math.nan, _power_of_two(s.clamp(1, 254) - 127))
    step = step.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)
    return (codes.view(FORMATS[format][3]).float() * step)[:, :cols]


# ---------------------------------------------------------------------------
# AdamW states in 8 bits: blocks of 128 consecutive elements; m in e4m3, u = sqrt(v) without a sign, four bits
# of exponent and four of mantissa, the same bias; the last code of each is a NaN; rounded up with the probability
# of the remainder, 16 bits of it, m by the low and u by the high half of the element's random word
# ---------------------------------------------------------------------------
def _words(places):
    """Philox-4x32-10 words of the buffer's elements: key (seed), counter (element / 4, step, tensor)."""
    c0, c3 = _counters(places)
    c1, c2 = c0 >> 32, torch.full_like(c0, STEP)
    c0 = c0 & 0xFFFFFFFF
    k0, k1 = SEED & 0xFFFFFFFF, SEED >> 32

    def high_low(a, b):
        low, high = b & 0xFFFF, b >> 16
        return (a * high + (a * low >> 16)) >> 16, (a * b) & 0xFFFFFFFF

    for _ in range(10):
        h0, l0 = high_low(0xD2511F53, c0)
        h1, l1 = high_low(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return torch.stack((c0, c1, c2, c3), 1).view(-1)


def _encode(y, bits, top, above, random):
    """Codes (magnitudes) and scales of y >= 0 [blocks, 128]; random [blocks, 128]: 16 bits each."""
    finite = torch.isfinite(y)
    s = _scale(torch.where(finite, y, 0.0).amax(1), top, above)
    t = torch.where(finite, y, 0.0) * _power_of_two(127 - s)[:, None]
    drop = 23 - bits
    normal = ((t.view(torch.int32) + (random << (drop - 16))) >> drop) - (120 << bits)
    small = ((t * (2.0 ** (6 + bits) * 65536)).to(torch.int32) + random) >> 16
    code = torch.where(t < 2.0 ** -6, small, normal)
    return torch.where(finite, code, 0x7F if bits == 3 else 0xFF), s.to(torch.uint8)


def _encode_state(m, u, words):
    """(codes of m, codes of u, scales [blocks, 2]) of two buffers."""
    m, u, words = m.view(-1, 128), u.view(-1, 128), words.view(-1, 128)
    cm, sm = _encode(m.abs(), 3, 448.0, 0x1FFFFF, (words & 0xFFFF).to(torch.int32))
    cu, su = _encode(u, 4, 480.0, 0x0FFFFF, (words >> 16).to(torch.int32))
    cm = cm | torch.where(torch.signbit(m), 0x80, 0)
    cu = torch.where(u > 0, cu.clamp(min=1), cu)  # what is not zero stays so
    return cm.to(torch.uint8).view(-1), cu.to(torch.uint8).view(-1), torch.stack((sm, su), 1)


def _decode_state(state):
    """m and u in 32 bits."""
    cm, cu, s = state
    s = _power_of_two(s.to(torch.int32) - 127)
    m = cm.view(torch.float8_e4m3fn).float().view(-1, 128) * s[:, :1]
    c = cu.to(torch.int32).view(-1, 128)
    u = torch.where(c < 16, c, (16 + (c & 15)) << ((c >> 4) - 1).clamp(min=0)).float() * 2.0 ** -10
    u = torch.where(c == 255, math.nan, u) * s[:, 1:]
    return m.view(-1), u.view(-1)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _shapes(case):
    """Tensors of the step: per block q, k, v, o, gate, up, down and the weights of its two norms."""
    h, kv, i = case["hidden"], case["kv"], case["inter"]
    return [(h, h), (kv, h), (kv, h), (h, h), (i, h), (i, h), (h, i), (h,), (h,)] * case["layers"]


def _elements(case):
    return sum(math.prod(s) for s in _shapes(case))


def _places(case):
    """(first element in the buffers, number of elements) of each tensor, and the buffers' length."""
    places, at = [], 0
    for shape in _shapes(case):
        places.append((at, math.prod(shape)))
        at += (places[-1][1] + 127) // 128 * 128
    return places, at


def _counters(places):
    """Element / 4 and tensor of every four elements of the buffers."""
    fours = [(n + 127) // 128 * 32 for _, n in places]
    return (torch.cat([torch.arange(k, device="cuda", dtype=torch.int64) for k in fours]),
            torch.cat([torch.full((k,), i, device="cuda", dtype=torch.int64) for i, k in enumerate(fours)]))


def _rows(g, rows, cols, gap, dtype):
    """[rows, cols] with `gap` elements between a row's end and the next one's start."""
    return torch.empty(rows, cols + gap, dtype=dtype, device="cuda").normal_(generator=g)[:, :cols]


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"] == "adamw":
        places, total = _places(case)
        keep = torch.zeros(total, device="cuda")
        for at, n in places:
            keep[at:at + n] = 1
        make = lambda: torch.empty(total, device="cuda").normal_(generator=g)  # noqa: E731
        # gradients of a spread of magnitudes from element to element, one in sixteen zero
        size = (1.5 * make() - 7).exp() * keep
        grad = size * make() * (torch.rand(total, generator=g, device="cuda") >= 0.0625)
        # moments as a few steps of such gradients leave them
        return dict(param=make() * keep, grad=grad.to(DTYPES[case["grad"]]), m=0.3 * size * make(),
                    u=size * torch.rand(total, generator=g, device="cuda"),
                    scale=torch.rand(1, generator=g, device="cuda") if case["scaled"] else None)
    T, rows, cols, dtype = case["T"], case["rows"], case["cols"], DTYPES[case["dtype"]]
    # masked weights: two in four kept in the main
    W = torch.empty(rows, cols, device="cuda").normal_(generator=g).mul_(0.02)
    W = (W * torch.rand(rows, cols, generator=g, device="cuda").round_()).to(torch.bfloat16)
    if case["kind"] == "fwd":
        # activations: unit spread around a small offset, one channel in a hundred 20 times as large
        x = _rows(g, T, cols, case["gap"], dtype)
        large = torch.rand(cols, generator=g, device="cuda") < 0.01
        x.mul_(torch.where(large, 20.0, 1.0).to(dtype)).add_((0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype))
    else:
        # one token in eight is padding or a prompt's, with no gradient
        x = _rows(g, T, rows, case["gap"], dtype)
        x.mul_((1e-2 * (torch.rand(T, 1, generator=g, device="cuda") >= 0.125)).to(dtype))
    return {"x": x, "W": W}


def _state(case, seed):
    d = _inputs(case, seed)
    empty = lambda *shape, dtype=torch.uint8: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    if case["kind"] == "adamw":
        s = dict(case=case, places=_places(case)[0], **d)
        total = d["param"].numel()
        if case["copy"] != "none":
            s["copy"] = empty(total, dtype=DTYPES[case["copy"]]).zero_()
        if case["bits"] == 32:
            s["v"] = s.pop("u").square_()
        else:
            s["state"] = _encode_state(s["m"], s.pop("u"), torch.full((total,), 0x80008000, dtype=torch.int64, device="cuda"))
            # where what the states stand for goes: m, and the root of v
            s["m"], s["u"] = (empty(total, dtype=torch.bfloat16).zero_() for _ in range(2))
        return s
    T, rows, cols = case["T"], case["rows"], case["cols"]
    width, out = (cols, rows) if case["kind"] == "fwd" else (rows, cols)
    pitch, scale_pitch = _pitches(width)
    s = dict(case=case, x=d["x"], x8=(empty(T, pitch), empty(T, scale_pitch)),
             out=empty(T, out + case["gap"], dtype=DTYPES[case["dtype"]])[:, :out])
    if case["fresh"]:
        pitch, scale_pitch = _pitches(cols)
        s["W"], s["w8"] = d["W"], (empty(rows, pitch), empty((rows + 127) // 128, scale_pitch))
    else:
        s["w8"] = _save_weight(d["W"])
    return s


def prepare(case, seed):
    s = _state(case, seed)
    if own and case["kind"] == "adamw":
        s["plan"] = _adamw_plan(s)
    return s


def _adamw_plan(s):
    """The library's lists of tensors and its settings, which a program keeps from step to step."""
    import paper_2608_23048_gb300 as roi
    opt = roi.AdamW(OPT["lr"], OPT["beta1"], OPT["beta2"], OPT["eps"], OPT["weight_decay"], STEP)

    def of(name, at, n):
        return s[name][at:at + n] if name in s else None

    if s["case"]["bits"] == 32:
        step = [tuple(of(k, *p) for k in ("param", "grad", "m", "v", "copy")) for p in s["places"]]
        return opt, roi.make_adamw_step_items(step), None
    step, load = [], []
    for i, (at, n) in enumerate(s["places"]):
        codes, blocks = slice(at, at + (n + 127) // 128 * 128), slice(at // 128, (at + n + 127) // 128)
        state = (s["state"][0][codes], s["state"][1][codes], s["state"][2][blocks])
        step.append((of("param", at, n), of("grad", at, n), state, of("copy", at, n), i))
        load.append((state, of("m", at, n), of("u", at, n)))
    return opt, roi.make_adamw_step8_items(step), roi.make_adamw_state8_items(load)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _adamw_outputs(s):
    return {k: s[k] for k in ("param", "m", "v", "u", "copy") if k in s}


def _run_own(s):
    import paper_2608_23048_gb300 as roi
    case = s["case"]
    if case["kind"] == "adamw":
        opt, step, load = s["plan"]
        if case["bits"] == 32:
            roi.roi_adamw_step(step, opt, s["scale"])
        else:
            roi.roi_adamw_step8(step, opt, SEED, s["scale"])
            roi.roi_adamw_state8_load(load)
        return _adamw_outputs(s)
    if case["fresh"]:
        roi.roi_fp8_save_weight(s["W"], *s["w8"])
    roi.roi_fp8_save(s["x"], case["format"], *s["x8"])
    product = roi.roi_fp8_linear_fwd if case["kind"] == "fwd" else roi.roi_fp8_linear_dgrad
    product(s["x8"], case["format"], s["w8"], s["out"])
    return {"out": s["out"]}


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "adamw":
        _adamw_plain(s)
        return _adamw_outputs(s)
    fwd = case["kind"] == "fwd"
    w8 = _save_weight(s["W"]) if case["fresh"] else s["w8"]
    W = _load(*w8, "e4m3", case["cols"], 128)
    x = _load(*_save(s["x"], case["format"]), case["format"], case["cols"] if fwd else case["rows"])
    return {"out": (x @ (W.T if fwd else W)).to(s["out"].dtype)}


def _adamw_plain(s):
    f = lambda x: torch.tensor(x, dtype=torch.float32).item()  # noqa: E731  (settings are held in 32 bits)
    b1, b2, lr = f(OPT["beta1"]), f(OPT["beta2"]), f(OPT["lr"])
    step, r = f(lr / (1 - b1 ** STEP)), f(1 / math.sqrt(1 - b2 ** STEP))
    g = s["grad"].float()
    if s["scale"] is not None:
        g = g * s["scale"]
    if "state" in s:
        m, u = _decode_state(s["state"])
        v = u * u
    else:
        m, v = s["m"], s["v"]
    p = s["param"] * (1 - f(lr * f(OPT["weight_decay"])))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * (g * g)
    u = v.sqrt()
    p = p - step * m / (u * r + f(OPT["eps"]))
    s["param"].copy_(p)
    if "copy" in s:
        s["copy"].copy_(p)
    if "state" not in s:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return
    for kept, new in zip(s["state"], _encode_state(m, u, _words(s["places"]))):
        kept.copy_(new)
    m, u = _decode_state(s["state"])
    s["m"].copy_(m)
    s["u"].copy_(u)


def work(case):
    if case["kind"] == "adamw":
        E, copy = _elements(case), 0 if case["copy"] == "none" else 2
        grad = 4 if case["grad"] == "fp32" else 2
        if case["bits"] == 32:
            return {"bytes": (24 + grad + copy) * E, "flops": 15 * E}
        # states in and out, and what they stand for
        return {"bytes": (8 + grad + copy + 2 * 2 + 4) * E + 4 * (E // 128), "flops": 40 * E}
    T, rows, cols, b = case["T"], case["rows"], case["cols"], 4 if case["dtype"] == "fp32" else 2
    return {"bytes": b * T * (rows + cols) + (2 if case["fresh"] else 1) * rows * cols, "flops": 2 * T * rows * cols}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_power(e):
    """2^e in 64 bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _least_exponent(largest, top):
    """The least e with largest <= top 2^e, no less than -126."""
    fraction, exponent = torch.frexp(largest / top)  # fraction in [1/2, 1)
    return torch.where(largest > 0, torch.where(fraction == 0.5, exponent - 1, exponent), -126).clamp(min=-126)


def _nearest(x, format, high):
    """What the copy of x (finite, in 64 bits) stands for, blocks of high x 128."""
    top, bits, least, _ = FORMATS[format]
    out = torch.empty_like(x)
    rows, cols = x.shape
    for c in range(0, cols, 128):
        part = x[:, c:c + 128]
        largest = part.abs().amax(1)
        if high > 1:
            largest = torch.cat([p.amax().expand(p.numel()) for p in largest.split(high)])
        unit = _exact_power(_least_exponent(largest, top))[:, None]
        t = part / unit
        step = _exact_power((torch.frexp(t)[1] - 1).clamp(min=least) - bits)
        out[:, c:c + 128] = torch.where(t == 0, 0.0, torch.round(t / step) * step) * unit
    return out


def _exact_words(places):
    """The same words, their products in pieces of 16 bits."""
    q, tensor = _counters(places)
    c = [q, torch.zeros_like(q), torch.full_like(q, STEP), tensor]
    key = [SEED % 2 ** 32, SEED // 2 ** 32]

    def product(const, x):
        a, b = divmod(const, 65536)
        p, q = torch.div(x, 65536, rounding_mode="floor"), x % 65536
        middle = a * q + b * p
        low = b * q + (middle % 65536) * 65536
        return a * p + torch.div(middle, 65536, rounding_mode="floor") + torch.div(low, 2 ** 32, rounding_mode="floor"), low % 2 ** 32

    for _ in range(10):
        (h0, l0), (h1, l1) = product(3528531795, c[0]), product(3449720151, c[2])
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 2654435769) % 2 ** 32, (key[1] + 3144134277) % 2 ** 32]
    return torch.stack(c, 1).flatten()


def _exact_rounded(y, bits, top, random, least_code):
    """What the 8-bit form of y (finite, in 64 bits) stands for."""
    part = y.view(-1, 128)
    unit = _exact_power(_least_exponent(part.abs().amax(1), top))[:, None]
    t = part.abs() / unit
    step = _exact_power((torch.frexp(t)[1] - 1).clamp(min=-6) - bits)
    step = torch.where(t == 0, 2.0 ** (-6 - bits), step)
    code = torch.floor((torch.floor(t / step * 65536) + random.view(-1, 128)) / 65536)
    if least_code:
        code = torch.where(t > 0, code.clamp(min=1), code)
    return (torch.copysign(code * step, part) * unit).view(-1)


def exact(case, seed):
    if case["kind"] != "adamw":
        d = _inputs(case, seed)
        W = _nearest(d["W"].double(), "e4m3", 128)
        x = _nearest(d["x"].double(), case["format"], 1)
        return {"out": x @ (W.T if case["kind"] == "fwd" else W)}
    d = _state(case, seed)
    single = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    b1, b2, lr, wd, eps = (single(OPT[k]) for k in ("beta1", "beta2", "lr", "weight_decay", "eps"))
    g = d["grad"].double() * (1.0 if d["scale"] is None else d["scale"].double())
    if case["bits"] == 8:
        m, u = (x.double() for x in _decode_state(d["state"]))
        v = u.square()
    else:
        m, v = d["m"].double(), d["v"].double()
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g.square() - v)
    mh, vh = m / (1 - b1 ** STEP), v / (1 - b2 ** STEP)
    p = d["param"].double()
    p = p - lr * wd * p - lr * mh / (vh.sqrt() + eps)
    out = {"param": p, "m": m, "v": v}
    if case["bits"] == 8:
        words = _exact_words(d["places"])
        out = {"param": p, "m": _exact_rounded(m, 3, 448.0, words % 65536, False),
               "u": _exact_rounded(v.sqrt(), 4, 480.0, torch.div(words, 65536, rounding_mode="floor"), True)}
    if "copy" in d:
        out["copy"] = p
    return out
