"""The AdamW step over many tensors, with moments in 32 bits and in 8, against the oracle bit for bit: its operations are
stated one by one and each rounds in one way."""
import numpy as np
import pytest

from oracle import optim_oracle as O
from oracle import philox
from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

SETTINGS = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.05, t=7)
SEED = 0x1234567890ABCDEF
# one element, parts of a thread's four, of a block, of a tile; whole ones; tensors of several tiles
SIZES = [1, 2, 3, 4, 5, 127, 128, 129, 130, 1000, 1024, 1025, 4099, 70001]


def bits(x):
    x = x.detach().cpu().numpy() if hasattr(x, "detach") else np.ascontiguousarray(x)
    return x.view({1: np.uint8, 2: np.uint16, 4: np.uint32}[x.dtype.itemsize])


def same(got, want):
    """Bit for bit, NaN for NaN."""
    import torch
    want = torch.from_numpy(np.ascontiguousarray(want))
    got = got.detach().cpu().reshape(-1)
    return bool(((got == want) | (got.isnan() & want.isnan())).all()) if got.is_floating_point() else torch.equal(got, want.reshape(-1))


def tensors(n, dtype, seed):
    """param, grad (of that type), m, v of a tensor; zeros, a wide spread, and an element that is not finite."""
    import torch
    g = torch.Generator().manual_seed(seed * 1000 + n)
    size = torch.exp(3 * torch.randn(n, generator=g) - 6)
    grad = (size * torch.randn(n, generator=g) * (torch.rand(n, generator=g) > 0.1)).to(getattr(torch, dtype))
    m, v = 0.3 * size * torch.randn(n, generator=g), (size * torch.rand(n, generator=g)) ** 2
    if n > 4000:
        grad[3500], grad[10], m[20], v[30] = float("inf"), float("nan"), float("inf"), 0.0
    return torch.randn(n, generator=g), grad, m, v


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("scale", [None, 0.37])
@pytest.mark.parametrize("copy", [None, "bfloat16", "float16"])
def test_step(roi, dtype, scale, copy):  # noqa: F811
    """All sizes in one call, and twice in a row."""
    import torch
    host = [tensors(n, dtype, 1) for n in SIZES]
    items = [tuple(t.clone().cuda() for t in h) + (None if copy is None else torch.zeros(n, dtype=getattr(torch, copy), device="cuda"),)
             for n, h in zip(SIZES, host)]
    factor = None if scale is None else torch.full((1,), scale, device="cuda")
    arr = roi.make_adamw_step_items(items)
    want = [[t.float().numpy() for t in h] for h in host]
    for t in (7, 8):
        s = dict(SETTINGS, t=t)
        before = roi.roi_launch_count()
        roi.roi_adamw_step(arr, roi.AdamW(*s.values()), factor)
        assert roi.roi_launch_count() == before + 1
        for w in want:
            w[0], w[2], w[3], _ = O.step(*w, O.constants(**s), scale)
    roi.roi_device_status()
    for item, w in zip(items, want):
        assert same(item[0], w[0]) and same(item[2], w[2]) and same(item[3], w[3]), len(w[0])
        assert same(item[1], w[1])
        if copy is not None:
            half = torch.from_numpy(w[0]).to(getattr(torch, copy))
            assert torch.equal(item[4].cpu().nan_to_num(1.5), half.nan_to_num(1.5))


def test_step_is_the_fused_one(roi):  # noqa: F811
    """On the gradient that roi_mask_bwd gives, the bits of roi_mask_bwd_adamw."""
    import torch

    import workloads as WL
    W, phi, dWm = WL.make_inputs(40, 264, "normal", 5, device="cuda")
    st = roi.NoiseState(3, 4, 5, 1.0, 0)
    opt = roi.AdamW(*SETTINGS.values())
    m, v = (0.01 * torch.rand_like(phi) for _ in range(2))
    a, b = [t.clone() for t in (phi, m, v)], [t.clone() for t in (phi, m, v)]
    roi.roi_mask_bwd_adamw(a[0], W, st, 2, 4, dWm, 0.7, a[1], a[2], opt)
    g = torch.empty_like(phi)
    roi.roi_mask_bwd(phi, W, st, 2, 4, dWm, 0.7, g)
    roi.roi_adamw_step([(b[0], g, b[1], b[2], None)], opt)
    roi.roi_device_status()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def state_of(m, v, seed):
    """(codes, codes, scales) on the host of moments."""
    n = m.numel()
    whole = -(-n // 128) * 128
    pad = lambda x: np.concatenate([x.numpy(), np.zeros(whole - n, np.float32)])  # noqa: E731
    r = np.random.default_rng(seed).integers(0, 65536, whole)
    cm, sm = O.encode(pad(m), "m", r)
    cu, su = O.encode(pad(v.sqrt()), "u", r)
    return cm, cu, np.stack([sm, su], 1)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("scale", [None, 0.37])
def test_step8(roi, dtype, scale):  # noqa: F811
    """Codes, scales and parameters after two steps, and what the states stand for."""
    import torch
    host = [tensors(n, dtype, 2) for n in SIZES]
    states = [state_of(h[2], h[3], 1) for h in host]
    copies = [None if i % 3 == 0 else torch.zeros(n, dtype=torch.bfloat16 if i % 3 == 1 else torch.float16, device="cuda")
              for i, n in enumerate(SIZES)]
    items = [(h[0].clone().cuda(), h[1].cuda(), tuple(torch.from_numpy(s.copy()).cuda() for s in st), c, 11 + i)
             for i, (h, st, c) in enumerate(zip(host, states, copies))]
    factor = None if scale is None else torch.full((1,), scale, device="cuda")
    arr = roi.make_adamw_step8_items(items)
    params = [h[0].numpy() for h in host]
    for t in (7, 8):
        s = dict(SETTINGS, t=t)
        roi.roi_adamw_step8(arr, roi.AdamW(*s.values()), SEED, factor)
        for i, h in enumerate(host):
            params[i], states[i] = O.step8(params[i], h[1].float().numpy(), states[i], O.constants(**s), SEED, t, 11 + i, scale)
    loads = [(it[2], torch.full_like(it[0], 7.0), torch.full_like(it[0], 7.0)) for it in items]
    roi.roi_adamw_state8_load(loads)
    roi.roi_device_status()
    for it, st, p, ld, c in zip(items, states, params, loads, copies):
        n = p.size
        for got, want in zip(it[2], st):
            assert np.array_equal(got.cpu().numpy(), want), n
        assert same(it[0], p), n
        assert same(ld[1], O.decode(st[0], st[2][:, 0], "m")[:n]) and same(ld[2], O.decode(st[1], st[2][:, 1], "u")[:n])
        if c is not None:
            assert torch.equal(c.cpu().nan_to_num(1.5), torch.from_numpy(p).to(c.dtype).nan_to_num(1.5))


@pytest.mark.parametrize("kind", [0, 1])
def test_every_code(roi, kind):  # noqa: F811
    """Every pair of a code and a scale byte, loaded in every type; those that no step writes among them."""
    import torch
    codes = np.tile(np.arange(256, dtype=np.uint8), 256)
    scales = np.repeat(np.arange(256, dtype=np.uint8), 2)
    state = tuple(torch.from_numpy(x).cuda() for x in (codes, codes, np.stack([scales, scales], 1)))
    name = "mu"[kind]
    want = torch.from_numpy(O.decode(codes, scales, name))
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        out = torch.zeros(codes.size, dtype=dtype, device="cuda")
        roi.roi_adamw_state8_load([(state, out if kind == 0 else None, out if kind == 1 else None)])
        assert torch.equal(out.cpu().nan_to_num(1.5), want.to(dtype).nan_to_num(1.5))
        if dtype == torch.bfloat16:
            # a block's least code is 2^-10 or 2^-9 of its power of two 2^(s - 127), bfloat16's least number 2^-133
            held = torch.from_numpy(np.repeat(scales, 128) >= 4)
            assert torch.equal(out.cpu().float()[held].nan_to_num(1.5), want[held].nan_to_num(1.5))
    roi.roi_device_status()


def test_step8_extremes(roi):  # noqa: F811
    """Moments from the least to the largest numbers: blocks of float32's subnormals, of its largest numbers, of all
    magnitudes at once; gradients that are zero."""
    import torch
    n = 128 * 6
    g = np.zeros(n, np.float32)
    g[:128] = np.ldexp(1.0, -149) * np.arange(1, 129)
    g[128:256] = 1.5e38 * np.linspace(-1, 1, 128)
    g[256:384] = np.exp2(np.linspace(-149, 60, 128)) * (-1.0) ** np.arange(128)
    g[384:512] = 1e-30
    p = np.linspace(-1, 1, n).astype(np.float32)
    state = (np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros((6, 2), np.uint8))
    dev = [torch.from_numpy(p.copy()).cuda(), torch.from_numpy(g).cuda(), roi.new_adamw_state8(n)]
    for t in range(1, 5):
        s = dict(SETTINGS, t=t)
        roi.roi_adamw_step8([(dev[0], dev[1], dev[2], None, 3)], roi.AdamW(*s.values()), SEED)
        p, state = O.step8(p, g, state, O.constants(**s), SEED, t, 3)
        for got, want in zip(dev[2], state):
            assert np.array_equal(got.cpu().numpy(), want), t
        assert same(dev[0], p), t
        # (the next steps with other signs)
        g = -g
        dev[1].neg_()
    roi.roi_device_status()


def test_more_tensors_than_a_launch_takes(roi):  # noqa: F811
    """1000 tensors, some empty, in one call: as one by one."""
    import torch
    sizes = [(37 * i) % 300 for i in range(1000)]
    make = lambda: [tuple(t.cuda() for t in tensors(n, "float32", 3)) for n in sizes]  # noqa: E731
    a, b = make(), make()
    opt = roi.AdamW(*SETTINGS.values())
    roi.roi_adamw_step([x + (None,) for x in a], opt)
    for x in b:
        roi.roi_adamw_step([x + (None,)], opt)
    sa, sb = ([roi.new_adamw_state8(n) for n in sizes] for _ in range(2))
    roi.roi_adamw_step8([(x[0], x[1], s, None, i) for i, (x, s) in enumerate(zip(a, sa))], opt, SEED)
    for i, (x, s) in enumerate(zip(b, sb)):
        roi.roi_adamw_step8([(x[0], x[1], s, None, i)], opt, SEED)
    roi.roi_device_status()
    for x, y, s, q in zip(a, b, sa, sb):
        assert all(torch.equal(i, j) for i, j in zip(x, y)) and all(torch.equal(i, j) for i, j in zip(s, q))
    roi.roi_adamw_step([], opt)
    roi.roi_adamw_step8([], opt, 0)
    roi.roi_adamw_state8_load([])


def test_words_are_the_noise_of_the_mask(roi):  # noqa: F811
    """Elements 2^31 and on of a tensor draw their own words (only the last block's gradient is not zero)."""
    import torch
    n = 2 ** 31 + 2 ** 20 + 77
    if torch.cuda.mem_get_info()[0] < 6 * n + 12 * n:
        pytest.skip("needs 40 GB")
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = n // 128 * 128
    host = tensors(n - tail, "bfloat16", 4)[1]
    g[tail:] = host.cuda()
    state = roi.new_adamw_state8(n)
    roi.roi_adamw_step8([(p, g, state, None, 2)], roi.AdamW(*dict(SETTINGS, t=1).values()), SEED)
    roi.roi_device_status()
    k = O.constants(**dict(SETTINGS, t=1))
    zero = np.zeros(n - tail, np.float32)
    want, m, _, u = O.step(zero, host.float().numpy(), zero, zero, k)
    words = philox.noise_words(SEED, 1, 2, np.arange(tail, tail + 128, dtype=np.uint64)).astype(np.int64)
    pad = lambda x: np.concatenate([x, np.zeros(128 - x.size, np.float32)])  # noqa: E731
    assert np.array_equal(state[0][tail:].cpu().numpy(), O.encode(pad(m), "m", words & 0xFFFF)[0])
    assert np.array_equal(state[1][tail:].cpu().numpy(), O.encode(pad(u), "u", words >> 16)[0])
    assert same(p[tail:], want) and not p[:tail].any() and not state[0][:tail].any()
