"""Layer norm and RMS norm (roi_norm_fwd, roi_norm_bwd) against the CPU oracle in float64.

Tolerances, from the arithmetic (u = 2^-24, the rounding of one float32 operation; ut that of
the output's type).  A sum over a row or over rows is a chain of additions in a thread, then a
tree: with n additions one after another its error is at most n u times the sum of magnitudes.
Chains over a row are at most 16 (four pieces of 8, in pairs) + 10 (shuffles) + 16 (warps)
+ 1 (1 / n), under 48 up to 16384 columns; past those a thread adds cols / 512 elements.  So,
with S = 64 + cols / 512:
  mean   S u mean|x|
  rstd   its square's relative error is S u plus what the mean's error adds: (S u mean|x| rstd)^2,
         and rstd's half of it, plus 3 roundings: rel <= S u + (S u mean|x| rstd)^2
  y      |g| (|xh| (rel of rstd + 4 u) + rstd S u mean|x|) + 2 u |y|, then ut |y|
  dx     rstd (S u + 8 u)(|a| + mean|a| + |xh| mean|a xh|), then ut |dx|; x, mean and rstd are
         inputs here, so xh has 2 roundings
  dgamma, dbeta   a chain of rows / (CTAs x teams) per thread, the teams (15), the CTAs (152 / 8)
         and 8: at most rows / 152 + 64 additions, plus 3 roundings of each term
plus half the least subnormal of float16 outputs (2^-25).  Checkpoints of x are exact; those of
y are the oracle's of the y that came back, bit for bit.
"""
import numpy as np
import pytest

from oracle import layer_oracle as LO
from test_checkpoint_gpu import DTYPES, on_gpu, roi, same, values  # noqa: F401  (roi: the fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11, "float32": U}
EPS = 1e-6


def tiny(dtype):
    return 2.0 ** -25 if dtype == "float16" else 2.0 ** -134 if dtype == "bfloat16" else 2.0 ** -149


class Case:
    """Inputs of one call on the GPU, their values in float64 on the CPU."""

    def __init__(self, rows, cols, dtype, kind, seed=0, gap=0, offset=0, params="own", x=None):
        import torch
        self.rows, self.cols, self.dtype, self.kind, self.gap, self.offset = rows, cols, dtype, kind, gap, offset
        g = torch.Generator().manual_seed(1000 + seed)
        t = getattr(torch, dtype)
        pt = torch.float32 if params == "float32" else t
        x = values(rows, cols, dtype, seed) + 0.3 if x is None else x
        self.x = on_gpu(x, dtype, gap, offset)
        self.dy = on_gpu(torch.randn(rows, cols, generator=g), dtype, gap, offset)
        self.gamma = self.beta = None
        if params != "none":
            self.gamma = (1 + 0.3 * torch.randn(cols, generator=g)).to(pt).cuda()
            self.beta = torch.randn(cols, generator=g).to(pt).cuda() if kind == "layer" else None

    def new(self):
        import torch
        return on_gpu(torch.zeros(self.rows, self.cols), self.dtype, self.gap, self.offset)

    def f64(self, t):
        return None if t is None else t.double().cpu().numpy()


def check_fwd(roi, c, eps=EPS):
    import torch
    rows, cols = c.rows, c.cols
    y = c.new()
    mean = torch.full((rows,), 9.0, device="cuda") if c.kind == "layer" else None
    rstd = torch.full((rows,), 9.0, device="cuda")
    xq, yq = roi.new_checkpoint(rows, cols), roi.new_checkpoint(rows, cols)
    for t in xq + yq:
        t.fill_(99)
    roi.roi_norm_fwd(c.x, c.kind, c.gamma, c.beta, eps, y, mean, rstd, xq, yq)
    x, g = c.f64(c.x), c.f64(c.gamma)
    yo, mo, ro = LO.norm_fwd(x, c.kind, g, c.f64(c.beta), eps)
    S = 64 + cols / 512
    mx = np.abs(x).mean(1)
    if c.kind == "layer":
        assert np.all(np.abs(c.f64(mean) - mo) <= S * U * mx + 2.0 ** -149)
    rel = S * U + ((S * U * mx * ro) ** 2 if c.kind == "layer" else 0 * ro)
    assert np.all(np.abs(c.f64(rstd) - ro) <= rel * ro)
    got = c.f64(y)
    xh = np.abs((x - mo[:, None]) * ro[:, None])
    w = np.ones(cols) if g is None else np.abs(g)
    bound = w * (xh * (rel + 4 * U)[:, None] + (ro * S * U * mx if c.kind == "layer" else 0 * ro)[:, None])
    bound = bound + 2 * U * np.abs(yo)
    bound = bound + UT[c.dtype] * (np.abs(yo) + bound) + tiny(c.dtype)
    assert np.all(np.abs(got - yo) <= bound), np.max(np.abs(got - yo) / bound)
    for (codes, scales), of in ((xq, x), (yq, got)):
        a, b = LO.checkpoint_save(of)
        assert same(codes.cpu().numpy(), a) and same(scales.cpu().numpy(), b)
    # without the further outputs, the same bits
    again = c.new()
    roi.roi_norm_fwd(c.x, c.kind, c.gamma, c.beta, eps, again)
    assert torch.equal(again, y)
    return mean, rstd


def check_bwd(roi, c, mean, rstd, source):
    import torch
    rows, cols = c.rows, c.cols
    x_in, x = c.x, c.f64(c.x)
    if source == "checkpoint":
        x_in = roi.new_checkpoint(rows, cols)
        roi.roi_checkpoint_save(c.x, *x_in)
        x = LO.checkpoint_load(x_in[0].cpu().numpy(), x_in[1].cpu().numpy(), cols)
    ws = torch.empty(max(16, roi.roi_norm_bwd_workspace_size(rows, cols)), dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        dx, dg = c.new(), torch.full((cols,), 9.0, device="cuda")
        db = torch.full((cols,), 9.0, device="cuda") if c.kind == "layer" else None
        ws.fill_(255)
        roi.roi_norm_bwd(c.dy, x_in, c.kind, c.gamma, mean, rstd, dx, dg, db, ws)
        out.append((dx, dg, db))
    dx, dg, db = out[0]
    assert torch.equal(dx, out[1][0]) and torch.equal(dg, out[1][1]) and (db is None or torch.equal(db, out[1][2]))
    dy, g = c.f64(c.dy), c.f64(c.gamma)
    mo, ro = (c.f64(mean) if mean is not None else np.zeros(rows)), c.f64(rstd)
    dxo, dgo, dbo = LO.norm_bwd(dy, x, c.kind, g, mo, ro)
    xh, a = (x - mo[:, None]) * ro[:, None], dy * (1 if g is None else g)
    S = 64 + cols / 512
    m = lambda v: np.abs(v).mean(1, keepdims=True)  # noqa: E731
    bound = ro[:, None] * (S + 8) * U * (np.abs(a) + m(a) + np.abs(xh) * m(a * xh))
    bound = bound + UT[c.dtype] * (np.abs(dxo) + bound) + tiny(c.dtype)
    assert np.all(np.abs(c.f64(dx) - dxo) <= bound), np.max(np.abs(c.f64(dx) - dxo) / bound)
    n = rows / 152 + 64 + 3
    assert np.all(np.abs(c.f64(dg) - dgo) <= n * U * np.abs(dy * xh).sum(0) + 1e-40)
    if db is not None:
        assert np.all(np.abs(c.f64(db) - dbo) <= n * U * np.abs(dy).sum(0))
    # dx alone, and one of the sums alone
    alone, dg2 = c.new(), torch.empty_like(dg)
    roi.roi_norm_bwd(c.dy, x_in, c.kind, c.gamma, mean, rstd, alone)
    assert torch.equal(alone, dx)
    roi.roi_norm_bwd(c.dy, x_in, c.kind, c.gamma, mean, rstd, alone, dg2, None, ws)
    assert torch.equal(dg2, dg)
    if db is not None:
        roi.roi_norm_bwd(c.dy, x_in, c.kind, c.gamma, mean, rstd, alone, None, dg2, ws)
        assert torch.equal(dg2, db)


def check(roi, c):
    mean, rstd = check_fwd(roi, c)
    for source in ("x", "checkpoint"):
        check_bwd(roi, c, mean, rstd, source)
    roi.roi_device_status()


SIZES = [(1, 1), (1, 7), (3, 32), (2, 40), (5, 127), (700, 64), (1, 3584), (33, 896), (400, 1001), (20, 1531), (310, 1536),
         (9, 4096), (7, 4104), (320, 4111), (5, 8192), (3, 8200), (4, 9001), (2, 16384), (2, 16390), (2, 40000)]


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(roi, rows, cols, dtype, kind):  # noqa: F811
    check(roi, Case(rows, cols, dtype, kind, seed=rows + cols))


@pytest.mark.parametrize("gap,offset,params", [(8, 0, "own"), (3, 0, "float32"), (0, 1, "none"), (4, 8, "float32")])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(37, 328), (160, 1000), (3, 5000)])
def test_strides_and_parameters(roi, rows, cols, dtype, gap, offset, params):  # noqa: F811
    for kind in ("layer", "rms"):
        check(roi, Case(rows, cols, dtype, kind, 7, gap, offset, params))


def test_many_rows(roi):  # noqa: F811
    check(roi, Case(9000, 256, "bfloat16", "layer", 1))
    check(roi, Case(5001, 72, "float16", "rms", 2))


def test_rows_that_say_nothing(roi):  # noqa: F811
    """Zero rows and constant rows (no deviation: rstd = eps^-1/2), rows of large magnitude, and
    rows of padding with a zero gradient."""
    import torch
    for kind in ("layer", "rms"):
        x = values(12, 200, "float32", 3)
        x[1], x[2], x[3], x[4] = 0, 5, 1e18, 1e-18
        c = Case(12, 200, "float32", kind, 4, x=x)
        c.dy[5:7] = 0
        mean, rstd = check_fwd(roi, c, eps=1e-5)
        check_bwd(roi, c, mean, rstd, "x")
        dx = c.new()
        roi.roi_norm_bwd(c.dy, c.x, kind, c.gamma, mean, rstd, dx)
        assert not dx[5:7].any()


def test_non_finite_rows_stay_by_themselves(roi):  # noqa: F811
    """A NaN or infinity makes its own row NaN, its own blocks NaN in the checkpoint, its column of
    the weight's gradient NaN, and leaves everything else what it is without that row."""
    import torch
    x = values(20, 160, "bfloat16", 5)
    x[4, 7], x[11, 100] = float("nan"), float("inf")
    c = Case(20, 160, "bfloat16", "layer", 6, x=x)
    y, mean, rstd, q = c.new(), torch.empty(20, device="cuda"), torch.empty(20, device="cuda"), roi.new_checkpoint(20, 160)
    roi.roi_norm_fwd(c.x, "layer", c.gamma, c.beta, EPS, y, mean, rstd, q)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda")
    bad[4] = bad[11] = True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()
    s = q[1].cpu()
    assert (s == 255).nonzero().tolist() == [[4, 0], [11, 3]]
    dx, dg, ws = c.new(), torch.empty(160, device="cuda"), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    roi.roi_norm_bwd(c.dy, q, "layer", c.gamma, mean, rstd, dx, dg, None, ws)
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[~bad]).all()
    keep = (~bad).nonzero().flatten()
    want = c.new()[keep]
    roi.roi_norm_bwd(c.dy[keep], c.x[keep], "layer", c.gamma, mean[keep], rstd[keep], want)
    roi.roi_norm_bwd(c.dy, c.x, "layer", c.gamma, mean, rstd, dx, dg, None, ws)
    assert torch.equal(dx[keep], want)


def test_gradient_against_differences(roi):  # noqa: F811
    """The float32 gradients against central differences of the float64 forward: their own error
    is h^2 times a third derivative, under 1e-8 here; the rest is the bound of check_bwd, which is
    under 2e-5 of the largest gradient."""
    import torch
    for kind in ("layer", "rms"):
        c = Case(2, 24, "float32", kind, 8, x=values(2, 24, "float32", 9).clamp(-3, 3))
        x, g, dy = c.f64(c.x), c.f64(c.gamma), c.f64(c.dy)
        mean = torch.empty(2, device="cuda") if kind == "layer" else None
        rstd, y, dx, dg = torch.empty(2, device="cuda"), c.new(), c.new(), torch.empty(24, device="cuda")
        ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        roi.roi_norm_fwd(c.x, kind, c.gamma, c.beta, 1e-3, y, mean, rstd)
        roi.roi_norm_bwd(c.dy, c.x, kind, c.gamma, mean, rstd, dx, dg, None, ws)
        loss = lambda x, g: float((LO.norm_fwd(x, kind, g, None, 1e-3)[0] * dy).sum())  # noqa: E731
        h = 1e-5
        fd = np.zeros_like(x)
        for at in np.ndindex(*x.shape):
            d = np.zeros_like(x)
            d[at] = h
            fd[at] = (loss(x + d, g) - loss(x - d, g)) / (2 * h)
        assert np.max(np.abs(c.f64(dx) - fd)) <= 2e-5 * np.max(np.abs(fd)) + 1e-7
        fd = np.array([(loss(x, g + h * np.eye(24)[k]) - loss(x, g - h * np.eye(24)[k])) / (2 * h) for k in range(24)])
        assert np.max(np.abs(c.f64(dg) - fd)) <= 2e-5 * np.max(np.abs(fd)) + 1e-7


def test_past_32_bits(roi):  # noqa: F811
    """Element offsets past 2^32: the last rows of a long call are those of a short one."""
    import torch
    rows, cols = 1_060_000, 4096
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-8:] = values(8, cols, "bfloat16", 1).to("cuda", torch.bfloat16)
    y, q, rstd = torch.empty_like(x), roi.new_checkpoint(rows, cols), torch.empty(rows, device="cuda")
    roi.roi_norm_fwd(x, "rms", None, None, EPS, y, None, rstd, None, q)
    y8, q8, r8 = torch.empty_like(x[-8:]), roi.new_checkpoint(8, cols), torch.empty(8, device="cuda")
    roi.roi_norm_fwd(x[-8:], "rms", None, None, EPS, y8, None, r8, None, q8)
    # (a short call adds in another order)
    assert torch.allclose(y[-8:].float(), y8.float(), rtol=2 ** -7) and torch.allclose(rstd[-8:], r8, rtol=1e-5)
    assert not y[:-8].any() and bool((q[1][:-8] == 7).all())
    dx, dg, ws = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(8 << 20, dtype=torch.uint8, device="cuda")
    dx8, dg8 = torch.empty_like(y8), torch.empty_like(dg)
    roi.roi_norm_bwd(y, q, "rms", None, None, rstd, dx, dg, None, ws)
    roi.roi_norm_bwd(y[-8:], (q[0][-8:], q[1][-8:]), "rms", None, None, rstd[-8:], dx8, dg8, None, ws)
    assert torch.equal(dx[-8:], dx8) and torch.allclose(dg, dg8, rtol=1e-5, atol=1e-5) and not dx[:-8].any()


def test_empty_and_refusals(roi):  # noqa: F811
    import torch
    c = Case(4, 64, "bfloat16", "layer", 1)
    y, mean, rstd = c.new(), torch.ones(4, device="cuda"), torch.ones(4, device="cuda")
    dg, db = torch.full((64,), 9.0, device="cuda"), torch.full((64,), 9.0, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    roi.roi_norm_fwd(c.x[:0], "layer", c.gamma, c.beta, EPS, y[:0])
    roi.roi_norm_bwd(c.dy[:0], c.x[:0], "layer", c.gamma, mean[:0], rstd[:0], y[:0], dg, db)
    assert not dg.any() and not db.any()   # empty sums

    def fails(code, f, *a, **k):
        with pytest.raises(roi.RoiError) as e:
            f(*a, **k)
        assert e.value.status == code, e.value
    fails(10, roi.roi_norm_fwd, c.x, "rms", c.gamma, c.beta, EPS, y)          # a bias, and none in the RMS norm
    fails(10, roi.roi_norm_fwd, c.x, "rms", c.gamma, None, EPS, y, mean)
    fails(10, roi.roi_norm_fwd, c.x, "layer", c.gamma, None, -1.0, y)
    fails(10, roi.roi_norm_fwd, c.x, "layer", c.gamma, None, float("nan"), y)
    fails(6, roi.roi_norm_fwd, c.x, "layer", c.gamma, None, EPS, c.x)
    fails(10, roi.roi_norm_bwd, c.dy, c.x, "rms", c.gamma, mean, rstd, y)
    fails(1, roi.roi_norm_bwd, c.dy, c.x, "layer", c.gamma, None, rstd, y)
    fails(1, roi.roi_norm_bwd, c.dy, c.x, "layer", c.gamma, mean, rstd, y, dg)  # no workspace
    fails(2, roi.roi_norm_bwd, c.dy, c.x, "layer", c.gamma, mean, rstd, y, dg, None, ws[:16])
    fails(6, roi.roi_norm_bwd, c.dy, c.x, "layer", c.gamma, mean, rstd, c.dy)
    with pytest.raises(ValueError):
        roi.roi_norm_fwd(c.x, "batch", None, None, EPS, y)
    with pytest.raises(TypeError):
        roi.roi_norm_fwd(c.x, "layer", c.gamma.half(), None, EPS, y)
    with pytest.raises(TypeError):
        roi.roi_norm_fwd(c.x, "layer", c.gamma, c.beta.float(), EPS, y)
    with pytest.raises(TypeError):
        roi.roi_norm_bwd(c.dy, c.x.float(), "layer", c.gamma, mean, rstd, y)
    # columns between those of an input are no overlap
    room = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    room[:, :64] = c.x
    roi.roi_norm_fwd(room[:, :64], "layer", c.gamma, c.beta, EPS, room[:, 64:])
    roi.roi_norm_fwd(c.x, "layer", c.gamma, c.beta, EPS, y)
    assert torch.equal(room[:, 64:], y) and torch.equal(room[:, :64], c.x)
