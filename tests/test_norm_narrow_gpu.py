"""Norms of rows so short that several lie in one granule of 16 bytes, and backward passes from
checkpoints whose rows of scales do (up to 128 columns), at every place in it.  Bounds: those of
test_norm_gpu.py."""
import numpy as np
import pytest

from oracle import layer_oracle as LO
from test_checkpoint_gpu import DTYPES, roi  # noqa: F401  (the fixture)
from test_norm_gpu import U, UT, Case, check, check_bwd, check_fwd, tiny

pytestmark = pytest.mark.gpu


def check_past_half(roi, c):  # noqa: F811
    """check, for a layer norm of one column in float16: rstd is eps^-1/2, and from a checkpoint, whose x is not
    the mean, dx can lie past float16's largest number: infinite, of that sign, from 65520 on."""
    mean, rstd = check_fwd(roi, c)
    check_bwd(roi, c, mean, rstd, "x")
    q, dx = roi.new_checkpoint(c.rows, 1), c.new()
    roi.roi_checkpoint_save(c.x, *q)
    x = LO.checkpoint_load(q[0].cpu().numpy(), q[1].cpu().numpy(), 1)
    roi.roi_norm_bwd(c.dy, q, "layer", c.gamma, mean, rstd, dx)
    dy, g, mo, ro = c.f64(c.dy), c.f64(c.gamma), c.f64(mean), c.f64(rstd)
    want, got = LO.norm_bwd(dy, x, "layer", g, mo, ro)[0], c.f64(dx)
    a, xh = np.abs(dy * (1 if g is None else g)), np.abs((x - mo[:, None]) * ro[:, None])
    bound = ro[:, None] * 72 * U * (2 * a + xh * a * xh)
    past = np.abs(want) >= 65520 + bound
    assert np.all(np.isinf(got[past]) & (np.sign(got[past]) == np.sign(want[past])))
    bound = bound + UT["float16"] * (np.abs(want) + bound) + tiny("float16")
    inside = np.abs(want) < 65520 - bound
    assert np.all(np.abs(got - want)[inside] <= bound[inside])


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_short_rows(roi, dtype, kind):  # noqa: F811
    for rows in range(2, 10):
        for cols in range(1, 8):
            c = Case(rows, cols, dtype, kind, seed=10 * rows + cols, gap=(rows + cols) % 3, offset=rows % 5)
            (check_past_half if (dtype, kind, cols) == ("float16", "layer", 1) else check)(roi, c)
    check(roi, Case(1000, 3, dtype, kind, seed=1, offset=1))


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("cols", [32, 64, 100, 128, 130, 300])
def test_scales_at_any_place(roi, cols, kind):  # noqa: F811
    """The backward from slices of a checkpoint's rows gives the bits of the backward from their copies."""
    import torch
    c = Case(12, cols, "bfloat16", kind, seed=cols)
    y, mean, rstd = c.new(), torch.empty(12, device="cuda") if kind == "layer" else None, torch.empty(12, device="cuda")
    q = roi.new_checkpoint(12, cols)
    roi.roi_norm_fwd(c.x, kind, c.gamma, c.beta, 1e-6, y, mean, rstd, q)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for a in range(8):
        for b in range(a + 1, 13):
            dy = c.dy[a:b].clone()
            out = []
            for pair in ((q[0][a:b], q[1][a:b]), (q[0][a:b].clone(), q[1][a:b].clone())):
                dx, dg = torch.empty_like(dy), torch.empty(cols, device="cuda")
                roi.roi_norm_bwd(dy, pair, kind, c.gamma, None if mean is None else mean[a:b].clone(), rstd[a:b].clone(), dx, dg, None, ws)
                out.append((dx, dg))
            assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    roi.roi_device_status()
