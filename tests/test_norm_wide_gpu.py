"""Norms of rows too wide for a ring, with more rows than their kernels take at once (two CTAs an SM) and than
there are partial rows of sums (64); and what a row that is not finite does to the gradients of weight and
bias.  Bounds: those of test_norm_gpu.py."""
import pytest

from test_checkpoint_gpu import roi, values  # noqa: F401  (roi: the fixture)
from test_norm_gpu import EPS, Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols,dtype", [(70, 24000, "bfloat16"), (70, 16400, "float16"), (65, 16400, "float32"), (310, 24001, "bfloat16")])
def test_many_wide_rows(roi, rows, cols, dtype, kind):  # noqa: F811
    check(roi, Case(rows, cols, dtype, kind, seed=rows))


@pytest.mark.parametrize("cols", [160, 24000])
@pytest.mark.parametrize("source", ["x", "checkpoint"])
def test_gradients_of_rows_that_are_not_finite(roi, cols, source):  # noqa: F811
    """A NaN, or an infinity in a layer norm, makes rstd NaN, and so the whole row's normalised values, its dx and all
    of dgamma; dbeta is the sum of dy still.  An infinity in an RMS norm makes rstd 0: the row adds nothing to dgamma
    but NaN at the infinity, or in its block where x is a checkpoint."""
    import torch
    rows = 20
    ws = torch.empty(8 << 20, dtype=torch.uint8, device="cuda")

    def backward(c, x, kind, dy, mean, rstd):
        q = roi.new_checkpoint(rows, cols)
        roi.roi_checkpoint_save(x, *q)
        dx, dg, db = c.new(), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda") if kind == "layer" else None
        roi.roi_norm_bwd(dy, x if source == "x" else q, kind, c.gamma, mean, rstd, dx, dg, db, ws)
        return dx, dg, db

    def forward(c, x, kind):
        mean, rstd = torch.empty(rows, device="cuda") if kind == "layer" else None, torch.empty(rows, device="cuda")
        roi.roi_norm_fwd(x, kind, c.gamma, c.beta, EPS, c.new(), mean, rstd)
        return mean, rstd

    for kind, bad in (("layer", float("nan")), ("layer", float("inf")), ("rms", float("nan")), ("rms", float("inf"))):
        c = Case(rows, cols, "bfloat16", kind, 6, x=values(rows, cols, "bfloat16", 5))
        clean = backward(c, c.x, kind, c.dy, *forward(c, c.x, kind))
        x = c.x.clone()
        x[11, 100] = bad
        mean, rstd = forward(c, x, kind)
        dx, dg, db = backward(c, x, kind, c.dy, mean, rstd)
        others = torch.arange(rows) != 11
        assert torch.isnan(dx[11]).all() and torch.equal(dx[others], clean[0][others])
        if kind == "layer":
            assert torch.equal(db, clean[2])
        if kind == "rms" and bad == float("inf"):
            assert float(rstd[11]) == 0
            at = torch.zeros(cols, dtype=torch.bool)
            at[100 if source == "x" else slice(96, 128)] = True
            dy = c.dy.clone()
            dy[11] = 0
            without = backward(c, c.x, kind, dy, *forward(c, c.x, kind))[1]
            assert torch.isnan(dg[at]).all() and torch.equal(dg[~at], without[~at])
        else:
            assert torch.isnan(dg).all()
    roi.roi_device_status()
