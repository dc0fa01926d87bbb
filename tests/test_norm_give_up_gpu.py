"""Norms whose bounded waits run out, with more than one row a team.  Every copy is valid and every wait
bounded: a call that gives up says so in the device status, leaves when its copies have landed, and what
comes after it is right."""
import pytest

from test_checkpoint_gpu import roi, values  # noqa: F401  (roi: the fixture)

pytestmark = pytest.mark.gpu


class Calls:
    def __init__(self, roi, rows, cols, kind, dtype="bfloat16", gap=0):  # noqa: F811
        import torch
        t = getattr(torch, dtype)
        g = torch.Generator("cuda").manual_seed(rows + cols)
        new = lambda: torch.randn(rows, cols + gap, device="cuda", generator=g).to(t)[:, :cols]  # noqa: E731
        self.roi, self.kind, self.x, self.dy = roi, kind, new(), new()
        self.gamma = (1 + 0.1 * torch.randn(cols, device="cuda", generator=g)).to(t)
        self.q = roi.new_checkpoint(rows, cols)
        self.y, self.dx = torch.empty(rows, cols, dtype=t, device="cuda"), torch.empty(rows, cols, dtype=t, device="cuda")
        self.mean = torch.empty(rows, device="cuda") if kind == "layer" else None
        self.rstd, self.dg = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        self.ws = torch.empty(roi.roi_norm_bwd_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
        roi.roi_checkpoint_save(self.x, *self.q)
        self.calls = [self.fwd, lambda: self.bwd(self.x), lambda: self.bwd(self.q)]
        self.fwd()
        # (of the backward: the statistics as they are now)
        self.stats = None if self.mean is None else self.mean.clone(), self.rstd.clone()

    def fwd(self):
        self.roi.roi_norm_fwd(self.x, self.kind, self.gamma, None, 1e-5, self.y, self.mean, self.rstd)
        return self.y, self.rstd

    def bwd(self, x):
        self.roi.roi_norm_bwd(self.dy, x, self.kind, self.gamma, *self.stats, self.dx, self.dg, None, self.ws)
        return self.dx, self.dg


def same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


def others(m):
    """Work of other kernels that lives in shared memory."""
    import torch
    return torch.softmax(m, 1), m @ m.T, m.cumsum(1), m.sort(1).values


# 2 to 5 rows a team, all of which fit its ring
@pytest.mark.parametrize("rows,cols,kind,gap", [(760, 8192, "rms", 0), (760, 8192, "layer", 0), (600, 8001, "rms", 3), (450, 6000, "layer", 0)])
def test_copies_land_before_the_next_kernel(roi, rows, cols, kind, gap):  # noqa: F811
    import torch
    c = Calls(roi, rows, cols, kind, gap=gap)
    m = torch.randn(1024, 1500, device="cuda")
    for call in c.calls:
        want, beside = [t.clone() for t in call()], others(m)
        roi.roi_device_status()
        got = []
        roi.roi_set_ring_wait_limit_ns(0)
        try:
            for _ in range(20):
                call()
                got.append(others(m))
            with pytest.raises(roi.RoiError) as err:
                roi.roi_device_status()
            assert err.value.status == 8
        finally:
            roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
        assert all(same(beside, g) for g in got)
        assert same(want, call())
        roi.roi_device_status()


# teams with many more rows than their rings are deep; every warp gives up at its first row
@pytest.mark.parametrize("rows,cols,kind,gap,dtype", [(8000, 8192, "rms", 0, "bfloat16"), (8000, 8192, "layer", 0, "bfloat16"),
                                                      (9000, 4100, "rms", 3, "float16"), (4000, 4096, "layer", 0, "float32"),
                                                      (90000, 256, "layer", 0, "bfloat16"), (60000, 1001, "rms", 0, "float32")])
def test_long_rings(roi, rows, cols, kind, gap, dtype):  # noqa: F811
    c = Calls(roi, rows, cols, kind, dtype, gap)
    for call in c.calls:
        want = [t.clone() for t in call()]
        roi.roi_device_status()
        roi.roi_set_ring_wait_limit_ns(0)
        try:
            for _ in range(5):
                call()
            with pytest.raises(roi.RoiError) as err:
                roi.roi_device_status()
            assert err.value.status == 8
        finally:
            roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
        assert same(want, call())
        roi.roi_device_status()


# teams of one, two and many warps
@pytest.mark.parametrize("rows,cols,kind,gap,dtype", [(8000, 8192, "layer", 0, "bfloat16"), (9000, 4100, "rms", 3, "float16"),
                                                      (3000, 9000, "layer", 0, "bfloat16"), (90000, 256, "rms", 0, "bfloat16"),
                                                      (60000, 1001, "layer", 0, "float32"), (300, 3584, "layer", 0, "bfloat16")])
def test_small_limits(roi, rows, cols, kind, gap, dtype):  # noqa: F811
    """Limits around the time that a copy takes, so that some waits of a team run out and some do not, at any
    row: every call returns, and either says that it gave up or is right.  (Which of the two is the clock's
    affair.)"""
    c = Calls(roi, rows, cols, kind, dtype, gap)
    for call in c.calls:
        want = [t.clone() for t in call()]
        roi.roi_device_status()
        try:
            for ns in (1, 50, 200, 500, 1000, 2000, 3000, 5000, 10000, 30000, 100000):
                roi.roi_set_ring_wait_limit_ns(ns)
                for _ in range(10):
                    got = call()
                    try:
                        roi.roi_device_status()
                    except roi.RoiError as err:
                        assert err.status == 8
                    else:
                        assert same(want, got), ns
        finally:
            roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
        assert same(want, call())
        roi.roi_device_status()
