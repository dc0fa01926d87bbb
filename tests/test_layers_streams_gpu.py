"""Checkpoints and norms: stream order and capture, and their bounded waits running out.  (The weight
gradient's are in test_wgrad_gpu.py.)"""
import pytest

from test_checkpoint_gpu import on_gpu, roi, values  # noqa: F401  (roi: the fixture)

pytestmark = pytest.mark.gpu


class Calls:
    """Every kind of call on one input, writing fresh outputs."""

    def __init__(self, roi, rows, cols, kind, dtype, gap):  # noqa: F811
        import torch
        self.roi, self.rows, self.cols, self.kind = roi, rows, cols, kind
        self.x = on_gpu(values(rows, cols, dtype, 5), dtype, gap)
        self.dy = on_gpu(values(rows, cols, dtype, 6), dtype, gap)
        self.gamma = torch.full((cols,), 1.5, dtype=self.x.dtype, device="cuda")
        self.ws = torch.empty(max(16, roi.roi_norm_bwd_workspace_size(rows, cols)), dtype=torch.uint8, device="cuda")

    def outputs(self):
        import torch
        new = lambda: torch.zeros(self.rows, self.cols, dtype=self.x.dtype, device="cuda")  # noqa: E731
        vec = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
        q = [t.zero_() for _ in range(2) for t in self.roi.new_checkpoint(self.rows, self.cols)]
        return [new(), new(), new(), vec(self.rows), vec(self.rows), vec(self.cols), vec(self.cols)] + q

    def run(self, out, x, stream=None):
        roi, layer = self.roi, self.kind == "layer"  # noqa: F811
        y, back, dx, mean, rstd, dg, db, yq, ys, xq, xs = out
        mean, db = (mean, db) if layer else (None, None)
        roi.roi_norm_fwd(x, self.kind, self.gamma, None, 1e-5, y, mean, rstd, None, (yq, ys), stream=stream)
        roi.roi_checkpoint_save(x, xq, xs, stream=stream)
        roi.roi_checkpoint_load(yq, ys, back, stream=stream)
        roi.roi_norm_bwd(self.dy, (xq, xs), self.kind, self.gamma, mean, rstd, dx, dg, db, self.ws, stream=stream)
        return out


def same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


CASES = [(300, 896, "rms", "bfloat16", 0), (700, 1001, "layer", "float16", 3), (40, 3584, "layer", "float32", 0), (3, 64, "rms", "bfloat16", 5)]


@pytest.mark.parametrize("rows,cols,kind,dtype,gap", CASES)
def test_calls_wait_for_other_streams(roi, rows, cols, kind, dtype, gap):  # noqa: F811
    import torch
    c = Calls(roi, rows, cols, kind, dtype, gap)
    want = c.run(c.outputs(), c.x)
    torch.cuda.synchronize()
    side, main = torch.cuda.Stream(), torch.cuda.Stream()
    for rep in range(6):
        x, out, other = torch.full_like(c.x, float(rep)), c.outputs(), c.outputs()
        torch.cuda.synchronize()
        with torch.cuda.stream(main):
            c.run(other, c.x, main)   # launches that let their successors in before they end
            with torch.cuda.stream(side):
                torch.cuda._sleep(300_000)
                x.copy_(c.x)
            main.wait_stream(side)
            c.run(out, x, main)
            copies = [t.clone() for t in out]
        main.synchronize()
        assert same(want, copies) and same(want, out), rep
    roi.roi_device_status()


@pytest.mark.parametrize("rows,cols,kind,dtype,gap", CASES)
def test_captured_calls_replay(roi, rows, cols, kind, dtype, gap):  # noqa: F811
    import torch
    c = Calls(roi, rows, cols, kind, dtype, gap)
    want = c.run(c.outputs(), c.x)
    x, out = c.x.clone(), c.outputs()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(out, x)
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(want, out)
    roi.roi_device_status()


@pytest.mark.parametrize("rows,cols,kind,dtype,gap", CASES[:3])
def test_norms_time_out_then_recover(roi, rows, cols, kind, dtype, gap):  # noqa: F811
    """With the limit of the ring's waits at 0 every team gives up at its first row, with copies in
    flight; the status says so, and the next calls give what they gave before."""
    import torch
    c = Calls(roi, rows, cols, kind, dtype, gap)
    want = c.run(c.outputs(), c.x)
    for call in (lambda o: roi.roi_norm_fwd(c.x, kind, c.gamma, None, 1e-5, o[0], None, o[4]),
                 lambda o: roi.roi_norm_bwd(c.dy, c.x, kind, c.gamma, want[3] if kind == "layer" else None, want[4], o[2], o[5],
                                            None, c.ws)):
        roi.roi_device_status()
        roi.roi_set_ring_wait_limit_ns(0)
        try:
            call(c.outputs())
            with pytest.raises(roi.RoiError) as err:
                roi.roi_device_status()
            assert err.value.status == 8
        finally:
            roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
        roi.roi_device_status()
    again = c.run(c.outputs(), c.x)
    roi.roi_device_status()
    assert same(want, again)
    torch.cuda.synchronize()
