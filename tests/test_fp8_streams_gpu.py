"""The products in 8-bit floating point and the AdamW steps: stream order, capture, overlapping streams, and a step of
mask learning made of them."""
import numpy as np
import pytest

from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


class Calls:
    """A layer's calls of a step on one input, writing fresh outputs: copies, both products, AdamW in 32 and 8 bits."""

    def __init__(self, roi, T, rows, cols, dtype, gap):  # noqa: F811
        import torch
        self.roi, self.T, self.rows, self.cols, self.gap = roi, T, rows, cols, gap
        self.dtype = getattr(torch, dtype)
        g = torch.Generator("cuda").manual_seed(T)
        rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
        self.x = self.wide(T, cols).copy_(rand(T, cols))
        self.dy = self.wide(T, rows).copy_(rand(T, rows))
        self.W = (0.02 * rand(rows, cols)).bfloat16()
        self.param, self.grad, self.m, self.v = rand(rows, cols), 1e-3 * rand(rows, cols), 1e-3 * rand(rows, cols), 1e-6 * rand(rows, cols).square()
        self.opt = roi.AdamW(1e-3, 0.9, 0.95, 1e-8, 0.05, 3)

    def wide(self, rows, cols):
        import torch
        return torch.zeros(rows, cols + self.gap, dtype=self.dtype, device="cuda")[:, :cols]

    def outputs(self):
        import torch
        r = self.roi
        new = [t.zero_() for t in (*r.new_fp8(self.T, self.cols), *r.new_fp8(self.T, self.rows), *r.new_fp8_weight(self.rows, self.cols))]
        state = [*r.new_adamw_state8(self.rows * self.cols)]
        return new + [self.wide(self.T, self.rows), self.wide(self.T, self.cols)] + [torch.zeros_like(self.param) for _ in range(4)] + state

    def run(self, out, x, stream=None):
        r = self.roi
        xq, xs, dq, ds, wq, ws, y, dx, p, m, v, p8, *state = out
        r.roi_fp8_save_weight(self.W, wq, ws, stream=stream)
        r.roi_fp8_save(x, "e4m3", xq, xs, stream=stream)
        r.roi_fp8_linear_fwd((xq, xs), "e4m3", (wq, ws), y, stream=stream)
        r.roi_fp8_save(self.dy, "e5m2", dq, ds, stream=stream)
        r.roi_fp8_linear_dgrad((dq, ds), "e5m2", (wq, ws), dx, stream=stream)
        for t, s in ((p, self.param), (m, self.m), (v, self.v), (p8, self.param)):
            t.copy_(s)
        for t in state:
            t.zero_()
        r.roi_adamw_step([(p, self.grad, m, v, None)], self.opt, stream=stream)
        r.roi_adamw_step8([(p8, self.grad, tuple(state), None, 4)], self.opt, 9, stream=stream)
        return out


def same(a, b):
    import torch
    return all(torch.equal(x, y) for x, y in zip(a, b))


CASES = [(300, 896, 640, "bfloat16", 0), (777, 1001, 1531, "float32", 3), (1, 3584, 4864, "float16", 0), (2048, 3584, 1536, "bfloat16", 8)]


@pytest.mark.parametrize("T,rows,cols,dtype,gap", CASES)
def test_calls_wait_for_other_streams(roi, T, rows, cols, dtype, gap):  # noqa: F811
    import torch
    c = Calls(roi, T, rows, cols, dtype, gap)
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


@pytest.mark.parametrize("T,rows,cols,dtype,gap", CASES)
def test_captured_calls_replay(roi, T, rows, cols, dtype, gap):  # noqa: F811
    """Two graphs of the same calls, replayed in turn and side by side."""
    import torch
    c = Calls(roi, T, rows, cols, dtype, gap)
    want = c.run(c.outputs(), c.x)
    outs, graphs = [c.outputs(), c.outputs()], []
    torch.cuda.synchronize()
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run(out, c.x)
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for out in outs:
            for t in out:
                t.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert same(want, outs[0]) and same(want, outs[1])
    roi.roi_device_status()


def test_threads_on_their_own_streams(roi):  # noqa: F811
    import threading

    import torch
    cases = [Calls(roi, *CASES[i]) for i in (0, 1, 2)]
    want = [c.run(c.outputs(), c.x) for c in cases]
    torch.cuda.synchronize()
    got = [None] * 3

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got[i] = cases[i].run(cases[i].outputs(), cases[i].x)
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    roi.roi_device_status()
    assert all(same(a, b) for a, b in zip(want, got))


def test_far_rows(roi):  # noqa: F811
    """Matrices past 2^31 elements: the rows at both ends are those of a call on them alone."""
    import torch
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    T, rows, cols = 270000, 8200, 130
    g = torch.Generator("cuda").manual_seed(1)
    x = torch.randn(T, cols, device="cuda", generator=g).bfloat16()
    W = torch.randn(rows, cols, device="cuda", generator=g).bfloat16()
    x8, w8, y = roi.new_fp8(T, cols), roi.new_fp8_weight(rows, cols), torch.empty(T, rows, dtype=torch.bfloat16, device="cuda")
    roi.roi_fp8_save(x, "e4m3", *x8)
    roi.roi_fp8_save_weight(W, *w8)
    roi.roi_fp8_linear_fwd(x8, "e4m3", w8, y)
    y8 = roi.new_fp8(T, rows)
    roi.roi_fp8_save(y, "e5m2", *y8)
    dx = torch.empty(T, cols, dtype=torch.float32, device="cuda")
    roi.roi_fp8_linear_dgrad(y8, "e5m2", w8, dx)
    for at in (slice(0, 300), slice(T - 300, T)):
        part, q, dpart = torch.empty(300, rows, dtype=torch.bfloat16, device="cuda"), roi.new_fp8(300, rows), torch.empty(300, cols, device="cuda")
        roi.roi_fp8_linear_fwd((x8[0][at], x8[1][at]), "e4m3", w8, part)
        # (the order of the sums is another, so the last bit may be)
        assert float((part.double() - y[at].double()).norm()) <= 2e-4 * float(part.double().norm())
        roi.roi_fp8_save(y[at], "e5m2", *q)
        assert torch.equal(q[0], y8[0][at]) and torch.equal(q[1], y8[1][at])
        roi.roi_fp8_linear_dgrad(q, "e5m2", w8, dpart)
        assert float((dpart - dx[at]).double().norm()) <= 2e-6 * float(dpart.double().norm())
    # a row of the output far from the next
    wide = torch.full((300, 1 << 23), 7.0, dtype=torch.bfloat16, device="cuda")[:, :rows]
    roi.roi_fp8_linear_fwd((x8[0][:300], x8[1][:300]), "e4m3", w8, wide)
    roi.roi_device_status()
    assert float((wide.double() - y[:300].double()).norm()) <= 2e-4 * float(wide.double().norm())


def test_a_step_of_mask_learning(roi):  # noqa: F811
    """Mask, copies, both products, weight gradient, logit gradient and the optimizer's step, as a data-parallel run makes them,
    against the same formulas in float64 on the masked weights and the copies' values, and the optimizer's oracle."""
    import torch

    import workloads as WL
    from oracle import fp8_oracle as F8
    from oracle import optim_oracle as OO
    rows, cols, T, N, M, tau = 384, 640, 300, 2, 4, 0.7
    W, phi, _ = WL.make_inputs(rows, cols, "normal", 11, device="cuda")
    g = torch.Generator("cuda").manual_seed(3)
    x = torch.randn(T, cols, device="cuda", generator=g).bfloat16()
    dy = (1e-2 * torch.randn(T, rows, device="cuda", generator=g)).bfloat16()
    st = roi.NoiseState(5, 1, 2, 1.0, 0)
    Wm, dWm, dphi = torch.empty_like(W), torch.empty_like(W), torch.empty_like(phi)
    x8, d8, w8, ck = roi.new_fp8(T, cols), roi.new_fp8(T, rows), roi.new_fp8_weight(rows, cols), roi.new_checkpoint(T, cols)
    y, dx = torch.empty(T, rows, dtype=torch.bfloat16, device="cuda"), torch.empty(T, cols, dtype=torch.bfloat16, device="cuda")
    roi.roi_mask_fwd_ex(phi, W, N, M, tau, st, Wm)
    roi.roi_fp8_save_weight(Wm, *w8)
    roi.roi_fp8_save(x, "e4m3", *x8)
    roi.roi_checkpoint_save(x, *ck)
    roi.roi_fp8_linear_fwd(x8, "e4m3", w8, y)
    roi.roi_fp8_save(dy, "e4m3", *d8)
    roi.roi_fp8_linear_dgrad(d8, "e4m3", w8, dx)
    roi.roi_masked_linear_wgrad(dy, ck, dWm)
    roi.roi_mask_bwd(phi, W, st, N, M, dWm, tau, dphi)
    # two ranks with the same gradient: a sum, which the step halves
    half = torch.full((1,), 0.5, device="cuda")
    p32, p8, m, v, state = phi.clone(), phi.clone(), torch.zeros_like(phi), torch.zeros_like(phi), roi.new_adamw_state8(phi.numel())
    for t in (1, 2):
        opt = roi.AdamW(1e-2, 0.9, 0.95, 1e-8, 0.0, t)
        roi.roi_adamw_step([(p32, dphi + dphi, m, v, None)], opt, half)
        roi.roi_adamw_step8([(p8, dphi + dphi, state, None, 2)], opt, 5, half)
    m8, u8 = torch.empty_like(phi), torch.empty_like(phi)
    roi.roi_adamw_state8_load([(state, m8, u8)])
    roi.roi_device_status()
    xv, dv = (torch.from_numpy(F8.save(t.double().cpu().numpy())[2]).cuda() for t in (x, dy))
    wv = torch.from_numpy(F8.save(Wm.double().cpu().numpy(), "e4m3", 128)[2]).cuda()
    for got, want in ((y, xv @ wv.T), (dx, dv @ wv)):
        # one rounding to bfloat16
        assert float((got.double() - want).norm()) <= 2.0 ** -8 * float(want.norm())
    # copies are off by at most 2^-4 of a value (e4m3's half step), both factors' errors independent over hundreds of terms
    for got, want in ((y, x.double() @ Wm.double().T), (dx, dy.double() @ Wm.double())):
        assert float((got.double() - want).norm()) <= 2 * 2.0 ** -4 * float(want.norm())
    # the optimizer's part bit for bit, from the gradient that the library gave
    k = [OO.constants(1e-2, 0.9, 0.95, 1e-8, 0.0, t) for t in (1, 2)]
    grad = (dphi + dphi).cpu().numpy().reshape(-1)
    zero = np.zeros_like(grad)
    want = phi.cpu().numpy().reshape(-1)
    q8, s8 = want, tuple(t.numpy() for t in roi.new_adamw_state8(grad.size, "cpu"))
    mv = (zero, zero)
    for t in (1, 2):
        want, *mv, _ = OO.step(want, grad, *mv, k[t - 1], 0.5)
        q8, s8 = OO.step8(q8, grad, s8, k[t - 1], 5, t, 2, 0.5)
    for got, ref in ((p32, want), (m, mv[0]), (v, mv[1]), (p8, q8), (m8, OO.decode(s8[0], s8[2][:, 0], "m")), (u8, OO.decode(s8[1], s8[2][:, 1], "u"))):
        assert np.array_equal(got.cpu().numpy().reshape(-1), ref)
