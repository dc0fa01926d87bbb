"""The masked linear's weight gradient from 8-bit checkpoints (roi_masked_linear_wgrad) against the
CPU oracle.

Most cases have integer inputs whose sums stay below 2^24, times a power of two a block: products
and sums are exact in float32 in any order, so the results are compared bit for bit (after the one
rounding to bfloat16), with every token and every scale counted.  The others: a product of two
bfloat16 values is exact in float32; a tensor-core step aligns its terms and the running sum to
the largest and may drop what lies below 2^-23 of it, so T terms are at most T 2^-23 sum |dY x|
from their sum; adding acc and rounding to bfloat16 are one rounding each."""
import numpy as np
import pytest

from oracle import layer_oracle as LO
from test_checkpoint_gpu import on_gpu, roi, same, values  # noqa: F401  (roi: the fixture)

pytestmark = pytest.mark.gpu


def integers(T, rows, cols, seed, gap=0, top=127):
    """(dY on the GPU, its values, the checkpoint of x, x): every sum exact in float32."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dY = torch.randint(-8, 9, (T, rows), generator=g).float()
    x = torch.randint(-top, top + 1, (T, cols), generator=g).float()
    x *= torch.exp2(torch.randint(-2, 1, (T, -(-cols // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :cols]
    x[torch.rand(T, generator=g) < 0.1] = 0
    return on_gpu(dY, "bfloat16", gap), dY.double(), x.double()


def checkpoint(roi, x):
    q = roi.new_checkpoint(*x.shape)
    roi.roi_checkpoint_save(x.float().cuda(), *q)
    return q


def workspace(roi, T, rows, cols, ld, fill=255):
    import torch
    return torch.full((max(16, roi.roi_masked_linear_wgrad_workspace_size(T, rows, cols, ld)),), fill, dtype=torch.uint8,
                      device="cuda")


def exact_case(roi, T, rows, cols, seed, gap=0, ws=True, top=127):
    import torch
    dY, dy, x = integers(T, rows, cols, seed, gap, top)
    assert T * 8 * 127 < 2 ** 22
    q = checkpoint(roi, x)
    want = (dy.cuda().T @ x.cuda()).float() if T * rows * cols > 1 << 28 else (dy.T @ x).float().cuda()
    ld = dY.stride(0) if T > 1 else rows
    w = workspace(roi, T, rows, cols, ld) if ws or ld % 8 else None
    if not ws and w is not None:   # room for dY alone
        w = w[:T * ((rows + 7) // 8 * 8) * 2]
    out = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
    roi.roi_masked_linear_wgrad(dY, q, out, None, w)
    assert torch.equal(out, want.to(torch.bfloat16))
    # added to a sum over micro-batches, with and without the rounded copy
    acc = torch.randint(-1000, 1000, (rows, cols), device="cuda").float()
    total, only = acc + want, acc.clone()
    roi.roi_masked_linear_wgrad(dY, q, None, only, w)
    assert torch.equal(only, total)
    roi.roi_masked_linear_wgrad(dY, q, out, acc, w)
    assert torch.equal(acc, total) and torch.equal(out, total.to(torch.bfloat16))


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 200, 1000, 2047])
@pytest.mark.parametrize("rows,cols", [(1, 4), (8, 36), (100, 128), (129, 260), (300, 100), (520, 516)])
def test_exact(roi, T, rows, cols):  # noqa: F811
    for gap, ws in ((0, True), (0, False), (8, True), (3, True), (5, False)):
        exact_case(roi, T, rows, cols, T + rows + cols, gap, ws)
    roi.roi_device_status()


@pytest.mark.parametrize("T,rows,cols", [(4100, 128, 896), (4096, 512, 3584), (3000, 1215, 2504), (64, 4864, 896), (1, 3584, 18944),
                                         (700, 18944, 328), (2500, 40, 8960), (1500, 5000, 5000)])
def test_exact_large(roi, T, rows, cols):  # noqa: F811
    for ws in (True, False):
        exact_case(roi, T, rows, cols, T, 0, ws)
    roi.roi_device_status()


@pytest.mark.parametrize("T,rows,cols", [(300, 200, 300), (6000, 130, 520), (37, 128, 256)])
def test_real_values(roi, T, rows, cols):  # noqa: F811
    import torch
    x = values(T, cols, "bfloat16", T)
    dY = on_gpu(values(T, rows, "bfloat16", T + 1) * 1e-3, "bfloat16")
    dY[::8] = 0
    q = checkpoint(roi, x)
    back = LO.checkpoint_load(q[0].cpu().numpy(), q[1].cpu().numpy(), cols)
    dy = dY.double().cpu().numpy()
    acc0 = 1e-3 * torch.randn(rows, cols, device="cuda")
    acc, out = acc0.clone(), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    ws = workspace(roi, T, rows, cols, rows)
    roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
    roi.roi_masked_linear_wgrad(dY, q, None, acc, ws)
    want, size = LO.linear_wgrad(dy, back), T * 2.0 ** -23 * (np.abs(dy).T @ np.abs(back))
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= size + 2.0 ** -8 * (np.abs(want) + size))
    total = want + acc0.double().cpu().numpy()
    assert np.all(np.abs(acc.double().cpu().numpy() - total) <= size + 2.0 ** -24 * (np.abs(total) + size))
    # the same bits again, from a workspace of other contents
    again, ws2 = torch.empty_like(out), workspace(roi, T, rows, cols, rows, 7)
    roi.roi_masked_linear_wgrad(dY, q, again, None, ws2)
    assert torch.equal(out, again)


def test_against_differences(roi):  # noqa: F811
    """L(Wm) = sum dY * (x Wm^T) is linear in Wm: a central difference is its gradient up to the
    rounding of float64, and the integers here have exact sums."""
    dY, dy, x = integers(70, 9, 12, 3)
    q = checkpoint(roi, x)
    import torch
    acc = torch.zeros(9, 12, device="cuda")
    roi.roi_masked_linear_wgrad(dY, q, None, acc, None if dY.stride(0) % 8 == 0 else workspace(roi, 70, 9, 12, 9))
    loss = lambda W: float((dy.numpy() * (x.numpy() @ W.T)).sum())  # noqa: E731
    for at in np.ndindex(9, 12):
        W = np.zeros((9, 12))
        W[at] = 0.5
        assert loss(W) - loss(-W) == float(acc[at])


def test_non_finite_values_stay_where_they_are(roi):  # noqa: F811
    """A NaN or infinity in x makes its block's columns NaN (a zero gradient times NaN included),
    one in dY its row; nothing else changes."""
    import torch
    T, rows, cols = 150, 140, 300
    dY, dy, x = integers(T, rows, cols, 4)
    clean = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    ws = workspace(roi, T, rows, cols, dY.stride(0))
    roi.roi_masked_linear_wgrad(dY, checkpoint(roi, x), clean, None, ws)
    x[149, 70], x[3, 299], dY[100, 17] = float("nan"), float("inf"), float("inf")
    dY[149] = 0
    out = torch.empty_like(clean)
    roi.roi_masked_linear_wgrad(dY, checkpoint(roi, x), out, None, ws)
    bad = torch.zeros(rows, cols, dtype=torch.bool, device="cuda")
    bad[:, 64:96] = True
    bad[:, 288:] = True
    assert torch.isnan(out[:, 64:96]).all() and torch.isnan(out[:, 288:]).all()
    assert not torch.isfinite(out[17]).any()
    bad[17] = True
    # (token 149's gradient was zeroed: the others' sums without it)
    dy2 = dy.clone()
    dy2[149] = 0
    want = (dy2.T @ torch.nan_to_num(x, nan=0, posinf=0)).float().to(torch.bfloat16).cuda()
    assert torch.equal(out[~bad], want[~bad])


def test_streams_and_capture(roi):  # noqa: F811
    """On another stream, after that stream's copies; recorded and replayed; two calls in a row on
    one workspace."""
    import torch
    T, rows, cols = 2000, 130, 520
    dY, dy, x = integers(T, rows, cols, 6)
    q, ld = checkpoint(roi, x), dY.stride(0)
    want = (dy.T @ x).float().cuda()
    ws = workspace(roi, T, rows, cols, ld)
    late, out, acc = torch.zeros_like(dY), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(want)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(300_000)
        late.copy_(dY)
        for _ in range(3):
            roi.roi_masked_linear_wgrad(late, q, out, acc, ws)
        copy = acc.clone()
    side.synchronize()
    assert torch.equal(copy, 3 * want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
        roi.roi_masked_linear_wgrad(dY, q, None, acc, ws)
    for _ in range(3):
        out.zero_(), acc.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want.to(torch.bfloat16)) and torch.equal(acc, want)
    roi.roi_device_status()


def test_times_out_then_recovers(roi):  # noqa: F811
    """With the limit of its waits at 0 every role gives up at once, with copies in flight; the status
    says so, and the next call is right."""
    import torch
    T, rows, cols = 1000, 600, 700
    dY, dy, x = integers(T, rows, cols, 7)
    q, ws = checkpoint(roi, x), workspace(roi, T, rows, cols, rows)
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    roi.roi_device_status()
    roi.roi_set_ring_wait_limit_ns(0)
    try:
        roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
        with pytest.raises(roi.RoiError) as err:
            roi.roi_device_status()
        assert err.value.status == 8
    finally:
        roi.roi_set_ring_wait_limit_ns(roi.ROI_DEFAULT_RING_WAIT_NS)
    roi.roi_device_status()
    roi.roi_masked_linear_wgrad(dY, q, out, None, ws)
    roi.roi_device_status()
    assert torch.equal(out, (dy.T @ x).float().to(torch.bfloat16).cuda())


def test_empty_and_refusals(roi):  # noqa: F811
    import torch
    dY, dy, x = integers(5, 16, 64, 8)
    q = checkpoint(roi, x)
    out, acc = torch.full((16, 64), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((16, 64), 2.5, device="cuda")
    none = (q[0][:0], q[1][:0])
    roi.roi_masked_linear_wgrad(dY[:0], none, out)
    assert not out.any()
    roi.roi_masked_linear_wgrad(dY[:0], none, out, acc)
    assert bool((out == 2.5).all()) and bool((acc == 2.5).all())

    def fails(code, *a):
        with pytest.raises(roi.RoiError) as e:
            roi.roi_masked_linear_wgrad(*a)
        assert e.value.status == code, e.value
    odd = on_gpu(dy.float(), "bfloat16", 3)
    fails(1, odd, q, out)                                                     # rows to be laid out again: no workspace
    fails(2, odd, q, out, None, torch.empty(64, dtype=torch.uint8, device="cuda"))
    fails(5, on_gpu(dy.float(), "bfloat16", 0, 4), q, out)
    room = torch.empty(16 * 64 * 4, dtype=torch.uint8, device="cuda")
    fails(6, dY, q, room[:2048].view(torch.bfloat16).view(16, 64), room.view(torch.float32).view(16, 64))
    with pytest.raises(ValueError):
        roi.roi_masked_linear_wgrad(dY, q)
    with pytest.raises(ValueError):
        roi.roi_masked_linear_wgrad(dY[:4], q, out)
    with pytest.raises(TypeError):
        roi.roi_masked_linear_wgrad(dY.float(), q, out)
    with pytest.raises(TypeError):
        roi.roi_masked_linear_wgrad(dY, q, out.float())
