"""Argument checks of the calls around the masked linear layers, on the C ABI: they return before
any CUDA call, so this runs without a GPU."""
import ctypes

import pytest

A, B, C, D, E, F = 0x10000000, 0x20000000, 0x30000000, 0x40000000, 0x50000000, 0x60000000
OK, NULL, SHAPE, ALIGN, ALIAS, TYPE = 0, 1, 2, 5, 6, 10
BF16, FP16, FP32 = 0, 1, 2
LAYER, RMS = 0, 1


@pytest.fixture(scope="module")
def L():
    from paper_2608_23048_gb300 import _build
    _build.build()
    import paper_2608_23048_gb300 as roi
    return roi.lib()


def P(a):
    return ctypes.c_void_p(a) if a else None


def test_sizes(L):
    assert [L.roi_checkpoint_pitch(c) for c in (-1, 0, 1, 32, 33, 3584)] == [0, 0, 32, 32, 64, 3584]
    assert [L.roi_checkpoint_scale_pitch(c) for c in (-1, 0, 1, 128, 129, 3584)] == [0, 0, 4, 4, 8, 112]
    assert L.roi_norm_bwd_workspace_size(0, 64) == 0 and L.roi_norm_bwd_workspace_size(4, 0) == 0
    assert L.roi_masked_linear_wgrad_workspace_size(0, 8, 8, 8) == 0
    assert L.roi_masked_linear_wgrad_workspace_size(4, 8, 8, 7) == 0
    assert L.roi_masked_linear_wgrad_workspace_size(4, 9, 8, 9) == 4 * 16 * 2   # dY laid out again
    assert b"type" in L.roi_status_string(TYPE)


def test_checkpoint(L):
    def save(x=A, dt=BF16, rows=4, cols=64, ld=64, q=B, s=C):
        return L.roi_checkpoint_save(P(x), dt, rows, cols, ld, P(q), P(s), None)

    def load(q=B, s=C, dt=BF16, rows=4, cols=64, x=A, ld=64):
        return L.roi_checkpoint_load(P(q), P(s), dt, rows, cols, P(x), ld, None)
    for f in (save, load):
        assert f(x=0) == NULL and f(q=0) == NULL and f(s=0) == NULL
        assert f(dt=3) == TYPE and f(dt=-1) == TYPE
        assert f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(ld=63) == SHAPE and f(rows=1 << 62) == SHAPE
        assert f(x=A + 1) == ALIGN and f(x=A + 2, dt=FP32) == ALIGN and f(q=B + 8) == ALIGN and f(s=C + 2) == ALIGN
        assert f(q=A + 64) == ALIAS and f(s=A) == ALIAS
        assert f(rows=0, x=0, q=0, s=0) == OK
    assert save(s=B + 128) == ALIAS


def test_norm_fwd(L):
    def f(x=A, dt=BF16, rows=4, cols=64, ldx=64, kind=LAYER, g=B, b=C, pt=BF16, eps=1e-6, y=D, ldy=64, mean=E, rstd=F, xq=0,
          xs=0, yq=0, ys=0):
        return L.roi_norm_fwd(P(x), dt, rows, cols, ldx, kind, P(g), P(b), pt, eps, P(y), ldy, P(mean), P(rstd), P(xq), P(xs),
                              P(yq), P(ys), None)
    assert f(dt=5) == TYPE and f(pt=FP16) == TYPE and f(kind=2) == TYPE
    assert f(eps=-1.0) == TYPE and f(eps=float("nan")) == TYPE and f(eps=float("inf")) == TYPE
    assert f(kind=RMS) == TYPE and f(kind=RMS, b=0) == TYPE          # a bias, a mean
    assert f(ldx=63) == SHAPE and f(ldy=3) == SHAPE and f(cols=-4) == SHAPE and f(rows=-1) == SHAPE
    assert f(x=0) == NULL and f(y=0) == NULL and f(xq=0x70000000) == NULL and f(ys=0x70000000) == NULL
    assert f(x=A + 1) == ALIGN and f(g=B + 4) == ALIGN and f(rstd=F + 2) == ALIGN and f(xq=0x70000008, xs=0x71000000) == ALIGN
    assert f(y=A) == ALIAS and f(y=A + 64) == ALIAS and f(mean=F) == ALIAS and f(yq=D, ys=0x70000000) == ALIAS
    assert f(rows=0, x=0, y=0) == OK


def test_norm_bwd(L):
    def f(dy=A, dt=BF16, rows=4, cols=64, lddy=64, x=B, ldx=64, q=0, s=0, kind=LAYER, g=C, pt=BF16, mean=D, rstd=D + 0x1000,
          dx=E, lddx=64, dg=F, db=F + 0x1000, ws=0x70000000, n=1 << 20):
        return L.roi_norm_bwd(P(dy), dt, rows, cols, lddy, P(x), ldx, P(q), P(s), kind, P(g), pt, P(mean), P(rstd), P(dx), lddx,
                              P(dg), P(db), P(ws), n, None)
    assert f(dt=9) == TYPE and f(pt=FP16) == TYPE and f(kind=-1) == TYPE
    assert f(kind=RMS) == TYPE and f(kind=RMS, db=0) == TYPE and f(kind=RMS, mean=0) == TYPE
    assert f(lddy=8) == SHAPE and f(ldx=8) == SHAPE and f(lddx=8) == SHAPE and f(cols=0) == SHAPE
    assert f(dy=0) == NULL and f(dx=0) == NULL and f(rstd=0) == NULL and f(mean=0) == NULL
    assert f(x=0) == NULL and f(q=0x71000000, s=0x72000000) == NULL and f(x=0, q=0x71000000) == NULL
    assert f(ws=0) == NULL and f(n=16) == SHAPE
    assert f(dy=A + 1) == ALIGN and f(ws=0x70000008) == ALIGN and f(dg=F + 2) == ALIGN and f(x=0, q=0x71000008, s=0x72000000) == ALIGN
    assert f(dx=A) == ALIAS and f(dx=B + 16) == ALIAS and f(dg=D) == ALIAS and f(db=F) == ALIAS and f(ws=C) == ALIAS


def test_wgrad(L):
    def f(dY=A, ld=64, q=B, s=C, T=4, rows=64, cols=96, out=D, acc=E, ws=0, n=0):
        return L.roi_masked_linear_wgrad(P(dY), ld, P(q), P(s), T, rows, cols, P(out), P(acc), P(ws), n, None)
    assert f(ld=63) == SHAPE and f(T=-1) == SHAPE and f(cols=0) == SHAPE and f(rows=-1) == SHAPE and f(T=1 << 40) == SHAPE
    assert f(out=0, acc=0) == NULL and f(dY=0) == NULL and f(q=0) == NULL and f(s=0) == NULL
    assert f(ld=65) == NULL and f(ld=65, ws=F, n=256) == SHAPE      # rows to be laid out again
    assert f(dY=A + 8) == ALIGN and f(q=B + 4) == ALIGN and f(s=C + 1) == ALIGN and f(out=D + 4) == ALIGN and f(acc=E + 8) == ALIGN
    assert f(ws=F + 8, n=64) == ALIGN
    assert f(out=A) == ALIAS and f(acc=D) == ALIAS and f(out=B + 16) == ALIAS and f(ld=65, ws=A, n=1 << 20) == ALIAS
    assert f(rows=0, dY=0, q=0, s=0, out=0, acc=0) == OK


def test_registers_of_the_weight_gradient():
    """18 warps on four schedulers leave a thread 96 registers; the converting warps hold 64 of them as
    outputs, and a spill in their loop costs more than any tile shape gains."""
    import os
    import re

    from paper_2608_23048_gb300 import _build
    try:
        _build.nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    if not os.path.exists(_build.log_of("roi_wgrad.cu")):
        _build.build(force=True)
    with open(_build.log_of("roi_wgrad.cu")) as f:
        found = re.findall(r"Compiling entry function '\w*roi_wgrad_kernel\w*'[^\n]*\n[^\n]*\n\s*(\d+) bytes stack frame, (\d+) "
                           r"bytes spill stores[^\n]*\n[^\n]*Used (\d+) registers", f.read())
    # (the form that stores whole sectors, and two for other widths)
    assert len(found) == 3 and all(int(f[2]) <= 96 and int(f[1]) <= 16 for f in found) and ("0", "0") in [f[:2] for f in found], found
