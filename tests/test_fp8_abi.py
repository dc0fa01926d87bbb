"""Argument checks of the products in 8-bit floating point, on the C ABI and in the binding: they return before any
CUDA call, so this runs without a GPU."""
import ctypes

import pytest

A, B, C, D, E = 0x10000000, 0x20000000, 0x30000000, 0x40000000, 0x50000000
OK, NULL, SHAPE, ALIGN, ALIAS, TYPE = 0, 1, 2, 5, 6, 10
BF16, FP16, FP32 = 0, 1, 2
E4M3, E5M2 = 0, 1
BIG = (1 << 30) + 1


@pytest.fixture(scope="module")
def roi():
    from paper_2608_23048_gb300 import _build
    _build.build()
    import paper_2608_23048_gb300 as roi
    return roi


@pytest.fixture(scope="module")
def L(roi):
    return roi.lib()


def P(a):
    return ctypes.c_void_p(a) if a else None


def test_sizes(L):
    assert [L.roi_fp8_pitch(c) for c in (-1, 0, 1, 128, 129, 3584)] == [0, 0, 128, 128, 256, 3584]
    assert [L.roi_fp8_scale_pitch(c) for c in (-1, 0, 1, 2048, 2049, 18944)] == [0, 0, 16, 16, 32, 160]


def test_save(L):
    def f(x=A, dt=BF16, rows=4, cols=64, ld=64, fmt=E4M3, q=B, s=C):
        return L.roi_fp8_save(P(x), dt, rows, cols, ld, fmt, P(q), P(s), None)
    assert f(x=0) == NULL and f(q=0) == NULL and f(s=0) == NULL
    assert f(dt=3) == TYPE and f(dt=-1) == TYPE and f(fmt=2) == TYPE and f(fmt=-1) == TYPE
    assert f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(ld=63) == SHAPE and f(rows=BIG) == SHAPE and f(cols=BIG, ld=BIG) == SHAPE
    assert f(x=A + 1) == ALIGN and f(x=A + 2, dt=FP32) == ALIGN and f(q=B + 8) == ALIGN and f(s=C + 4) == ALIGN
    assert f(q=A + 64) == ALIAS and f(s=A) == ALIAS and f(s=B + 256) == ALIAS
    assert f(rows=0, x=0, q=0, s=0) == OK


def test_save_weight(L):
    def f(x=A, rows=200, cols=64, q=B, s=C):
        return L.roi_fp8_save_weight(P(x), rows, cols, P(q), P(s), None)
    assert f(x=0) == NULL and f(q=0) == NULL and f(s=0) == NULL
    assert f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(rows=BIG) == SHAPE
    assert f(x=A + 8) == ALIGN and f(q=B + 8) == ALIGN and f(s=C + 8) == ALIGN
    assert f(q=A + 128) == ALIAS and f(s=A + 16) == ALIAS and f(s=B) == ALIAS
    assert f(rows=0, x=0, q=0, s=0) == OK


def test_products(L):
    for name in ("roi_fp8_linear_fwd", "roi_fp8_linear_dgrad"):
        def f(x=A, xs=B, fmt=E4M3, w=C, ws=D, T=4, rows=128, cols=128, out=E, dt=BF16, ld=128):
            return getattr(L, name)(P(x), P(xs), fmt, P(w), P(ws), T, rows, cols, P(out), dt, ld, None)
        assert f(fmt=2) == TYPE and f(dt=3) == TYPE and f(dt=-1) == TYPE
        assert f(T=-1) == SHAPE and f(rows=-1) == SHAPE and f(cols=0) == SHAPE and f(ld=127) == SHAPE
        assert f(T=BIG) == SHAPE and f(rows=BIG, ld=BIG) == SHAPE and f(cols=BIG, ld=BIG) == SHAPE
        assert all(f(**{k: 0}) == NULL for k in ("x", "xs", "w", "ws", "out"))
        assert all(f(**{k: A0 + 8}) == ALIGN for k, A0 in (("x", A), ("xs", B), ("w", C), ("ws", D)))
        assert f(out=E + 1) == ALIGN and f(out=E + 2, dt=FP32) == ALIGN
        assert f(out=A) == ALIAS and f(out=B) == ALIAS and f(out=C + 64) == ALIAS and f(out=D) == ALIAS
        assert f(T=0, x=0, xs=0, w=0, ws=0, out=0) == OK
    assert L.roi_fp8_linear_fwd(None, None, E4M3, None, None, 4, 0, 128, None, BF16, 0, None) == OK


def test_binding(roi):
    import torch
    cpu = torch.zeros(4, 128)
    with pytest.raises(ValueError, match="CUDA"):
        roi.roi_fp8_save(cpu, "e4m3", *roi.new_fp8(4, 128, "cpu"))
    with pytest.raises(ValueError, match="format"):
        roi._format("e3m4")
    w8 = roi.new_fp8_weight(130, 200, "cpu")
    assert w8[0].shape == (130, 256) and w8[1].shape == (2, 16)
    with pytest.raises(ValueError, match="expected shape|CUDA"):
        roi.roi_fp8_linear_fwd(roi.new_fp8(4, 128, "cpu"), "e4m3", w8, torch.zeros(4, 130))
