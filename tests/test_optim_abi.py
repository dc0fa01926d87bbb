"""Argument checks of the AdamW steps over many tensors, on the C ABI and in the binding: they return before any CUDA
call, so this runs without a GPU."""
import ctypes

import pytest

A, B, C, D, E, S = 0x10000000, 0x20000000, 0x30000000, 0x40000000, 0x50000000, 0x60000000
OK, NULL, SHAPE, ALIGN, ALIAS, OPT, TYPE = 0, 1, 2, 5, 6, 9, 10
GOOD = (1e-3, 0.9, 0.95, 1e-8, 0.05, 1)


@pytest.fixture(scope="module")
def roi():
    from paper_2608_23048_gb300 import _build
    _build.build()
    import paper_2608_23048_gb300 as roi
    return roi


def settings(f):
    """What every step refuses of its settings."""
    for i, bad in ((0, -1.0), (0, float("nan")), (1, 1.0), (2, -0.1), (3, 0.0), (4, float("inf")), (5, 0)):
        assert f(opt=GOOD[:i] + (bad,) + GOOD[i + 1:]) == OPT
    assert f(opt=None) == NULL and f(count=-1) == SHAPE and f(items=False) == NULL
    assert f(scale=S + 2) == ALIGN
    assert f(count=0) == OK and f(count=0, items=False) == OK


def test_step(roi):
    L = roi.lib()

    def f(p=A, g=B, m=C, v=D, copy=E, n=100, gt=2, ct=0, opt=GOOD, count=1, items=True, scale=S):
        arr = (roi.AdamWStepItem * 1)(roi.AdamWStepItem(p, g, m, v, copy, n, gt, ct))
        return L.roi_adamw_step(arr if items else None, count, None if opt is None else ctypes.byref(roi.AdamW(*opt)), scale, None)
    settings(f)
    assert all(f(**{k: 0}) == NULL for k in "pgmv")
    assert all(f(**{k: x + 8}) == ALIGN for k, x in (("p", A), ("g", B), ("m", C), ("v", D), ("copy", E)))
    assert f(gt=3) == TYPE and f(ct=2) == TYPE and f(ct=-1) == TYPE and f(n=-1) == SHAPE and f(n=1 << 62) == SHAPE
    assert f(g=A) == ALIAS and f(m=A + 384) == ALIAS and f(v=C) == ALIAS and f(copy=B) == ALIAS and f(scale=A + 4) == ALIAS
    assert f(p=0, g=0, m=0, v=0, copy=0, n=0) == OK
    two = (roi.AdamWStepItem * 2)(roi.AdamWStepItem(A, B, C, D, 0, 100, 2, 0), roi.AdamWStepItem(A + 4096, B, C + 4096, D + 384, 0, 100, 2, 0))
    assert L.roi_adamw_step(two, 2, ctypes.byref(roi.AdamW(*GOOD)), None, None) == ALIAS     # v of the two


def test_step8(roi):
    L = roi.lib()

    def f(p=A, g=B, m=C, u=D, s=E, copy=0x70000000, n=130, gt=2, ct=0, opt=GOOD, count=1, items=True, scale=S):
        arr = (roi.AdamWStep8Item * 1)(roi.AdamWStep8Item(p, g, m, u, s, copy, n, gt, ct, 0))
        return L.roi_adamw_step8(arr if items else None, count, None if opt is None else ctypes.byref(roi.AdamW(*opt)), 1, scale, None)
    settings(f)
    assert all(f(**{k: 0}) == NULL for k in "pgmus")
    assert all(f(**{k: x + 8}) == ALIGN for k, x in (("p", A), ("g", B), ("m", C), ("u", D), ("copy", 0x70000000)))
    assert f(s=E + 1) == ALIGN
    assert f(gt=-1) == TYPE and f(ct=2) == TYPE and f(n=-1) == SHAPE
    # a state's padding counts
    assert f(u=C + 240) == ALIAS and f(g=A) == ALIAS and f(s=C + 254) == ALIAS and f(copy=A + 512) == ALIAS
    assert f(p=0, g=0, m=0, u=0, s=0, n=0) == OK


def test_load(roi):
    L = roi.lib()

    def f(m=A, u=B, s=C, om=D, ou=E, n=130, dt=0, count=1, items=True):
        arr = (roi.AdamWState8Item * 1)(roi.AdamWState8Item(m, u, s, om, ou, n, dt))
        return L.roi_adamw_state8_load(arr if items else None, count, None)
    assert f(count=-1) == SHAPE and f(items=False) == NULL and f(dt=3) == TYPE and f(n=-1) == SHAPE
    assert f(m=0) == NULL and f(u=0) == NULL and f(s=0) == NULL and f(om=0, ou=0) == NULL
    assert f(m=A + 4) == ALIGN and f(s=C + 1) == ALIGN and f(om=D + 2) == ALIGN
    assert f(om=A) == ALIAS and f(ou=D + 256) == ALIAS and f(ou=C) == ALIAS
    assert f(n=0, m=0, u=0, s=0, om=0, ou=0) == OK


def test_binding(roi):
    import torch
    t = torch.zeros(8)
    for make, item in ((roi.make_adamw_step_items, (t, t, t, t, None)),
                       (roi.make_adamw_step8_items, (t, t, roi.new_adamw_state8(8, "cpu"), None, 0)),
                       (roi.make_adamw_state8_items, (roi.new_adamw_state8(8, "cpu"), t, t))):
        with pytest.raises(ValueError, match="CUDA"):
            make([item])
    assert [tuple(x.shape) for x in roi.new_adamw_state8(129, "cpu")] == [(256,), (256,), (2, 2)]
    with pytest.raises(TypeError, match="copy"):
        roi._half(t, "copy", t.shape)
