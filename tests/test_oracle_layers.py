"""Pins of oracle/layer_oracle.py that do not use its own formulas: the definition of the
checkpoint by search, torch's norms and their autograd in float64, differences, and planted
mistakes."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as LO


def _values(rng, n):
    v = rng.standard_normal(n) * np.exp2(rng.integers(-140, 120, n))
    v[rng.random(n) < 0.05] = 0.0
    return v.astype(np.float32).astype(np.float64)


def test_checkpoint_is_the_best_of_its_kind():
    """By search over every exponent: the least that holds the block, and the nearest code."""
    rng = np.random.default_rng(1)
    for n in (1, 7, 31, 32):
        for _ in range(60):
            x = rng.standard_normal(n) * 2.0 ** rng.integers(-135, 126)
            x = np.clip(x, -3.4028234e38, 3.4028234e38).astype(np.float32).astype(np.float64)
            codes, scales = LO.checkpoint_save(x[None])
            a = np.max(np.abs(x))
            fits = [e for e in range(-126, 122) if a <= 127.5 * 2.0 ** e]
            e = fits[0] if fits else 121
            assert scales[0, 0] == e + 133
            back = LO.checkpoint_load(codes, scales, n)[0]
            for v, q in zip(x, codes[0]):
                every = np.arange(-127, 128) * 2.0 ** e
                assert abs(q * 2.0 ** e - v) == np.min(np.abs(every - v))
            # (past 127.5 * 2^121 the last code stands for what is over)
            assert np.all(np.abs(back - x) <= np.maximum(2.0 ** (e - 1), np.abs(x) - 127 * 2.0 ** e))


def test_checkpoint_layout_and_special_values():
    assert LO.pitches(1) == (32, 4) and LO.pitches(128) == (128, 4) and LO.pitches(129) == (160, 8)
    x = np.zeros((4, 70))
    x[0, 3], x[1, 40], x[2, 69] = np.nan, np.inf, -np.inf
    codes, scales = LO.checkpoint_save(x)
    assert codes.shape == (4, 96) and scales.shape == (4, 4)
    assert scales.tolist() == [[255, 7, 7, 7], [7, 255, 7, 7], [7, 7, 255, 7], [7] * 4] and not codes.any()
    back = LO.checkpoint_load(codes, scales, 70)
    assert np.array_equal(np.isnan(back), np.repeat(scales == 255, 32, 1)[:, :70])
    # ties go to the even code, and half a step past the last code is the last code
    x = np.array([[127.5, 0.5, 1.5, 2.5, -0.5, -1.5, -127.5, 126.5]])
    assert LO.checkpoint_save(x)[0][0, :8].tolist() == [127, 0, 2, 2, 0, -2, -127, 126]
    assert LO.checkpoint_save(x)[1][0, 0] == 133 and LO.checkpoint_save(x * 1.001)[1][0, 0] == 134
    # held exactly by bfloat16
    x = _values(np.random.default_rng(2), 4096).reshape(8, 512)
    back = torch.from_numpy(LO.checkpoint_load(*LO.checkpoint_save(x), 512))
    assert torch.equal(back.to(torch.bfloat16).double(), back)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("affine", [True, False])
def test_norm_against_torch_autograd(kind, affine):
    rng = np.random.default_rng(3)
    x = torch.from_numpy(rng.standard_normal((5, 33)) + 0.3).requires_grad_()
    g = torch.from_numpy(1 + 0.3 * rng.standard_normal(33)).requires_grad_()
    b = torch.from_numpy(0.2 * rng.standard_normal(33)).requires_grad_()
    dy = torch.from_numpy(rng.standard_normal((5, 33)))
    layer = kind == "layer"
    w, c = (g, b if layer else None) if affine else (None, None)
    y = torch.nn.functional.layer_norm(x, (33,), w, c, 1e-5) if layer else torch.nn.functional.rms_norm(x, (33,), w, 1e-5)
    y.backward(dy)
    n = lambda t: None if t is None else t.detach().numpy()  # noqa: E731
    yo, mean, rstd = LO.norm_fwd(n(x), kind, n(w), n(c), 1e-5)
    dx, dg, db = LO.norm_bwd(n(dy), n(x), kind, n(w), mean, rstd)
    np.testing.assert_allclose(yo, n(y), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(dx, n(x.grad), rtol=1e-10, atol=1e-12)
    if affine:
        np.testing.assert_allclose(dg, n(g.grad), rtol=1e-11, atol=1e-12)
        if layer:
            np.testing.assert_allclose(db, n(b.grad), rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_against_differences(kind):
    rng = np.random.default_rng(4)
    x, g, dy = rng.standard_normal((2, 9)), rng.standard_normal(9), rng.standard_normal((2, 9))
    loss = lambda x, g: float((LO.norm_fwd(x, kind, g, None, 1e-3)[0] * dy).sum())  # noqa: E731
    _, mean, rstd = LO.norm_fwd(x, kind, g, None, 1e-3)
    dx, dg, _ = LO.norm_bwd(dy, x, kind, g, mean, rstd)
    h = 1e-5
    for at in np.ndindex(2, 9):
        d = np.zeros_like(x)
        d[at] = h
        assert abs((loss(x + d, g) - loss(x - d, g)) / (2 * h) - dx[at]) < 1e-8
    for c in range(9):
        d = np.zeros_like(g)
        d[c] = h
        assert abs((loss(x, g + d) - loss(x, g - d)) / (2 * h) - dg[c]) < 1e-8


def test_wgrad_against_autograd():
    rng = np.random.default_rng(5)
    x, W = rng.standard_normal((11, 7)), torch.from_numpy(rng.standard_normal((5, 7))).requires_grad_()
    dY = rng.standard_normal((11, 5))
    (torch.from_numpy(x) @ W.T).backward(torch.from_numpy(dY))
    np.testing.assert_allclose(LO.linear_wgrad(dY, x), W.grad.numpy(), rtol=1e-12)
    np.testing.assert_allclose(LO.linear_wgrad(dY, x, np.ones((5, 7))), W.grad.numpy() + 1, rtol=1e-12)


def test_planted_mistakes_are_caught():
    """What the pins above must tell apart: each wrong form differs by far more than they allow."""
    rng = np.random.default_rng(6)
    x, g, dy = rng.standard_normal((3, 40)) + 0.5, 1 + rng.standard_normal(40), rng.standard_normal((3, 40))
    _, mean, rstd = LO.norm_fwd(x, "layer", g, None, 1e-5)
    dx, dg, _ = LO.norm_bwd(dy, x, "layer", g, mean, rstd)
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy * g
    no_mean = rstd[:, None] * (a - xh * (a * xh).mean(1, keepdims=True))
    no_weight = rstd[:, None] * (dy - dy.mean(1, keepdims=True) - xh * (dy * xh).mean(1, keepdims=True))
    uncentred = (dy * x * rstd[:, None]).sum(0)
    assert np.abs(no_mean - dx).max() > 1e-3 and np.abs(no_weight - dx).max() > 1e-3 and np.abs(uncentred - dg).max() > 1e-3
    codes, scales = LO.checkpoint_save(x)
    back = LO.checkpoint_load(codes, scales, 40)
    assert np.abs(LO.checkpoint_load(codes, np.roll(scales, 1, 1), 40) - back).max() > 1e-3
    assert np.abs(LO.checkpoint_load(np.roll(codes, 1, 0), scales, 40) - back).max() > 1e-3
