"""The oracle of the AdamW step with moments in 8 bits."""
import numpy as np
import pytest

from oracle import optim_oracle as O
from oracle import roi_oracle


def test_step_is_adamw():
    rng = np.random.default_rng(1)
    p, g, m = (rng.normal(0, s, 512).astype(np.float32) for s in (1, 1e-2, 1e-3))
    v = rng.uniform(0, 1e-5, 512).astype(np.float32)
    k = O.constants(1e-3, 0.9, 0.95, 1e-8, 0.05, 7)
    got = O.step(p, g, m, v, k)
    want = roi_oracle.adamw_step(p, g, m, v, 1e-3, 0.9, 0.95, 1e-8, 0.05, 7)
    for a, b in zip(got, want):
        assert np.allclose(a, b, rtol=4e-6, atol=1e-9)
    assert np.array_equal(O.step(p, g * np.float32(0.5), m, v, k)[0], O.step(p, g, m, v, k, 0.5)[0])


@pytest.mark.parametrize("kind", ["m", "u"])
def test_every_code_is_its_own(kind):
    """All codes of a block whose largest is the largest, whatever the random bits: nothing to round."""
    bits, top, nan = O.KINDS[kind]
    every = np.arange(0, nan, dtype=np.uint8)
    for s in (1, 127, 240):
        for part in (every[::2], every[1::2]):
            codes = np.zeros(256, np.uint8)
            codes[:part.size] = part
            codes[[127, 255]] = nan - 1
            scales = np.full(2, s, np.uint8)
            v = O.decode(codes, scales, kind)
            for r in (0, 1, 65535):
                back = O.encode(v, kind, np.full(256, r))
                assert np.array_equal(back[0], codes) and np.array_equal(back[1], scales)
    assert O.decode(np.full(128, nan - 1, np.uint8), np.array([127], np.uint8), kind)[0] == top


@pytest.mark.parametrize("kind", ["m", "u"])
def test_rounding_keeps_the_mean(kind):
    """Over all random numbers a code's mean is the value, to 2^-16 of its spacing."""
    x = np.zeros(128 * 4096, np.float32).reshape(4096, 128)
    x[:, 0] = O.KINDS[kind][1]
    x[:, 1:] = np.exp(np.linspace(np.log(0.004), np.log(400), 127)).astype(np.float32)
    r = (np.arange(4096) * 16)[:, None] + np.zeros((1, 128), np.int64)
    codes, scales = O.encode(x.reshape(-1), kind, r.reshape(-1))
    mean = O.decode(codes, scales, kind).reshape(4096, 128).astype(np.float64).mean(0)
    spacing = np.exp2(np.maximum(np.frexp(x[0])[1] - 1, -6) - float(O.KINDS[kind][0]))
    assert np.all(np.abs(mean - x[0]) <= spacing / 4096)


def test_u_follows_a_vanishing_gradient_down():
    """With no gradient v falls by beta2 a step: over 100 steps as much as in float32, to a few parts in a hundred."""
    n = 128 * 64
    p, g = np.zeros(n, np.float32), np.zeros(n, np.float32)
    u0 = np.linspace(0.5, 1, n).astype(np.float32)
    r = np.random.default_rng(2).integers(0, 65536, n)
    cm, sm = O.encode(np.zeros(n, np.float32), "m", r)
    cu, su = O.encode(u0, "u", r)
    state = (cm, cu, np.stack([sm, su], 1))
    for t in range(1, 101):
        p, state = O.step8(p, g, state, O.constants(1e-3, 0.9, 0.95, 1e-8, 0.0, t), 5, t, 0)
    u = O.decode(state[1], state[2][:, 1], "u").astype(np.float64)
    # 100 roundings of at most 1/16 of a step of the value, independent: 2^-4 / sqrt(6) * 10 each, averaged over n
    assert abs(u.mean() / (u0.mean() * 0.95 ** 50) - 1) < 4 * 0.26 / np.sqrt(n)
    assert not np.array_equal(cu, state[1])


def test_what_is_not_finite_stays():
    x = np.zeros(256, np.float32)
    x[3], x[4], x[130], x[131] = np.inf, 1.0, np.nan, 2.0
    for kind in ("m", "u"):
        codes, scales = O.encode(x, kind, np.zeros(256, np.int64))
        v = O.decode(codes, scales, kind)
        assert np.isnan(v[[3, 130]]).all() and v[4] == 1 and v[131] == 2
