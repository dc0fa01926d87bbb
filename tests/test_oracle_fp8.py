"""The oracle of the copies in 8-bit floating point, against torch's own conversions and hand-made numbers."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as O

TYPES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_every_code_is_its_own(fmt):
    """All finite codes as values, rounded and encoded again."""
    every = torch.arange(256, dtype=torch.uint8)
    v = every.view(TYPES[fmt]).double().numpy()
    keep = np.isfinite(v)
    assert np.array_equal(O._byte(O._round(v[keep], fmt), fmt), every.numpy()[keep])
    one = np.full((1, 16), 127, np.uint8)
    back = np.concatenate([O.load(every.numpy()[None, 128 * h:128 * h + 128], one, fmt, 128)[0] for h in range(2)])
    assert np.array_equal(back[keep], v[keep])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("high", [1, 128])
def test_against_torch(fmt, high):
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(130, 300, generator=g) * torch.exp(4 * torch.randn(130, 1, generator=g))).double()
    codes, scales, values = O.save(x.numpy(), fmt, high)
    step = torch.from_numpy(np.repeat(np.repeat(scales[:, :3].astype(np.int64), high, 0)[:130], 128, 1)[:, :300])
    q = (x * torch.exp2(127.0 - step)).float().to(TYPES[fmt])
    assert np.array_equal(q.view(torch.uint8).numpy(), codes[:, :300]) and not codes[:, 300:].any()
    assert np.array_equal(values, O.load(codes, scales, fmt, 300, high))
    # no block could do with a smaller power of two
    top = O.FORMATS[fmt][0]
    for i in range(scales.shape[0]):
        a = float(x[i * high:(i + 1) * high, :128].abs().max())
        assert top * 2.0 ** (int(scales[i, 0]) - 128) < a <= top * 2.0 ** (int(scales[i, 0]) - 127)
    assert (scales[:, 3:] == 1).all()


def test_borders():
    x = np.zeros((5, 128))
    x[0, 0], x[1, 0], x[2, 0], x[3, 5], x[4, 9] = 448.0, np.nextafter(np.float32(448), np.float32(500)), 2.0 ** -140, np.inf, np.nan
    codes, scales, values = O.save(x)
    assert list(scales[:, 0]) == [127, 128, 1, 255, 255]
    assert values[0, 0] == 448 and values[1, 0] == 448 and values[2, 0] == 0
    assert np.isnan(values[3:]).all() and not codes[3:].any()
