"""The AdamW step with moments in 8 bits at the ends of its settings' ranges: the quotient's quick form is taken only where it
is right, and the step is the oracle's bit for bit."""
import numpy as np
import pytest

from oracle import optim_oracle as O
from test_checkpoint_gpu import roi  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lr", [1e-3, 1e6, 1e30])
@pytest.mark.parametrize("eps", [2.0 ** -60, 2.0 ** -41, 2.0 ** -40, 1e-8, 1.0, 2.0 ** 40, 2.0 ** 41, 2.0 ** 100, 2.0 ** 126, 2.0 ** 127, 3e38])
def test_eps_and_lr(roi, eps, lr):  # noqa: F811
    """Parameters at zero, so that the quotient alone is what they become; whole significands and magnitudes from 2^-20 to 2^20."""
    import torch
    n = 128 * 40
    rng = np.random.default_rng(3)
    g = (np.exp2(rng.uniform(-20, 20, n)) * rng.choice((-1, 1), n)).astype(np.float32)
    p = np.zeros(n, np.float32)
    state = (np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros((n // 128, 2), np.uint8))
    dev = [torch.zeros(n, device="cuda"), torch.from_numpy(g).cuda(), roi.new_adamw_state8(n)]
    for t in (1, 2):
        s = dict(lr=lr, beta1=0.9, beta2=0.95, eps=eps, weight_decay=0.0, t=t)
        roi.roi_adamw_step8([(dev[0], dev[1], dev[2], None, 3)], roi.AdamW(*s.values()), 77)
        p, state = O.step8(p, g, state, O.constants(**s), 77, t, 3)
        roi.roi_device_status()
        assert np.array_equal(dev[0].cpu().numpy(), p), t
        for got, want in zip(dev[2], state):
            assert np.array_equal(got.cpu().numpy(), want), t
