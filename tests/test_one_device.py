"""The tensors of a call lie on one device: the binding refuses others before any CUDA call (no GPU)."""
import pytest
import torch

from test_fp8_abi import roi  # noqa: F401  (the fixture)


class On:
    """A tensor that says it is on a CUDA device."""

    def __init__(self, tensor, device):
        self.tensor, self.is_cuda, self.device = tensor, True, torch.device("cuda", device)

    def get_device(self):
        return self.device.index

    def __getattr__(self, name):
        return getattr(self.tensor, name)


def pair(p, a, b=None):
    return On(p[0], a), On(p[1], a if b is None else b)


# which of (x or out, codes, scales) is on the other device
@pytest.mark.parametrize("where", [(1, 0, 0), (0, 1, 0), (0, 0, 1)])
def test_copies(roi, where):  # noqa: F811
    a, b, c = where
    with pytest.raises(ValueError, match="cuda:"):
        roi.roi_fp8_save(On(torch.zeros(4, 128), a), "e4m3", *pair(roi.new_fp8(4, 128, "cpu"), b, c))
    with pytest.raises(ValueError, match="cuda:"):
        roi.roi_fp8_save_weight(On(torch.zeros(4, 128, dtype=torch.bfloat16), a), *pair(roi.new_fp8_weight(4, 128, "cpu"), b, c))


@pytest.mark.parametrize("where", [(1, 0, 0, 0, 0), (0, 1, 0, 0, 0), (0, 0, 1, 0, 0), (0, 0, 0, 1, 0), (0, 0, 0, 0, 1), (0, 1, 1, 0, 0)])
def test_products(roi, where):  # noqa: F811
    out, xq, xs, wq, ws = where
    x8, w8 = pair(roi.new_fp8(4, 128, "cpu"), xq, xs), pair(roi.new_fp8_weight(128, 128, "cpu"), wq, ws)
    for call in (roi.roi_fp8_linear_fwd, roi.roi_fp8_linear_dgrad):
        with pytest.raises(ValueError, match="cuda:"):
            call(x8, "e4m3", w8, On(torch.zeros(4, 128), out))


def test_items_of_a_step(roi):  # noqa: F811
    """Tensor by tensor, and item by item."""
    t = lambda d: On(torch.zeros(8), d)  # noqa: E731
    s = lambda d: tuple(On(x, d) for x in roi.new_adamw_state8(8, "cpu"))  # noqa: E731
    for make, item, mixed in ((roi.make_adamw_step_items, lambda d: (t(d), t(d), t(d), t(d), None), (t(0), t(1), t(0), t(0), None)),
                              (roi.make_adamw_step8_items, lambda d: (t(d), t(d), s(d), None, 0), (t(0), t(0), s(1), None, 0)),
                              (roi.make_adamw_state8_items, lambda d: (s(d), t(d), t(d)), (s(0), t(0), t(1)))):
        assert len(make([item(0), item(0)])) == 2
        with pytest.raises(ValueError, match="cuda:"):
            make([mixed])
        with pytest.raises(ValueError, match="cuda:"):
            make([item(0), item(1)])


def test_gradient_factor(roi):  # noqa: F811
    """The list of tensors knows its device."""
    t = lambda d: On(torch.zeros(8), d)  # noqa: E731
    opt, factor = roi.AdamW(1e-3, 0.9, 0.95, 1e-8, 0.0, 1), On(torch.ones(1), 1)
    with pytest.raises(ValueError, match="cuda:"):
        roi.roi_adamw_step(roi.make_adamw_step_items([(t(0), t(0), t(0), t(0), None)]), opt, factor)
    state = tuple(On(x, 0) for x in roi.new_adamw_state8(8, "cpu"))
    with pytest.raises(ValueError, match="cuda:"):
        roi.roi_adamw_step8([(t(0), t(0), state, None, 0)], opt, 1, factor)
