"""The example's two uses of the library's noise: what draws its masks and what rounds its moments in 8 bits are different
words.  (With the same words a logit's root of v is rounded up where its noise in a mask is large.)"""
import pytest

from test_example_fp8_gpu import example  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def test_masks_and_rounding_draw_different_words(example, monkeypatch):  # noqa: F811
    masks, rounded = set(), set()

    class Recorder:
        """The library, noting which words are drawn."""

        def __getattr__(self, name):
            return getattr(library, name)

        def NoiseState(self, seed, step, tensor_id, *rest):
            masks.add((seed, step, tensor_id))
            return library.NoiseState(seed, step, tensor_id, *rest)

        def roi_adamw_step8(self, items, opt, seed, *rest, **kw):
            rounded.update((seed, opt.t, item[4]) for item in items)
            return library.roi_adamw_step8(items, opt, seed, *rest, **kw)

    library = example.roi
    monkeypatch.setattr(example, "roi", Recorder())
    example.train(256, 512, 64, 4, fp8=True)
    assert len(masks) == len(rounded) == 12
    assert not masks & rounded
