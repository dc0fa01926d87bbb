"""What ptxas reports of the kernels of the 8-bit products and of the AdamW steps (the library's own compile, no GPU)."""
import os
import re

import pytest

from paper_2608_23048_gb300 import _build


def kernels(source, name):
    """[(registers, bytes of spill stores)] of the kernels called `name`."""
    try:
        _build.nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    if not os.path.exists(_build.log_of(source)):
        _build.build(force=True)
    with open(_build.log_of(source)) as f:
        found = re.findall(r"Compiling entry function '\w*" + name + r"\w*'[^\n]*\n[^\n]*\n[^\n]*?(\d+) bytes spill stores[^\n]*\n[^\n]*Used "
                           r"(\d+) registers", f.read())
    return [(int(regs), int(spill)) for spill, regs in found]


def test_products():
    """The sums of a tile stay in registers while they are written: nothing spills."""
    one, pair = kernels("roi_fp8_linear.cu", "roi_fp8_linear_kernel"), kernels("roi_fp8_pair.cu", "roi_fp8_pair_kernel")
    assert len(one) == 6 and len(pair) == 9
    assert all(spill == 0 for _, spill in one + pair) and all(regs <= 168 for regs, _ in pair)


def test_copies():
    assert all(spill == 0 for _, spill in kernels("roi_fp8.cu", "roi_fp8_save"))


def test_adamw():
    """Nothing spills, with as many CTAs of 128 threads an SM as the launches count on."""
    for name, ctas in (("roi_adamw_step_kernel", 10), ("roi_adamw_step8_kernel", 5), ("roi_adamw_state8_load_kernel", 12)):
        found = kernels("roi_optim.cu", name)
        assert len(found) == 2 and all(spill == 0 and -(-regs // 8) * 8 * 128 * ctas <= 65536 for regs, spill in found), (name, found)


def test_copies_are_found():
    """Rows whole sectors apart and anywhere, two formats and three types each, and weights of either kind."""
    found = kernels("roi_fp8.cu", "roi_fp8_save")
    assert len(found) == 14 and all(spill == 0 for _, spill in found)
    assert len(kernels("roi_fp8.cu", "roi_fp8_save_weight_kernel")) == 2
