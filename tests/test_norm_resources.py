"""What ptxas reports of the norms' kernels (the library's own compile, no GPU): the forms that most calls take
keep their rows and sums in registers."""
import os
import re

import pytest

from paper_2608_23048_gb300 import _build


@pytest.fixture(scope="module")
def kernels():
    """{(pass, template arguments): (registers, bytes of spill stores)}; arguments as numbers, in their order."""
    try:
        _build.nvcc()
    except RuntimeError:
        pytest.skip("needs nvcc")
    if not os.path.exists(_build.log_of("roi_norm.cu")):
        _build.build(force=True)
    with open(_build.log_of("roi_norm.cu")) as f:
        found = re.findall(r"Compiling entry function '\w*roi_norm_(fwd|bwd)_kernelI(\w*)EEv\w*'[^\n]*\n[^\n]*\n[^\n]*?(\d+) bytes spill "
                           r"stores[^\n]*\n[^\n]*Used (\d+) registers", f.read())
    return {(way, tuple(int(v) for v in re.findall(r"(?:ElemE|Lb|Li)(\d+)E", args + "E"))): (int(regs), int(spill))
            for way, args, spill, regs in found}


def test_forward(kernels):
    """(type, layer, rows anywhere, pieces): nothing to speak of, whichever the form."""
    forms = {k[1]: v for k, v in kernels.items() if k[0] == "fwd"}
    assert len(forms) == 24 and all(spill <= 8 for _, spill in forms.values()), forms


def test_backward_of_whole_granules(kernels):
    """(type, layer, checkpoint, rows anywhere, pieces, threads): two pieces a thread in fewer than 1024 threads,
    and one piece in 1024, at most 32 bytes; none where x is in 16 bits and most used (3584 columns)."""
    forms = {k[1]: v for k, v in kernels.items() if k[0] == "bwd" and k[1][3] == 0}
    few = {k: v for k, v in forms.items() if k[4] == 1 or k[5] < 1024}
    assert len(few) >= 24 and all(spill <= 32 for _, spill in few.values()), few
    for dtype in (0, 1):
        for ckpt in (0, 1):
            assert few[dtype, 0, ckpt, 0, 2, 768][1] <= 8 and few[dtype, 1, ckpt, 0, 2, 512][1] == 0


def test_rows_that_start_anywhere(kernels):
    """They spill, for the words of their shifts: what they do now is the most they may."""
    forms = {k[1]: v for k, v in kernels.items() if k[0] == "bwd" and k[1][3] == 1 and (k[1][4] == 1 or k[1][5] < 1024)}
    assert len(forms) >= 24 and all(spill <= (176 if k[0] < 2 else 304) for k, (_, spill) in forms.items()), forms
