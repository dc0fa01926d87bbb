"""The reach of the norms' row copies (csrc/roi_extent.h, plain C++), on the CPU: over rows, strides and
starting addresses, a row's copy takes whole granules inside the matrix, and with the bytes it leaves
out the row is whole in its stage."""
import ctypes
import shutil
import subprocess

import numpy as np
import pytest

from paper_2608_23048_gb300 import _build

SHIM = r"""
#include <cstring>
#include "roi_extent.h"
using namespace roi;
// Row by row as the kernels copy it; what of it went wrong (0: nothing).
extern "C" int copy_rows(const uint8_t* p, int rows, int pitch, int width, int any, uint8_t* stage, int room) {
  const Bounds all = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + uintptr_t((rows - 1) * pitch) + width};
  for (int r = 0; r < rows; ++r) {
    const uint8_t* row = p + r * pitch;
    const Extent x(row, width, any, all);
    memset(stage, 0xee, room);
    if (any && x.cut()) x.ends(stage);
    if (x.bytes() > 0) {
      if (x.from % 16 || x.bytes() % 16 || x.offset() % 16) return 1;
      if (x.from < all.begin || x.to > all.end) return 2;
      if (x.offset() + x.bytes() > unsigned(room)) return 3;
      memcpy(stage + x.offset(), reinterpret_cast<const void*>(x.from), x.bytes());
    }
    if (memcmp(stage + (any ? reinterpret_cast<uintptr_t>(row) & 15 : 0), row, width)) return 4;
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def copy_rows(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("needs a C++ compiler")
    d = tmp_path_factory.mktemp("extents")
    (d / "shim.cc").write_text(SHIM)
    subprocess.run([cxx, "-O1", "-std=c++17", "-shared", "-fPIC", "-I", _build.CSRC, "-o", str(d / "shim.so"), str(d / "shim.cc")],
                   check=True)
    f = ctypes.CDLL(str(d / "shim.so")).copy_rows
    f.argtypes = [ctypes.c_void_p] + [ctypes.c_int] * 4 + [ctypes.c_void_p, ctypes.c_int]
    room = np.random.default_rng(0).integers(0, 255, 1 << 14, dtype=np.uint8)
    base = room.ctypes.data + (-room.ctypes.data) % 16 + 64
    stage = np.zeros(1024, np.uint8)

    def call(offset, rows, pitch, width, any_=1):
        # a row's room in the ring: whole runs of 8 columns, and two granules
        return f(base + offset, rows, pitch, width, any_, stage.ctypes.data, (width + 15) // 16 * 16 + 32)
    return call


# 4 to 16 bytes a row are the scales of checkpoints of up to 512 columns
@pytest.mark.parametrize("width", [2, 4, 6, 8, 10, 12, 14, 16, 18, 28, 30, 32, 46, 100])
def test_copies_stay_inside_the_matrix(copy_rows, width):
    for gap in (0, 2, 4, 6, 10, 14, 16, 30, 64):
        for offset in range(0, 16, 2):
            for rows in (1, 2, 3, 4, 5, 6, 7, 8, 9, 17):
                assert copy_rows(offset, rows, width + gap, width) == 0, (offset, rows, gap)


def test_rows_of_whole_granules(copy_rows):
    for width, gap in ((16, 0), (48, 16), (256, 0)):
        assert copy_rows(0, 5, width + gap, width, 0) == 0
        assert copy_rows(0, 5, width + gap, width, 1) == 0
