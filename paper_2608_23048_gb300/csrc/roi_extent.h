// What a bulk copy takes of a matrix row that starts anywhere (plain C++, on the host and the device).
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define ROI_HD __host__ __device__ __forceinline__
#else
#define ROI_HD inline
#endif

namespace roi {

// A matrix's first byte, and the one after its last.
struct Bounds {
  uintptr_t begin, end;
};

// Bulk copies move granules of 16 bytes.  Of a row: the granules around it that lie inside the matrix;
// what is in the matrix's first or last granule, only part of which may be the caller's, goes byte by
// byte.  Several rows lie in such a granule where rows are shorter than 16 bytes.  A row's byte
// i lies i + (address mod 16) bytes after the place it is copied to.
struct Extent {
  uintptr_t row, end, from, to;
  // (rows of whole granules, ANY false, are copied as they are)
  ROI_HD Extent(const void* p, uint32_t bytes, bool any, const Bounds& of) {
    constexpr uintptr_t kMask = ~uintptr_t(15);
    row = reinterpret_cast<uintptr_t>(p), end = row + bytes, from = row, to = end;
    if (any) {
      from = row & kMask, to = (end + 15) & kMask;
      const uintptr_t first = (of.begin + 15) & kMask, last = of.end & kMask;
      if (from < first) from = first;
      if (to > last) to = last;
    }
  }
  ROI_HD uint32_t bytes() const { return to > from ? uint32_t(to - from) : 0u; }
  // whether the copy leaves out some of the row
  ROI_HD bool cut() const { return from > row || to < end; }
  // (one thread) what the copy leaves out
  ROI_HD void ends(uint8_t* place) const {
    uint8_t* at = place + (row & 15);
    for (uintptr_t p = row; p < from && p < end; ++p) at[p - row] = *reinterpret_cast<const uint8_t*>(p);
    uintptr_t p = to > from ? to : from;
    for (p = p < row ? row : p; p < end; ++p) at[p - row] = *reinterpret_cast<const uint8_t*>(p);
  }
  // where the copy's first byte goes
  ROI_HD uint32_t offset() const { return uint32_t(from - (row & ~uintptr_t(15))); }
};

}  // namespace roi
