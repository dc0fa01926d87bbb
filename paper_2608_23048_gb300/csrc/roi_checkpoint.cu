// Activation checkpoints in 8 bits (the layout is in roi_block8.cuh): save and load.
//
// Bound by memory: a save reads b bytes an element and writes 33/32, a load the reverse.  A
// thread takes 16 consecutive columns (one 16-byte access of codes), so a block is two
// neighbouring lanes, whose largest magnitudes meet in one shuffle; kUnits such pieces are
// loaded before the first is used.  Where rows are whole 32-byte sectors apart, the pieces of
// all rows follow one another and every access is whole sectors; elsewhere a warp, or a part of
// one, has a row of its own and goes by granules (roi_rows.cuh).
//
// Measured, 8192 x 18944 (of 6.79 TB/s copied): bf16 save 82 us (5.75 TB/s), load 77 to 84; fp32 save 115 (6.79),
// load 121 to 128 (6.1 to 6.4; stores alone run at 3.9 TB/s here).  A save in bf16 issues in 60 % of the cycles, a load waits
// for memory.  Rows that start anywhere, 8192 x 18943 bf16: 93 and 131 us.  The same aligned matrices through the kernels
// of rows that start anywhere: bf16 91 and 102 us, fp32 125 and 156.
#include "roi_block8.cuh"
#include "roi_launch.h"
#include "roi_rows.cuh"

namespace roi {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 2;        // pieces of 16 columns a thread has in flight

struct SaveArgs {
  const void* x;
  int8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, ld;
  int64_t pitch, spitch;
  int64_t pieces;  // of 16 columns in a row, the scales' padding included
  int width, segments;  // rows anywhere: lanes of a row, and how often they go over it
  bool wait;
};

struct LoadArgs {
  const int8_t* codes;
  const uint8_t* scales;
  void* x;
  int64_t rows, cols, ld;
  int64_t pitch, spitch;
  int64_t pieces;  // of 16 columns in a row
  int width, segments;
  bool wait;
};

// Row and place in the row of the `i`-th item of a row-major walk over rows of `per_row`
// items, from the row and the place of the walk's start (one division of 64 bits a tile).
__device__ __forceinline__ void walk(int64_t row0, int64_t rem0, uint32_t i, int64_t per_row, int64_t& row, int64_t& j) {
  j = rem0 + i;
  row = row0;
  if (j >= per_row) {
    if (per_row <= 0x3fffffff) {
      const uint32_t q = uint32_t(j) / uint32_t(per_row);
      row += q;
      j -= int64_t(q) * per_row;
    } else {
      ++row;
      j -= per_row;
    }
  }
}

// Codes and scale of a piece (all lanes of the warp); `q` is its place in the row.
template <Elem E>
__device__ __forceinline__ void save_piece(const SaveArgs& a, const RowWords<E, 16>& r, int64_t row, int64_t q) {
  uint32_t top = max_bits(r);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const uint32_t s = block8_scale(top);
  uint32_t w[4];
  block8_codes(r, top, s, w);
  if (row < a.rows && q < a.pieces) {
    if (16 * q < a.pitch) *reinterpret_cast<uint4*>(a.codes + row * a.pitch + 16 * q) = make_uint4(w[0], w[1], w[2], w[3]);
    if ((q & 1) == 0) a.scales[row * a.spitch + (q >> 1)] = uint8_t(s);
  }
}
template <Elem E>
__device__ __forceinline__ void load_piece(const uint4& q, uint32_t s, RowWords<E, 16>& r) {
  const float step = block8_step(s);
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  float v[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    F2 a, b;
    block8_pairs(w[i], step, a, b);
    v[4 * i] = block8_clip<E>(lo(a)), v[4 * i + 1] = block8_clip<E>(hi(a));
    v[4 * i + 2] = block8_clip<E>(lo(b)), v[4 * i + 3] = block8_clip<E>(hi(b));
  }
  r.set(v);
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_save_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  constexpr int kWords = RowWords<E, 16>::kWords;
  pdl_begin(a.wait);
  const T* x = static_cast<const T*>(a.x);
  const int64_t total = a.rows * a.pieces;
  constexpr int kTile = kThreads * kUnits;
  for (int64_t base = int64_t(blockIdx.x) * kTile; base < total; base += int64_t(gridDim.x) * kTile) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    RowWords<E, 16> r[kUnits];
    int64_t row[kUnits], j[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      walk(row0, rem0, uint32_t(u * kThreads) + threadIdx.x, a.pieces, row[u], j[u]);
      const T* p = x + row[u] * a.ld + 16 * j[u];
      if (row[u] < a.rows && a.cols - 16 * j[u] >= 16) {
#pragma unroll
        for (int i = 0; i < kWords / 8; ++i) load32(reinterpret_cast<const uint4*>(p) + 2 * i, r[u].u + 8 * i);
      } else if (row[u] < a.rows) {
        r[u].load_elements(x + row[u] * a.ld, 16 * j[u], a.cols);
      } else {
        r[u].zero();
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      save_piece<E>(a, r[u], row[u], j[u]);
    }
  }
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_load_kernel(LoadArgs a) {
  using T = typename ElemType<E>::T;
  constexpr int kWords = RowWords<E, 16>::kWords;
  pdl_begin(a.wait);
  T* x = static_cast<T*>(a.x);
  const int64_t total = a.rows * a.pieces;
  constexpr int kTile = kThreads * kUnits;
  for (int64_t base = int64_t(blockIdx.x) * kTile; base < total; base += int64_t(gridDim.x) * kTile) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    uint4 q[kUnits];
    uint32_t s[kUnits];
    int64_t row[kUnits], j[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      walk(row0, rem0, uint32_t(u * kThreads) + threadIdx.x, a.pieces, row[u], j[u]);
      q[u] = make_uint4(0, 0, 0, 0), s[u] = 0;
      if (row[u] < a.rows) {
        q[u] = __ldg(reinterpret_cast<const uint4*>(a.codes + row[u] * a.pitch + 16 * j[u]));
        s[u] = __ldg(a.scales + row[u] * a.spitch + (j[u] >> 1));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (row[u] >= a.rows) continue;
      RowWords<E, 16> r;
      load_piece<E>(q[u], s[u], r);
      T* p = x + row[u] * a.ld + 16 * j[u];
      const int64_t left = a.cols - 16 * j[u];
      if (left >= 16) {
#pragma unroll
        for (int i = 0; i < kWords / 8; ++i) store32(reinterpret_cast<uint4*>(p) + 2 * i, r.u + 8 * i);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i < left) p[i] = r.at(i);
      }
    }
  }
}

// Rows anywhere.  A warp's task: 32 / width rows, or one segment of a row.
__device__ __forceinline__ void row_task(int64_t task, int width, int segments, int64_t& row, int64_t& piece) {
  const int lane = threadIdx.x & 31;
  if (segments > 1) {
    row = task / segments;
    piece = (task - row * segments) * 32 + lane;
  } else {
    row = task * (32 / width) + lane / width;
    piece = lane & (width - 1);
  }
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_save_rows_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const int64_t per = 32 / a.width, tasks = (a.rows + per - 1) / per * a.segments;
  const int64_t stride = int64_t(gridDim.x) * (kThreads / 32) * kUnits;
  for (int64_t t = (int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * kUnits; t < tasks; t += stride) {
    Window<E, 16> x[kUnits];
    int64_t row[kUnits], j[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      row_task(t + u, a.width, a.segments, row[u], j[u]);
      x[u].load(static_cast<const T*>(a.x) + row[u] * a.ld, 16 * j[u], row[u] < a.rows ? a.cols : 0);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      RowWords<E, 16> r;
      x[u].get(r);
      save_piece<E>(a, r, row[u], j[u]);
    }
  }
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_load_rows_kernel(LoadArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const int64_t per = 32 / a.width, tasks = (a.rows + per - 1) / per * a.segments;
  const int64_t stride = int64_t(gridDim.x) * (kThreads / 32) * kUnits;
  for (int64_t t = (int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * kUnits; t < tasks; t += stride) {
    uint4 q[kUnits];
    uint32_t s[kUnits];
    int64_t row[kUnits], j[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      row_task(t + u, a.width, a.segments, row[u], j[u]);
      q[u] = make_uint4(0, 0, 0, 0), s[u] = 0;
      if (row[u] < a.rows && j[u] < a.pieces) {
        q[u] = __ldg(reinterpret_cast<const uint4*>(a.codes + row[u] * a.pitch + 16 * j[u]));
        s[u] = __ldg(a.scales + row[u] * a.spitch + (j[u] >> 1));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      RowWords<E, 16> r;
      load_piece<E>(q[u], s[u], r);
      const int64_t none = -(int64_t(1) << 40);
      store_row<E, 16, false>(static_cast<T*>(a.x) + row[u] * a.ld, 16 * j[u], row[u] < a.rows ? a.cols : none, r, a.width);
    }
  }
}

template <class Args>
int launch(void (*kern)(Args), const Args& a, int64_t total, int tile, cudaStream_t stream) {
  int64_t grid = (total + tile - 1) / tile;
  const int64_t cap = int64_t(sm_count()) * 8;  // what an SM holds at once
  if (grid > cap) grid = cap;
  return launch_maybe_pdl(kern, int(grid), kThreads, 0, stream, a.wait, a);
}

// Rows that are whole 32-byte sectors apart.
bool in_sectors(const void* p, int64_t ld, int64_t rows, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 31u) == 0 && (rows <= 1 || ld * bytes % 32 == 0);
}
// Rows anywhere: the lanes of a row, a power of two that holds its pieces, or a whole warp that
// goes over it in segments.  Returns the tiles of the launch.
template <class Args>
int64_t by_rows(Args& a) {
  a.width = 8;
  while (a.width < 32 && a.width < a.pieces) a.width *= 2;
  a.segments = int((a.pieces + 31) / 32);
  const int64_t per = 32 / a.width;
  return (a.rows + per - 1) / per * a.segments;
}

template <Elem E>
int save(const CheckpointCall& c) {
  SaveArgs a{c.x_in, c.codes, c.scales, c.rows, c.cols, c.ld, block8_pitch(c.cols), block8_scale_pitch(c.cols), 0, 0, 0,
             lone_pdl(c.stream)};
  if (!in_sectors(c.x_in, c.ld, c.rows, elem_bytes<E>())) {
    a.pieces = a.spitch * 2;
    return launch(roi_checkpoint_save_rows_kernel<E>, a, by_rows(a), kThreads / 32 * kUnits, c.stream);
  }
  if (a.ld == a.cols && a.cols % 128 == 0) {  // the rows follow one another in every array: one long row
    a.cols *= a.rows, a.pitch *= a.rows, a.spitch *= a.rows, a.ld = a.cols, a.rows = 1;
  }
  a.pieces = a.spitch * 2;
  return launch(roi_checkpoint_save_kernel<E>, a, a.rows * a.pieces, kThreads * kUnits, c.stream);
}

template <Elem E>
int load(const CheckpointCall& c) {
  LoadArgs a{c.codes, c.scales, c.x_out, c.rows, c.cols, c.ld, block8_pitch(c.cols), block8_scale_pitch(c.cols), 0, 0, 0,
             lone_pdl(c.stream)};
  a.pieces = (a.cols + 15) / 16;
  if (!in_sectors(c.x_out, c.ld, c.rows, elem_bytes<E>()))
    return launch(roi_checkpoint_load_rows_kernel<E>, a, by_rows(a), kThreads / 32 * kUnits, c.stream);
  if (a.ld == a.cols && a.cols % 128 == 0) {
    a.cols *= a.rows, a.pitch *= a.rows, a.spitch *= a.rows, a.ld = a.cols, a.rows = 1;
    a.pieces = a.cols / 16;
  }
  return launch(roi_checkpoint_load_kernel<E>, a, a.rows * a.pieces, kThreads * kUnits, c.stream);
}

}  // namespace

int launch_checkpoint_save(const CheckpointCall& c) {
  switch (c.dtype) {
    case Elem::kBf16: return save<Elem::kBf16>(c);
    case Elem::kFp16: return save<Elem::kFp16>(c);
    default: return save<Elem::kFp32>(c);
  }
}

int launch_checkpoint_load(const CheckpointCall& c) {
  switch (c.dtype) {
    case Elem::kBf16: return load<Elem::kBf16>(c);
    case Elem::kFp16: return load<Elem::kFp16>(c);
    default: return load<Elem::kFp32>(c);
  }
}

}  // namespace roi
