// Activation checkpoints in 8 bits (the layout is in roi_block8.cuh): save and load.
//
// Bound by memory: a save reads b bytes an element and writes 33/32, a load the reverse.
// Vector kernels: a thread takes 16 consecutive columns (two or four 16-byte loads, one
// 16-byte store of codes), so a block is two neighbouring lanes, whose largest magnitudes
// meet in one shuffle; kUnits such pieces are loaded before the first is used.  Rows whose
// start or stride is not a multiple of 16 bytes go to the element kernels, where a warp
// takes a block, a lane a column.
#include "roi_block8.cuh"
#include "roi_launch.h"

namespace roi {
namespace {

constexpr int kThreads = 256;
constexpr int kUnits = 2;        // pieces of 16 columns a thread has in flight
constexpr int kBlocksAWarp = 8;  // element kernels: blocks a warp has in flight

struct SaveArgs {
  const void* x;
  int8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, ld;
  int64_t pitch, spitch;
  int64_t pieces;  // of 16 columns in a row, the scales' padding included
  bool wait;
};

struct LoadArgs {
  const int8_t* codes;
  const uint8_t* scales;
  void* x;
  int64_t rows, cols, ld;
  int64_t pitch, spitch;
  int64_t pieces;  // of 16 columns in a row
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

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_save_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const T* x = static_cast<const T*>(a.x);
  const int64_t total = a.rows * a.pieces;
  constexpr int kTile = kThreads * kUnits;
  for (int64_t base = int64_t(blockIdx.x) * kTile; base < total; base += int64_t(gridDim.x) * kTile) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    Raw8<E> r[kUnits][2];
    int64_t row[kUnits], j[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      walk(row0, rem0, uint32_t(u * kThreads) + threadIdx.x, a.pieces, row[u], j[u]);
      const T* p = x + row[u] * a.ld + 16 * j[u];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t left = a.cols - 16 * j[u] - 8 * h;
        if (row[u] < a.rows && left >= 8) {
          r[u][h].load(p + 8 * h);
        } else if (row[u] < a.rows && left > 0) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = i < left ? to_f32<E>(p[8 * h + i]) : 0.0f;
          r[u][h].set(v);
        } else {
          r[u][h].zero();
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      float v[16];
      {
        float lo[8], hi[8];
        r[u][0].get(lo), r[u][1].get(hi);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lo[i], v[8 + i] = hi[i];
      }
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = max(top, abs_bits(v[i]));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      const uint32_t s = block8_scale(top);
      const float inverse = block8_inverse(min(s, kScaleMax));
      const uint32_t keep = s == kScaleNaN ? 0u : 0xffffffffu;
      if (row[u] < a.rows) {
        if (16 * j[u] < a.pitch)
          *reinterpret_cast<uint4*>(a.codes + row[u] * a.pitch + 16 * j[u]) =
              make_uint4(block8_codes4(v, inverse, keep), block8_codes4(v + 4, inverse, keep),
                         block8_codes4(v + 8, inverse, keep), block8_codes4(v + 12, inverse, keep));
        if ((j[u] & 1) == 0) a.scales[row[u] * a.spitch + (j[u] >> 1)] = uint8_t(s);
      }
    }
  }
}

// A warp a block of 32 columns, a lane a column (`pieces`: blocks in a row here).
template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_save_elem_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const T* x = static_cast<const T*>(a.x);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t total = a.rows * a.pieces;
  constexpr int kTile = kThreads / 32 * kBlocksAWarp;
  for (int64_t base = int64_t(blockIdx.x) * kTile; base < total; base += int64_t(gridDim.x) * kTile) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    float v[kBlocksAWarp];
    int64_t row[kBlocksAWarp], b[kBlocksAWarp];
#pragma unroll
    for (int u = 0; u < kBlocksAWarp; ++u) {
      walk(row0, rem0, uint32_t(warp * kBlocksAWarp + u), a.pieces, row[u], b[u]);
      const int64_t c = 32 * b[u] + lane;
      v[u] = row[u] < a.rows && c < a.cols ? to_f32<E>(x[row[u] * a.ld + c]) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < kBlocksAWarp; ++u) {
      const uint32_t s = block8_scale(__reduce_max_sync(0xffffffffu, abs_bits(v[u])));
      const uint32_t q = block8_code(v[u], block8_inverse(min(s, kScaleMax)));
      if (row[u] < a.rows) {
        if (32 * b[u] < a.pitch) a.codes[row[u] * a.pitch + 32 * b[u] + lane] = s == kScaleNaN ? int8_t(0) : int8_t(q);
        if (lane == 0) a.scales[row[u] * a.spitch + b[u]] = uint8_t(s);
      }
    }
  }
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_load_kernel(LoadArgs a) {
  using T = typename ElemType<E>::T;
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
      const float step = block8_step(s[u]);
      T* p = x + row[u] * a.ld + 16 * j[u];
      const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = block8_clip<E>(block8_value(w[2 * h + i / 4], i % 4, step));
        const int64_t left = a.cols - 16 * j[u] - 8 * h;
        if (left >= 8) {
          Raw8<E> r;
          r.set(v);
          r.store(p + 8 * h);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < left) p[8 * h + i] = from_f32<E>(v[i]);
        }
      }
    }
  }
}

template <Elem E>
__global__ void __launch_bounds__(kThreads) roi_checkpoint_load_elem_kernel(LoadArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  T* x = static_cast<T*>(a.x);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t total = a.rows * a.pieces;
  constexpr int kTile = kThreads / 32 * kBlocksAWarp;
  for (int64_t base = int64_t(blockIdx.x) * kTile; base < total; base += int64_t(gridDim.x) * kTile) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    int8_t q[kBlocksAWarp];
    uint8_t s[kBlocksAWarp];
    int64_t row[kBlocksAWarp], b[kBlocksAWarp];
#pragma unroll
    for (int u = 0; u < kBlocksAWarp; ++u) {
      walk(row0, rem0, uint32_t(warp * kBlocksAWarp + u), a.pieces, row[u], b[u]);
      q[u] = 0, s[u] = 0;
      if (row[u] < a.rows) {
        q[u] = a.codes[row[u] * a.pitch + 32 * b[u] + lane];
        s[u] = a.scales[row[u] * a.spitch + b[u]];
      }
    }
#pragma unroll
    for (int u = 0; u < kBlocksAWarp; ++u) {
      const int64_t c = 32 * b[u] + lane;
      if (row[u] < a.rows && c < a.cols)
        x[row[u] * a.ld + c] = from_f32<E>(block8_clip<E>(float(q[u]) * block8_step(s[u])));
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

bool rows_aligned(const void* p, int64_t ld, int64_t rows, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * bytes % 16 == 0);
}

template <Elem E>
int save(const CheckpointCall& c) {
  SaveArgs a{c.x_in, c.codes, c.scales, c.rows, c.cols, c.ld, block8_pitch(c.cols), block8_scale_pitch(c.cols), 0,
             lone_pdl(c.stream)};
  if (!rows_aligned(c.x_in, c.ld, c.rows, elem_bytes<E>())) {
    a.pieces = a.spitch;
    return launch(roi_checkpoint_save_elem_kernel<E>, a, a.rows * a.pieces, kThreads / 32 * kBlocksAWarp, c.stream);
  }
  if (a.ld == a.cols && a.cols % 128 == 0) {  // the rows follow one another in every array: one long row
    a.cols *= a.rows, a.pitch *= a.rows, a.spitch *= a.rows, a.ld = a.cols, a.rows = 1;
  }
  a.pieces = a.spitch * 2;
  return launch(roi_checkpoint_save_kernel<E>, a, a.rows * a.pieces, kThreads * kUnits, c.stream);
}

template <Elem E>
int load(const CheckpointCall& c) {
  LoadArgs a{c.codes, c.scales, c.x_out, c.rows, c.cols, c.ld, block8_pitch(c.cols), block8_scale_pitch(c.cols), 0,
             lone_pdl(c.stream)};
  if (!rows_aligned(c.x_out, c.ld, c.rows, elem_bytes<E>())) {
    a.pieces = a.pitch / 32;
    return launch(roi_checkpoint_load_elem_kernel<E>, a, a.rows * a.pieces, kThreads / 32 * kBlocksAWarp, c.stream);
  }
  if (a.ld == a.cols && a.cols % 128 == 0) {
    a.cols *= a.rows, a.pitch *= a.rows, a.spitch *= a.rows, a.ld = a.cols, a.rows = 1;
  }
  a.pieces = (a.cols + 15) / 16;
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
