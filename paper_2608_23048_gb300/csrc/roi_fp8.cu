// Copies in 8-bit floating point (the layout is in roi_fp8.cuh) of activations and of weights.
//
// Bound by memory: b bytes an element are read and 129/128 written.  A thread takes 16 consecutive columns (one 16-byte
// store of codes), so eight neighbouring lanes hold a block of a row and its largest magnitude takes three shuffles.  A
// weight's block of 128 x 128 is a CTA's, four such pieces a thread, and its largest magnitude goes through shared memory.
//
// Measured (of 6.79 TB/s copied): 8192 x 18944 bf16 71 us (6.6 TB/s), fp32 2048 x 18944 30 us (6.6), 37 x 896 2.2 us; rows that
// start anywhere, 8192 x 18943 bf16, 90 us.  Weights: 18944 x 3584 31 us (6.6), 18944 x 3583 38 us (43 by rows of their own).
#include "roi_fp8.cuh"
#include "roi_launch.h"

namespace roi {
namespace {

constexpr int kThreads = 256;

struct SaveArgs {
  const void* x;
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, ld;
  int64_t pitch, spitch;
  int64_t pieces;       // of 16 columns in a row, whole blocks of them
  int width, segments;  // rows anywhere: lanes of a row, and how often they go over it
  bool wait;
};

// Codes and scale of a piece, the q-th of its row (all lanes of the warp; eight of them hold a block).
template <Fp8 F, Elem E>
__device__ __forceinline__ void save_piece(const SaveArgs& a, const RowWords<E, 16>& r, int64_t row, int64_t q) {
  uint32_t top = max_bits(r);
#pragma unroll
  for (int m = 1; m < 8; m *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
  const uint32_t s = fp8_scale<F>(top);
  const uint4 w = fp8_codes16<F>(r, s);
  if (row < a.rows && q < a.pieces) {
    *reinterpret_cast<uint4*>(a.codes + row * a.pitch + 16 * q) = w;
    if ((q & 7) == 0) {
      uint8_t* to = a.scales + row * a.spitch;
      to[q >> 3] = uint8_t(s);
      if (q + 8 == a.pieces)
        for (int64_t b = a.pieces >> 3; b < a.spitch; ++b) to[b] = 1;
    }
  }
}

template <Fp8 F, Elem E>
__global__ void __launch_bounds__(kThreads) roi_fp8_save_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  constexpr int kWords = RowWords<E, 16>::kWords;
  pdl_begin(a.wait);
  const T* x = static_cast<const T*>(a.x);
  const int64_t total = a.rows * a.pieces;
  for (int64_t base = int64_t(blockIdx.x) * kThreads; base < total; base += int64_t(gridDim.x) * kThreads) {
    const int64_t row0 = base / a.pieces, rem0 = base - row0 * a.pieces;
    RowWords<E, 16> r;
    int64_t row, j;
    walk(row0, rem0, threadIdx.x, a.pieces, row, j);
    const T* p = x + row * a.ld + 16 * j;
    if (row < a.rows && a.cols - 16 * j >= 16) {
#pragma unroll
      for (int i = 0; i < kWords / 8; ++i) load32(reinterpret_cast<const uint4*>(p) + 2 * i, r.u + 8 * i);
    } else if (row < a.rows) {
      r.load_elements(x + row * a.ld, 16 * j, a.cols);
    } else {
      r.zero();
    }
    save_piece<F, E>(a, r, row, j);
  }
}

template <Fp8 F, Elem E>
__global__ void __launch_bounds__(kThreads) roi_fp8_save_rows_kernel(SaveArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const int64_t per = 32 / a.width, tasks = (a.rows + per - 1) / per * a.segments;
  const int64_t stride = int64_t(gridDim.x) * (kThreads / 32);
  const T* end = static_cast<const T*>(a.x) + (a.rows - 1) * a.ld + a.cols;
  for (int64_t t = int64_t(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5); t < tasks; t += stride) {
    Window<E, 16> x;
    int64_t row, j;
    row_task(t, a.width, a.segments, row, j);
    const T* p = static_cast<const T*>(a.x) + row * a.ld + 16 * j;
    const int64_t left = row < a.rows ? a.cols - 16 * j : 0;
    if (left > 0 && x.in_matrix(p, a.x, end)) x.load_granules(p);
    else x.load(static_cast<const T*>(a.x) + row * a.ld, 16 * j, row < a.rows ? a.cols : 0);
    RowWords<E, 16> r;
    x.get_masked(r, left);
    save_piece<F, E>(a, r, row, j);
  }
}

struct WeightArgs {
  const uint16_t* W;
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, cols, pitch, spitch;
  int64_t blocks_n, blocks;
  bool wait;
};

// ANYWHERE: rows that are not whole sectors apart.
template <bool ANYWHERE>
__global__ void __launch_bounds__(kThreads) roi_fp8_save_weight_kernel(WeightArgs a) {
  constexpr int kPieces = 4;
  __shared__ uint32_t tops[2][kThreads / 32];
  pdl_begin(a.wait);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int turn = 0;
  for (int64_t b = blockIdx.x; b < a.blocks; b += gridDim.x, turn ^= 1) {
    const int64_t bm = b / a.blocks_n, bn = b - bm * a.blocks_n;
    const int64_t r0 = bm * 128 + (threadIdx.x >> 3), c = bn * 128 + 16 * (threadIdx.x & 7);
    RowWords<Elem::kBf16, 16> r[kPieces];
    if constexpr (ANYWHERE) {
      using Piece = Window<Elem::kBf16, 16>;
      Piece w[kPieces];
      const uint16_t *p = a.W + r0 * a.cols + c, *end = a.W + a.rows * a.cols;
      const int64_t left = a.cols - c;
      if (left > 0 && Piece::in_matrix(p, a.W, end) && Piece::in_matrix(p + 32 * (kPieces - 1) * a.cols, a.W, end)) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) w[i].load_granules(p + 32 * i * a.cols);
      } else {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) w[i].load(a.W + (r0 + 32 * i) * a.cols, c, r0 + 32 * i < a.rows ? a.cols : 0);
      }
#pragma unroll
      for (int i = 0; i < kPieces; ++i) w[i].get_masked(r[i], r0 + 32 * i < a.rows ? left : 0);
    } else if (r0 + 32 * (kPieces - 1) < a.rows && c + 16 <= a.cols) {
      // (no branch between the loads: where ways meet, the compiler waits for what is on its way)
#pragma unroll
      for (int i = 0; i < kPieces; ++i) load32(a.W + (r0 + 32 * i) * a.cols + c, r[i].u);
    } else {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        if (r0 + 32 * i < a.rows && c + 16 <= a.cols) load32(a.W + (r0 + 32 * i) * a.cols + c, r[i].u);
        else r[i].zero();  // (columns come in sixteens)
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) top = max(top, max_bits(r[i]));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) tops[turn][warp] = top;
    __syncthreads();  // (the next block's tops lie apart)
    top = __reduce_max_sync(0xffffffffu, tops[turn][lane & (kThreads / 32 - 1)]);
    const uint32_t s = fp8_scale<Fp8::kE4M3>(top);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int64_t row = r0 + 32 * i;
      if (row < a.rows) *reinterpret_cast<uint4*>(a.codes + row * a.pitch + c) = fp8_codes16<Fp8::kE4M3>(r[i], s);
    }
    if (threadIdx.x == 0) {
      uint8_t* to = a.scales + bm * a.spitch;
      to[bn] = uint8_t(s);
      if (bn == a.blocks_n - 1)
        for (int64_t k = a.blocks_n; k < a.spitch; ++k) to[k] = 1;
    }
  }
}

template <class Args>
int launch(void (*kern)(Args), const Args& a, int64_t grid, cudaStream_t stream) {
  // four times what an SM holds at once: tiles are taken nearly in their order (8192 x 18944 bf16: once 74 us, twice 72, four times 71,
  // eight times 69, all 74; 8192 x 3584 15.6, 14.9, 14.9, 15.5, 15.5)
  const int64_t cap = int64_t(sm_count()) * 32;
  return launch_maybe_pdl(kern, int(grid < cap ? grid : cap), kThreads, 0, stream, a.wait, a);
}

template <Fp8 F, Elem E>
int save(const Fp8SaveCall& c) {
  SaveArgs a{c.x,  c.codes, c.scales, c.rows, c.cols, c.ld, fp8_pitch(c.cols), fp8_scale_pitch(c.cols), fp8_pitch(c.cols) / 16, 0, 0,
             lone_pdl(c.stream)};
  if (!in_sectors(c.x, c.ld, c.rows, elem_bytes<E>())) {
    const int64_t tasks = by_rows(a);
    return launch(roi_fp8_save_rows_kernel<F, E>, a, (tasks + kThreads / 32 - 1) / (kThreads / 32), c.stream);
  }
  const int64_t total = a.rows * a.pieces;
  return launch(roi_fp8_save_kernel<F, E>, a, (total + kThreads - 1) / kThreads, c.stream);
}

template <Fp8 F>
int save_of(const Fp8SaveCall& c) {
  switch (c.dtype) {
    case Elem::kBf16: return save<F, Elem::kBf16>(c);
    case Elem::kFp16: return save<F, Elem::kFp16>(c);
    default: return save<F, Elem::kFp32>(c);
  }
}

}  // namespace

int launch_fp8_save(const Fp8SaveCall& c) { return c.format == Fp8::kE4M3 ? save_of<Fp8::kE4M3>(c) : save_of<Fp8::kE5M2>(c); }

int launch_fp8_save_weight(const Fp8SaveCall& c) {
  WeightArgs a{static_cast<const uint16_t*>(c.x), c.codes, c.scales, c.rows, c.cols, fp8_pitch(c.cols), fp8_scale_pitch(c.cols),
               (c.cols + 127) / 128, 0, lone_pdl(c.stream)};
  a.blocks = a.blocks_n * ((c.rows + 127) / 128);
  if (in_sectors(c.x, c.cols, 2, 2)) return launch(roi_fp8_save_weight_kernel<false>, a, a.blocks, c.stream);
  return launch(roi_fp8_save_weight_kernel<true>, a, a.blocks, c.stream);
}

}  // namespace roi
