// Layer norm and RMS norm, forward and backward, with the reduction of the gradients of
// weight and bias, and with activation checkpoints in 8 bits as the forward's further outputs
// and as the backward's input.
//
//   mu = mean(x) (layer norm; 0 for the RMS norm), r = 1 / sqrt(mean((x - mu)^2) + eps)
//   xh = (x - mu) r,  y = xh gamma + beta
//   a = dy gamma,  dx = r (a - mean(a) [layer norm] - xh mean(a xh))
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// Bound by memory (one read of every input, one write of every output).  Everything is
// computed in 32 bits, two columns an instruction; outputs are rounded once.
//
// A team of warps takes a row at a time.  Its rows come through a ring in shared memory, which a warp of
// its own fills by bulk copies far ahead of their use, so that threads hold no rows on their way: an SM
// keeps some 200 KB in flight.  A lane has runs of 8 consecutive columns; its warp's runs follow one
// another.  gamma and beta lie in shared memory as fp32, for all rows of a CTA.
//  - forward: the row in registers as it was read (RUN pieces a lane), so the squares are summed around
//    the mean already known;
//  - backward: a thread has the same columns of every row it sees, so that the sums of dgamma and dbeta
//    stay in its registers.  The teams' and then the CTAs' sums are added in a fixed order (through
//    shared memory, and by a second launch): no atomics, the same bits every time.
// Rows that start anywhere are copied by the 16-byte granules around them (those at the matrix's own
// ends byte by byte) and shifted as they are read; they are written as roi_rows.cuh does.  Rows so wide that
// two of them do not fit go to kernels that read them again for each step.
//
// Measured, 8192 x 3584 bf16 (of 6.79 TB/s copied): RMS norm forward 22.8 us (5.2 TB/s), with y's checkpoint
// 35.8, layer norm 31.4; RMS norm backward 39.4 us from x (4.5 TB/s), 42.0 from its checkpoint, 7 of which are the
// sums' (their places in memory and the second launch), layer norm 45.2 and 49.0.  fp32: RMS norm 44.3 (5.3 TB/s) forward,
// 67.4 and 55.8 backward; layer norm 51.9, 68.0 and 59.4.  With rows loaded
// by the threads that use them: RMS norm forward 48 us, layer norm 46, RMS norm backward from the checkpoint 52.
// The forward with y's checkpoint issues in 57 % of the cycles and the backward in 59 %, with 20 to 22 warps an SM, which
// wait for instructions before (`wait`), shared memory and their teams' meetings.  Rows that start anywhere (8192
// x 3583) take 1.5 to 1.8 times as long, for the shifts and, in the backward, for registers (roi_norm_bwd_kernel).
// Rows too wide for a ring, 2048 x 16384: backward 186 to 243 us, 6 to 10 times its floor, three passes over everything.
#include <atomic>

#include "roi_block8.cuh"
#include "roi_extent.h"
#include "roi_launch.h"
#include "roi_rows.cuh"

namespace roi {
namespace {

// The division of a launch's rows among teams, and of shared memory.
struct Shape {
  int nt;         // threads of a team
  int teams;      // of a CTA
  int fillers;    // warps that fill the rings, after the teams
  int depth;      // rows of a team's ring, 0 where two do not fit
  int grid;
  uint32_t stage; // bytes of a row in the ring
  uint32_t params; // bytes of gamma (and beta) before the rings
  size_t smem;
};

struct FwdArgs {
  const void* x;
  void* y;
  const void* gamma;
  const void* beta;
  float* mean;
  float* rstd;
  int8_t* xcodes;
  uint8_t* xscales;
  int8_t* ycodes;
  uint8_t* yscales;
  int64_t rows, cols, ldx, ldy;
  int64_t pitch, spitch;
  Shape shape;
  unsigned int* status;
  float eps;
  bool params32;  // gamma and beta in fp32, else in the type of x
  bool wait;
};

struct BwdArgs {
  const void* dy;
  const void* x;
  const int8_t* codes;
  const uint8_t* scales;
  const void* gamma;
  const float* mean;
  const float* rstd;
  void* dx;
  float* dgamma;
  float* dbeta;
  float* part;  // [gridDim][1 or 2][part_cols] sums of a CTA's rows
  int64_t rows, cols, lddy, ldx, lddx;
  int64_t pitch, spitch, part_cols;
  Shape shape;
  unsigned int* status;
  bool params32;
  bool wait;
};

template <Elem E>
__device__ __forceinline__ float param1(const void* p, bool p32, int64_t c, float none) {
  using T = typename ElemType<E>::T;
  return p == nullptr ? none : p32 ? __ldg(static_cast<const float*>(p) + c) : to_f32<E>(__ldg(static_cast<const T*>(p) + c));
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// Eight columns in pairs.
struct Piece {
  F2 v[4];
};
__device__ __forceinline__ Piece pairs(const float (&f)[8]) {
  Piece p;
#pragma unroll
  for (int k = 0; k < 4; ++k) p.v[k] = f2(f[2 * k], f[2 * k + 1]);
  return p;
}
__device__ __forceinline__ float total(F2 s) { return lo(s) + hi(s); }
// gamma or beta as fp32 in shared memory (the whole CTA; `n` is cols rounded up to a warp's pieces),
// `none` where it is not given and past the last column.  Each 256 columns lie as the first four of
// every lane's eight, then the others, so that a warp's loads meet on no bank.
template <Elem E>
__device__ __forceinline__ void stage_param(float* to, const void* p, bool p32, int cols, int n, float none) {
  for (int c = threadIdx.x; c < n; c += blockDim.x)
    to[(c & ~255) + (c & 4) * 32 + ((c & 255) >> 3) * 4 + (c & 3)] = c < cols ? param1<E>(p, p32, c, none) : none;
}
// Of the lane whose first column is c = 256 q + 8 lane.
__device__ __forceinline__ Piece param(const float* p, int c) {
  const float* at = p + (c & ~255) + ((c & 255) >> 1);
  const float4 a = *reinterpret_cast<const float4*>(at), b = *reinterpret_cast<const float4*>(at + 128);
  Piece q;
  q.v[0] = f2(a.x, a.y), q.v[1] = f2(a.z, a.w), q.v[2] = f2(b.x, b.y), q.v[3] = f2(b.z, b.w);
  return q;
}

// ---- a row in the ring ----
// A matrix row's place: `m` bytes after the stage's start, as after a 16-byte boundary in memory.
template <bool ANY>
__device__ __forceinline__ uint32_t row_shift(const void* row) {
  return ANY ? uint32_t(reinterpret_cast<uintptr_t>(row) & 15u) : 0u;
}
__device__ __forceinline__ void copy_row(const Extent& x, uint8_t* st, uint64_t* bar) {
  if (x.bytes() > 0) bulk_g2s(st + x.offset(), reinterpret_cast<const void*>(x.from), x.bytes(), bar);
}
__device__ __forceinline__ Bounds bounds(const void* p, int64_t rows, int64_t pitch, uint32_t width) {
  const uintptr_t begin = reinterpret_cast<uintptr_t>(p);
  return {begin, begin + uintptr_t((rows - 1) * pitch) + width};
}
// Zeros past the last column.
template <Elem E>
__device__ __forceinline__ void clear_past(RowWords<E, 8>& r, int c, int cols) {
#pragma unroll
  for (int i = 0; i < RowWords<E, 8>::kWords; ++i) {
    const int k = E == Elem::kFp32 ? i : 2 * i;  // the word's first column
    if (c + k >= cols) r.u[i] = 0;
    else if (E != Elem::kFp32 && c + k + 1 >= cols) r.u[i] &= 0xffffu;
  }
}
// Columns c .. c + 7 of a row whose stage starts at st (zeros past the last column).
template <Elem E, bool ANY>
__device__ __forceinline__ RowWords<E, 8> read_row(const uint8_t* st, uint32_t m, int c, int cols) {
  constexpr int W = RowWords<E, 8>::kWords;
  RowWords<E, 8> r;
  if (c >= cols) {
    r.zero();
    return r;
  }
  const uint4* q = reinterpret_cast<const uint4*>(st + c * elem_bytes<E>());
  uint32_t w[ANY ? W + 4 : W];
#pragma unroll
  for (int i = 0; i < (ANY ? W / 4 + 1 : W / 4); ++i) {
    const uint4 v = q[i];
    w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
  }
  if constexpr (ANY) {
    shift_words<W>(w, m, r.u);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) r.u[i] = w[i];
  }
  // (a whole number of granules is one of pieces in 16 bits, and of half pieces in 32)
  if ((ANY || E == Elem::kFp32) && c + 8 > cols) clear_past<E>(r, c, cols);
  return r;
}

// One piece's part of a checkpoint row (all lanes of the warp call it; values past the last column
// are 0): a block is four neighbouring lanes.
template <Elem E>
__device__ __forceinline__ void save_piece(int8_t* codes, uint8_t* scales, int64_t pitch, int64_t spitch, int c, const RowWords<E, 8>& r) {
  uint32_t top = max_bits(r);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  const uint32_t s = block8_scale(top);
  uint32_t w[2];
  block8_codes(r, top, s, w);
  if (c < pitch) *reinterpret_cast<uint2*>(codes + c) = make_uint2(w[0], w[1]);
  if (c % 32 == 0 && c / 32 < spitch) scales[c / 32] = uint8_t(s);
}

__device__ __forceinline__ void team_sync(int team, int nt) {
  if (nt == 32) {
    __syncwarp();
  } else {
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(nt) : "memory");
  }
}

// Pieces a lane of the forward holds, and the most threads of a CTA: what keeps the registers that a
// thread then has from spilling.
template <Elem E>
constexpr int kRun = E == Elem::kFp32 ? 2 : 4;
template <bool LAYER, bool ANY>
constexpr int kFwdThreads = LAYER && ANY ? 640 : 768;
constexpr int kThreads = 1024, kMostTeams = 32, kMostNamed = 15, kMostDepth = 8;
// Barriers, slots and lost rows of the teams.
struct TeamState {
  uint64_t full[kMostTeams][kMostDepth];   // the row has landed
  uint64_t empty[kMostTeams][kMostDepth];  // every warp has read it
  float slots[3][kThreads / 32][2];  // a set is written again two meetings later
  // Whether the row of a turn did not land for a warp of the team, written before the row's meeting and read
  // after it, so that the team breaks off together.  (A warp that has gone on to its next row may write while the others
  // still read for this one; with one flag for all rows they would part, and one part would wait for ever.)
  int lost[3][kMostTeams];
};
// The barriers of the rings (the whole CTA).
__device__ __forceinline__ void init_teams(TeamState& ts, const Shape& s) {
  for (int i = threadIdx.x; i < s.teams * s.depth; i += blockDim.x) {
    mbar_init(&ts.full[i / s.depth][i % s.depth], 1);
    mbar_init(&ts.empty[i / s.depth][i % s.depth], s.nt / 32);
  }
  for (int i = threadIdx.x; i < 3 * kMostTeams; i += blockDim.x) ts.lost[i / kMostTeams][i % kMostTeams] = 0;
  fence_mbar_init();
  __syncthreads();
}
// Whether a row has landed, one answer for the warp.
__device__ __forceinline__ bool row_landed(uint64_t* full, uint32_t parity, uint64_t lim) {
  return __all_sync(0xffffffffu, mbar_wait_ring(full, parity, lim));
}
// A warp that fills rings, a lane a team: `copy(team, stage, row, barrier)` sends a row's copies off.  It
// gives up when no stage has become free for `lim`; what was sent off lands before it leaves, and
// before what comes after the rings takes their place.  (A copy takes a warp some 70 cycles to send
// off, so the many teams of narrow rows have several.)
template <class Copy>
__device__ __forceinline__ void fill_rings(TeamState& ts, const Shape& s, int64_t rows, uint64_t lim, unsigned int* status, Copy copy) {
  const int team = int(threadIdx.x & 31) * s.fillers + (int(threadIdx.x) - s.teams * s.nt) / 32;
  const int64_t all = int64_t(gridDim.x) * s.teams;
  int64_t row = team < s.teams ? int64_t(blockIdx.x) * s.teams + team : rows;
  int at = 0, k = 0;
  uint32_t pass = 0;  // parity of the phase that frees the stage
  uint64_t since = 0;
  while (__any_sync(0xffffffffu, row < rows)) {
    const bool go = row < rows && (k < s.depth || mbar_test_wait(&ts.empty[team][at], pass));
    if (go) {
      copy(team, at, row, &ts.full[team][at]);
      row += all;
      if (k++ >= s.depth && at == s.depth - 1) pass ^= 1u;
      at = at == s.depth - 1 ? 0 : at + 1;
    }
    if (__any_sync(0xffffffffu, go)) {
      since = 0;
    } else if (since == 0) {
      since = global_timer_ns();
    } else if (global_timer_ns() - since > lim) {
      break;
    }
  }
  if (__any_sync(0xffffffffu, row < rows) && (threadIdx.x & 31) == 0) atomicOr(status, kStatusTimeout);
  // What was sent off lands, whether or not a team gives up on it, now or later (a stage's phases end one after
  // another, so the last rows of the ring stand for all).
  for (int q = k > s.depth ? k - s.depth : 0; q < k; ++q) mbar_wait_bounded(&ts.full[team][q % s.depth], uint32_t(q / s.depth) & 1u);
  __syncwarp();
}

// RUN pieces a lane.
template <Elem E, bool LAYER, bool ANY, int RUN>
__global__ void __launch_bounds__(RUN == 1 ? kThreads : kFwdThreads<LAYER, ANY>) roi_norm_fwd_kernel(FwdArgs a) {
  using T = typename ElemType<E>::T;
  extern __shared__ __align__(128) uint8_t smem[];  // gamma, beta; [teams][depth][stage]
  __shared__ TeamState ts;
  const int nt = a.shape.nt, team = threadIdx.x / nt, t = threadIdx.x - team * nt;
  const int warps = nt >> 5, warp0 = team * warps, warp = t >> 5, lane = t & 31, depth = a.shape.depth;
  const int cols = int(a.cols), padded = (cols + 255) / 256 * 256;
  init_teams(ts, a.shape);
  pdl_begin(a.wait);
  const uint64_t lim = ring_wait_limit(a.status);
  float* gamma = reinterpret_cast<float*>(smem);
  float* beta = gamma + padded;
  stage_param<E>(gamma, a.gamma, a.params32, cols, padded, 1.0f);
  if constexpr (LAYER) stage_param<E>(beta, a.beta, a.params32, cols, padded, 0.0f);
  __syncthreads();
  if (team >= a.shape.teams) {
    const uint32_t row_bytes = uint32_t(cols) * elem_bytes<E>();
    const Bounds whole = bounds(a.x, a.rows, a.ldx * elem_bytes<E>(), row_bytes);
    fill_rings(ts, a.shape, a.rows, lim, a.status, [&](int of, int stage, int64_t row, uint64_t* bar) {
      uint8_t* st = smem + a.shape.params + (size_t(of) * depth + stage) * a.shape.stage;
      const Extent x(static_cast<const T*>(a.x) + row * a.ldx, row_bytes, ANY, whole);
      if (ANY && x.cut()) x.ends(st);
      mbar_arrive_expect_tx(bar, x.bytes());
      copy_row(x, st, bar);
    });
    return;
  }
  const int64_t all = int64_t(gridDim.x) * a.shape.teams, row0 = int64_t(blockIdx.x) * a.shape.teams + team;
  const uint8_t* ring = smem + a.shape.params + size_t(team) * depth * a.shape.stage;
  const int base = warp * RUN * 256, c0 = base + lane * 8;  // the warp's and the lane's first column
  // columns that the pieces go up to: the row's, and a checkpoint's padding
  const int end = a.xcodes != nullptr || a.ycodes != nullptr ? int(a.spitch) * 32 : cols;
  const float inv_cols = 1.0f / float(cols);
  int at = 0, turn = 0;
  uint32_t pass = 0;
  // sum over the team, the same bits in every thread
  auto meet = [&](float v) {
    v = warp_sum(v);
    if (nt > 32 && lane == 0) ts.slots[turn][warp0 + warp][0] = v;
    team_sync(team, nt);
    if (nt > 32) v = warp_sum(lane < warps ? ts.slots[turn][warp0 + lane][0] : 0.0f);
    turn = turn == 2 ? 0 : turn + 1;
    return v;
  };
  for (int64_t row = row0; row < a.rows; row += all) {
    const bool landed = row_landed(&ts.full[team][at], pass, lim);
    const int of = turn;
    if (!landed) ts.lost[of][team] = 1;
    const uint8_t* st = ring + at * a.shape.stage;
    const uint32_t m = row_shift<ANY>(static_cast<const T*>(a.x) + row * a.ldx);
    RowWords<E, 8> x[RUN];
    F2 sum = f2(0.0f);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      x[i] = read_row<E, ANY>(st, m, c0 + 256 * i, cols);
      if constexpr (LAYER) {
        float f[8];
        x[i].get(f);
        const Piece v = pairs(f);
        sum = sum + ((v.v[0] + v.v[1]) + (v.v[2] + v.v[3]));
      }
    }
    // (the stage of a row that did not land stays taken: its copy may still be on its way)
    __syncwarp();
    if (landed && lane == 0) mbar_arrive(&ts.empty[team][at]);
    float mean = 0.0f;
    if constexpr (LAYER) mean = meet(total(sum)) * inv_cols;
    const F2 minus = f2(-mean);
    F2 squares = f2(0.0f);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      if (base + 256 * i >= cols) break;
      float f[8];
      x[i].get(f);
      Piece v = pairs(f);
      if constexpr (LAYER) {
        // (columns past the last hold 0, which is not at distance 0 from the mean)
        const int left = cols - (c0 + 256 * i);
#pragma unroll
        for (int k = 0; k < 4; ++k) v.v[k] = v.v[k] + minus;
        if (left < 8) {
#pragma unroll
          for (int k = 0; k < 4; ++k) v.v[k] = f2(2 * k < left ? lo(v.v[k]) : 0.0f, 2 * k + 1 < left ? hi(v.v[k]) : 0.0f);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) squares = vfma(v.v[k], v.v[k], squares);
    }
    const float rstd = 1.0f / sqrtf(meet(total(squares)) * inv_cols + a.eps);
    if (ts.lost[of][team] != 0) {  // (the whole team)
      if (t == 0) atomicOr(a.status, kStatusTimeout);
      break;
    }
    if (t == 0) {
      if (LAYER && a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    if (a.xcodes != nullptr) {
#pragma unroll
      for (int i = 0; i < RUN; ++i)
        if (base + 256 * i < end) save_piece<E>(a.xcodes + row * a.pitch, a.xscales + row * a.spitch, a.pitch, a.spitch, c0 + 256 * i, x[i]);
    }
    T* to = static_cast<T*>(a.y) + row * a.ldy;
    const F2 r2 = f2(rstd);
#pragma unroll
    for (int i = 0; i < RUN; ++i) {
      if (base + 256 * i >= cols) break;
      const int c = c0 + 256 * i;
      float f[8];
      x[i].get(f);
      Piece v = pairs(f);
      const Piece g = param(gamma, c);
      Piece b;
      if constexpr (LAYER) b = param(beta, c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (LAYER) v.v[k] = vfma((v.v[k] + minus) * r2, g.v[k], b.v[k]);
        else v.v[k] = v.v[k] * r2 * g.v[k];
        f[2 * k] = lo(v.v[k]), f[2 * k + 1] = hi(v.v[k]);
      }
      RowWords<E, 8> y;
      y.set(f);
      store_row<E, 8, !ANY>(to, c, cols, y, 32, i > 0 ? &x[i - 1] : nullptr, i + 1 < RUN && base + 256 * (i + 1) < cols);
      x[i] = y;
    }
    if (a.ycodes != nullptr) {
#pragma unroll
      for (int i = 0; i < RUN; ++i) {
        const int c = c0 + 256 * i;
        if (base + 256 * i >= end) break;
        if (base + 256 * i >= cols) x[i].zero();
        // (a bias or a NaN may stand past the last column)
        if (c + 8 > cols) clear_past<E>(x[i], c, cols);
        save_piece<E>(a.ycodes + row * a.pitch, a.yscales + row * a.spitch, a.pitch, a.spitch, c, x[i]);
      }
    }
    if (++at == depth) at = 0, pass ^= 1u;
  }
}

// First column of run i of a team's thread t, with NP runs a thread.
template <int NP>
__device__ __forceinline__ int column(int i, int t) { return ((t >> 5) * NP + i) * 256 + (t & 31) * 8; }

// What a thread keeps of dy until dx is written: dy as it was read where that is half the registers (16
// bits) and they are short, else its product with gamma.  bf16, x from memory: RMS norm 8192 x 3584 39.4 us
// with dy in 768 threads (46 in 640) and 50 with the product in 640; layer norm 8192 x 8192 98 us with dy
// and 130 with the product in 640; 8192 x 3584 46 us with the product and 53 with dy, both in 512.
template <Elem E, bool LAYER, int THREADS>
constexpr bool kKeepDy = E != Elem::kFp32 && (!LAYER || THREADS > 512);

// THREADS: 1024 for one piece; for two pieces what leaves them their registers where rows are whole granules (spills of 0
// to 28 bytes).  These numbers were chosen by such rows; rows that start anywhere have the same and spill 20 to 300 bytes (RMS
// norm in 16 bits 116, layer norm in 640 threads 140 to 172), and so does one piece, up to 124.  Rows too wide for
// these take two pieces in 1024 threads (RMS norm in 16 bits from 11777 columns on, layer norm and fp32 from 9729) and spill
// 152 to 584 bytes: RMS norm 4096 x 12288 bf16 94 us from x, layer norm 152, against 83 and 99 at 8192 x 8192.
template <Elem E, bool LAYER, bool CKPT, bool ANY, int NP, int THREADS>
__global__ void __launch_bounds__(THREADS) roi_norm_bwd_kernel(BwdArgs a) {
  using T = typename ElemType<E>::T;
  extern __shared__ __align__(128) uint8_t smem[];  // gamma; [teams][depth][stage]; at the end the teams' sums
  __shared__ TeamState ts;
  const int nt = a.shape.nt, team = threadIdx.x / nt, t = threadIdx.x - team * nt;
  const int warps = nt >> 5, warp0 = team * warps, warp = t >> 5, lane = t & 31, depth = a.shape.depth;
  const int cols = int(a.cols), padded = (cols + 255) / 256 * 256;
  init_teams(ts, a.shape);
  pdl_begin(a.wait);
  const uint64_t lim = ring_wait_limit(a.status);
  const uint32_t room = (uint32_t(cols + 7) / 8 * 8) * elem_bytes<E>() + (ANY ? 32u : 0u);  // of dy, before x
  float* gamma = reinterpret_cast<float*>(smem);
  stage_param<E>(gamma, a.gamma, a.params32, cols, padded, 1.0f);
  __syncthreads();
  const int teams = a.shape.teams;
  const bool sums_wanted = a.dgamma != nullptr || a.dbeta != nullptr;
  if (team >= teams) {
    const uint32_t row_bytes = uint32_t(cols) * elem_bytes<E>();
    const Bounds all_dy = bounds(a.dy, a.rows, a.lddy * elem_bytes<E>(), row_bytes);
    const Bounds all_x = CKPT ? bounds(a.scales, a.rows, a.spitch, uint32_t(a.spitch)) : bounds(a.x, a.rows, a.ldx * elem_bytes<E>(), row_bytes);
    fill_rings(ts, a.shape, a.rows, lim, a.status, [&](int of, int stage, int64_t row, uint64_t* bar) {
      uint8_t* st = smem + a.shape.params + (size_t(of) * depth + stage) * a.shape.stage;
      const Extent dy(static_cast<const T*>(a.dy) + row * a.lddy, row_bytes, ANY, all_dy);
      if (ANY && dy.cut()) dy.ends(st);
      if constexpr (CKPT) {
        const Extent scales(a.scales + row * a.spitch, uint32_t(a.spitch), true, all_x);
        if (scales.cut()) scales.ends(st + room + a.pitch);
        mbar_arrive_expect_tx(bar, dy.bytes() + uint32_t(a.pitch) + scales.bytes());
        bulk_g2s(st + room, a.codes + row * a.pitch, uint32_t(a.pitch), bar);
        copy_row(scales, st + room + a.pitch, bar);
      } else {
        const Extent x(static_cast<const T*>(a.x) + row * a.ldx, row_bytes, ANY, all_x);
        if (ANY && x.cut()) x.ends(st + room);
        mbar_arrive_expect_tx(bar, dy.bytes() + x.bytes());
        copy_row(x, st + room, bar);
      }
      copy_row(dy, st, bar);
    });
    // the barriers of the others' sums
    if (sums_wanted) {
      __syncthreads();
      for (int q = 0; q < teams && teams > 1; ++q) __syncthreads();
    }
    return;
  }
  const float inv_cols = 1.0f / float(cols);
  const int64_t all = int64_t(gridDim.x) * teams, row0 = int64_t(blockIdx.x) * teams + team;
  const uint8_t* ring = smem + a.shape.params + size_t(team) * depth * a.shape.stage;

  Piece dg[NP], db[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) dg[i].v[k] = db[i].v[k] = f2(0.0f);
  float next_mean = LAYER && row0 < a.rows ? __ldg(a.mean + row0) : 0.0f, next_rstd = row0 < a.rows ? __ldg(a.rstd + row0) : 0.0f;
  int at = 0, turn = 0;
  uint32_t pass = 0;
  T* to = static_cast<T*>(a.dx) + row0 * a.lddx;
  for (int64_t row = row0; row < a.rows; row += all) {
    const float rstd = next_rstd;
    const F2 r2 = f2(rstd), minus = f2(-next_mean);
    const int64_t after = row + all;
    if (after < a.rows) {
      next_rstd = __ldg(a.rstd + after);
      if constexpr (LAYER) next_mean = __ldg(a.mean + after);
    }
    const bool landed = row_landed(&ts.full[team][at], pass, lim);
    if (!landed) ts.lost[turn][team] = 1;
    const uint8_t* st = ring + at * a.shape.stage;
    const uint32_t m = row_shift<ANY>(static_cast<const T*>(a.dy) + row * a.lddy);
    const uint32_t ms = CKPT ? row_shift<true>(a.scales + row * a.spitch) : 0u;
    const uint32_t mx = CKPT ? 0u : row_shift<ANY>(static_cast<const T*>(a.x) + row * a.ldx);
    // this thread's columns: dy, and xh (past the last column dy is 0)
    constexpr bool KEEP = kKeepDy<E, LAYER, THREADS>;
    auto get = [&](int i, RowWords<E, 8>& dy, Piece& xh) {
      const int c = column<NP>(i, t);
      float f[8];
      dy = read_row<E, ANY>(st, m, c, cols);
      if constexpr (CKPT) {
        uint2 w = make_uint2(0, 0);
        float step = 0.0f;
        if (c < int(a.pitch)) {
          w = *reinterpret_cast<const uint2*>(st + room + c);
          step = block8_step(st[room + a.pitch + ms + c / 32]);
        }
        block8_pairs(w.x, step, xh.v[0], xh.v[1]);
        block8_pairs(w.y, step, xh.v[2], xh.v[3]);
      } else {
        read_row<E, ANY>(st + room, mx, c, cols).get(f);
        xh = pairs(f);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (LAYER) xh.v[k] = xh.v[k] + minus;
        xh.v[k] = xh.v[k] * r2;
      }
    };
    F2 s1 = f2(0.0f), s2 = f2(0.0f);
    RowWords<E, 8> raw[KEEP ? NP : 1];
    Piece w[KEEP ? 1 : NP], xh[NP];  // dy gamma, and the normalised input
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (column<NP>(i, t) - lane * 8 >= cols) break;  // (the whole warp)
      RowWords<E, 8> words;
      get(i, words, xh[i]);
      float f[8];
      words.get(f);
      const Piece g = param(gamma, column<NP>(i, t)), dy = pairs(f);
      Piece p;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p.v[k] = dy.v[k] * g.v[k];
        dg[i].v[k] = vfma(dy.v[k], xh[i].v[k], dg[i].v[k]);
        s1 = vfma(p.v[k], xh[i].v[k], s1);
        if constexpr (LAYER) {
          db[i].v[k] = db[i].v[k] + dy.v[k];
          s2 = s2 + p.v[k];
        }
      }
      if constexpr (KEEP) raw[i] = words;
      else w[i] = p;
    }
    // (the stage of a row that did not land stays taken: its copy may still be on its way)
    __syncwarp();
    if (landed && lane == 0) mbar_arrive(&ts.empty[team][at]);
    float c1 = warp_sum(total(s1)), c2 = LAYER ? warp_sum(total(s2)) : 0.0f;
    if (nt > 32 && lane == 0) {
      ts.slots[turn][warp0 + warp][0] = c1;
      if constexpr (LAYER) ts.slots[turn][warp0 + warp][1] = c2;
    }
    team_sync(team, nt);
    if (ts.lost[turn][team] != 0) {  // (the whole team)
      if (t == 0) atomicOr(a.status, kStatusTimeout);
      break;
    }
    if (nt > 32) {
      c1 = warp_sum(lane < warps ? ts.slots[turn][warp0 + lane][0] : 0.0f);
      if constexpr (LAYER) c2 = warp_sum(lane < warps ? ts.slots[turn][warp0 + lane][1] : 0.0f);
    }
    turn = turn == 2 ? 0 : turn + 1;
    // dx = rstd a - rstd mean(a) - xh (rstd mean(a xh))
    const F2 k1 = f2(-(c1 * inv_cols) * rstd), k2 = f2(-(c2 * inv_cols) * rstd);
    RowWords<E, 8> before;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int c = column<NP>(i, t);
      if (c - lane * 8 >= cols) break;
      float o[8];
      Piece p;
      if constexpr (KEEP) {
        raw[i].get(o);
        const Piece g = param(gamma, c);
        p = pairs(o);
#pragma unroll
        for (int k = 0; k < 4; ++k) p.v[k] = p.v[k] * g.v[k];
      } else {
        p = w[i];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const F2 d = vfma(xh[i].v[k], k1, LAYER ? vfma(p.v[k], r2, k2) : p.v[k] * r2);
        o[2 * k] = lo(d), o[2 * k + 1] = hi(d);
      }
      RowWords<E, 8> d;
      d.set(o);
      store_row<E, 8, !ANY>(to, c, cols, d, 32, i > 0 ? &before : nullptr, i + 1 < NP && column<NP>(i + 1, t) - lane * 8 < cols);
      if (ANY) before = d;
    }
    to += all * a.lddx;
    if (++at == depth) at = 0, pass ^= 1u;
  }
  if (!sums_wanted) return;
  __syncthreads();  // the rings are done with
  // the teams' sums in their order, then this CTA's to its place among the partial sums (the outputs
  // themselves where it is the only CTA)
  float* sums = reinterpret_cast<float*>(smem);  // [1 or 2][NP][8][nt]
  float* part = a.part + int64_t(blockIdx.x) * (LAYER ? 2 : 1) * a.part_cols;
  const bool only = gridDim.x == 1;
  float* to_g = only ? a.dgamma : part;
  float* to_b = only ? a.dbeta : part + a.part_cols;
  float g8[NP][8], b8[NP][8];
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      g8[i][k] = k % 2 == 0 ? lo(dg[i].v[k / 2]) : hi(dg[i].v[k / 2]);
      b8[i][k] = k % 2 == 0 ? lo(db[i].v[k / 2]) : hi(db[i].v[k / 2]);
    }
  for (int q = 0; q < teams && teams > 1; ++q) {
    if (q == team) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int s = (8 * i + k) * nt + t;
          if (q > 0) {
            g8[i][k] += sums[s];
            if constexpr (LAYER) b8[i][k] += sums[8 * NP * nt + s];
          }
          sums[s] = g8[i][k];
          if constexpr (LAYER) sums[8 * NP * nt + s] = b8[i][k];
        }
      }
    }
    __syncthreads();
  }
  if (team == teams - 1) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        const int c = column<NP>(i, t) + k;
        if (!only) {
          // (a partial row has whole fours)
          if (c < cols) *reinterpret_cast<float4*>(to_g + c) = make_float4(g8[i][k], g8[i][k + 1], g8[i][k + 2], g8[i][k + 3]);
          if (LAYER && c < cols) *reinterpret_cast<float4*>(to_b + c) = make_float4(b8[i][k], b8[i][k + 1], b8[i][k + 2], b8[i][k + 3]);
          continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (c + e < cols && to_g != nullptr) to_g[c + e] = g8[i][k + e];
          if (LAYER && c + e < cols && to_b != nullptr) to_b[c + e] = b8[i][k + e];
        }
      }
    }
  }
}

// 152 partial rows of 3584 columns: 2.2 MB, which a launch of 112 CTAs reads in one go of ten loads a thread.
constexpr int kSumSegments = 16;
// out[c] = the sum of the `parts` partial rows at c, in a fixed order: sixteen threads a column
// take every sixteenth row, and their sums are added in their order.  kinds: 1 (dgamma) or 2.
__global__ void __launch_bounds__(32 * kSumSegments) roi_norm_sum_kernel(const float* part, int parts, int kinds, int64_t part_cols, int64_t cols,
                                                           float* dgamma, float* dbeta) {
  __shared__ float sums[kSumSegments][33];
  pdl_begin(true);  // the partial sums of the launch before
  const int lane = threadIdx.x & 31, seg = threadIdx.x >> 5;
  const int64_t blocks = (cols + 31) / 32;
  const int64_t kind = blockIdx.x / blocks, c = (blockIdx.x - kind * blocks) * 32 + lane;
  float s = 0.0f;
  if (c < cols) {
    const float* p = part + kind * part_cols + c;
    const int64_t stride = kinds * part_cols;
#pragma unroll 10
    for (int q = seg; q < parts; q += kSumSegments) s += p[q * stride];
  }
  sums[seg][lane] = s;
  __syncthreads();
  if (seg == 0 && c < cols) {
    for (int q = 1; q < kSumSegments; ++q) s += sums[q][lane];
    float* out = kind == 0 ? dgamma : dbeta;
    if (out != nullptr) out[c] = s;
  }
}

// ---- rows too wide for a ring ----
// Sum over the CTA, the same bits in every thread.  Two sets of slots in turn: a set is written
// again only after the barrier of the sum in between.
__device__ __forceinline__ float cta_sum(float v, float (&slots)[2][32], int& turn) {
  v = warp_sum(v);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) slots[turn][warp] = v;
  __syncthreads();
  v = warp_sum(lane < int(blockDim.x >> 5) ? slots[turn][lane] : 0.0f);
  turn ^= 1;
  return v;
}

template <Elem E, bool LAYER>
__global__ void __launch_bounds__(kThreads) roi_norm_fwd_wide_kernel(FwdArgs a) {
  using T = typename ElemType<E>::T;
  __shared__ float slots[2][32];
  pdl_begin(a.wait);
  const int cols = int(a.cols), lane = threadIdx.x & 31;
  const int end = a.xcodes != nullptr || a.ycodes != nullptr ? int(a.spitch) * 32 : cols;
  const float inv_cols = 1.0f / float(cols);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    T* y = static_cast<T*>(a.y) + row * a.ldy;
    float mean = 0.0f;
    if constexpr (LAYER) {
      float s = 0.0f;
#pragma unroll 4
      for (int c = threadIdx.x; c < cols; c += blockDim.x) s += to_f32<E>(x[c]);
      mean = cta_sum(s, slots, turn) * inv_cols;
    }
    float s = 0.0f;
#pragma unroll 4
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
      const float d = to_f32<E>(x[c]) - mean;
      s = __fmaf_rn(d, d, s);
    }
    const float rstd = 1.0f / sqrtf(cta_sum(s, slots, turn) * inv_cols + a.eps);
    if (threadIdx.x == 0) {
      if (LAYER && a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    // a warp a block of 32 columns, a lane a column
    for (int c = threadIdx.x; c - lane < end; c += blockDim.x) {
      const float v = c < cols ? to_f32<E>(x[c]) : 0.0f;
      float o = 0.0f;
      if (c < cols) {
        const T r = from_f32<E>(__fmaf_rn((v - mean) * rstd, param1<E>(a.gamma, a.params32, c, 1.0f),
                                          LAYER ? param1<E>(a.beta, a.params32, c, 0.0f) : 0.0f));
        y[c] = r;
        o = to_f32<E>(r);
      }
      auto save = [&](int8_t* codes, uint8_t* scales, float w) {
        const uint32_t q = block8_scale(__reduce_max_sync(0xffffffffu, abs_bits(w)));
        if (c < a.pitch) codes[row * a.pitch + c] = q == kScaleNaN ? int8_t(0) : int8_t(block8_code(w, block8_inverse(min(q, kScaleMax))));
        if (lane == 0) scales[row * a.spitch + c / 32] = uint8_t(q);
      };
      if (a.xcodes != nullptr) save(a.xcodes, a.xscales, v);
      if (a.ycodes != nullptr) save(a.ycodes, a.yscales, o);
    }
  }
}

template <Elem E, bool CKPT>
__device__ __forceinline__ float x_at(const BwdArgs& a, int64_t row, int64_t c) {
  using T = typename ElemType<E>::T;
  if constexpr (CKPT) return float(a.codes[row * a.pitch + c]) * block8_step(a.scales[row * a.spitch + c / 32]);
  return to_f32<E>(static_cast<const T*>(a.x)[row * a.ldx + c]);
}

template <Elem E, bool LAYER, bool CKPT>
__global__ void __launch_bounds__(1024) roi_norm_bwd_wide_kernel(BwdArgs a) {
  using T = typename ElemType<E>::T;
  __shared__ float slots[2][32];
  pdl_begin(a.wait);
  const float inv_cols = 1.0f / float(a.cols);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const float mean = LAYER ? a.mean[row] : 0.0f, rstd = a.rstd[row];
    float c1 = 0.0f, c2 = 0.0f;
#pragma unroll 4
    for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float d = to_f32<E>(dy[c]) * param1<E>(a.gamma, a.params32, c, 1.0f);
      c1 = __fmaf_rn(d, (x_at<E, CKPT>(a, row, c) - mean) * rstd, c1);
      if constexpr (LAYER) c2 += d;
    }
    const float m1 = cta_sum(c1, slots, turn) * inv_cols;
    const float m2 = LAYER ? cta_sum(c2, slots, turn) * inv_cols : 0.0f;
#pragma unroll 4
    for (int64_t c = threadIdx.x; c < a.cols; c += blockDim.x) {
      const float xh = (x_at<E, CKPT>(a, row, c) - mean) * rstd;
      const float d = __fmaf_rn(-xh, m1, to_f32<E>(dy[c]) * param1<E>(a.gamma, a.params32, c, 1.0f));
      static_cast<T*>(a.dx)[row * a.lddx + c] = from_f32<E>((d - m2) * rstd);
    }
  }
}

// A thread a column, a CTA (256 columns) every gridDim.y-th row: partial row blockIdx.y.
template <Elem E, bool LAYER, bool CKPT>
__global__ void __launch_bounds__(256) roi_norm_bwd_wide_sums_kernel(BwdArgs a) {
  using T = typename ElemType<E>::T;
  pdl_begin(a.wait);
  const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float dg = 0.0f, db = 0.0f;
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float dy = to_f32<E>(static_cast<const T*>(a.dy)[row * a.lddy + c]);
    dg = __fmaf_rn(dy, (x_at<E, CKPT>(a, row, c) - (LAYER ? a.mean[row] : 0.0f)) * a.rstd[row], dg);
    if constexpr (LAYER) db += dy;
  }
  float* part = a.part + int64_t(blockIdx.y) * (LAYER ? 2 : 1) * a.part_cols;
  part[c] = dg;
  if constexpr (LAYER) part[a.part_cols + c] = db;
}

// Rows of whole granules.
bool on_granules(const void* p, int64_t ld, int64_t rows, int64_t cols, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && cols * bytes % 16 == 0 && (rows <= 1 || ld * bytes % 16 == 0);
}

// Shared memory that a CTA may take, less what the kernels declare.
constexpr size_t kMostSmem = 232448 - 1024 - sizeof(TeamState);

// `run` pieces of 256 columns a warp, at most `threads` threads; `least`: bytes that must be there.
Shape shape_of(int64_t rows, int64_t cols, int64_t pieces, int run, int threads, size_t stage, size_t params, size_t least) {
  Shape s;
  s.stage = uint32_t(stage);
  s.params = uint32_t(params);
  const int64_t warps = (pieces + run - 1) / run;
  s.depth = 0;
  if (warps * 32 > threads - 32 || params + 2 * stage > kMostSmem || least > kMostSmem) return s;
  s.nt = int(warps) * 32;
  int64_t teams = (threads - 32) / s.nt;  // (a warp fills the rings)
  const int64_t most = s.nt == 32 ? kMostTeams : kMostNamed, fit = int64_t((kMostSmem - params) / (2 * stage));
  if (teams > most) teams = most;
  if (teams > fit) teams = fit;
  // no more teams than rows need
  const int64_t cap = sm_count();
  const int64_t need = (rows + cap - 1) / cap;
  if (teams > need) teams = need;
  // a filling warp for every eight teams
  s.fillers = int((teams + 7) / 8);
  while (teams * s.nt + s.fillers * 32 > threads) --teams;
  s.teams = int(teams);
  const int64_t depth = int64_t((kMostSmem - params) / (stage * size_t(teams)));
  s.depth = int(depth > kMostDepth ? kMostDepth : depth);
  const int64_t want = (rows + teams - 1) / teams;
  s.grid = int(want < cap ? want : cap);
  // no deeper than a team has rows
  const int64_t each = (rows + s.grid * teams - 1) / (s.grid * teams);
  if (s.depth > each) s.depth = int(each);
  s.smem = params + stage * size_t(s.depth) * size_t(teams);
  if (s.smem < least) s.smem = least;
  return s;
}

// Dynamic shared memory past the default limit, once for a kernel and device.
template <class K>
bool allow_smem(K kern, std::atomic<bool> (&done)[64]) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (done[dev].load(std::memory_order_acquire)) return true;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMostSmem)) != cudaSuccess) return false;
  done[dev].store(true, std::memory_order_release);
  return true;
}

template <Elem E, bool LAYER, bool ANY, int RUN>
int fwd_run(const NormFwdCall& c, const FwdArgs& a) {
  static std::atomic<bool> done[64];
  auto kern = roi_norm_fwd_kernel<E, LAYER, ANY, RUN>;
  if (!allow_smem(kern, done)) return -1;
  return launch_maybe_pdl(kern, a.shape.grid, a.shape.nt * a.shape.teams + a.shape.fillers * 32, a.shape.smem, c.stream, a.wait, a);
}

template <Elem E, bool LAYER, bool ANY>
int fwd(const NormFwdCall& c, FwdArgs& a) {
  // the padding of a checkpoint's scales is written too
  const int64_t end = c.xcodes != nullptr || c.ycodes != nullptr ? a.spitch * 32 : a.cols;
  const int64_t pieces = (end + 255) / 256;
  const size_t stage = size_t(a.cols + 7) / 8 * 8 * elem_bytes<E>() + (ANY ? 32 : 0);
  const size_t params = size_t((a.cols + 255) / 256 * 256) * 4 * (LAYER ? 2 : 1);
  // few rows, where a row's own time counts: as many warps as there are pieces.  RMS norm of 3584 columns in a graph,
  // one piece a lane against four: 1 row 3.9 and 6.7 us, 304 rows 4.2 and 5.3, 600 rows 5.2 and 4.6, 1200 rows
  // 7.4 and 6.1.
  const bool few = a.rows <= 2 * sm_count() && pieces < 32;
  a.shape = shape_of(a.rows, a.cols, pieces, few ? 1 : kRun<E>, few ? kThreads : kFwdThreads<LAYER, ANY>, stage, params, 0);
  if (a.shape.depth > 0) return few ? fwd_run<E, LAYER, ANY, 1>(c, a) : fwd_run<E, LAYER, ANY, kRun<E>>(c, a);
  const int64_t cap = int64_t(sm_count()) * 2;
  return launch_maybe_pdl(roi_norm_fwd_wide_kernel<E, LAYER>, int(a.rows < cap ? a.rows : cap), kThreads, 0, c.stream, a.wait, a);
}

template <Elem E>
int fwd_type(const NormFwdCall& c) {
  FwdArgs a;
  a.x = c.x, a.y = c.y, a.gamma = c.gamma, a.beta = c.beta, a.mean = c.mean, a.rstd = c.rstd;
  a.xcodes = c.xcodes, a.xscales = c.xscales, a.ycodes = c.ycodes, a.yscales = c.yscales;
  a.rows = c.rows, a.cols = c.cols, a.ldx = c.ldx, a.ldy = c.ldy;
  a.pitch = block8_pitch(c.cols), a.spitch = block8_scale_pitch(c.cols);
  a.status = c.status;
  a.eps = c.eps;
  a.params32 = c.params32;
  a.wait = lone_pdl(c.stream);
  const int b = elem_bytes<E>();
  const bool any = !on_granules(c.x, c.ldx, c.rows, c.cols, b) || !on_granules(c.y, c.ldy, c.rows, c.cols, b);
  if (c.layer) return any ? fwd<E, true, true>(c, a) : fwd<E, true, false>(c, a);
  return any ? fwd<E, false, true>(c, a) : fwd<E, false, false>(c, a);
}

int64_t wide_parts(int64_t rows) { return rows < 64 ? rows : 64; }

int sum_parts(const BwdArgs& a, int parts, int kinds, cudaStream_t stream) {
  const int64_t grid = (a.cols + 31) / 32 * kinds;
  return launch_maybe_pdl(roi_norm_sum_kernel, int(grid), 32 * kSumSegments, 0, stream, true, static_cast<const float*>(a.part), parts,
                          kinds, a.part_cols, a.cols, a.dgamma, a.dbeta);
}

template <Elem E, bool LAYER, bool CKPT, bool ANY, int NP, int THREADS>
int bwd_run(const NormBwdCall& c, const BwdArgs& a) {
  static std::atomic<bool> done[64];
  auto kern = roi_norm_bwd_kernel<E, LAYER, CKPT, ANY, NP, THREADS>;
  if (!allow_smem(kern, done)) return -1;
  return launch_maybe_pdl(kern, a.shape.grid, a.shape.nt * a.shape.teams + a.shape.fillers * 32, a.shape.smem, c.stream, a.wait, a);
}

template <Elem E, bool LAYER, bool CKPT, bool ANY>
int bwd(const NormBwdCall& c, BwdArgs& a) {
  const bool sums = a.dgamma != nullptr || a.dbeta != nullptr;
  const int kinds = LAYER ? 2 : 1;
  const size_t rowb = size_t(a.cols + 7) / 8 * 8 * elem_bytes<E>() + (ANY ? 32 : 0);
  const size_t stage = rowb + (CKPT ? (size_t(a.pitch + a.spitch) + 15) / 16 * 16 + 32 : rowb);
  const size_t params = size_t((a.cols + 255) / 256 * 256) * 4;
  const int64_t pieces = (a.cols + 255) / 256;
  const int np = pieces > 1 ? 2 : 1;
  // (the teams' sums take the place of the rings)
  const size_t least = size_t(kinds) * 8 * size_t((pieces + np - 1) / np * np) * 32 * 4;
  const int64_t nt = (pieces + np - 1) / np * 32;
  // (layer norm, 8192 rows, from the checkpoint, 512 threads against 640: 3584 columns 49 and 54 us, 2048 columns
  // 31.5 and 31.7, from x 45 and 52, 28 and 31; the sums of dbeta take registers, and 512 hold no two teams of more than 240 threads)
  constexpr int kFew = E != Elem::kFp32 && !LAYER ? 768 : 640;
  const int threads = np == 1 || nt > kFew - 32 ? 1024 : LAYER && nt <= 240 ? 512 : kFew;
  a.shape = shape_of(a.rows, a.cols, pieces, np, threads, stage, params, least);
  if (a.shape.depth == 0) {
    const int64_t cap = int64_t(sm_count()) * 2;
    const int n = launch_maybe_pdl(roi_norm_bwd_wide_kernel<E, LAYER, CKPT>, int(a.rows < cap ? a.rows : cap), 1024, 0, c.stream, a.wait, a);
    if (n < 0 || !sums) return n;
    const int parts = int(wide_parts(a.rows));
    roi_norm_bwd_wide_sums_kernel<E, LAYER, CKPT><<<dim3(unsigned((a.cols + 255) / 256), unsigned(parts)), 256, 0, c.stream>>>(a);
    if (cudaGetLastError() != cudaSuccess || sum_parts(a, parts, kinds, c.stream) < 0) return -1;
    return 3;
  }
  int n;
  if (np == 1) n = bwd_run<E, LAYER, CKPT, ANY, 1, 1024>(c, a);
  else if (threads == 1024) n = bwd_run<E, LAYER, CKPT, ANY, 2, 1024>(c, a);
  else if (!LAYER || threads == kFew) n = bwd_run<E, LAYER, CKPT, ANY, 2, kFew>(c, a);
  else n = bwd_run<E, true, CKPT, ANY, 2, 512>(c, a);
  if (n < 0 || !sums || a.shape.grid == 1) return n;
  return sum_parts(a, a.shape.grid, kinds, c.stream) < 0 ? -1 : 2;
}

template <Elem E>
int bwd_type(const NormBwdCall& c) {
  BwdArgs a;
  a.dy = c.dy, a.x = c.x, a.codes = c.codes, a.scales = c.scales, a.gamma = c.gamma, a.mean = c.mean, a.rstd = c.rstd;
  a.dx = c.dx, a.dgamma = c.dgamma, a.dbeta = c.dbeta, a.part = static_cast<float*>(c.workspace);
  a.rows = c.rows, a.cols = c.cols, a.lddy = c.lddy, a.ldx = c.ldx, a.lddx = c.lddx;
  a.pitch = block8_pitch(c.cols), a.spitch = block8_scale_pitch(c.cols), a.part_cols = (c.cols + 3) / 4 * 4;
  a.status = c.status;
  a.params32 = c.params32;
  a.wait = lone_pdl(c.stream);
  const int b = elem_bytes<E>();
  const bool any = !on_granules(c.dy, c.lddy, c.rows, c.cols, b) || !on_granules(c.dx, c.lddx, c.rows, c.cols, b) ||
                   (c.x != nullptr && !on_granules(c.x, c.ldx, c.rows, c.cols, b));
  if (c.layer) {
    if (c.x == nullptr) return any ? bwd<E, true, true, true>(c, a) : bwd<E, true, true, false>(c, a);
    return any ? bwd<E, true, false, true>(c, a) : bwd<E, true, false, false>(c, a);
  }
  if (c.x == nullptr) return any ? bwd<E, false, true, true>(c, a) : bwd<E, false, true, false>(c, a);
  return any ? bwd<E, false, false, true>(c, a) : bwd<E, false, false, false>(c, a);
}

}  // namespace

// (one partial row a CTA, at most one CTA an SM; 64 for the widest rows)
size_t norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  const int64_t most = sm_count() > 64 ? sm_count() : 64;
  return size_t(rows < most ? rows : most) * 2 * size_t((cols + 3) / 4 * 4) * 4;
}

int launch_norm_fwd(const NormFwdCall& c) {
  switch (c.dtype) {
    case Elem::kBf16: return fwd_type<Elem::kBf16>(c);
    case Elem::kFp16: return fwd_type<Elem::kFp16>(c);
    default: return fwd_type<Elem::kFp32>(c);
  }
}

int launch_norm_bwd(const NormBwdCall& c) {
  switch (c.dtype) {
    case Elem::kBf16: return bwd_type<Elem::kBf16>(c);
    case Elem::kFp16: return bwd_type<Elem::kFp16>(c);
    default: return bwd_type<Elem::kFp32>(c);
  }
}

}  // namespace roi
