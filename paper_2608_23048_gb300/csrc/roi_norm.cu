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
// computed in 32 bits; outputs are rounded once.
//
// Forward: a CTA a row, the row in registers (each thread holds NV pieces of 8 elements), so
// the squares are summed around the mean already known and x is read once.  Rows past 16384
// columns are read again for each step instead.
// Backward: a team of threads a row, each thread with the same 8 columns of every row it
// sees, so that the sums of dgamma and dbeta stay in its registers; two rows are reduced at a
// time and the next two are loaded before.  The teams' and then the CTAs' sums are added in a
// fixed order (through shared memory, and by a second launch): no atomics, the same bits every
// time.  Rows past 8192 columns go to a kernel for dx and one for the sums over rows.
// Pieces are 8 consecutive columns where the rows allow 16-byte loads (VEC); elsewhere a
// thread takes every blockDim-th column, so that a warp still reads 32 neighbours.
#include "roi_block8.cuh"
#include "roi_launch.h"

namespace roi {
namespace {

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
  int teams;
  bool params32;
  bool wait;
};

// gamma or beta at 8 consecutive columns from c on, or at one column; `none` where not given.
template <Elem E>
__device__ __forceinline__ void param8(const void* p, bool p32, int64_t c, int64_t cols, float none, float (&v)[8]) {
  using T = typename ElemType<E>::T;
  if (p == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = none;
  } else if (c + 8 <= cols) {
    if (p32) {
      Raw8<Elem::kFp32> r;
      r.load(static_cast<const float*>(p) + c);
      r.get(v);
    } else {
      Raw8<E> r;
      r.load(static_cast<const T*>(p) + c);
      r.get(v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      v[i] = c + i >= cols ? none : p32 ? __ldg(static_cast<const float*>(p) + c + i) : to_f32<E>(__ldg(static_cast<const T*>(p) + c + i));
  }
}
template <Elem E>
__device__ __forceinline__ float param1(const void* p, bool p32, int64_t c, float none) {
  using T = typename ElemType<E>::T;
  return p == nullptr ? none : p32 ? __ldg(static_cast<const float*>(p) + c) : to_f32<E>(__ldg(static_cast<const T*>(p) + c));
}

// Column of element k of piece i of thread `t` of `nt`.
template <bool VEC>
__device__ __forceinline__ int64_t column(int i, int k, int t, int nt) {
  return VEC ? (int64_t(i) * nt + t) * 8 + k : (int64_t(i) * 8 + k) * nt + t;
}

template <Elem E, bool VEC>
__device__ __forceinline__ void load_piece(const typename ElemType<E>::T* row, int64_t cols, int i, int t, int nt, float (&v)[8]) {
  if constexpr (VEC) {
    const int64_t c = column<true>(i, 0, t, nt);
    if (c + 8 <= cols) {
      Raw8<E> r;
      r.load(row + c);
      r.get(v);
      return;
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t c = column<VEC>(i, k, t, nt);
    v[k] = c < cols ? to_f32<E>(row[c]) : 0.0f;
  }
}

template <Elem E, bool VEC>
__device__ __forceinline__ void store_piece(typename ElemType<E>::T* row, int64_t cols, int i, int t, int nt, const float (&v)[8]) {
  if constexpr (VEC) {
    const int64_t c = column<true>(i, 0, t, nt);
    if (c + 8 <= cols) {
      Raw8<E> r;
      r.set(v);
      r.store(row + c);
      return;
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t c = column<VEC>(i, k, t, nt);
    if (c < cols) row[c] = from_f32<E>(v[k]);
  }
}

// One piece's part of a checkpoint row (all lanes of the warp call it; values past the last
// column are 0).  VEC: a block is four neighbouring lanes; else a lane's k-th element belongs
// to the warp's k-th block.
template <bool VEC>
__device__ __forceinline__ void save_piece(int8_t* codes, uint8_t* scales, int64_t pitch, int64_t spitch, int i, int t, int nt,
                                           const float (&v)[8]) {
  if constexpr (VEC) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, abs_bits(v[k]));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t s = block8_scale(top);
    const float inverse = block8_inverse(min(s, kScaleMax));
    const uint32_t keep = s == kScaleNaN ? 0u : 0xffffffffu;
    const int64_t c = column<true>(i, 0, t, nt);
    if (c < pitch)
      *reinterpret_cast<uint2*>(codes + c) = make_uint2(block8_codes4(v, inverse, keep), block8_codes4(v + 4, inverse, keep));
    if (c % 32 == 0 && c / 32 < spitch) scales[c / 32] = uint8_t(s);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t s = block8_scale(__reduce_max_sync(0xffffffffu, abs_bits(v[k])));
      const uint32_t q = block8_code(v[k], block8_inverse(min(s, kScaleMax)));
      const int64_t c = column<false>(i, k, t, nt);
      if (c < pitch) codes[c] = s == kScaleNaN ? int8_t(0) : int8_t(q);
      if (c % 32 == 0 && c / 32 < spitch) scales[c / 32] = uint8_t(s);
    }
  }
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
// Sum over the CTA, the same bits in every thread.  Two sets of slots in turn: a set is written
// again only after the barrier of the sum in between.
__device__ __forceinline__ float cta_sum(float v, float (&slots)[2][32], int& turn) {
  v = warp_sum(v);
  if (blockDim.x == 32) return v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) slots[turn][warp] = v;
  __syncthreads();
  v = warp_sum(lane < int(blockDim.x >> 5) ? slots[turn][lane] : 0.0f);
  turn ^= 1;
  return v;
}

constexpr int kFwdThreads = 512, kTeamThreads = 512;  // at most, of a CTA
// NV > 0: the row in registers; NV = 0: read again for each step, `pieces` pieces a thread.
template <Elem E, bool LAYER, bool VEC, int NV>
__global__ void __launch_bounds__(kFwdThreads) roi_norm_fwd_kernel(FwdArgs a, int pieces) {
  using T = typename ElemType<E>::T;
  __shared__ float slots[2][32];
  pdl_begin(a.wait);
  const int t = threadIdx.x, nt = blockDim.x;
  const int n = NV > 0 ? NV : pieces;
  constexpr int kHeld = NV > 0 ? NV : 1;
  const float inv_cols = 1.0f / float(a.cols);
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    float v[kHeld][8];
    auto piece = [&](int i) -> float(&)[8] {
      if (NV == 0) load_piece<E, VEC>(x, a.cols, i, t, nt, v[0]);
      return v[NV > 0 ? i : 0];
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) load_piece<E, VEC>(x, a.cols, i, t, nt, v[i]);
    }
    float mean = 0.0f;
    if constexpr (LAYER) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < n; ++i) {
        float(&p)[8] = piece(i);
        sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      }
      mean = cta_sum(sum, slots, turn) * inv_cols;
    }
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      float(&p)[8] = piece(i);
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // columns past the last hold 0, which is not at distance 0 from the mean
        const float d = LAYER && column<VEC>(i, k, t, nt) >= a.cols ? 0.0f : p[k] - mean;
        s = __fmaf_rn(d, d, s);
      }
      squares += s;
    }
    const float rstd = 1.0f / sqrtf(cta_sum(squares, slots, turn) * inv_cols + a.eps);
    if (t == 0) {
      if (LAYER && a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(a.y) + row * a.ldy;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      float(&p)[8] = piece(i);
      float o[8];
      if (a.xcodes != nullptr)
        save_piece<VEC>(a.xcodes + row * a.pitch, a.xscales + row * a.spitch, a.pitch, a.spitch, i, t, nt, p);
      if constexpr (VEC) {
        const int64_t c = column<true>(i, 0, t, nt);
        float g[8], b[8];
        param8<E>(a.gamma, a.params32, c, a.cols, 1.0f, g);
        param8<E>(a.beta, a.params32, c, a.cols, 0.0f, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = __fmaf_rn((p[k] - mean) * rstd, g[k], b[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int64_t c = column<false>(i, k, t, nt);
          const bool in = c < a.cols;
          o[k] = __fmaf_rn((p[k] - mean) * rstd, in ? param1<E>(a.gamma, a.params32, c, 1.0f) : 1.0f,
                           in ? param1<E>(a.beta, a.params32, c, 0.0f) : 0.0f);
        }
      }
      store_piece<E, VEC>(y, a.cols, i, t, nt, o);
      if (a.ycodes != nullptr) {
        // of y as it was rounded
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = column<VEC>(i, k, t, nt) < a.cols ? to_f32<E>(from_f32<E>(o[k])) : 0.0f;
        save_piece<VEC>(a.ycodes + row * a.pitch, a.yscales + row * a.spitch, a.pitch, a.spitch, i, t, nt, o);
      }
    }
  }
}

__device__ __forceinline__ void team_sync(int team, int nt) {
  if (nt == 32) {
    __syncwarp();
  } else {
    asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(nt) : "memory");
  }
}

// A thread's piece of one row of the backward's inputs, as it lies in memory.
template <Elem E, bool VEC, bool CKPT>
struct RowIn {
  using T = typename ElemType<E>::T;
  static constexpr int kEl = VEC ? 1 : 8;
  Raw8<E> dy8, x8;
  T dy1[kEl], x1[kEl];
  uint2 q8;
  int8_t q1[kEl];
  uint8_t s1[kEl];

  __device__ __forceinline__ void load(const BwdArgs& a, int64_t row, int piece, int t, int nt) {
    const bool in = row < a.rows;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    if constexpr (VEC) {
      const int64_t c = column<true>(piece, 0, t, nt);
      const bool whole = in && c + 8 <= a.cols;
      if (whole) {
        dy8.load(dy + c);
        if constexpr (!CKPT) x8.load(x + c);
      } else {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = in && c + k < a.cols ? to_f32<E>(dy[c + k]) : 0.0f;
        dy8.set(v);
        if constexpr (!CKPT) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = in && c + k < a.cols ? to_f32<E>(x[c + k]) : 0.0f;
          x8.set(v);
        }
      }
      if constexpr (CKPT) {
        q8 = make_uint2(0, 0), s1[0] = 0;
        if (in && c < a.pitch) {
          q8 = __ldg(reinterpret_cast<const uint2*>(a.codes + row * a.pitch + c));
          s1[0] = __ldg(a.scales + row * a.spitch + c / 32);
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t c = column<false>(piece, k, t, nt);
        const bool ok = in && c < a.cols;
        dy1[k] = ok ? dy[c] : T(0);
        if constexpr (CKPT) {
          q1[k] = ok ? a.codes[row * a.pitch + c] : int8_t(0);
          s1[k] = ok ? a.scales[row * a.spitch + c / 32] : uint8_t(0);
        } else {
          x1[k] = ok ? x[c] : T(0);
        }
      }
    }
  }
  __device__ __forceinline__ void get(float (&dy)[8], float (&x)[8]) const {
    if constexpr (VEC) {
      dy8.get(dy);
      if constexpr (CKPT) {
        const float step = block8_step(s1[0]);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = block8_value(k < 4 ? q8.x : q8.y, k % 4, step);
      } else {
        x8.get(x);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        dy[k] = to_f32<E>(dy1[k]);
        x[k] = CKPT ? float(q1[k]) * block8_step(s1[k]) : to_f32<E>(x1[k]);
      }
    }
  }
};

// NP: pieces a thread; PAIR: rows a team reduces at a time.
template <Elem E, bool LAYER, bool VEC, bool CKPT, int NP, int PAIR>
__global__ void __launch_bounds__(kTeamThreads) roi_norm_bwd_kernel(BwdArgs a) {
  using T = typename ElemType<E>::T;
  extern __shared__ float sums[];  // [1 or 2][NP][8][nt], the teams' sums (more than one team)
  __shared__ float slots[2][kTeamThreads / 32][2 * PAIR];
  pdl_begin(a.wait);
  const int nt = blockDim.x / a.teams;
  const int team = threadIdx.x / nt, t = threadIdx.x - team * nt;
  const int warps = nt >> 5, warp0 = team * warps, lane = t & 31;
  const float inv_cols = 1.0f / float(a.cols);
  auto weight = [&](int i, float(&g)[8]) {
    if constexpr (VEC) {
      param8<E>(a.gamma, a.params32, column<true>(i, 0, t, nt), a.cols, 1.0f, g);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t c = column<false>(i, k, t, nt);
        g[k] = c < a.cols ? param1<E>(a.gamma, a.params32, c, 1.0f) : 1.0f;
      }
    }
  };
  // with one piece a thread the weight stays in registers
  float held[8], dg[NP][8], db[NP][8];
  if constexpr (NP == 1) weight(0, held);
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) dg[i][k] = db[i][k] = 0.0f;

  const int64_t all = int64_t(gridDim.x) * a.teams;
  int64_t row = int64_t(blockIdx.x) * a.teams + team;
  RowIn<E, VEC, CKPT> next[PAIR][NP];
  float next_mean[PAIR], next_rstd[PAIR];
  auto load = [&](int64_t from) {
#pragma unroll
    for (int r = 0; r < PAIR; ++r) {
      const int64_t at = from + r * all;
      next_mean[r] = LAYER && at < a.rows ? __ldg(a.mean + at) : 0.0f;
      next_rstd[r] = at < a.rows ? __ldg(a.rstd + at) : 0.0f;
#pragma unroll
      for (int i = 0; i < NP; ++i) next[r][i].load(a, at, i, t, nt);
    }
  };
  load(row);
  int turn = 0;
  for (; row < a.rows; row += PAIR * all) {
    RowIn<E, VEC, CKPT> cur[PAIR][NP];
    float mean[PAIR], rstd[PAIR];
#pragma unroll
    for (int r = 0; r < PAIR; ++r) {
      mean[r] = next_mean[r], rstd[r] = next_rstd[r];
#pragma unroll
      for (int i = 0; i < NP; ++i) cur[r][i] = next[r][i];
    }
    load(row + PAIR * all);
    float c[2 * PAIR];
#pragma unroll
    for (int r = 0; r < PAIR; ++r) {
      float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        float dy[8], x[8], g[8];
        if constexpr (NP > 1) weight(i, g);
        cur[r][i].get(dy, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float gk = NP > 1 ? g[k] : held[k];
          const float p = dy[k] * ((x[k] - mean[r]) * rstd[r]);
          dg[i][k] += p;
          if constexpr (LAYER) db[i][k] += dy[k];
          c1 = __fmaf_rn(p, gk, c1);
          if constexpr (LAYER) c2 = __fmaf_rn(dy[k], gk, c2);
        }
      }
      c[2 * r] = warp_sum(c1);
      c[2 * r + 1] = LAYER ? warp_sum(c2) : 0.0f;
    }
    if (nt > 32) {
      if (lane == 0) {
#pragma unroll
        for (int q = 0; q < 2 * PAIR; ++q) slots[turn][warp0 + (t >> 5)][q] = c[q];
      }
      team_sync(team, nt);
#pragma unroll
      for (int q = 0; q < 2 * PAIR; ++q) c[q] = 0.0f;
      for (int w = 0; w < warps; ++w) {
#pragma unroll
        for (int q = 0; q < 2 * PAIR; ++q) c[q] += slots[turn][warp0 + w][q];
      }
      turn ^= 1;
    }
#pragma unroll
    for (int r = 0; r < PAIR; ++r) {
      const int64_t at = row + r * all;
      if (at >= a.rows) break;
      const float m1 = c[2 * r] * inv_cols, m2 = c[2 * r + 1] * inv_cols;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        float dy[8], x[8], g[8], o[8];
        if constexpr (NP > 1) weight(i, g);
        cur[r][i].get(dy, x);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float d = __fmaf_rn((mean[r] - x[k]) * rstd[r], m1, dy[k] * (NP > 1 ? g[k] : held[k]));
          if constexpr (LAYER) d -= m2;
          o[k] = d * rstd[r];
        }
        store_piece<E, VEC>(static_cast<T*>(a.dx) + at * a.lddx, a.cols, i, t, nt, o);
      }
    }
  }

  if (a.dgamma == nullptr && a.dbeta == nullptr) return;
  // the teams' sums in their order, then this CTA's to its place among the partial sums (the
  // outputs themselves where it is the only CTA)
  float* part = a.part + int64_t(blockIdx.x) * (LAYER ? 2 : 1) * a.part_cols;
  float* to_g = gridDim.x == 1 ? a.dgamma : part;
  float* to_b = gridDim.x == 1 ? a.dbeta : part + a.part_cols;
  for (int q = 0; q < a.teams && a.teams > 1; ++q) {
    if (q == team) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = (8 * i + k) * nt + t;
          if (q > 0) {
            dg[i][k] += sums[at];
            if constexpr (LAYER) db[i][k] += sums[8 * NP * nt + at];
          }
          sums[at] = dg[i][k];
          if constexpr (LAYER) sums[8 * NP * nt + at] = db[i][k];
        }
      }
    }
    __syncthreads();
  }
  if (team == a.teams - 1) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int64_t c = column<VEC>(i, k, t, nt);
        if (c < a.cols) {
          if (to_g != nullptr) to_g[c] = dg[i][k];
          if (LAYER && to_b != nullptr) to_b[c] = db[i][k];
        }
      }
    }
  }
}

// out[c] = the sum of the `parts` partial rows at c, in a fixed order: eight threads a column
// take every eighth row, and their sums are added in their order.  kinds: 1 (dgamma) or 2.
__global__ void __launch_bounds__(256) roi_norm_sum_kernel(const float* part, int parts, int kinds, int64_t part_cols, int64_t cols,
                                                           float* dgamma, float* dbeta) {
  __shared__ float sums[8][33];
  pdl_begin(true);  // the partial sums of the launch before
  const int lane = threadIdx.x & 31, seg = threadIdx.x >> 5;
  const int64_t blocks = (cols + 31) / 32;
  const int64_t kind = blockIdx.x / blocks, c = (blockIdx.x - kind * blocks) * 32 + lane;
  float s = 0.0f;
  if (c < cols) {
    const float* p = part + kind * part_cols + c;
    const int64_t stride = kinds * part_cols;
#pragma unroll 8
    for (int q = seg; q < parts; q += 8) s += p[q * stride];
  }
  sums[seg][lane] = s;
  __syncthreads();
  if (seg == 0 && c < cols) {
    for (int q = 1; q < 8; ++q) s += sums[q][lane];
    float* out = kind == 0 ? dgamma : dbeta;
    if (out != nullptr) out[c] = s;
  }
}

// ---- rows past 8192 columns ----
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

bool aligned_rows(const void* p, int64_t ld, int64_t rows, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld * bytes % 16 == 0);
}

constexpr int64_t kHeldPieces = 4 * kFwdThreads;    // forward: what a CTA holds in registers
constexpr int64_t kTeamCols = 2 * kTeamThreads * 8;  // backward: two pieces a thread

// Threads of a CTA or team for so many pieces, a whole number of warps.
int threads_for(int64_t pieces, int most) {
  const int64_t t = (pieces + 31) / 32 * 32;
  return int(t < 32 ? 32 : t > most ? most : t);
}

template <Elem E, bool LAYER, bool VEC>
int fwd(const NormFwdCall& c, const FwdArgs& a) {
  // the padding of a checkpoint's scales is written too
  const int64_t pieces = c.xcodes != nullptr || c.ycodes != nullptr ? a.spitch * 4 : (a.cols + 7) / 8;
  int64_t grid = a.rows;
  if (pieces > kHeldPieces) {
    const int64_t cap = int64_t(sm_count()) * 4;
    return launch_maybe_pdl(roi_norm_fwd_kernel<E, LAYER, VEC, 0>, int(grid < cap ? grid : cap), kFwdThreads, 0, c.stream,
                            a.wait, a, int((pieces + kFwdThreads - 1) / kFwdThreads));
  }
  // few rows: one piece a thread, so that a row's loads and sums take the least time
  const bool few = a.rows <= 2 * sm_count() && pieces <= kFwdThreads;
  const int threads = threads_for(few ? pieces : (pieces + 3) / 4, kFwdThreads);
  const int64_t cap = int64_t(sm_count()) * 32;
  if (grid > cap) grid = cap;
  return few ? launch_maybe_pdl(roi_norm_fwd_kernel<E, LAYER, VEC, 1>, int(grid), threads, 0, c.stream, a.wait, a, 1)
             : launch_maybe_pdl(roi_norm_fwd_kernel<E, LAYER, VEC, 4>, int(grid), threads, 0, c.stream, a.wait, a, 4);
}

template <Elem E>
int fwd_type(const NormFwdCall& c) {
  FwdArgs a;
  a.x = c.x, a.y = c.y, a.gamma = c.gamma, a.beta = c.beta, a.mean = c.mean, a.rstd = c.rstd;
  a.xcodes = c.xcodes, a.xscales = c.xscales, a.ycodes = c.ycodes, a.yscales = c.yscales;
  a.rows = c.rows, a.cols = c.cols, a.ldx = c.ldx, a.ldy = c.ldy;
  a.pitch = block8_pitch(c.cols), a.spitch = block8_scale_pitch(c.cols);
  a.eps = c.eps;
  a.params32 = c.params32;
  a.wait = lone_pdl(c.stream);
  const bool vec = aligned_rows(c.x, c.ldx, c.rows, elem_bytes<E>()) && aligned_rows(c.y, c.ldy, c.rows, elem_bytes<E>());
  if (c.layer) return vec ? fwd<E, true, true>(c, a) : fwd<E, true, false>(c, a);
  return vec ? fwd<E, false, true>(c, a) : fwd<E, false, false>(c, a);
}

// CTAs of the backward, the teams in each (as many as 512 threads hold) and the pieces a
// thread takes.  The partial sums are as many rows as there are CTAs.
struct BwdShape {
  int pieces, nt, teams, grid;
};
BwdShape bwd_shape(int64_t rows, int64_t cols) {
  BwdShape s;
  const int64_t pieces = (cols + 7) / 8;
  s.pieces = pieces > kTeamThreads ? 2 : 1;
  s.nt = threads_for((pieces + s.pieces - 1) / s.pieces, kTeamThreads);
  s.teams = kTeamThreads / s.nt > 15 ? 15 : kTeamThreads / s.nt;
  const int64_t want = (rows + s.teams - 1) / s.teams;
  const int64_t cap = sm_count();
  s.grid = int(want < cap ? want : cap);
  return s;
}
int64_t wide_parts(int64_t rows) { return rows < 64 ? (rows < 1 ? 1 : rows) : 64; }

int sum_parts(const BwdArgs& a, int parts, int kinds, cudaStream_t stream) {
  const int64_t grid = (a.cols + 31) / 32 * kinds;
  return launch_maybe_pdl(roi_norm_sum_kernel, int(grid), 256, 0, stream, true, static_cast<const float*>(a.part), parts, kinds,
                          a.part_cols, a.cols, a.dgamma, a.dbeta);
}

template <Elem E, bool LAYER, bool CKPT>
int bwd(const NormBwdCall& c, BwdArgs a, bool vec) {
  const bool sums = a.dgamma != nullptr || a.dbeta != nullptr;
  const int kinds = LAYER ? 2 : 1;
  if (a.cols > kTeamCols) {
    const int64_t cap = int64_t(sm_count()) * 2;
    int n = launch_maybe_pdl(roi_norm_bwd_wide_kernel<E, LAYER, CKPT>, int(a.rows < cap ? a.rows : cap), 1024, 0, c.stream, a.wait, a);
    if (n < 0 || !sums) return n;
    const int parts = int(wide_parts(a.rows));
    roi_norm_bwd_wide_sums_kernel<E, LAYER, CKPT><<<dim3(unsigned((a.cols + 255) / 256), unsigned(parts)), 256, 0, c.stream>>>(a);
    if (cudaGetLastError() != cudaSuccess || sum_parts(a, parts, kinds, c.stream) < 0) return -1;
    return 3;
  }
  const BwdShape s = bwd_shape(a.rows, a.cols);
  a.teams = s.teams;
  const size_t smem = s.teams > 1 && sums ? size_t(kinds) * 8 * s.pieces * s.nt * 4 : 0;
  auto kern = s.pieces == 1 ? (vec ? roi_norm_bwd_kernel<E, LAYER, true, CKPT, 1, 2> : roi_norm_bwd_kernel<E, LAYER, false, CKPT, 1, 1>)
                            : (vec ? roi_norm_bwd_kernel<E, LAYER, true, CKPT, 2, 1> : roi_norm_bwd_kernel<E, LAYER, false, CKPT, 2, 1>);
  const int n = launch_maybe_pdl(kern, s.grid, s.nt * s.teams, smem, c.stream, a.wait, a);
  if (n < 0 || !sums || s.grid == 1) return n;
  return sum_parts(a, s.grid, kinds, c.stream) < 0 ? -1 : 2;
}

template <Elem E>
int bwd_type(const NormBwdCall& c) {
  BwdArgs a;
  a.dy = c.dy, a.x = c.x, a.codes = c.codes, a.scales = c.scales, a.gamma = c.gamma, a.mean = c.mean, a.rstd = c.rstd;
  a.dx = c.dx, a.dgamma = c.dgamma, a.dbeta = c.dbeta, a.part = static_cast<float*>(c.workspace);
  a.rows = c.rows, a.cols = c.cols, a.lddy = c.lddy, a.ldx = c.ldx, a.lddx = c.lddx;
  a.pitch = block8_pitch(c.cols), a.spitch = block8_scale_pitch(c.cols), a.part_cols = (c.cols + 3) / 4 * 4;
  a.teams = 1;
  a.params32 = c.params32;
  a.wait = lone_pdl(c.stream);
  const int b = elem_bytes<E>();
  const bool vec = aligned_rows(c.dy, c.lddy, c.rows, b) && aligned_rows(c.dx, c.lddx, c.rows, b) &&
                   (c.x == nullptr || aligned_rows(c.x, c.ldx, c.rows, b));
  if (c.layer) return c.x == nullptr ? bwd<E, true, true>(c, a, vec) : bwd<E, true, false>(c, a, vec);
  return c.x == nullptr ? bwd<E, false, true>(c, a, vec) : bwd<E, false, false>(c, a, vec);
}

}  // namespace

size_t norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  const int64_t part_cols = (cols + 3) / 4 * 4;
  const int64_t parts = cols > kTeamCols ? wide_parts(rows) : bwd_shape(rows, cols).grid;
  return size_t(parts) * 2 * size_t(part_cols) * 4;
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
