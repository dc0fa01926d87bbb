// The products of roi_fp8_linear.cu for many tokens: a pair of CTAs shares its MMAs (cta_group::2) and owns a tile of 256 tokens
// by n outputs, n a multiple of 32 up to 224; each CTA holds 128 tokens, half of the outputs, and in TMEM the
// sums of its 128 tokens.  The sums are double: 2 x 224 columns, and the scales of four chunks of four blocks take the other 64.
//
// Roles of the 8 warps of a CTA, each a loop over the same list of tiles and blocks of 128:
//   warp 0      stages tokens and weight by TMA; both CTAs' copies end on the even CTA's barrier
//   warp 1      of the even CTA: copies of scales to TMEM, and four MMAs a block, for both; commits them to `empty`
//               and, after the last block, to `sum`
//   warp 2      stages scales: words of four blocks, of the CTA's 128 tokens and of the tile's outputs
//   warps 4 - 7 read the sums from TMEM and write them out, `free`, while the next tile's MMAs go to the other half
// Every wait is bounded; a CTA that gives up lets its copies and MMAs end before it leaves.
#include <atomic>

#include "roi_fp8.cuh"
#include "roi_launch.h"
#include "roi_tc.cuh"
#include "roi_tmap.h"

namespace roi {
namespace {

constexpr int kThreads = 256;
constexpr int kSide = 256;                 // tokens of a tile
constexpr int kStep = 128;                 // of the sum a stage holds: a block
constexpr int kMaxN = 224;
constexpr int kStages = 6;
constexpr uint32_t kABytes = 128 * kStep, kStageBytes = 2 * kABytes;
constexpr int kScaleSlots = 4;             // of four blocks' scales: 128 tokens, up to 256 outputs
constexpr uint32_t kScaleBytes = 512 + 1024;
constexpr uint32_t kOffScales = kStages * kStageBytes, kOffBlocks = kOffScales + kScaleSlots * kScaleBytes;
constexpr int kBlockPitch = 33;            // 32 rows of 32 sums for each of the warps that write, where rows are not whole sectors
constexpr uint32_t kOffBars = kOffBlocks + 4 * 32 * kBlockPitch * 4;
constexpr int kBars = 2 * kStages + 2 * kScaleSlots + 4;
constexpr uint32_t kOffMisc = kOffBars + kBars * 8, kSmem = kOffMisc + 8;
static_assert(kSmem + 1024 <= 232448, "shared memory");
constexpr uint32_t kTmemCols = 512, kTmemScales = 2 * kMaxN;

struct PairArgs {
  const uint8_t* w_scales;
  const uint8_t* x_scales;
  void* out;
  int64_t T, outs, ldo;
  int64_t w_spitch, x_spitch;
  int w_blocks;    // rows of the weight's scales
  int n;           // outputs of a tile
  int tiles_m, tiles;
  int groups;      // pairs of CTAs
  int blocks;      // of the sum
  int pieces;      // of the sum, added in out
  uint32_t idesc;
  bool sectors;    // rows of out are whole sectors apart
  unsigned int* status;
  bool wait;
};

// A sum in TMEM: blocks k0 .. k1 of a tile; pieces after the first are added to out.
struct Work {
  int64_t m0, n0;
  int k0, k1;
  bool first;
};
__device__ __forceinline__ bool work_of(const PairArgs& a, int g, int i, Work& w) {
  const int round = i / a.pieces, piece = i - round * a.pieces;
  const int tile = round * a.groups + g;
  if (tile >= a.tiles) return false;
  const int n = tile / a.tiles_m;
  w.m0 = int64_t(tile - n * a.tiles_m) * kSide;
  w.n0 = int64_t(n) * a.n;
  w.k0 = int(int64_t(a.blocks) * piece / a.pieces);
  w.k1 = int(int64_t(a.blocks) * (piece + 1) / a.pieces);
  w.first = piece == 0;
  return true;
}

// 32 columns of a row of the sums from column n on, where rows are whole sectors (the last may end inside one).
template <Elem E>
__device__ __forceinline__ void store_sectors(const PairArgs& a, bool first, int64_t m, int64_t n, const float (&v)[32], int width) {
  using T = typename ElemType<E>::T;
  constexpr int kPer = 32 / int(sizeof(T));  // columns of a sector
  T* out = static_cast<T*>(a.out) + m * a.ldo + n;
#pragma unroll
  for (int q = 0; q < 32 / kPer; ++q) {
    if (kPer * q + kPer <= width) {
      uint32_t w[8];
      if constexpr (E == Elem::kFp32) {
        if (!first) {
          asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                       : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                       : "l"(out + 8 * q)
                       : "memory");
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) + v[8 * q + e]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[8 * q + e]);
        }
      } else {
        RowWords<E, 16> r;
        float x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = v[16 * q + e];
        r.set(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = r.u[e];
      }
      store32(out + kPer * q, w);
    } else {
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        if (kPer * q + e >= width) break;
        float x = v[kPer * q + e];
        if (E == Elem::kFp32 && !first) x += to_f32<E>(out[kPer * q + e]);
        out[kPer * q + e] = from_f32<E>(x);
      }
    }
  }
}
// Any other rows (the whole warp, rows m0 on): through shared memory, so that a warp writes consecutive columns of a row.
template <Elem E>
__device__ __forceinline__ void store_block(const PairArgs& a, bool first, float* block, int64_t m0, int64_t n, const float (&v)[32],
                                            int width) {
  using T = typename ElemType<E>::T;
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll
  for (int e = 0; e < 32; ++e) block[lane * kBlockPitch + e] = v[e];
  __syncwarp();
  const int64_t below = a.T - m0;
  const int rows = lane >= width || below <= 0 ? 0 : below > 32 ? 32 : int(below);
  T* out = static_cast<T*>(a.out) + m0 * a.ldo + n + lane;
#pragma unroll 8
  for (int r = 0; r < rows; ++r, out += a.ldo) {
    float x = block[r * kBlockPitch + lane];
    if (E == Elem::kFp32 && !first) x += to_f32<E>(*out);
    *out = from_f32<E>(x);
  }
}

template <bool DGRAD, Elem E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    roi_fp8_pair_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, PairArgs a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  // `full`, `scale_full` and `free` are the even CTA's, on which both arrive; the others each CTA's own
  uint64_t *full = bars, *empty = full + kStages, *scale_full = empty + kStages, *scale_empty = scale_full + kScaleSlots;
  uint64_t *sum = scale_empty + kScaleSlots, *free = sum + 2;
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + kOffMisc);  // [0] TMEM base, [1] ok
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int g = blockIdx.x / 2;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      mbar_init(scale_full + s, 2);
      mbar_init(scale_empty + s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(sum + b, 1);
      mbar_init(free + b, 4 * 2);
    }
    misc[1] = 1u;
    fence_mbar_init();
  }
  if (warp == 0) tc_alloc_pair(misc, kTmemCols);
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  pdl_begin(a.wait);

  const uint64_t lim = ring_wait_limit(a.status);
  bool ok = true;
  int issued = 0, committed = 0;
  Work w;
  TcRing<kStages> ring;
  TcRing<kScaleSlots> slot;
  // (a warp goes on or gives up as one)
  auto agreed = [](bool mine) { return __all_sync(0xffffffffu, mine) != 0; };
  const int half = a.n / 2;
  if (warp == 0) {
    const uint32_t b_bytes = DGRAD ? kABytes : uint32_t(half) * kStep;
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int m = int(w.m0) + int(rank) * 128, n = int(w.n0) + int(rank) * half;
      for (int k = w.k0; k < w.k1; ++k, ++issued, ring.next()) {
        ok = agreed(mbar_wait_ring_cluster(empty + ring.at, ring.pass ^ 1u, lim));
        if (!ok) break;
        uint8_t* st = smem + ring.at * kStageBytes;
        if (elect_one()) {
          if (rank == 0) mbar_arrive_expect_tx(full + ring.at, 2 * (kABytes + b_bytes));
          const uint32_t bar = cluster_addr(full + ring.at, 0);
          tma_load_2d_pair(st, &tm_x, k * kStep, m, bar);
          if constexpr (DGRAD) tma_load_2d_pair(st + kABytes, &tm_w, n, k * kStep, bar);
          else tma_load_2d_pair(st + kABytes, &tm_w, k * kStep, n, bar);
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint64_t x0 = tc_smem_desc_k128(smem_addr(smem));
      const uint64_t w0 = DGRAD ? tc_smem_desc_mn128(smem_addr(smem + kABytes), kABytes) : tc_smem_desc_k128(smem_addr(smem + kABytes));
      const uint32_t scales0 = smem_addr(smem + kOffScales);
      for (int i = 0; ok && work_of(a, g, i, w); ++i) {
        const int b = i & 1;
        ok = agreed(mbar_wait_ring_cluster(free + b, (uint32_t(i >> 1) & 1u) ^ 1u, lim));
        const uint32_t d = tmem + uint32_t(b) * kMaxN;
        for (int k = w.k0; ok && k < w.k1; ++k, ++committed, ring.next()) {
          const bool fresh = k == w.k0 || (k & 3) == 0, last = (k & 3) == 3 || k == w.k1 - 1;
          if (fresh) ok = agreed(mbar_wait_ring_cluster(scale_full + slot.at, slot.pass, lim));
          if (ok) ok = agreed(mbar_wait_ring_cluster(full + ring.at, ring.pass, lim));
          if (!ok) break;
          tc_fence_after();
          const uint64_t x = x0 + uint32_t(ring.at) * (kStageBytes / 16), v = w0 + uint32_t(ring.at) * (kStageBytes / 16);
          const uint32_t idesc = tc_idesc_scale_byte(a.idesc, uint32_t(k) & 3u);
          const uint32_t sa = tmem + kTmemScales + uint32_t(slot.at) * 16, sb = sa + 4;
          if (elect_one()) {
            if (fresh) {
              const uint32_t from = scales0 + slot.at * kScaleBytes;
              tc_copy_scales_pair(sa, from);
              tc_copy_scales_pair(sb, from + 512);
              tc_copy_scales_pair(sb + 4, from + 1024);
            }
#pragma unroll
            for (int s = 0; s < kStep / 32; ++s)
              tc_mma_mxf8_pair(d, x + s * (32 / 16), v + s * (DGRAD ? 4096 / 16 : 32 / 16), idesc, sa, sb, s > 0 || k > w.k0);
            tc_commit_pair(empty + ring.at);
            if (last) tc_commit_pair(scale_empty + slot.at);
            if (k == w.k1 - 1) tc_commit_pair(sum + b);
          }
          __syncwarp();
          if (last) slot.next();
        }
      }
    }
  } else if (warp == 2) {
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int64_t t = w.m0 + int64_t(rank) * 128 + lane, b0 = w.n0 / 128;
      for (int k = w.k0 & ~3; k < w.k1; k += 4, slot.next()) {
        uint32_t x[4], word[3] = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
#pragma unroll
        for (int q = 0; q < 4; ++q)
          x[q] = t + 32 * q < a.T ? *reinterpret_cast<const uint32_t*>(a.x_scales + (t + 32 * q) * a.x_spitch + k) : 0x7f7f7f7fu;
        // the tile's outputs lie in three blocks of 128 at most
        if constexpr (DGRAD) {
          const int block = lane >> 2, row = k + (lane & 3);
          uint32_t byte = 0x7fu;
          if (block < 3 && b0 + block < a.w_spitch && row < a.w_blocks) byte = a.w_scales[int64_t(row) * a.w_spitch + b0 + block];
          byte <<= 8 * (lane & 3);
          byte |= __shfl_xor_sync(0xffffffffu, byte, 1);
          byte |= __shfl_xor_sync(0xffffffffu, byte, 2);
#pragma unroll
          for (int j = 0; j < 3; ++j) word[j] = __shfl_sync(0xffffffffu, byte, 4 * j);
        } else {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (b0 + j < a.w_blocks) word[j] = *reinterpret_cast<const uint32_t*>(a.w_scales + (b0 + j) * a.w_spitch + k);
        }
        uint32_t o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int64_t j = (w.n0 + 32 * q + lane) / 128 - b0;
          o[q] = j == 0 ? word[0] : j == 1 ? word[1] : word[2];
        }
        ok = agreed(mbar_wait_ring_cluster(scale_empty + slot.at, slot.pass ^ 1u, lim));
        if (!ok) break;
        uint8_t* to = smem + kOffScales + slot.at * kScaleBytes + 16 * lane;
        *reinterpret_cast<uint4*>(to) = make_uint4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<uint4*>(to + 512) = make_uint4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<uint4*>(to + 1024) = make_uint4(o[4], o[5], o[6], o[7]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(scale_full + slot.at, 0);
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    float* block = reinterpret_cast<float*>(smem + kOffBlocks) + quarter * 32 * kBlockPitch;
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int b = i & 1;
      const int64_t m = w.m0 + int64_t(rank) * 128 + quarter * 32 + lane;
      ok = agreed(mbar_wait_ring_cluster(sum + b, uint32_t(i >> 1) & 1u, lim));
      if (!ok) break;
      tc_fence_after();
      const int64_t left = a.outs - w.n0;
      const int width = left < a.n ? int(left) : a.n;
      for (int c = 0; c < width; c += 32) {
        uint32_t u[32];
        tc_ld32(tmem + (uint32_t(quarter * 32) << 16) + uint32_t(b * kMaxN + c), u);
        float v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(u[e]);
        const int cols = width - c < 32 ? width - c : 32;
        if (a.sectors) {
          if (m < a.T) store_sectors<E>(a, w.first, m, w.n0 + c, v, cols);
        } else {
          store_block<E>(a, w.first, block, m - lane, w.n0 + c, v, cols);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(free + b, 0);
    }
  }
  if (!ok) misc[1] = 0u;
  __syncthreads();
  if (misc[1] == 0u) {
    // a wait gave up: MMAs end, and the copies that were sent off land, before it leaves (on the even CTA's barriers,
    // where both CTAs' land; a stage that only one of them filled runs out of time)
    if (warp == 0 && rank == 0)
      for (int c = issued > kStages ? issued - kStages : 0; c < issued; ++c)
        if (!mbar_wait_bounded(full + c % kStages, uint32_t(c / kStages) & 1u)) break;
    if (warp == 1 && committed > 0)
      mbar_wait_bounded(empty + (committed - 1) % kStages, uint32_t((committed - 1) / kStages) & 1u);
    if (tid == 0) atomicOr(a.status, kStatusTimeout);
    __syncthreads();
  }
  tc_fence_after();
  cluster_sync();
  if (warp == 0) tc_dealloc_pair(tmem, kTmemCols);
}

template <bool DGRAD, Elem E>
int launch(const CUtensorMap& tm_x, const CUtensorMap& tm_w, const PairArgs& a, int grid, cudaStream_t stream) {
  auto kern = roi_fp8_pair_kernel<DGRAD, E>;
  constexpr size_t smem = kSmem + 1024;
  static std::atomic<bool> set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  if (!set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return -1;
    set[dev].store(true, std::memory_order_release);
  }
  return launch_maybe_pdl(kern, grid, kThreads, smem, stream, a.wait, tm_x, tm_w, a);
}

template <bool DGRAD>
int launch_of(Elem e, const CUtensorMap& tm_x, const CUtensorMap& tm_w, const PairArgs& a, int grid, cudaStream_t stream) {
  switch (e) {
    case Elem::kBf16: return launch<DGRAD, Elem::kBf16>(tm_x, tm_w, a, grid, stream);
    case Elem::kFp16: return launch<DGRAD, Elem::kFp16>(tm_x, tm_w, a, grid, stream);
    default: return launch<DGRAD, Elem::kFp32>(tm_x, tm_w, a, grid, stream);
  }
}

// The fewest rounds of tiles over the pairs, each as long as its outputs (and what a tile costs besides, in outputs).
constexpr int kTileCost = 16;
int outputs_of(int64_t tiles_m, int64_t outs, int groups) {
  int best = kMaxN;
  int64_t least = INT64_MAX;
  for (int n = kMaxN; n >= 64; n -= 32) {
    const int64_t tiles = tiles_m * ((outs + n - 1) / n), rounds = (tiles + groups - 1) / groups;
    if (rounds * (n + kTileCost) < least) least = rounds * (n + kTileCost), best = n;
  }
  return best;
}

// The most blocks of an unbroken sum for fp32 results (the tensor cores drop what is below a sum's last bit).
constexpr int kMostBlocks = 16;

}  // namespace

int launch_fp8_pair(const Fp8LinearCall& c) {
  PairArgs a;
  const int64_t outs = c.dgrad ? c.cols : c.rows, width = c.dgrad ? c.rows : c.cols;
  a.w_scales = c.w_scales;
  a.x_scales = c.x_scales;
  a.out = c.out;
  a.T = c.T;
  a.outs = outs;
  a.ldo = c.ldo;
  a.w_spitch = fp8_scale_pitch(c.cols);
  a.x_spitch = fp8_scale_pitch(width);
  a.w_blocks = int((c.rows + 127) / 128);
  a.blocks = int((width + kStep - 1) / kStep);
  a.pieces = c.dtype == Elem::kFp32 ? (a.blocks + kMostBlocks - 1) / kMostBlocks : 1;
  a.groups = sm_count() / 2;
  a.tiles_m = int((c.T + kSide - 1) / kSide);
  a.n = outputs_of(a.tiles_m, outs, a.groups);
  a.tiles = int(a.tiles_m * ((outs + a.n - 1) / a.n));
  a.idesc = tc_idesc_mxf8(kSide, a.n, int(c.format), int(Fp8::kE4M3), false, c.dgrad);
  const int b = c.dtype == Elem::kFp32 ? 4 : 2;
  a.sectors = (reinterpret_cast<uintptr_t>(c.out) & 31u) == 0 && c.ldo * b % 32 == 0;
  a.status = c.status;
  a.wait = lone_pdl(c.stream);
  CUtensorMap tm_w, tm_x;
  const int64_t w_pitch = fp8_pitch(c.cols), x_pitch = fp8_pitch(width);
  if (!make_tensor_map(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.w_codes, uint64_t(w_pitch), uint64_t(c.rows), uint64_t(w_pitch), 128,
                       c.dgrad ? kStep : uint32_t(a.n) / 2, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      !make_tensor_map(&tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.x_codes, uint64_t(x_pitch), uint64_t(c.T), uint64_t(x_pitch), kStep, 128,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
    return -1;
  const int grid = 2 * (a.tiles < a.groups ? a.tiles : a.groups);
  return c.dgrad ? launch_of<true>(c.dtype, tm_x, tm_w, a, grid, c.stream) : launch_of<false>(c.dtype, tm_x, tm_w, a, grid, c.stream);
}

}  // namespace roi
