// The products of roi_fp8_linear.cu for many tokens: a pair of CTAs shares its MMAs (cta_group::2) and owns a tile of 256 by n, n
// a multiple of 32 up to 224.  Either tokens or outputs are the 256, A's rows: each CTA holds 128 of them and half of B's
// n, and in TMEM the sums of its 128 rows.  The sums are double, 2 x 224 columns, and the scales of four chunks of four blocks
// take the other 64.
//
// Roles of the 12 warps of a CTA, each a loop over the same list of tiles and blocks of 128:
//   warp 0       stages tokens and weight by TMA; both CTAs' copies end on the even CTA's barrier
//   warp 1       of the even CTA: copies of scales to TMEM, and four MMAs a block, for both; commits them to `empty`
//                and, after the last block, to `sum`
//   warps 2, 3   stage scales, every other chunk each: words of four blocks, of the CTA's 128 rows of A and of all n of B
//   warps 4 - 11 read the sums from TMEM and write them out, `free`, while the next tile's MMAs go to the other half; two
//                warps share 32 rows
// Every wait is bounded; a pair of which one gives up lets its copies and MMAs end before it leaves.
//
// Bound by what an SM takes in (64 bytes a cycle) and by the clock under load.  8192 tokens, us (at twice the measured cuBLAS
// bf16 rate, 3764 TFLOP/s, 296): 18944 x 3584 forward 305 (3645 TFLOP/s), 3584 x 18944 330, its input gradient 315, 331 to 344
// for the gradient of 18944 inputs.  On the way: one CTA a tile 480; pairs 320; the weight as A in the gradient 395 -> 331
// (as B, its tiles of 112 columns began between sectors); two warps for the scales 319 -> 305.  Six stages are as good but for
// 2048 tokens of 3584 x 18944 in fp32 (100, 94 with seven); five take 1 to 2 % more, four 3 to 12 %.
#include <atomic>
#include <type_traits>

#include "roi_fp8.cuh"
#include "roi_launch.h"
#include "roi_tc.cuh"
#include "roi_tmap.h"

namespace roi {
namespace {

constexpr int kThreads = 384;
constexpr int kSide = 256;                 // rows of A of a tile
constexpr int kStep = 128;                 // of the sum a stage holds: a block
constexpr int kMaxN = 224;
constexpr int kStages = 7;
constexpr uint32_t kABytes = 128 * kStep, kStageBytes = kABytes + kMaxN / 2 * kStep;
constexpr int kScaleSlots = 4;             // of four blocks' scales: 128 rows of A, up to 256 of B
constexpr uint32_t kScaleBytes = 512 + 1024;
constexpr uint32_t kOffScales = kStages * kStageBytes, kOffBars = kOffScales + kScaleSlots * kScaleBytes;
constexpr int kBars = 2 * kStages + 2 * kScaleSlots + 4;
constexpr uint32_t kOffMisc = kOffBars + kBars * 8, kSmem = kOffMisc + 24;
static_assert(kSmem + 1024 <= 232448, "shared memory");
constexpr uint32_t kTmemCols = 512, kTmemScales = 2 * kMaxN;

struct PairArgs {
  const uint8_t* w_scales;
  const uint8_t* x_scales;
  void* out;
  int64_t T, outs, ldo;
  int64_t w_spitch, x_spitch;
  int w_blocks;    // rows of the weight's scales
  int n;           // rows of B of a tile
  int tiles_m, tiles;
  int groups;      // pairs of CTAs
  int blocks;      // of the sum
  int pieces;      // of the sum, added by the warps that write
  int unbroken;    // blocks of a piece, whole chunks
  uint32_t idesc;
  unsigned int* status;
  bool wait;
};

// A sum in TMEM: blocks k0 .. k1 of a tile.
struct Work {
  int64_t m0, n0;
  int k0, k1;
  bool first, last;  // of a tile's pieces
};
__device__ __forceinline__ bool work_of(const PairArgs& a, int g, int i, Work& w) {
  const int round = i / a.pieces, piece = i - round * a.pieces;
  const int tile = round * a.groups + g;
  if (tile >= a.tiles) return false;
  const int n = tile / a.tiles_m;
  w.m0 = int64_t(tile - n * a.tiles_m) * kSide;
  w.n0 = int64_t(n) * a.n;
  w.k0 = a.unbroken * piece;
  w.k1 = piece == a.pieces - 1 ? a.blocks : w.k0 + a.unbroken;
  w.first = piece == 0;
  w.last = piece == a.pieces - 1;
  return true;
}

// 16 columns of sums, from column c of the tile on, as the warps that write have them: lanes are A's rows, columns B's.
// Tokens in the lanes: a lane writes its token's outputs, whole sectors (rows of out are whole sectors apart; the last of
// a row may end inside one).
template <Elem E>
struct TokenLanes {
  using T = typename ElemType<E>::T;
  T* out;      // the lane's row of out at the tile's first column
  bool there;  // whether it has one
  int width;   // columns of the tile
  __device__ __forceinline__ TokenLanes(const PairArgs& a, const Work& w, int row) {
    const int64_t t = w.m0 + row, left = a.outs - w.n0;
    out = static_cast<T*>(a.out) + t * a.ldo + w.n0;
    there = t < a.T;
    width = left < a.n ? int(left) : a.n;
  }
  __device__ __forceinline__ void store(int c, const RowWords<E, 16>& r) const {
    if (!there) return;
    T* p = out + c;
    if (c + 16 <= width) {
#pragma unroll
      for (int q = 0; q < RowWords<E, 16>::kWords / 8; ++q) store32(reinterpret_cast<uint32_t*>(p) + 8 * q, r.u + 8 * q);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (c + e < width) p[e] = r.at(e);
    }
  }
};
// Outputs in the lanes: a warp writes 32 outputs of a token side by side, wherever rows start.
template <Elem E>
struct OutputLanes {
  using T = typename ElemType<E>::T;
  T* out;  // the lane's output of the tile's first token
  bool there;
  int width;
  int64_t ldo;
  __device__ __forceinline__ OutputLanes(const PairArgs& a, const Work& w, int row) {
    const int64_t o = w.m0 + row, left = a.T - w.n0;
    out = static_cast<T*>(a.out) + w.n0 * a.ldo + o;
    there = o < a.outs;
    width = left < a.n ? int(left) : a.n;
    ldo = a.ldo;
  }
  __device__ __forceinline__ void store(int c, const RowWords<E, 16>& r) const {
    if (!there) return;
    T* p = out + c * ldo;
#pragma unroll
    for (int e = 0; e < 16; ++e, p += ldo)
      if (c + e < width) *p = r.at(e);
  }
};

// OUTPUTS: A is the weight (MN-major in the input gradient), B the tokens; else A is the tokens (forward only).
template <bool DGRAD, bool OUTPUTS, Elem E>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    roi_fp8_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b, PairArgs a) {
  static_assert(OUTPUTS || !DGRAD, "the weight is A where it is MN-major: whole tiles of 128 columns are aligned");
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  // `full`, `scale_full` and `free` are the even CTA's, on which both arrive; the others each CTA's own
  uint64_t *full = bars, *empty = full + kStages, *scale_full = empty + kStages, *scale_empty = scale_full + kScaleSlots;
  uint64_t *sum = scale_empty + kScaleSlots, *free = sum + 2;
  // [0] TMEM base; [1] ok; blocks whose copies were sent off, and ok, of CTA 0 in [2] and [3], of CTA 1 in [4] and [5]
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + kOffMisc);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int g = blockIdx.x / 2;

  if (tid == 32) prefetch_tensor_map(&tm_a), prefetch_tensor_map(&tm_b);
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
      mbar_init(free + b, 8 * 2);
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
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int m = int(w.m0) + int(rank) * 128, n = int(w.n0) + int(rank) * half;
      for (int k = w.k0; k < w.k1; ++k, ++issued, ring.next()) {
        ok = agreed(mbar_wait_ring_cluster(empty + ring.at, ring.pass ^ 1u, lim));
        if (!ok) break;
        uint8_t* st = smem + ring.at * kStageBytes;
        if (elect_one()) {
          if (rank == 0) mbar_arrive_expect_tx(full + ring.at, 2 * (kABytes + uint32_t(half) * kStep));
          const uint32_t bar = cluster_addr(full + ring.at, 0);
          if constexpr (DGRAD) tma_load_2d_pair(st, &tm_a, m, k * kStep, bar);
          else tma_load_2d_pair(st, &tm_a, k * kStep, m, bar);
          tma_load_2d_pair(st + kABytes, &tm_b, k * kStep, n, bar);
        }
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint64_t a0 = DGRAD ? tc_smem_desc_mn128(smem_addr(smem), kABytes) : tc_smem_desc_k128(smem_addr(smem));
      const uint64_t b0 = tc_smem_desc_k128(smem_addr(smem + kABytes));
      const uint32_t scales0 = smem_addr(smem + kOffScales);
      for (int i = 0; ok && work_of(a, g, i, w); ++i) {
        const int b = i & 1;
        ok = agreed(mbar_wait_ring_cluster(free + b, (uint32_t(i >> 1) & 1u) ^ 1u, lim));
        const uint32_t d = tmem + uint32_t(b) * kMaxN;
        for (int k = w.k0; ok && k < w.k1; ++k, ++committed, ring.next()) {
          const bool fresh = (k & 3) == 0, last = (k & 3) == 3 || k == w.k1 - 1;
          if (fresh) ok = agreed(mbar_wait_ring_cluster(scale_full + slot.at, slot.pass, lim));
          if (ok) ok = agreed(mbar_wait_ring_cluster(full + ring.at, ring.pass, lim));
          if (!ok) break;
          tc_fence_after();
          const uint64_t ad = a0 + uint32_t(ring.at) * (kStageBytes / 16), bd = b0 + uint32_t(ring.at) * (kStageBytes / 16);
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
              tc_mma_mxf8_pair(d, ad + s * (DGRAD ? 4096 / 16 : 32 / 16), bd + s * (32 / 16), idesc, sa, sb, s > 0 || k > w.k0);
            tc_commit_pair(empty + ring.at);
            if (last) tc_commit_pair(scale_empty + slot.at);
            if (k == w.k1 - 1) tc_commit_pair(sum + b);
          }
          __syncwarp();
          if (last) slot.next();
        }
      }
    }
  } else if (warp < 4) {
    uint32_t chunk = 0;  // of all
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int64_t row = w.m0 + int64_t(rank) * 128;  // A's first here
      // the weight's blocks of 128 outputs: A's one here, or the three at most that B's n lie in
      constexpr int kWords = OUTPUTS ? 1 : 3;
      const int64_t block = (OUTPUTS ? row : w.n0) / 128, t0 = OUTPUTS ? w.n0 : row;
      for (int k = w.k0; k < w.k1; k += 4, slot.next(), ++chunk) {
        if ((chunk & 1u) != uint32_t(warp & 1)) continue;
        uint32_t word[kWords];
        if constexpr (DGRAD) {
          // (a block of the sum is a row of scales)
          uint32_t byte = 0x7fu;
          if (lane < 4 && k + lane < a.w_blocks && block < a.w_spitch) byte = a.w_scales[int64_t(k + lane) * a.w_spitch + block];
          byte <<= 8 * (lane & 3);
          byte |= __shfl_xor_sync(0xffffffffu, byte, 1);
          byte |= __shfl_xor_sync(0xffffffffu, byte, 2);
          word[0] = __shfl_sync(0xffffffffu, byte, 0);
        } else {
#pragma unroll
          for (int j = 0; j < kWords; ++j)
            word[j] = block + j < a.w_blocks ? *reinterpret_cast<const uint32_t*>(a.w_scales + (block + j) * a.w_spitch + k) : 0x7f7f7f7fu;
        }
        uint32_t x[8], o[8];
#pragma unroll
        for (int q = 0; q < (OUTPUTS ? 8 : 4); ++q) {
          const int64_t t = t0 + 32 * q + lane;
          x[q] = t < a.T && (!OUTPUTS || 32 * q < a.n) ? *reinterpret_cast<const uint32_t*>(a.x_scales + t * a.x_spitch + k) : 0x7f7f7f7fu;
        }
#pragma unroll
        for (int q = 0; q < (OUTPUTS ? 4 : 8); ++q) {
          if constexpr (OUTPUTS) {
            o[q] = word[0];
          } else {
            const int64_t j = (w.n0 + 32 * q + lane) / 128 - block;
            o[q] = j == 0 ? word[0] : j == 1 ? word[1] : word[2];
          }
        }
        ok = agreed(mbar_wait_ring_cluster(scale_empty + slot.at, slot.pass ^ 1u, lim));
        if (!ok) break;
        uint8_t* to = smem + kOffScales + slot.at * kScaleBytes + 16 * lane;
        const uint32_t(&ra)[8] = OUTPUTS ? o : x, (&rb)[8] = OUTPUTS ? x : o;
        *reinterpret_cast<uint4*>(to) = make_uint4(ra[0], ra[1], ra[2], ra[3]);
        *reinterpret_cast<uint4*>(to + 512) = make_uint4(rb[0], rb[1], rb[2], rb[3]);
        *reinterpret_cast<uint4*>(to + 1024) = make_uint4(rb[4], rb[5], rb[6], rb[7]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(scale_full + slot.at, 0);
      }
    }
  } else if (warp >= 4) {
    using Lanes = std::conditional_t<OUTPUTS, OutputLanes<E>, TokenLanes<E>>;
    const int quarter = warp & 3, part = (warp - 4) >> 2;  // 32 rows, and every other 16 columns
    constexpr int kChunks = kMaxN / 32;
    // They leave TMEM before any is written: in 16 bits, or, fp32, added to what earlier pieces left.
    RowWords<E, 16> kept[kChunks];
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int b = i & 1;
      const Lanes out(a, w, int(rank) * 128 + quarter * 32 + lane);
      ok = agreed(mbar_wait_ring_cluster(sum + b, uint32_t(i >> 1) & 1u, lim));
      if (!ok) break;
      tc_fence_after();
      const uint32_t from = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(b * kMaxN + 16 * part);
#pragma unroll
      for (int q = 0; q < kChunks; ++q) {
        // (columns past the tile's are read, and not written)
        uint32_t u[16];
        tc_ld16(from + 32 * q, u);
        if constexpr (E == Elem::kFp32) {
#pragma unroll
          for (int e = 0; e < 16; ++e) kept[q].u[e] = __float_as_uint(__uint_as_float(w.first ? 0u : kept[q].u[e]) + __uint_as_float(u[e]));
        } else {
          float v[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(u[e]);
          kept[q].set(v);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_tmem(free + b, 0);
      if (!w.last) continue;
#pragma unroll
      for (int q = 0; q < kChunks; ++q) {
        const int c = 16 * (2 * q + part);
        if (c < out.width) out.store(c, kept[q]);
      }
    }
  }
  if (!ok) misc[1] = 0u;
  __syncthreads();
  tc_fence_after();
  if (tid < 2) {  // (of warp 0, which sent the copies off)
    const uint32_t at = cluster_addr(misc + 2 + 2 * rank, uint32_t(tid));
    store_cluster(at, uint32_t(issued));
    store_cluster(at + 4, misc[1]);
  }
  cluster_sync();
  if ((misc[3] & misc[5]) == 0u) {
    // a wait gave up: MMAs end, and the copies that were sent off land, before the pair leaves.  Both CTAs' land on
    // the even CTA's barriers; a stage that only one of them filled is done without the other's bytes.
    if (rank == 0 && tid == 0) {
      const uint32_t bytes = kABytes + uint32_t(half) * kStep;
      const int n0 = int(misc[2]), n1 = int(misc[4]), n = n0 > n1 ? n0 : n1;
      for (int c = n > kStages ? n - kStages : 0; c < n; ++c) {
        uint64_t* bar = full + c % kStages;
        if (c >= n1) mbar_complete_tx(bar, bytes);
        else if (c >= n0) mbar_arrive_expect_tx(bar, bytes);
        mbar_wait_bounded(bar, uint32_t(c / kStages) & 1u);
      }
    }
    if (warp == 1 && committed > 0)
      mbar_wait_bounded(empty + (committed - 1) % kStages, uint32_t((committed - 1) / kStages) & 1u);
    if (tid == 0) atomicOr(a.status, kStatusTimeout);
    __syncthreads();
    cluster_sync();
  }
  if (warp == 0) tc_dealloc_pair(tmem, kTmemCols);
}

template <bool DGRAD, bool OUTPUTS, Elem E>
int launch(const CUtensorMap& tm_a, const CUtensorMap& tm_b, const PairArgs& a, int grid, cudaStream_t stream) {
  auto kern = roi_fp8_pair_kernel<DGRAD, OUTPUTS, E>;
  constexpr size_t smem = kSmem + 1024;
  static std::atomic<bool> set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  if (!set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return -1;
    set[dev].store(true, std::memory_order_release);
  }
  return launch_maybe_pdl(kern, grid, kThreads, smem, stream, a.wait, tm_a, tm_b, a);
}

template <bool DGRAD, bool OUTPUTS>
int launch_of(Elem e, const CUtensorMap& tm_a, const CUtensorMap& tm_b, const PairArgs& a, int grid, cudaStream_t stream) {
  switch (e) {
    case Elem::kBf16: return launch<DGRAD, OUTPUTS, Elem::kBf16>(tm_a, tm_b, a, grid, stream);
    case Elem::kFp16: return launch<DGRAD, OUTPUTS, Elem::kFp16>(tm_a, tm_b, a, grid, stream);
    default: return launch<DGRAD, OUTPUTS, Elem::kFp32>(tm_a, tm_b, a, grid, stream);
  }
}

// A block's stage brings an SM 128 rows of A and n / 2 of B, 64 bytes a cycle: 256 + n cycles, where its MMAs take 2 n.  Measured
// a round of tiles (8192 tokens, 3584 x 18944), n = 128, 160, 192, 224: 39.1, 42.0, 46.1, 48.9 us, 0.10 us per 256 + n.
// What a tile, and the launch, cost besides is from a sweep over 1 to 4096 tokens of seven layers.
constexpr int kTileCycles = 2000, kLaunchCycles = 4000;
// Finds the n of the least time for tiles of `m` by n outputs; returns that time in cycles.
int64_t rows_of_b(int64_t m, int64_t n, int blocks, int groups, int& best) {
  int64_t least = INT64_MAX;
  for (int b = kMaxN; b >= 64; b -= 32) {
    const int64_t tiles = ((m + kSide - 1) / kSide) * ((n + b - 1) / b);
    const int64_t time = (tiles + groups - 1) / groups * (int64_t(256 + b) * blocks + kTileCycles) + kLaunchCycles;
    if (time < least) least = time, best = b;
  }
  return least;
}

// The most blocks of an unbroken sum for fp32 results.  The tensor cores drop the bits below their sum's last instead of
// rounding, an error that grows with the sum: 1.4e-6 of the result's norm over 18944, where an fp32 product has 2.1e-7.
// Pieces of 64, 32, 16 blocks: 3.5e-7, 2.0e-7, 1.2e-7.
constexpr int kMostBlocks = 16;

}  // namespace

// Tokens in the lanes need whole sectors of out and K-major weights.
bool fp8_pair_tokens(const Fp8LinearCall& c) {
  const int b = c.dtype == Elem::kFp32 ? 4 : 2;
  return !c.dgrad && (reinterpret_cast<uintptr_t>(c.out) & 31u) == 0 && c.ldo * b % 32 == 0;
}

int64_t fp8_pair_cycles(int64_t T, int64_t outs, int64_t width, bool tokens, int groups, Fp8PairPlan& plan) {
  const int blocks = int((width + kStep - 1) / kStep);
  const int64_t by_outputs = rows_of_b(outs, T, blocks, groups, plan.n);
  plan.outputs = true;
  if (!tokens) return by_outputs;
  int n;
  const int64_t by_tokens = rows_of_b(T, outs, blocks, groups, n);
  if (by_tokens > by_outputs) return by_outputs;
  plan = {n, false};
  return by_tokens;
}

int launch_fp8_pair(const Fp8LinearCall& c, const Fp8PairPlan& plan) {
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
  a.unbroken = c.dtype == Elem::kFp32 ? kMostBlocks : (a.blocks + 3) / 4 * 4;
  a.pieces = (a.blocks + a.unbroken - 1) / a.unbroken;
  a.groups = sm_count() / 2;
  a.n = plan.n;
  const bool outputs = plan.outputs;
  const int64_t m = outputs ? outs : c.T, n = outputs ? c.T : outs;
  a.tiles_m = int((m + kSide - 1) / kSide);
  a.tiles = int(a.tiles_m * ((n + a.n - 1) / a.n));
  a.idesc = outputs ? tc_idesc_mxf8(kSide, a.n, int(Fp8::kE4M3), int(c.format), c.dgrad, false)
                    : tc_idesc_mxf8(kSide, a.n, int(c.format), int(Fp8::kE4M3), false, false);
  a.status = c.status;
  a.wait = lone_pdl(c.stream);
  const int64_t w_pitch = fp8_pitch(c.cols), x_pitch = fp8_pitch(width);
  auto map = [](CUtensorMap* t, const uint8_t* codes, int64_t pitch, int64_t rows, int box) {
    return make_tensor_map(t, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, uint64_t(pitch), uint64_t(rows), uint64_t(pitch), 128, uint32_t(box),
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
  };
  CUtensorMap tm_w, tm_x;
  if (!map(&tm_w, c.w_codes, w_pitch, c.rows, outputs ? 128 : a.n / 2) || !map(&tm_x, c.x_codes, x_pitch, c.T, outputs ? a.n / 2 : 128))
    return -1;
  const int grid = 2 * (a.tiles < a.groups ? a.tiles : a.groups);
  if (c.dgrad) return launch_of<true, true>(c.dtype, tm_w, tm_x, a, grid, c.stream);
  return outputs ? launch_of<false, true>(c.dtype, tm_w, tm_x, a, grid, c.stream)
                 : launch_of<false, false>(c.dtype, tm_x, tm_w, a, grid, c.stream);
}

}  // namespace roi
