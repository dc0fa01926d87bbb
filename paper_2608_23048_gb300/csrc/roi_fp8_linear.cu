// Products of a masked layer's weight with activations, both in 8-bit floating point with a power of two for each
// block of 128 (roi_fp8.cuh):
//   forward         Y[t, o]  = sum_i x^[t, i] w^[o, i]
//   input gradient  dX[t, i] = sum_o dy^[t, o] w^[o, i]
// on the fifth-generation tensor cores' block-scaled instructions, which multiply 32 products by both blocks' powers of two
// and add them to fp32 sums: a scale byte serves four steps.
//
// The weight is the product's A (128 outputs of the tile in the lanes of TMEM), the tokens are B, so that few tokens
// make narrow tiles.  A's tile is K-major in the forward and MN-major in the input gradient (one copy of the weight serves
// both); tokens are K-major.  A CTA has one tile of 128 outputs by `n` tokens, or, where the tiles are
// fewer than the SMs, a range of its sum: the CTAs of a tile are a cluster, copy their sums into one another's shared memory and
// add them in the order of the ranges, each for some of the tokens.  Many tokens go to roi_fp8_pair.cu.
//
// One token of 18944 x 3584 is bound by the weight's bytes, 10 us of 12.8 from memory, call after call; the rest is a call's start
// and end.  What ranges of a sum give, call after call in a graph, weights in L2, by the ranges that plan() takes: one token of
// 3584 x 18944 in five 16.0 us, in one 46.3; 200 tokens of 640 x 6000 (fp32) in eight 10.8, in one 16.9, in five 9.7; 37 tokens of
// 896 x 4864 in eight 9.0, in one 14.2, in five 8.6; 37 of 1565 x 1941 in eight 8.5, in one 7.8, in four 7.2: what a range costs is
// more for many of them than plan() counts.  One range, as taken: the gradient of 777 tokens, 1001 x 1531, 6.5 (in two 10.0), 37
// tokens of 128 x 896 5.0 (6.3 to 6.9 in two to seven).
#include <atomic>

#include "roi_fp8.cuh"
#include "roi_launch.h"
#include "roi_tc.cuh"
#include "roi_tmap.h"

namespace roi {
namespace {

constexpr int kThreads = 128;
constexpr int kStep = 128;                      // of the sum a stage holds: a block
constexpr uint32_t kABytes = 128 * kStep;
constexpr uint32_t kRingBytes = 204800;         // for the stages
constexpr int kMaxStages = 11;                  // 16 tokens
constexpr int kScaleSlots = 4;                  // of four blocks' scales: 128 outputs, 256 tokens
constexpr uint32_t kScaleBytes = 512 + 1024;
constexpr uint32_t kOffScales = kRingBytes, kOffBars = kOffScales + kScaleSlots * kScaleBytes;
constexpr int kBars = 2 * kMaxStages + 2 * kScaleSlots + 2;
constexpr uint32_t kOffMisc = kOffBars + kBars * 8, kSmem = kOffMisc + 40;
static_assert(kSmem + 1024 <= 232448, "shared memory");

struct LinearArgs {
  const uint8_t* w_scales;
  const uint8_t* x_scales;
  void* out;
  int64_t T, outs, ldo;
  int64_t w_spitch, x_spitch;
  int w_blocks;   // rows of the weight's scales
  int n;          // tokens of a tile
  int tiles_o;
  int splits;     // ranges of a tile's sum: CTAs of a cluster
  int blocks;     // of the sum
  int unbroken;   // the most blocks of a sum in TMEM: the next ones have columns of their own
  int stages;
  int ahead;      // blocks of the weight that are sent for before the work before this call is done
  uint32_t idesc, tmem_cols;
  unsigned int* status;
  bool wait;
};

constexpr uint32_t kGroupBytes = 16 * 128 * 4;  // the sums of 16 tokens

template <bool DGRAD, Elem E>
__global__ void __launch_bounds__(kThreads, 1)
    roi_fp8_linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, LinearArgs a) {
  using T = typename ElemType<E>::T;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t *full = bars, *empty = full + kMaxStages, *scale_full = empty + kMaxStages, *scale_empty = scale_full + kScaleSlots;
  uint64_t *done = scale_empty + kScaleSlots, *joined = done + 1;
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + kOffMisc);  // [0] TMEM base, [1] ok, [2 + r] whether CTA r of the cluster has sums
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = a.splits > 1 ? int(cluster_rank()) : 0;
  const int tile = blockIdx.x / a.splits;
  const int64_t o0 = int64_t(tile % a.tiles_o) * 128, t0 = int64_t(tile / a.tiles_o) * a.n;
  const int k0 = int(int64_t(a.blocks) * rank / a.splits), k1 = int(int64_t(a.blocks) * (rank + 1) / a.splits);
  const uint32_t stage_bytes = kABytes + uint32_t(a.n) * kStep;

  // The weight's first blocks come into L2, where the work before this call may still write them, while it ends.
  if (tid == 32) {
    prefetch_tensor_map(&tm_x);
    for (int k = k0; k < k1 && k < k0 + a.ahead; ++k) {
      if constexpr (DGRAD) tma_prefetch_2d(&tm_w, int(o0), k * kStep);
      else tma_prefetch_2d(&tm_w, k * kStep, int(o0));
    }
  }
  if (tid == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < kScaleSlots; ++s) {
      mbar_init(scale_full + s, 1);
      mbar_init(scale_empty + s, 1);
    }
    mbar_init(done, 1);
    mbar_init(joined, 1);
    misc[1] = 1u;
    fence_mbar_init();
  }
  if (warp == 0) tc_alloc(misc, a.tmem_cols);
  tc_fence_before();
  __syncthreads();
  if (a.splits > 1) cluster_arrive();  // this CTA has started: the others may write into its memory
  tc_fence_after();
  const uint32_t tmem = misc[0], scales_at = tmem + a.tmem_cols - 32;
  pdl_begin(a.wait);

  const uint64_t lim = ring_wait_limit(a.status);
  bool ok = true;
  int issued = 0, committed = 0;
  // (a warp goes on or gives up as one)
  auto agreed = [](bool mine) { return __all_sync(0xffffffffu, mine) != 0; };
  int stage = 0;
  uint32_t pass = 0;
  if (warp == 0) {
    for (int k = k0; k < k1; ++k, ++issued) {
      ok = agreed(mbar_wait_ring(empty + stage, pass ^ 1u, lim));
      if (!ok) break;
      uint8_t* st = smem + stage * stage_bytes;
      if (elect_one()) {
        mbar_arrive_expect_tx(full + stage, stage_bytes);
        if constexpr (DGRAD) tma_load_2d(st, &tm_w, int(o0), k * kStep, full + stage);
        else tma_load_2d(st, &tm_w, k * kStep, int(o0), full + stage);
        tma_load_2d(st + kABytes, &tm_x, k * kStep, int(t0), full + stage);
      }
      __syncwarp();
      if (++stage == a.stages) stage = 0, pass ^= 1u;
    }
  } else if (warp == 1) {
    int slot = 0, chunk = 0;
    uint32_t slot_pass = 0;
    int piece_end = k0 + a.unbroken;
    uint32_t d = tmem;
    bool first = true;
    for (int k = k0; k < k1; ++k, ++committed) {
      if (k == piece_end) piece_end += a.unbroken, d += uint32_t(a.n), first = true;
      const bool fresh = k == k0 || (k & 3) == 0, last = (k & 3) == 3 || k == k1 - 1;
      if (fresh) ok = agreed(mbar_wait_ring(scale_full + slot, slot_pass, lim));
      if (ok) ok = agreed(mbar_wait_ring(full + stage, pass, lim));
      if (!ok) break;
      tc_fence_after();
      const uint32_t sa = scales_at + uint32_t(chunk & 1) * 16, sb = sa + 4;
      const uint32_t at = smem_addr(smem + stage * stage_bytes);
      const uint64_t x = tc_smem_desc_k128(at + kABytes);
      const uint64_t w = DGRAD ? tc_smem_desc_mn128(at, kABytes) : tc_smem_desc_k128(at);
      const uint32_t idesc = tc_idesc_scale_byte(a.idesc, uint32_t(k) & 3u);
      if (elect_one()) {
        if (fresh) {
          const uint32_t from = smem_addr(smem + kOffScales + slot * kScaleBytes);
          tc_copy_scales(sa, from);
          tc_copy_scales(sb, from + 512);
          if (a.n > 128) tc_copy_scales(sb + 4, from + 1024);
        }
#pragma unroll
        for (int s = 0; s < kStep / 32; ++s)
          tc_mma_mxf8(d, w + s * (DGRAD ? 4096 / 16 : 32 / 16), x + s * (32 / 16), idesc, sa, sb, s > 0 || !first);
        tc_commit(empty + stage);
        if (last) tc_commit(scale_empty + slot);
        if (k == k1 - 1) tc_commit(done);
      }
      __syncwarp();
      first = false;
      if (++stage == a.stages) stage = 0, pass ^= 1u;
      if (last) {
        ++chunk;
        if (++slot == kScaleSlots) slot = 0, slot_pass ^= 1u;
      }
    }
  } else {
    // two warps, every other chunk each: words of four blocks' scales, the weight's, the same for the tile's 128 outputs,
    // and each token's
    int slot = warp & 1;
    uint32_t slot_pass = 0;
    for (int k = (k0 & ~3) + 4 * slot; k < k1; k += 8) {
      uint32_t w = 0x7f7f7f7fu;
      if constexpr (DGRAD) {
        uint32_t byte = 0x7fu;
        if (lane < 4 && k + lane < a.w_blocks) byte = a.w_scales[int64_t(k + lane) * a.w_spitch + o0 / 128];
        w = __shfl_sync(0xffffffffu, byte, 0) | __shfl_sync(0xffffffffu, byte, 1) << 8 | __shfl_sync(0xffffffffu, byte, 2) << 16 |
            __shfl_sync(0xffffffffu, byte, 3) << 24;
      } else {
        w = *reinterpret_cast<const uint32_t*>(a.w_scales + o0 / 128 * a.w_spitch + k);
      }
      uint32_t x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t t = t0 + 32 * i + lane;
        x[i] = 32 * i < a.n && t < a.T ? *reinterpret_cast<const uint32_t*>(a.x_scales + t * a.x_spitch + k) : 0x7f7f7f7fu;
      }
      ok = agreed(mbar_wait_ring(scale_empty + slot, slot_pass ^ 1u, lim));
      if (!ok) break;
      uint8_t* to = smem + kOffScales + slot * kScaleBytes + 16 * lane;
      *reinterpret_cast<uint4*>(to) = make_uint4(w, w, w, w);
      *reinterpret_cast<uint4*>(to + 512) = make_uint4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<uint4*>(to + 1024) = make_uint4(x[4], x[5], x[6], x[7]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(scale_full + slot);
      if ((slot += 2) >= kScaleSlots) slot -= kScaleSlots, slot_pass ^= 1u;
    }
  }
  if (ok) ok = agreed(mbar_wait_ring(done, 0, lim));
  if (!ok) misc[1] = 0u;
  __syncthreads();
  const bool whole = misc[1] != 0u;
  if (!whole) {
    // a wait gave up: the copies this CTA sent off land, and its MMAs end, before it leaves
    if (warp == 0)
      for (int c = issued > a.stages ? issued - a.stages : 0; c < issued; ++c)
        mbar_wait_bounded(full + c % a.stages, uint32_t(c / a.stages) & 1u);
    if (warp == 1 && committed > 0)
      mbar_wait_bounded(empty + (committed - 1) % a.stages, uint32_t((committed - 1) / a.stages) & 1u);
    if (tid == 0) atomicOr(a.status, kStatusTimeout);
    __syncthreads();
  }
  tc_fence_after();
  // a lane's output, and the tokens of the tile sixteen at a time
  const int64_t o = o0 + 32 * warp + lane;
  T* out = static_cast<T*>(a.out) + t0 * a.ldo + o;
  const uint32_t sums = tmem + (uint32_t(warp * 32) << 16);
  const int groups = a.n / 16, pieces = (k1 - k0 + a.unbroken - 1) / a.unbroken;
  const int64_t left = o < a.outs ? a.T - t0 : 0;  // tokens, of which this lane writes
  auto read = [&](int g, float (&v)[16]) {
    uint32_t u[16];
    tc_ld16(sums + 16 * g, u);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(u[e]);
    for (int p = 1; p < pieces; ++p) {
      tc_ld16(sums + p * a.n + 16 * g, u);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] += __uint_as_float(u[e]);
    }
  };
  auto write = [&](int g, const float (&v)[16]) {
    T* to = out + int64_t(16 * g) * a.ldo;
#pragma unroll
    for (int e = 0; e < 16; ++e, to += a.ldo)
      if (16 * g + e < left) *to = from_f32<E>(v[e]);
  };
  if (a.splits == 1) {
    for (int g = 0; whole && g < groups; ++g) {
      float v[16];
      read(g, v);
      write(g, v);
    }
  } else {
    // Group g of sixteen tokens is added by CTA g % splits.  A CTA's sums lie at the start, group after group ([16 tokens][128
    // outputs]), then the other CTAs' of its groups: [CTA, itself left out][g / splits].
    const int each = (groups + a.splits - 1) / a.splits, mine = (groups - rank + a.splits - 1) / a.splits;
    float* own = reinterpret_cast<float*>(smem);
    const int place = 32 * warp + lane;
    for (int g = 0; whole && g < groups; ++g) {
      float v[16];
      read(g, v);
#pragma unroll
      for (int e = 0; e < 16; ++e) own[(g * 16 + e) * 128 + place] = v[e];
    }
    fence_proxy_async_smem();
    if (tid == 0) mbar_arrive_expect_tx(joined, uint32_t((a.splits - 1) * mine) * kGroupBytes);
    __syncwarp();
    cluster_wait();  // (they have long started)
    if (tid < a.splits) store_cluster(cluster_addr(misc + 2 + rank, uint32_t(tid)), whole ? 1u : 0u);
    __syncwarp();
    cluster_sync();  // every CTA is done with its stages, and its sums lie there
    int missing = 0;  // CTAs that gave up and send nothing
    for (int r = 0; r < a.splits; ++r) missing += r != rank && misc[2 + r] == 0u ? 1 : 0;
    if (tid == 0 && missing > 0 && mine > 0) mbar_complete_tx(joined, uint32_t(missing * mine) * kGroupBytes);
    if (warp == 0 && whole) {
      for (int g = lane; g < groups; g += 32) {
        const int to = g % a.splits;
        if (to == rank) continue;
        const uint32_t at = uint32_t(groups + (rank - (rank > to ? 1 : 0)) * each + g / a.splits) * kGroupBytes;
        bulk_s2s(cluster_addr(smem + at, uint32_t(to)), smem + uint32_t(g) * kGroupBytes, kGroupBytes, cluster_addr(joined, uint32_t(to)));
      }
    }
    const bool all = agreed(mbar_wait_ring_cluster(joined, 0, lim)) && whole && missing == 0;
    if (!all) {
      mbar_wait_bounded(joined, 0);  // what the others send has landed
      if (lane == 0) atomicOr(a.status, kStatusTimeout);
    }
    for (int g = rank; all && g < groups; g += a.splits) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = 0.0f;
      for (int r = 0; r < a.splits; ++r) {
        const int at = r == rank ? g : groups + (r - (r > rank ? 1 : 0)) * each + g / a.splits;
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] += own[(at * 16 + e) * 128 + place];
      }
      write(g, v);
    }
    cluster_sync();  // what this CTA copied to the others has been read
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tc_dealloc(tmem, a.tmem_cols);
}

// Bytes in which a CTA of a split tile has its own sums and takes the others'.
uint32_t join_bytes(int n, int splits) {
  const int groups = n / 16, each = (groups + splits - 1) / splits;
  return uint32_t(groups + (splits - 1) * each) * kGroupBytes;
}

// Blocks of the weight sent for ahead, where it is read once and a CTA's share is more than the ring holds.  Twelve to sixteen are
// best, by what stands before the call.  Weights from memory, us with 8, 12, 16 blocks:
//   1 token of 18944 x 3584, copied before it, other inputs each time   15.6, 15.3, 15.1 (4: 15.9)
//     the same input, 4 weights in turn                                 14.9, 14.6, 15.1; the product alone 13.0, 12.7, 12.8
//     in a graph, the product alone                                     14.0, 14.0, 14.9 (none 15.0, 4: 14.3, 24: 16.3)
//   16 and 64 tokens of it, alone                                       12.9, 12.6, 12.9 and 13.0, 13.3, 13.7
//   1 token of 3584 x 18944, alone                                      17.6, 17.3, 17.9; in a graph 18.2, 17.5, 17.7 (none 18.6)
//   input gradient of 16 tokens, 18944 x 3584, alone                    13.0, 13.4, 13.6
constexpr int kAhead = 16;

template <bool DGRAD, Elem E>
int launch(const CUtensorMap& tm_w, const CUtensorMap& tm_x, const LinearArgs& a, int64_t grid, cudaStream_t stream) {
  auto kern = roi_fp8_linear_kernel<DGRAD, E>;
  constexpr size_t smem = kSmem + 1024;
  static std::atomic<bool> set[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  if (!set[dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return -1;
    set[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (a.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = unsigned(a.splits);
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (a.wait) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kern, tm_w, tm_x, a) == cudaSuccess ? 1 : -1;
}

template <bool DGRAD>
int launch_of(Elem e, const CUtensorMap& tm_w, const CUtensorMap& tm_x, const LinearArgs& a, int64_t grid, cudaStream_t stream) {
  switch (e) {
    case Elem::kBf16: return launch<DGRAD, Elem::kBf16>(tm_w, tm_x, a, grid, stream);
    case Elem::kFp16: return launch<DGRAD, Elem::kFp16>(tm_w, tm_x, a, grid, stream);
    default: return launch<DGRAD, Elem::kFp32>(tm_w, tm_x, a, grid, stream);
  }
}

// The most blocks of an unbroken sum for fp32 results (roi_fp8_pair.cu says why).
constexpr int kMostBlocks = 16;

// Clusters of `size` CTAs of this kernel that the device holds at once: a cluster lies within one of its GPCs, so that
// they do not use every SM (7 CTAs to a cluster, 21 clusters, 147 CTAs on 152 SMs: two waves).
// (`dev` the current device.)
int clusters_at_once(int dev, int size) {
  if (size == 1) return sm_count();
  static std::atomic<int> known[64][9];
  if (dev < 0 || dev >= 64) return 1;
  int n = known[dev][size].load(std::memory_order_acquire);
  if (n == 0) {
    auto kern = roi_fp8_linear_kernel<false, Elem::kBf16>;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = unsigned(size);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(unsigned(size));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem + 1024;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmem + 1024)) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
      cudaGetLastError();
      n = 1;
    }
    known[dev][size].store(n, std::memory_order_release);
  }
  return n;
}

// Tokens of a tile, ranges of its sum and their pieces, for the least time; returns that in cycles.  An SM takes in 64 bytes
// a cycle: 2 (128 + n) cycles a block.  Filling the ring and writing the tile come once a tile, joining ranges once a range.
constexpr int kTileCycles = 2000, kTokenCycles = 12, kJoinCycles = 2000;
int64_t plan(int64_t T, int64_t tiles_o, int blocks, bool fp32, LinearArgs& a, int64_t& tiles_t) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) dev = -1;
  int64_t least = INT64_MAX;
  int64_t last = 0;
  for (int64_t t = (T + 255) / 256, tries = 0; tries < 16; ++t, ++tries) {
    const int64_t n = ((T + t - 1) / t + 15) / 16 * 16;
    if (n == last) continue;
    last = n;
    for (int s = 1; s <= 8 && s <= blocks; ++s) {
      const int64_t once = clusters_at_once(dev, s);
      if (s > 1 && (tiles_o * t > once || join_bytes(int(n), s) > kRingBytes)) break;
      const int range = (blocks + s - 1) / s;
      const int pieces = fp32 ? (range + kMostBlocks - 1) / kMostBlocks : 1;
      if (pieces * n > 480) continue;  // (columns of TMEM; pairs of CTAs take any number)
      const int64_t rounds = (tiles_o * t + once - 1) / once;
      const int64_t time = rounds * (range * 2 * (128 + n) + kTileCycles + kTokenCycles * n + (s > 1 ? kJoinCycles + kTokenCycles * n : 0));
      if (time >= least) continue;
      least = time;
      tiles_t = (T + n - 1) / n;
      a.n = int(n);
      a.splits = s;
      a.unbroken = (range + pieces - 1) / pieces;
      a.tmem_cols = 64;
      while (int(a.tmem_cols) < (int(n) * pieces + 31) / 32 * 32 + 32) a.tmem_cols *= 2;
    }
    if (n == 16) break;
  }
  return least;
}

}  // namespace

int launch_fp8_linear(const Fp8LinearCall& c) {
  LinearArgs a;
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
  a.tiles_o = int((outs + 127) / 128);
  int64_t tiles_t;
  // Pairs where they are quicker, on a way that is open to the call: counting the other, an input gradient of 4697 tokens, 896 x 896,
  // went to pairs, 9.3 us, 7.6 here; 4697 tokens, 4864 x 896, 23.9 and 19.5.
  Fp8PairPlan pair;
  const int64_t pair_cycles = fp8_pair_cycles(c.T, outs, width, fp8_pair_tokens(c), sm_count() / 2, pair);
  if (plan(c.T, a.tiles_o, a.blocks, c.dtype == Elem::kFp32, a, tiles_t) > pair_cycles) return launch_fp8_pair(c, pair);
  a.stages = int(kRingBytes / (kABytes + uint32_t(a.n) * kStep));
  if (a.stages > kMaxStages) a.stages = kMaxStages;
  a.idesc = tc_idesc_mxf8(128, a.n, int(Fp8::kE4M3), int(c.format), c.dgrad, false);
  a.ahead = tiles_t == 1 && (a.blocks + a.splits - 1) / a.splits > a.stages ? kAhead : 0;
  a.status = c.status;
  a.wait = lone_pdl(c.stream);
  CUtensorMap tm_w, tm_x;
  const int64_t w_pitch = fp8_pitch(c.cols), x_pitch = fp8_pitch(width);
  if (!make_tensor_map(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.w_codes, uint64_t(w_pitch), uint64_t(c.rows), uint64_t(w_pitch), 128, 128,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      !make_tensor_map(&tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.x_codes, uint64_t(x_pitch), uint64_t(c.T), uint64_t(x_pitch), kStep,
                       uint32_t(a.n), CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
    return -1;
  const int64_t grid = a.tiles_o * tiles_t * a.splits;
  return c.dgrad ? launch_of<true>(c.dtype, tm_w, tm_x, a, grid, c.stream) : launch_of<false>(c.dtype, tm_w, tm_x, a, grid, c.stream);
}

}  // namespace roi
