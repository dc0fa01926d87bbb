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
// fewer than the SMs, a range of its sum: the CTAs of a tile are a cluster, put their sums into one another's shared memory and
// add them in the order of the ranges, each for some of the tokens.
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
constexpr int kBars = 2 * kMaxStages + 2 * kScaleSlots + 1;
constexpr uint32_t kOffMisc = kOffBars + kBars * 8, kSmem = kOffMisc + 8;
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
  int stages;
  uint32_t idesc, tmem_cols;
  unsigned int* status;
  bool wait;
};

// Stores a float into the shared memory of CTA `rank` of the cluster at this CTA's `place`.
__device__ __forceinline__ void store_cluster(uint32_t place, uint32_t rank, float v) {
  asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %0, %1;\n\tst.shared::cluster.f32 [ra], %2;\n\t}" ::"r"(place),
               "r"(rank), "f"(v)
               : "memory");
}

template <bool DGRAD, Elem E>
__global__ void __launch_bounds__(kThreads, 1)
    roi_fp8_linear_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_x, LinearArgs a) {
  using T = typename ElemType<E>::T;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t *full = bars, *empty = full + kMaxStages, *scale_full = empty + kMaxStages, *scale_empty = scale_full + kScaleSlots;
  uint64_t* done = scale_empty + kScaleSlots;
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + kOffMisc);  // [0] TMEM base, [1] ok
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = a.splits > 1 ? int(cluster_rank()) : 0;
  const int tile = blockIdx.x / a.splits;
  const int64_t o0 = int64_t(tile % a.tiles_o) * 128, t0 = int64_t(tile / a.tiles_o) * a.n;
  const int k0 = int(int64_t(a.blocks) * rank / a.splits), k1 = int(int64_t(a.blocks) * (rank + 1) / a.splits);
  const uint32_t stage_bytes = kABytes + uint32_t(a.n) * kStep;

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
    misc[1] = 1u;
    fence_mbar_init();
  }
  if (warp == 0) tc_alloc(misc, a.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0], scales_at = tmem + uint32_t((a.n + 31) / 32 * 32);
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
    for (int k = k0; k < k1; ++k, ++committed) {
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
          tc_mma_mxf8(tmem, w + s * (DGRAD ? 4096 / 16 : 32 / 16), x + s * (32 / 16), idesc, sa, sb, s > 0 || k > k0);
        tc_commit(empty + stage);
        if (last) tc_commit(scale_empty + slot);
        if (k == k1 - 1) tc_commit(done);
      }
      __syncwarp();
      if (++stage == a.stages) stage = 0, pass ^= 1u;
      if (last) {
        ++chunk;
        if (++slot == kScaleSlots) slot = 0, slot_pass ^= 1u;
      }
    }
  } else if (warp == 2) {
    // words of four blocks' scales: the weight's, the same for the tile's 128 outputs, and each token's
    int slot = 0;
    uint32_t slot_pass = 0;
    for (int k = k0 & ~3; k < k1; k += 4) {
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
      if (++slot == kScaleSlots) slot = 0, slot_pass ^= 1u;
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
  T* out = static_cast<T*>(a.out) + o;
  const uint32_t sums = tmem + (uint32_t(warp * 32) << 16);
  const int groups = a.n / 16;
  if (a.splits == 1) {
    for (int g = 0; whole && g < groups; ++g) {
      uint32_t u[16];
      tc_ld16(sums + 16 * g, u);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t t = t0 + 16 * g + e;
        if (o < a.outs && t < a.T) out[t * a.ldo] = from_f32<E>(__uint_as_float(u[e]));
      }
    }
  } else {
    // Group g of tokens is added by CTA g % splits, where every CTA's sums lie one after another:
    // [CTA][g / splits][16 tokens][128 outputs].
    const int each = (groups + a.splits - 1) / a.splits;
    cluster_sync();  // every CTA is done with its stages
    for (int g = 0; whole && g < groups; ++g) {
      uint32_t u[16];
      tc_ld16(sums + 16 * g, u);
      const uint32_t place = smem_addr(smem) + uint32_t(((rank * each + g / a.splits) * 16) * 128 + 32 * warp + lane) * 4;
#pragma unroll
      for (int e = 0; e < 16; ++e) store_cluster(place + e * 512, uint32_t(g % a.splits), __uint_as_float(u[e]));
    }
    cluster_sync();
    const float* from = reinterpret_cast<const float*>(smem) + 32 * warp + lane;
    for (int g = rank; whole && g < groups; g += a.splits) {
#pragma unroll 4
      for (int e = 0; e < 16; ++e) {
        const int64_t t = t0 + 16 * g + e;
        if (o >= a.outs || t >= a.T) continue;
        float v = 0.0f;
        for (int r = 0; r < a.splits; ++r) v += from[((r * each + g / a.splits) * 16 + e) * 128];
        out[t * a.ldo] = from_f32<E>(v);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 0) tc_dealloc(tmem, a.tmem_cols);
}

// Bytes in which a CTA of a split tile takes its group's sums.
uint32_t join_bytes(int n, int splits) { return uint32_t(splits) * uint32_t((n / 16 + splits - 1) / splits) * 16 * 128 * 4; }

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

}  // namespace

int launch_fp8_linear(const Fp8LinearCall& c) {
  LinearArgs a;
  const int64_t outs = c.dgrad ? c.cols : c.rows, width = c.dgrad ? c.rows : c.cols;
  // tiles of a pair of CTAs where there are enough for half of the pairs
  if (((c.T + 255) / 256) * ((outs + 223) / 224) >= sm_count() / 4 && c.T > 128) return launch_fp8_pair(c);
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
  const int64_t tiles_t = (c.T + 255) / 256;
  a.n = int(((c.T + tiles_t - 1) / tiles_t + 15) / 16 * 16);
  const int64_t tiles = a.tiles_o * tiles_t;
  a.stages = int(kRingBytes / (kABytes + uint32_t(a.n) * kStep));
  if (a.stages > kMaxStages) a.stages = kMaxStages;
  a.splits = 1;
  while (a.splits < 8 && a.splits < a.blocks && tiles * (a.splits + 1) <= sm_count() && join_bytes(a.n, a.splits + 1) <= kRingBytes)
    ++a.splits;
  a.idesc = tc_idesc_mxf8(128, a.n, int(Fp8::kE4M3), int(c.format), c.dgrad, false);
  a.tmem_cols = 64;
  while (int(a.tmem_cols) < (a.n + 31) / 32 * 32 + 32) a.tmem_cols *= 2;
  a.status = c.status;
  a.wait = lone_pdl(c.stream);
  CUtensorMap tm_w, tm_x;
  const int64_t w_pitch = fp8_pitch(c.cols), x_pitch = fp8_pitch(width);
  if (!make_tensor_map(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.w_codes, uint64_t(w_pitch), uint64_t(c.rows), uint64_t(w_pitch), 128, 128,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      !make_tensor_map(&tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.x_codes, uint64_t(x_pitch), uint64_t(c.T), uint64_t(x_pitch), kStep,
                       uint32_t(a.n), CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
    return -1;
  const int64_t grid = tiles * a.splits;
  return c.dgrad ? launch_of<true>(c.dtype, tm_w, tm_x, a, grid, c.stream) : launch_of<false>(c.dtype, tm_w, tm_x, a, grid, c.stream);
}

}  // namespace roi
