// Weight gradient of a masked linear layer from the 8-bit checkpoint of its input:
//   dWm[o, i] = sum_t dY[t, o] x^[t, i]  (+ acc[o, i])
// on the fifth-generation tensor cores, the sums in fp32.  x^ is formed from codes and scales
// on the way into shared memory; its values have 7 bits and a sign, so bf16 holds them exactly
// and the product is that of dY with the checkpoint's own values.
//
// A pair of CTAs shares its MMAs (cta_group::2) and owns a tile of 256 outputs x 256 inputs; each CTA
// holds 128 outputs of dY, 128 inputs of x^ and, in TMEM, 128 rows of the sums, 256 columns wide.
// Both operands are MN-major (a token's row is contiguous along outputs or inputs), in tiles of 64
// tokens with 128-byte swizzle.
//
// Roles of the 18 warps of a CTA, each a loop over the same list of tiles and chunks of 64 tokens:
//   warp 0        stages dY by TMA (rows past the last token, columns past the last as zeros)
//   warp 12       stages the codes by TMA, and their scales by asynchronous copies of words
//   warps 2 - 11  five sets of two, each every fifth chunk: codes to bf16 in the layout of the MMA,
//                 into one of three slots; with warp 13, which says so of dY, they make a chunk `ready`
//   warp 1        of the even CTA: four MMAs of 16 tokens a chunk for both; commits them to `dy_empty`,
//                 which frees dY's stage and the slot, and after the last chunk to `sum`
//   warps 14 - 17 read the sums from TMEM and write them out, `free`, while the next tile's
//                 MMAs go to the other half of TMEM
// What it took to feed the tensor cores (8192 tokens, 18944 x 3584; the measured cuBLAS rate would be
// 589 us): codes and scales through registers of the converting warps, a cluster-wide release a
// chunk 1888 us; without that release 982; two sets of converting warps and the scales staged apart
// 867; even bytes converted where they are 727; rings of their own and loops of whole warps
// around the MMAs, so that descriptors stay in uniform registers, 631; whole sectors out 583 to 600,
// which is 1860 to 1910 TFLOP/s; waits that a whole warp answers as one 605; arrivals on the pair's barriers that release
// shared memory to the cluster 608 (with acc 785 -> 817; handed on by the warp that tells of dY alone, 622 and 816).  Under a
// long load the clock falls with the power (697 us).
// Every wait is bounded; a CTA that gives up lets its copies and MMAs end before it leaves.
//
// Tiles go to the pairs in rounds.  In the last, partial round the tokens of
// its tiles are cut into even ranges, one a pair, where that ends sooner: ranges that do not
// cover a whole tile leave fp32 partial sums in the workspace, which a second launch adds in
// the order of the tokens, so that results do not depend on timing.
#include <atomic>

#include "roi_launch.h"
#include "roi_rows.cuh"
#include "roi_tc.cuh"
#include "roi_tmap.h"

namespace roi {
namespace {

constexpr int kEdge = 128;                 // outputs, and inputs, that a CTA holds
constexpr int kSide = 2 * kEdge;           // of a pair's tile
constexpr int kChunk = 64;                 // tokens a stage
// Rings: codes and scales, dY, and converted x^ (where nothing waits for memory in between).  Stages of codes, of dY,
// slots, sets, warps of a set, 8192 tokens of 18944 x 3584: 10, 5, 3, 5, 2 583 to 599 us; 8, 5, 4, 4, 4 613; 10, 5, 3,
// 5, 4 627; 12, 4, 3, 4, 4 628; 8, 6, 3, 4, 4 625; 8, 6, 3, 4, 2 644.
constexpr int kCodeStages = 10, kDyStages = 5, kSlots = 3;
constexpr uint32_t kHalf = kChunk * 128;   // 64 tokens x 64 bf16
constexpr uint32_t kOperand = 2 * kHalf;   // 64 tokens x 128 bf16
constexpr uint32_t kCodes = kChunk * kEdge;
constexpr uint32_t kScales = kChunk * 4;   // a word of four blocks a token
constexpr uint32_t kOffSlots = kDyStages * kOperand, kOffCodes = kOffSlots + kSlots * kOperand;
constexpr uint32_t kOffScales = kOffCodes + kCodeStages * kCodes, kOffBars = kOffScales + kCodeStages * kScales;
constexpr int kSets = 5;            // sets of warps that turn codes into bf16, each every kSets-th chunk
constexpr int kConvertWarps = 2;    // of a set
// A wait for a phase of a barrier takes the one before to be over.  Copies may land out of their
// order, so a set waits for every phase of its code stages itself; dY's stages end in order, and a
// set that waits for one has seen a chunk end that is at most kSets before.
static_assert(kCodeStages % kSets == 0 && kSlots <= kDyStages && kSets <= kDyStages, "phases in turn");
constexpr int kUnits = 8 / kConvertWarps;        // blocks of 32 codes a thread takes of a chunk
// warp 0: dY; 1: MMA; 2 on: the sets; then codes and scales; the landed dY's notice; four that write
constexpr int kWarpCodes = 2 + kConvertWarps * kSets, kWarpNotice = kWarpCodes + 1;
constexpr int kThreads = 32 * (kWarpNotice + 1 + 4);
constexpr uint32_t kTmemCols = 512;
constexpr int kBars = 2 * kCodeStages + 2 * kDyStages + kSlots + 2 + 2;
constexpr uint32_t kOffMisc = kOffBars + kBars * 8;
// 16 rows of 32 sums for each of the four warps that write, where outputs are not whole sectors.
constexpr int kBlockPitch = 36;
constexpr uint32_t kOffBlocks = (kOffMisc + 8 + 15) / 16 * 16, kSmem = kOffBlocks + 4 * 16 * kBlockPitch * 4;  // from a 1024-byte boundary on
static_assert(kSmem + 1024 <= 232448, "shared memory");
// The fewest chunks of a range of the last round, and what a split costs in chunks: a tile of
// partial sums is written and read again.  With 8 and 8, 4 and 8, 4 and 4, 2 and 4: 1024 tokens of 896 x 896
// 14.8, 15.6, 15.5, 19.2 us; 2048 tokens of 128 x 896 14.0, 13.8, 13.9, 19.5; larger ones alike.
constexpr int kMinRange = 8, kSplitCost = 8;

// The most chunks that TMEM sums unbroken for acc.  The tensor cores drop the bits below their sum's last
// instead of rounding, all towards zero, which grows with the tokens: 4.3e-7 of the sum's norm at 2000
// tokens, 1.1e-6 at 4000, 6.8e-6 at 16000, where an fp32 product has 5e-7.  So longer sums are added to
// acc in pieces, rounded in fp32: at most 6.3e-7.  8192 tokens, 18944 x 3584: 846 us with acc, in three pieces, and 605
// without, where the result is rounded to bf16, 4000 times as coarse.
constexpr int kMostChunks = 44;
// The same for a bf16 result alone.  Unbroken, its error against the nearest bf16 number's (1.66e-3 of the norm) is
// 1.0001 times as large at 32768 tokens, 1.01 at 262144, 1.2 at a million and 3 at four million.  Longer sums are broken
// off at 32768 tokens and their total is kept in the other half of TMEM, so that the MMAs wait while a piece is added
// (65536 tokens of 9728 x 3584, one after another: 2723 to 2776 us whole, 2764 to 2775 in two pieces).
constexpr int kMostAlone = 512;

struct WgradArgs {
  const uint8_t* scales;
  uint16_t* dWm;  // nullable
  float* acc;     // nullable
  float* part;    // [2 * ranges][kSide / 4][kSide][4] (split): four columns of all rows after one another
  int64_t T, rows, cols, spitch;
  int tiles_m, tiles_n;
  bool n_first;   // consecutive tiles run along the inputs
  int chunks;     // of a whole tile
  int unbroken;   // the most chunks of a sum in TMEM
  int groups;     // pairs of CTAs
  int rounds;     // whole rounds of tiles
  int rest;       // tiles of the last round
  int ranges;     // ranges of its tokens, 0 where they are not cut
  unsigned int* status;
  bool wait;
};

// A sum in TMEM: some consecutive chunks of a tile.
struct Work {
  int tile, c0, c1;  // tile and chunks
  int slot;          // place of its partial sums, -1 where they go to the outputs
  bool first, last;  // of the pieces that are added to one place
};

__host__ __device__ inline int64_t range_start(const WgradArgs& a, int64_t r) {
  return r * (int64_t(a.rest) * a.chunks) / a.ranges;
}

// Piece `i` of the sum over chunks c0 .. c1, in even pieces; false, and `i` less their number, after the last.
__device__ __forceinline__ bool piece_of(const WgradArgs& a, int c0, int c1, int& i, Work& w) {
  const int n = (c1 - c0 + a.unbroken - 1) / a.unbroken;
  if (i >= n) {
    i -= n;
    return false;
  }
  const int each = (c1 - c0) / n, more = (c1 - c0) % n;
  w.c0 = c0 + each * i + (i < more ? i : more);
  w.c1 = w.c0 + each + (i < more ? 1 : 0);
  w.first = i == 0;
  w.last = i == n - 1;
  return true;
}

// The i-th sum of group g; false after the last.
__device__ __forceinline__ bool work_of(const WgradArgs& a, int g, int i, Work& w) {
  w.slot = -1;
  const int pieces = (a.chunks + a.unbroken - 1) / a.unbroken, round = i / pieces;
  if (a.ranges == 0 ? round < a.rounds + (g < a.rest ? 1 : 0) : round < a.rounds) {
    w.tile = round * a.groups + g;
    i -= round * pieces;
    return piece_of(a, 0, a.chunks, i, w);
  }
  if (g >= a.ranges) return false;
  i -= a.rounds * pieces;
  // a range is no longer than a tile: it touches two tiles at most
  const int64_t begin = range_start(a, g), end = range_start(a, g + 1);
  const int first = int(begin / a.chunks);
  for (int j = 0; j < 2; ++j) {
    const int64_t t0 = int64_t(first + j) * a.chunks;  // the tile's first chunk among all
    const int64_t from = begin > t0 ? begin : t0, to = end < t0 + a.chunks ? end : t0 + a.chunks;
    if (from >= to) return false;
    w.tile = a.rounds * a.groups + first + j;
    w.slot = to - from < a.chunks ? 2 * g + j : -1;
    if (piece_of(a, int(from - t0), int(to - t0), i, w)) return true;
  }
  return false;
}

__device__ __forceinline__ void tile_origin(const WgradArgs& a, int tile, int64_t& m0, int64_t& n0) {
  const int m = a.n_first ? tile / a.tiles_n : tile % a.tiles_m;
  const int n = a.n_first ? tile % a.tiles_n : tile / a.tiles_m;
  m0 = int64_t(m) * kSide;
  n0 = int64_t(n) * kSide;
}

// Two codes to two bf16, times the block's power of two: the codes in the low bytes of the
// halves of `w` (the high bytes are ignored).  A code byte b is (128 + (b & 127)) -
// (128 + (b & 128)): both terms are bf16 numbers whose mantissa holds the byte's bits, and
// difference and product are exact.
__device__ __forceinline__ uint32_t codes2_bf16(uint32_t w, __nv_bfloat162 step) {
  const uint32_t m = (w & 0x007f007fu) | 0x43004300u, n = (w & 0x00800080u) | 0x43004300u;
  const __nv_bfloat162 v = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&m), *reinterpret_cast<const __nv_bfloat162*>(&n)), step);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// Eight codes (two words) to eight bf16.  The even bytes of a word are taken where they are and
// the odd ones after one shift, which leaves each four in the order 0, 2, 1, 3: the order of the
// tile's columns in the sums, which the epilogue undoes (input_order) at no cost.
__device__ __forceinline__ uint4 codes8_bf16(uint32_t a, uint32_t b, __nv_bfloat162 step) {
  return make_uint4(codes2_bf16(a, step), codes2_bf16(a >> 8, step), codes2_bf16(b, step), codes2_bf16(b >> 8, step));
}
__device__ __forceinline__ void input_order(const uint32_t (&u)[32], float (&v)[32]) {
#pragma unroll
  for (int e = 0; e < 32; e += 4) {
    v[e] = __uint_as_float(u[e]), v[e + 1] = __uint_as_float(u[e + 2]);
    v[e + 2] = __uint_as_float(u[e + 1]), v[e + 3] = __uint_as_float(u[e + 3]);
  }
}
__device__ __forceinline__ __nv_bfloat162 step_bf16x2(uint32_t s) {
  const uint32_t h = __float_as_uint(block8_step(s)) >> 16;
  const uint32_t w = h | (h << 16);
  return *reinterpret_cast<const __nv_bfloat162*>(&w);
}

// A place in a ring of N, and the parity of the pass over it.
template <int N>
struct Ring {
  int at = 0;
  uint32_t pass = 0;
  __device__ __forceinline__ void next() {
    if (++at == N) at = 0, pass ^= 1u;
  }
};

// load32 of memory that this kernel writes as well.
__device__ __forceinline__ void load32_written(const void* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}

// (volatile: eight of them at once would take registers that the warps that write do not have)
__device__ __forceinline__ float4 load_written(const float4* p) {
  float4 x;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "l"(p) : "memory");
  return x;
}

// 32 columns of a row of the sums, from column n on (a multiple of 32): added to acc, and
// written out, where columns come in sixteens.  A lane has a row of its own and stores whole sectors.
__device__ __forceinline__ void store_sectors(const WgradArgs& a, bool last, int64_t m, int64_t n, float (&v)[32]) {
  const int64_t at = m * a.cols + n;
  if (a.acc != nullptr) {
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      if (n + 8 * q >= a.cols) break;  // (columns come in sixteens)
      uint32_t w[2][8];
      load32_written(a.acc + at + 8 * q, w[0]);
      load32_written(a.acc + at + 8 * q + 8, w[1]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[h][e] = __float_as_uint(v[8 * (q + h) + e] += __uint_as_float(w[h][e]));
        store32(a.acc + at + 8 * (q + h), w[h]);
      }
    }
  }
  if (last && a.dWm != nullptr) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (n + 16 * q >= a.cols) break;
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(v[16 * q + 2 * e], v[16 * q + 2 * e + 1]);
      store32(a.dWm + at + 16 * q, w);
    }
  }
}
// Any other width (the whole warp, rows m0 on): 16 rows at a time through shared memory, so that
// sixteen lanes write a row's 32 columns, two each (PAIRS: rows of an even width).  A store of 2
// bytes a lane to a row a lane would touch 32 lines.
template <bool PAIRS>
__device__ __forceinline__ void store_block(const WgradArgs& a, bool last, float* block, int64_t m0, int64_t n, const float (&v)[32]) {
  const int lane = threadIdx.x & 31, c = 2 * (lane & 15), odd = lane >> 4;
  const int64_t after = a.cols - n - c;
  const int left = after > 2 ? 2 : after < 0 ? 0 : int(after);  // of this lane's columns
  const int64_t step = 2 * a.cols;
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    __syncwarp();
    if (odd == h) {
#pragma unroll
      for (int e = 0; e < 32; e += 4)
        *reinterpret_cast<float4*>(block + (lane & 15) * kBlockPitch + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
    __syncwarp();
    const int64_t below = a.rows - m0 - 16 * h;
    const int rows = left == 0 ? 0 : below > 16 ? 16 : int(below);  // of the 16
    const int64_t at = (m0 + 16 * h + odd) * a.cols + n + c;
    const float* from = block + odd * kBlockPitch + c;
    uint16_t* out = a.dWm + at;
    if (a.acc == nullptr) {
#pragma unroll
      for (int r = 0; r < 8; ++r, out += step) {
        const float2 x = *reinterpret_cast<const float2*>(from + 2 * r * kBlockPitch);
        const uint32_t w = pack_bf16x2(x.x, x.y);
        if (2 * r + odd < rows) {
          if constexpr (PAIRS) {
            *reinterpret_cast<uint32_t*>(out) = w;
          } else {
            out[0] = uint16_t(w);
            if (left > 1) out[1] = uint16_t(w >> 16);
          }
        }
      }
    } else {
      float* acc = a.acc + at;
      const bool write = last && a.dWm != nullptr;
      float2 y[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        y[r] = make_float2(0.0f, 0.0f);
        const float* q = acc + r * step;
        if (2 * r + odd < rows) {
          if constexpr (PAIRS) y[r] = *reinterpret_cast<const float2*>(q);
          else y[r] = make_float2(q[0], left > 1 ? q[1] : 0.0f);
        }
      }
#pragma unroll
      for (int r = 0; r < 8; ++r, out += step, acc += step) {
        const float2 x = *reinterpret_cast<const float2*>(from + 2 * r * kBlockPitch);
        y[r].x += x.x, y[r].y += x.y;
        if (2 * r + odd < rows) {
          const uint32_t w = pack_bf16x2(y[r].x, y[r].y);
          if constexpr (PAIRS) {
            *reinterpret_cast<float2*>(acc) = y[r];
            if (write) *reinterpret_cast<uint32_t*>(out) = w;
          } else {
            acc[0] = y[r].x;
            if (write) out[0] = uint16_t(w);
            if (left > 1) {
              acc[1] = y[r].y;
              if (write) out[1] = uint16_t(w >> 16);
            }
          }
        }
      }
    }
  }
}

// How the outputs are written: whole sectors, pairs of columns, single columns (the last two through shared
// memory; 1999 tokens of 1215 x 2504 with acc 35 us, 45 element by element from registers).
enum class Out { kSectors, kPairs, kSingles };

// The half of TMEM of sum i, and the parity of its turn there.  KEPT: all sums in the first, totals in the second.
template <bool KEPT>
__device__ __forceinline__ int half_of(int i) {
  return KEPT ? 0 : i & 1;
}
template <bool KEPT>
__device__ __forceinline__ uint32_t turn_of(int i) {
  return uint32_t(KEPT ? i : i >> 1) & 1u;
}

template <Out OUT, bool KEPT>
__device__ __forceinline__ void wgrad(const CUtensorMap& tm_dy, const CUtensorMap& tm_codes, const WgradArgs& a) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBars);
  uint64_t *code_full = bars, *code_empty = code_full + kCodeStages, *dy_full = code_empty + kCodeStages, *dy_empty = dy_full + kDyStages;
  uint64_t *ready = dy_empty + kDyStages, *sum = ready + kSlots, *free = sum + 2;
  uint32_t* misc = reinterpret_cast<uint32_t*>(smem + kOffMisc);  // [0] TMEM base, [1] ok
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank();
  const int g = blockIdx.x / 2;

  if (tid == 0) {
    for (int s = 0; s < kCodeStages; ++s) {
      mbar_init(code_full + s, 1 + 32);  // the TMA copy, and each lane's copies of scales
      mbar_init(code_empty + s, kConvertWarps);
    }
    for (int s = 0; s < kDyStages; ++s) {
      mbar_init(dy_full + s, 1);
      mbar_init(dy_empty + s, 1);
    }
    for (int s = 0; s < kSlots; ++s) mbar_init(ready + s, (kConvertWarps + 1) * 2);
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
  int issued = 0, committed = 0;  // chunks whose copies, and whose MMAs, this thread has sent off
  Work w;
  int64_t m0, n0;
  Ring<kDyStages> ring;
  Ring<kCodeStages> code_ring;
  Ring<kSlots> slot;
  // A warp goes on or gives up as one: its loops have instructions of whole warps in them, at which lanes that
  // parted would wait for one another for ever.  (8192 tokens, 18944 x 3584: 605 us, 597 without, timed in turn.)
  auto agreed = [](bool mine) { return __all_sync(0xffffffffu, mine) != 0; };
  // A slot, and its `ready`, are free again once the MMAs of the chunk that had it are done: what
  // dy_empty of that chunk's stage says (whose next phase cannot end before this chunk is ready).
  auto slot_free = [&](uint32_t q) {
    return q < kSlots || mbar_wait_ring_cluster(dy_empty + (q - kSlots) % kDyStages, ((q - kSlots) / kDyStages) & 1u, lim);
  };
  if (warp == 0) {
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      tile_origin(a, w.tile, m0, n0);
      const int m = int(m0) + int(rank) * kEdge;
      for (int c = w.c0; c < w.c1; ++c, ++issued, ring.next()) {
        ok = agreed(mbar_wait_ring_cluster(dy_empty + ring.at, ring.pass ^ 1u, lim));
        if (!ok) break;
        uint8_t* st = smem + ring.at * kOperand;
        uint64_t* bar = dy_full + ring.at;
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, kOperand);
          tma_load_2d(st, &tm_dy, m, c * kChunk, bar);
          tma_load_2d(st + kHalf, &tm_dy, m + 64, c * kChunk, bar);
        }
        __syncwarp();
      }
    }
  } else if (warp == kWarpCodes) {
    // codes, and scales: two tokens a lane, a word of four blocks each
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      tile_origin(a, w.tile, m0, n0);
      const int64_t n = n0 + int64_t(rank) * kEdge;
      const bool in = n / 32 < a.spitch;  // (a row's scales end with whole words)
      int64_t row = int64_t(w.c0) * kChunk + lane;
      const uint8_t* from = a.scales + row * a.spitch + n / 32;
      for (int c = w.c0; c < w.c1; ++c, ++issued, code_ring.next()) {
        ok = agreed(mbar_wait_ring(code_empty + code_ring.at, code_ring.pass ^ 1u, lim));
        if (!ok) break;
        uint64_t* bar = code_full + code_ring.at;
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, kCodes);
          tma_load_2d(smem + kOffCodes + code_ring.at * kCodes, &tm_codes, int(n), c * kChunk, bar);
        }
        uint8_t* to = smem + kOffScales + code_ring.at * kScales + 4 * lane;
        const bool there = in && row < a.T, next = in && row + 32 < a.T;
        cp_async4_zfill(to, there ? from : a.scales, there ? 4u : 0u);
        cp_async4_zfill(to + 128, next ? from + 32 * a.spitch : a.scales, next ? 4u : 0u);
        cp_async_arrive(bar);
        row += kChunk;
        from += kChunk * a.spitch;
      }
    }
  } else if (warp == kWarpNotice) {
    // tells the thread that issues the MMAs, the pair's for both CTAs, that dY has landed
    uint32_t q = 0;
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      for (int c = w.c0; c < w.c1; ++c, ++q, ring.next(), slot.next()) {
        ok = agreed(mbar_wait_ring(dy_full + ring.at, ring.pass, lim) && slot_free(q));
        if (!ok) break;
        if (elect_one()) mbar_arrive_cluster(ready + slot.at, 0);
        __syncwarp();
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const uint32_t idesc = tc_idesc_bf16_f32_mn(kSide, kSide);
      // descriptors of the first stage and slot; addresses count in units of 16 bytes
      const uint64_t dy0 = tc_smem_desc_mn128(smem_addr(smem), kHalf), x0 = tc_smem_desc_mn128(smem_addr(smem + kOffSlots), kHalf);
      for (int i = 0; ok && work_of(a, g, i, w); ++i) {
        const int b = half_of<KEPT>(i);
        ok = agreed(mbar_wait_ring_cluster(free + b, turn_of<KEPT>(i) ^ 1u, lim));
        const uint32_t d = tmem + uint32_t(b) * kSide;
        for (int c = w.c0; ok && c < w.c1; ++c, ++committed, ring.next(), slot.next()) {
          ok = agreed(mbar_wait_ring_cluster(ready + slot.at, slot.pass, lim));
          if (!ok) break;
          tc_fence_after();
          const uint64_t dy = dy0 + uint32_t(ring.at) * (kOperand / 16), x = x0 + uint32_t(slot.at) * (kOperand / 16);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kChunk / 16; ++k)
              tc_mma_bf16_pair(d, dy + k * (2048 / 16), x + k * (2048 / 16), idesc, k > 0 || c > w.c0);
            tc_commit_pair(dy_empty + ring.at);
            if (c == w.c1 - 1) tc_commit_pair(sum + b);
          }
          __syncwarp();
        }
      }
    }
  } else if (warp < 2 + kConvertWarps * kSets) {
    // This thread's codes of a chunk: block b (of four) of every (64 / kUnits)-th token from k on.
    // The block's four 16-byte pieces of bf16 come in the order of its two 16-byte pieces of
    // codes, and which of those is first changes with the token and the half, so that neither the
    // loads nor the stores of eight neighbouring lanes meet on a bank.
    const int t = (tid - 64) % (32 * kConvertWarps), set = (warp - 2) / kConvertWarps, k = t >> 2, b = t & 3;
    constexpr int kStep = kChunk / kUnits;  // tokens from one unit to the next
    const uint32_t second = uint32_t((b >> 1) ^ (k & 1));  // whether the second piece of codes goes first
    const uint32_t codes_at = kOffCodes + k * kEdge + 32 * b + 16 * second, scale_at = kOffScales + 4 * k + b;
    const uint32_t row = kOffSlots + uint32_t(b >> 1) * kHalf + uint32_t(k) * 128;
    uint32_t piece[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) piece[e] = row + (((uint32_t(b & 1) * 4 + (uint32_t(e) ^ (2 * second))) ^ uint32_t(k & 7)) * 16);
    uint32_t n = 0;  // chunks of the tiles before
    for (int i = 0; ok && work_of(a, g, i, w); n += uint32_t(w.c1 - w.c0), ++i) {
      for (uint32_t q = n + (uint32_t(set) + kSets - n % kSets) % kSets; q < n + uint32_t(w.c1 - w.c0); q += kSets) {
        const uint32_t stage = q % kCodeStages, slot_at = q % kSlots;
        ok = agreed(mbar_wait_ring(code_full + stage, (q / kCodeStages) & 1u, lim));
        if (!ok) break;
        uint4 o[kUnits][4];
#pragma unroll
        for (int h = 0; h < kUnits; ++h) {
          const uint32_t at = stage * kCodes + codes_at + kStep * kEdge * h;
          const uint4 c0 = *reinterpret_cast<const uint4*>(smem + at), c1 = *reinterpret_cast<const uint4*>(smem + (at ^ 16u));
          const __nv_bfloat162 step = step_bf16x2(smem[stage * kScales + scale_at + 4 * kStep * h]);
          o[h][0] = codes8_bf16(c0.x, c0.y, step), o[h][1] = codes8_bf16(c0.z, c0.w, step);
          o[h][2] = codes8_bf16(c1.x, c1.y, step), o[h][3] = codes8_bf16(c1.z, c1.w, step);
        }
        ok = agreed(slot_free(q));
        if (!ok) break;
        uint8_t* to = smem + slot_at * kOperand;
#pragma unroll
        for (int h = 0; h < kUnits; ++h) {
#pragma unroll
          for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(to + piece[e] + kStep * 128 * h) = o[h][e];
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(code_empty + stage);
          mbar_arrive_cluster(ready + slot_at, 0);
        }
      }
    }
  } else {
    const int quarter = warp & 3;
    for (int i = 0; ok && work_of(a, g, i, w); ++i) {
      const int b = half_of<KEPT>(i);
      tile_origin(a, w.tile, m0, n0);
      const int r = int(rank) * kEdge + quarter * 32 + lane;  // row of the tile
      const int64_t m = m0 + r;
      if (a.acc != nullptr && w.slot < 0 && m < a.rows) {
        // acc's row comes into L2 while the sum is formed (with two loads at a time, 3000 tokens of 18944 x 3584:
        // 428 us, 488 with neither)
        for (int q = 0; q < kSide / 32 && n0 + 32 * q < a.cols; ++q)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(a.acc + m * a.cols + n0 + 32 * q));
      }
      ok = agreed(mbar_wait_ring_cluster(sum + b, turn_of<KEPT>(i), lim));
      if (!ok) break;
      tc_fence_after();
      float4* part = reinterpret_cast<float4*>(a.part) + int64_t(w.slot) * kSide * (kSide / 4) + r;
      for (int q = 0; q < kSide / 32; ++q) {
        uint32_t u[32];
        const uint32_t from = tmem + (uint32_t(quarter * 32) << 16) + uint32_t(b * kSide + 32 * q);
        tc_ld32(from, u);
        float v[32];
        input_order(u, v);
        if (KEPT && w.slot < 0 && !(w.first && w.last)) {
          // (the total's columns are as they are written out)
#pragma unroll
          for (int h = 0; h < 32; h += 16) {
            uint32_t t[16];
            if (!w.first) {
              tc_ld16(from + kSide + h, t);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[h + e] += __uint_as_float(t[e]);
            }
            if (!w.last) {
#pragma unroll
              for (int e = 0; e < 16; ++e) t[e] = __float_as_uint(v[h + e]);
              tc_st16(from + kSide + h, t);
            }
          }
          if (!w.last) continue;
        }
        if (w.slot >= 0) {
          if (!w.first) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 x = load_written(part + (8 * q + e / 4) * kSide);
              v[e] += x.x, v[e + 1] += x.y, v[e + 2] += x.z, v[e + 3] += x.w;
            }
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4) part[(8 * q + e / 4) * kSide] = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        } else if constexpr (OUT == Out::kSectors) {
          if (m < a.rows && n0 + 32 * q < a.cols) store_sectors(a, w.last, m, n0 + 32 * q, v);
        } else if (n0 + 32 * q < a.cols) {
          store_block<OUT == Out::kPairs>(a, w.last, reinterpret_cast<float*>(smem + kOffBlocks) + quarter * 16 * kBlockPitch, m - lane,
                                          n0 + 32 * q, v);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_tmem(free + b, 0);
    }
  }
  if (!ok) misc[1] = 0u;
  __syncthreads();
  if (misc[1] == 0u) {
    // a wait gave up: the copies this CTA sent off land, and its MMAs end, before it leaves
    if (warp == 0) {
      for (int c = issued > kDyStages ? issued - kDyStages : 0; c < issued; ++c)
        mbar_wait_bounded(dy_full + c % kDyStages, uint32_t(c / kDyStages) & 1u);
    }
    if (warp == kWarpCodes) {
      for (int c = issued > kCodeStages ? issued - kCodeStages : 0; c < issued; ++c)
        mbar_wait_bounded(code_full + c % kCodeStages, uint32_t(c / kCodeStages) & 1u);
    }
    if (warp == 1 && committed > 0)
      mbar_wait_bounded(dy_empty + (committed - 1) % kDyStages, uint32_t((committed - 1) / kDyStages) & 1u);
    if (tid == 0) atomicOr(a.status, kStatusTimeout);
    __syncthreads();
  }
  tc_fence_after();
  cluster_sync();
  if (warp == 0) tc_dealloc_pair(tmem, kTmemCols);
}

template <Out OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    roi_wgrad_kernel(const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_codes, WgradArgs a) {
  wgrad<OUT, false>(tm_dy, tm_codes, a);
}
// (a kernel of its own: where the other held both ways, its epilogue spilled more, 35.2 -> 36.4 us for 1999 tokens of
// 1215 x 2504 with acc)
template <Out OUT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    roi_wgrad_long_kernel(const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_codes, WgradArgs a) {
  wgrad<OUT, true>(tm_dy, tm_codes, a);
}

// The tiles of the last round whose tokens were cut: their partial sums in the order of the
// ranges.  A CTA takes 8 rows of a tile; a lane reads four columns of its row (eight lanes 128
// consecutive bytes), and the rows are written out through shared memory.
constexpr int kJoinRows = 8;
__global__ void __launch_bounds__(256) roi_wgrad_join_kernel(WgradArgs a) {
  constexpr int kQuads = kSide / 4, kEach = kQuads / 32, kAhead = 4;
  __shared__ float rows[kJoinRows][kSide + 4];
  pdl_begin(true);  // the partial sums of the launch before
  const int tile = blockIdx.x / (kSide / kJoinRows), r0 = blockIdx.x % (kSide / kJoinRows) * kJoinRows;
  int64_t m0, n0;
  tile_origin(a, a.rounds * a.groups + tile, m0, n0);
  m0 += r0;
  if (m0 >= a.rows) return;
  // the ranges that hold the tile's first and last chunk
  const int64_t t0 = int64_t(tile) * a.chunks, t1 = t0 + a.chunks - 1;
  int p0 = int(t0 * a.ranges / (int64_t(a.rest) * a.chunks)), p1 = int(t1 * a.ranges / (int64_t(a.rest) * a.chunks));
  while (range_start(a, p0 + 1) <= t0) ++p0;
  while (range_start(a, p1 + 1) <= t1) ++p1;
  if (p0 == p1) return;  // whole, and written already
  const int r = threadIdx.x & 7, quad = threadIdx.x >> 3;
  // (only the first range may have begun in the tile before, whose sums are in its other slot)
  const int first = 2 * p0 + (range_start(a, p0) < t0 ? 1 : 0);
  const float4* part = reinterpret_cast<const float4*>(a.part) + r0 + r + quad * kSide;
  float4 s[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) s[e] = __ldcs(part + int64_t(first) * kSide * kQuads + 32 * e * kSide);
  for (int p = p0 + 1; p <= p1; p += kAhead) {
    float4 v[kAhead][kEach];
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (p + q <= p1) v[q][e] = __ldcs(part + int64_t(2 * (p + q)) * kSide * kQuads + 32 * e * kSide);
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (p + q <= p1) s[e].x += v[q][e].x, s[e].y += v[q][e].y, s[e].z += v[q][e].z, s[e].w += v[q][e].w;
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) *reinterpret_cast<float4*>(&rows[r][4 * (quad + 32 * e)]) = s[e];
  __syncthreads();
  const bool fours = a.cols % 4 == 0;
  for (int i = threadIdx.x; i < kJoinRows * kQuads; i += 256) {
    const int w = i / kQuads, c = i % kQuads * 4;
    if (m0 + w >= a.rows || n0 + c >= a.cols) continue;
    float v[4] = {rows[w][c], rows[w][c + 1], rows[w][c + 2], rows[w][c + 3]};
    const int64_t at = (m0 + w) * a.cols + n0 + c;
    if (fours) {
      if (a.acc != nullptr) {
        float4* q = reinterpret_cast<float4*>(a.acc + at);
        const float4 x = *q;
        v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
        *q = make_float4(v[0], v[1], v[2], v[3]);
      }
      if (a.dWm != nullptr) *reinterpret_cast<uint2*>(a.dWm + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (n0 + c + k >= a.cols) break;
        if (a.acc != nullptr) a.acc[at + k] = v[k] += a.acc[at + k];
        if (a.dWm != nullptr) a.dWm[at + k] = __bfloat16_as_ushort(__float2bfloat16_rn(v[k]));
      }
    }
  }
}

// dY with rows that are not multiples of 16 bytes apart, laid out again with rows that are: `width` threads (a power of
// two) a row, each eight columns at a time by the granules around them.  16000 tokens of
// 3000 x 200: 81 us with this launch, 126 where it went element by element, 36 where dY's rows are aligned.
__global__ void __launch_bounds__(256) roi_wgrad_align_kernel(const uint16_t* src, int64_t ld, uint16_t* dst, int64_t pitch, int64_t T,
                                                              int64_t cols, int width, bool wait) {
  using E = ElemType<Elem::kBf16>::T;
  pdl_begin(wait);
  const int per = 256 / width, j = threadIdx.x & (width - 1);
  for (int64_t t = int64_t(blockIdx.x) * per + threadIdx.x / width; t < T; t += int64_t(gridDim.x) * per) {
#pragma unroll 2
    for (int64_t c = 8 * j; c < cols; c += 8 * width) {
      Window<Elem::kBf16, 8> x;
      x.load(reinterpret_cast<const E*>(src) + t * ld, c, cols);
      RowWords<Elem::kBf16, 8> r;
      x.get(r);
      *reinterpret_cast<uint4*>(dst + t * pitch + c) = make_uint4(r.u[0], r.u[1], r.u[2], r.u[3]);
    }
  }
}

// No tokens: an empty sum.
__global__ void __launch_bounds__(256) roi_wgrad_empty_kernel(uint16_t* dWm, const float* acc, int64_t n, bool wait) {
  pdl_begin(wait);
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
    dWm[i] = __bfloat16_as_ushort(__float2bfloat16_rn(acc == nullptr ? 0.0f : acc[i]));
}

// The division of the work among the groups, and the bytes of partial sums it needs.
size_t plan(int64_t T, int64_t rows, int64_t cols, WgradArgs& a) {
  constexpr int64_t side = kSide;
  a.T = T;
  a.rows = rows;
  a.cols = cols;
  a.tiles_m = int((rows + side - 1) / side);
  a.tiles_n = int((cols + side - 1) / side);
  // The larger operand (dY in 2 bytes, codes in one) is read through once, the other from L2.  Against the other
  // order, 8192 tokens: 18944 x 3584 601 and 737 us, 3584 x 18944 619 and 657, 2048 x 11008 218 and 231.
  a.n_first = 2 * rows >= cols;
  a.chunks = int((T + kChunk - 1) / kChunk);
  a.groups = sm_count() / 2;
  if (a.groups < 1) a.groups = 1;
  const int64_t tiles = int64_t(a.tiles_m) * a.tiles_n;
  a.rounds = int(tiles / a.groups);
  a.rest = int(tiles - int64_t(a.rounds) * a.groups);
  a.ranges = 0;
  const int64_t units = int64_t(a.rest) * a.chunks;
  const int64_t most = units / kMinRange < a.groups ? units / kMinRange : a.groups;
  if (most > a.rest && (units + most - 1) / most + kSplitCost < a.chunks) a.ranges = int(most);
  return a.ranges == 0 ? 0 : size_t(a.ranges) * 2 * side * side * 4;
}

int64_t aligned_pitch(int64_t rows) { return (rows + 7) / 8 * 8; }
bool needs_copy(int64_t T, int64_t ld) { return T > 1 && ld % 8 != 0; }

}  // namespace

size_t wgrad_workspace_bytes(int64_t T, int64_t rows, int64_t cols, int64_t lddy) {
  WgradArgs a;
  return plan(T, rows, cols, a) + (needs_copy(T, lddy) ? size_t(T) * size_t(aligned_pitch(rows)) * 2 : 0);
}
size_t wgrad_copy_bytes(int64_t T, int64_t rows, int64_t lddy) {
  return needs_copy(T, lddy) ? size_t(T) * size_t(aligned_pitch(rows)) * 2 : 0;
}

int launch_wgrad(const WgradCall& c) {
  bool wait = lone_pdl(c.stream);
  if (c.T == 0) {
    if (c.dWm == nullptr) return 0;
    const int64_t n = c.rows * c.cols, blocks = (n + 255) / 256, cap = int64_t(sm_count()) * 8;
    return launch_maybe_pdl(roi_wgrad_empty_kernel, int(blocks < cap ? blocks : cap), 256, 0, c.stream, wait, c.dWm,
                            static_cast<const float*>(c.acc), n, wait);
  }
  int launched = 0;
  const uint16_t* dY = c.dY;
  int64_t ld = c.T > 1 ? c.lddy : aligned_pitch(c.rows);
  uint8_t* ws = static_cast<uint8_t*>(c.workspace);
  size_t room = c.workspace_bytes;
  if (needs_copy(c.T, c.lddy)) {
    // the copy lies at the workspace's start, the partial sums behind it
    ld = aligned_pitch(c.rows);
    const int64_t cap = int64_t(sm_count()) * 8;
    int width = 8;
    while (width < 256 && width * 8 < c.rows) width *= 2;
    const int64_t blocks = (c.T + 256 / width - 1) / (256 / width);
    launched = launch_maybe_pdl(roi_wgrad_align_kernel, int(blocks < cap ? blocks : cap), 256, 0, c.stream, wait, c.dY, c.lddy,
                                reinterpret_cast<uint16_t*>(ws), ld, c.T, c.rows, width, wait);
    if (launched < 0) return -1;
    dY = reinterpret_cast<const uint16_t*>(ws);
    const size_t used = wgrad_copy_bytes(c.T, c.rows, c.lddy);
    ws += used;
    room -= used;
    wait = true;
  }
  WgradArgs a;
  const size_t need = plan(c.T, c.rows, c.cols, a);
  if (need > (ws == nullptr ? 0 : room)) a.ranges = 0;  // no room for partial sums: tiles stay whole
  a.scales = c.scales;
  a.dWm = c.dWm;
  a.acc = c.acc;
  const int most = c.acc != nullptr ? kMostChunks : kMostAlone;
  a.unbroken = a.chunks > most ? most : a.chunks;
  const bool kept = c.acc == nullptr && a.chunks > most;
  a.part = reinterpret_cast<float*>(ws);
  a.spitch = block8_scale_pitch(c.cols);
  a.status = c.status;
  a.wait = wait;
  CUtensorMap tm_dy, tm_codes;
  const int64_t pitch = block8_pitch(c.cols);
  if (!make_tensor_map(&tm_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dY, uint64_t(c.rows), uint64_t(c.T), uint64_t(ld) * 2, 64, kChunk,
                       CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B) ||
      !make_tensor_map(&tm_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, c.codes, uint64_t(pitch), uint64_t(c.T), uint64_t(pitch), kEdge,
                       kChunk, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B))
    return -1;
  // whole sectors where the outputs' rows are in sixteens of columns; else through shared memory
  const bool sectors = c.cols % 16 == 0 && ((reinterpret_cast<uintptr_t>(c.dWm) | reinterpret_cast<uintptr_t>(c.acc)) & 31u) == 0;
  const int form = (sectors ? 0 : c.cols % 2 == 0 ? 1 : 2) + (kept ? 3 : 0);
  constexpr decltype(&roi_wgrad_kernel<Out::kSectors>) forms[6] = {
      roi_wgrad_kernel<Out::kSectors>,      roi_wgrad_kernel<Out::kPairs>,      roi_wgrad_kernel<Out::kSingles>,
      roi_wgrad_long_kernel<Out::kSectors>, roi_wgrad_long_kernel<Out::kPairs>, roi_wgrad_long_kernel<Out::kSingles>};
  auto kern = forms[form];
  constexpr size_t smem = kSmem + 1024;
  static std::atomic<bool> set[6][64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return -1;
  if (!set[form][dev].load(std::memory_order_acquire)) {
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return -1;
    set[form][dev].store(true, std::memory_order_release);
  }
  const int64_t busy = a.rounds > 0 ? a.groups : a.ranges > 0 ? a.ranges : a.rest;
  if (launch_maybe_pdl(kern, int(busy) * 2, kThreads, smem, c.stream, wait, tm_dy, tm_codes, a) < 0) return -1;
  ++launched;
  if (a.ranges > 0) {
    if (launch_maybe_pdl(roi_wgrad_join_kernel, a.rest * (kSide / kJoinRows), 256, 0, c.stream, true, a) < 0) return -1;
    ++launched;
  }
  return launched;
}

}  // namespace roi
