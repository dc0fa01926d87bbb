// The AdamW step over many tensors at once (the one of roi_mask_bwd_adamw, on gradients that are there already: after a
// data-parallel reduction, or of norm weights), with moments in 32 bits, or in 8.
//
// Moments in 8 bits: m in e4m3 and u = sqrt(v) without a sign, four bits of exponent and four of mantissa with the same
// bias, in blocks of 128 consecutive elements with a power of two each (2^(s - 127), s - 127 the least exponent that keeps
// the block's largest under the largest code, 448 and 480).  The root halves v's range in octaves, so that 19 octaves under a
// block's largest stay.  Codes are rounded up with the probability of what they would drop: u moves by at most
// 1 - sqrt(b2) a step, 2.5 % at b2 = 0.95, less than half of a code's step, so that to the nearest it would never move down.
// The probability is compared in 16 bits, m's in the low and u's in the high half of the element's Philox word (counter
// as the mask's noise: element / 4, step, tensor).  The parameters take the step from the moments before they are rounded.
//
// Bound by memory in 32 bits (28 bytes an element, fp32 gradients); in 8 (16 bytes) near the rate of its instructions.
//
// Tensors are cut into tiles of 1024 elements that follow one another over all tensors; a CTA has a range of them.  A
// thread has four elements of a tile, so in 8 bits a warp has a block.
#include "roi_launch.h"

namespace roi {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 4 * kThreads;

struct Item {
  float* p;
  const void* g;
  void* a;          // m, or its codes
  void* b;          // v, or u's codes
  uint8_t* scales;  // (8 bits) two bytes a block: m's and u's
  void* copy;       // nullable
  int64_t n;
  int64_t tile0;    // its first tile among all
  uint32_t id;
  uint8_t grad, copied;  // roi_dtype
};
constexpr int kMost = 400;  // items a launch
struct Args {
  int count;
  bool wait;
  AdamW opt;
  uint32_t k0, k1, step;
  const float* scale;  // nullable: a factor of the gradients
  int64_t tiles;
  Item it[kMost];
};
static_assert(sizeof(Args) <= 32764, "kernel parameter block");

__device__ __forceinline__ float element(uint32_t word, int half, bool fp16) {
  const uint16_t h = uint16_t(half ? word >> 16 : word);
  return fp16 ? to_f32<Elem::kFp16>(h) : to_f32<Elem::kBf16>(h);
}
// Four gradients from element e on (a multiple of 4), zeros past the last.
__device__ __forceinline__ void load_grad(const Item& it, int64_t e, float (&g)[4]) {
  const bool whole = e + 4 <= it.n;
  if (it.grad == uint8_t(Elem::kFp32)) {
    const float* p = static_cast<const float*>(it.g) + e;
    if (whole) {
      const float4 x = __ldcs(reinterpret_cast<const float4*>(p));
      g[0] = x.x, g[1] = x.y, g[2] = x.z, g[3] = x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = e + i < it.n ? p[i] : 0.0f;
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(it.g) + e;
    const bool fp16 = it.grad == uint8_t(Elem::kFp16);
    uint2 x = make_uint2(0u, 0u);
    if (whole) {
      x = __ldcs(reinterpret_cast<const uint2*>(p));
    } else {
      if (e < it.n) x.x = p[0];
      if (e + 1 < it.n) x.x |= uint32_t(p[1]) << 16;
      if (e + 2 < it.n) x.y = p[2];
    }
    g[0] = element(x.x, 0, fp16), g[1] = element(x.x, 1, fp16), g[2] = element(x.y, 0, fp16), g[3] = element(x.y, 1, fp16);
  }
}
__device__ __forceinline__ void load4(const float* p, int64_t e, int64_t n, float (&v)[4]) {
  if (e + 4 <= n) {
    const float4 x = *reinterpret_cast<const float4*>(p + e);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = e + i < n ? p[e + i] : 0.0f;
  }
}
__device__ __forceinline__ void store4(float* p, int64_t e, int64_t n, const float (&v)[4]) {
  if (e + 4 <= n) {
    *reinterpret_cast<float4*>(p + e) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + i < n) p[e + i] = v[i];
  }
}
// Rounded to bf16 or fp16.
__device__ __forceinline__ void store_half4(void* to, bool fp16, int64_t e, int64_t n, const float (&v)[4]) {
  uint16_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = fp16 ? from_f32<Elem::kFp16>(v[i]) : from_f32<Elem::kBf16>(v[i]);
  uint16_t* p = static_cast<uint16_t*>(to) + e;
  if (e + 4 <= n) {
    *reinterpret_cast<uint2*>(p) = make_uint2(h[0] | uint32_t(h[1]) << 16, h[2] | uint32_t(h[3]) << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + i < n) p[i] = h[i];
  }
}

// ---------------------------------------------------------------------------
// moments in 8 bits
// ---------------------------------------------------------------------------
// A code's bits at the place of a float's are the code's value times 2^-120, subnormals among them.
constexpr int kMBits = 3, kUBits = 4;
template <int BITS>
__device__ __forceinline__ float decode(uint32_t code, float step) {
  constexpr uint32_t kNaN = BITS == kMBits ? 0x7fu : 0xffu;
  const uint32_t c = BITS == kMBits ? code & 0x7fu : code;
  float v = __uint_as_float(c << (23 - BITS)) * __uint_as_float((120u + 127u) << 23) * step;
  if (c == kNaN) v = __uint_as_float(0x7fc00000u);
  return BITS == kMBits && (code & 0x80u) != 0u ? -v : v;
}
// 2^(s - 127), and 2^(127 - s); scale bytes that no step writes stand for the nearest that one does.
__device__ __forceinline__ float scale_step(uint32_t s) { return __uint_as_float(min(max(s, 1u), 247u) << 23); }
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __uint_as_float((254u - s) << 23); }
// The scale byte from the bits of the largest finite magnitude (largest codes 1.75 2^8 and 1.875 2^8).
template <int BITS>
__device__ __forceinline__ uint32_t state_scale(uint32_t top_bits) {
  constexpr uint32_t kAbove = BITS == kMBits ? 0x1fffffu : 0x0fffffu;
  return uint32_t(max(int((top_bits + kAbove) >> 23) - 8, 1));
}
// The code of a magnitude: what is below its last bit decides with 16 random bits whether it is rounded up.
template <int BITS>
__device__ __forceinline__ uint32_t encode(float x, float inverse, uint32_t random) {
  constexpr int kDrop = 23 - BITS;
  const uint32_t bits = abs_bits(x);
  // (towards zero: what is under 2^-149 is dropped)
  const uint32_t t = __float_as_uint(__fmul_rz(__uint_as_float(bits) * inverse, __uint_as_float((127u - 120u) << 23)));
  const uint32_t code = (t + (random << (kDrop - 16))) >> kDrop;
  return bits >= kInfBits ? (BITS == kMBits ? 0x7fu : 0xffu) : code;
}
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = abs_bits(x);
  return b >= kInfBits ? 0u : b;
}

// One element's step; u is the root of the new v.  (adamw_elem, operation for operation.)
__device__ __forceinline__ void step_elem(float& p, float g, float& m, float& v, float& u, const AdamW& o) {
  p = __fmul_rn(p, o.decay);
  m = __fadd_rn(__fmul_rn(o.b1, m), __fmul_rn(o.omb1, g));
  v = __fadd_rn(__fmul_rn(o.b2, v), __fmul_rn(o.omb2, __fmul_rn(g, g)));
  u = __fsqrt_rn(v);
  p = __fsub_rn(p, __fdiv_rn(__fmul_rn(o.step, m), __fadd_rn(__fmul_rn(u, o.r), o.eps)));
}

// The range of tiles of this CTA, and the item of its first.
struct Walk {
  int64_t tile, end;
  int item;
  __device__ __forceinline__ explicit Walk(const Args& a) {
    tile = int64_t(blockIdx.x) * a.tiles / gridDim.x;
    end = int64_t(blockIdx.x + 1) * a.tiles / gridDim.x;
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.it[mid].tile0 <= tile) lo = mid;
      else hi = mid - 1;
    }
    item = lo;
  }
};

__global__ void __launch_bounds__(kThreads) roi_adamw_step_kernel(const __grid_constant__ Args a) {
  pdl_begin(a.wait);
  const float scale = a.scale != nullptr ? __ldg(a.scale) : 1.0f;
  for (Walk w(a); w.tile < w.end; ++w.tile) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * kTile + 4 * threadIdx.x;
    if (e >= it.n) continue;
    float p[4], g[4], m[4], v[4], u;
    load4(it.p, e, it.n, p);
    load4(static_cast<const float*>(it.a), e, it.n, m);
    load4(static_cast<const float*>(it.b), e, it.n, v);
    load_grad(it, e, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) step_elem(p[i], a.scale != nullptr ? __fmul_rn(g[i], scale) : g[i], m[i], v[i], u, a.opt);
    store4(it.p, e, it.n, p);
    store4(static_cast<float*>(it.a), e, it.n, m);
    store4(static_cast<float*>(it.b), e, it.n, v);
    if (it.copy != nullptr) store_half4(it.copy, it.copied == uint8_t(Elem::kFp16), e, it.n, p);
  }
}

__global__ void __launch_bounds__(kThreads) roi_adamw_step8_kernel(const __grid_constant__ Args a) {
  pdl_begin(a.wait);
  const float scale = a.scale != nullptr ? __ldg(a.scale) : 1.0f;
  const int lane = threadIdx.x & 31;
  for (Walk w(a); w.tile < w.end; ++w.tile) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * kTile + 4 * threadIdx.x;
    if (e - 4 * lane >= it.n) continue;  // (a warp has a block)
    uint32_t* mc = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(it.a) + e);
    uint32_t* uc = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(it.b) + e);
    uint16_t* sc = reinterpret_cast<uint16_t*>(it.scales) + (e >> 7);
    float p[4], g[4], m[4], u[4];
    load4(it.p, e, it.n, p);
    load_grad(it, e, g);
    const uint32_t mw = *mc, uw = *uc, sw = *sc;
    const uint4 random = philox4x32_10(make_uint4(uint32_t(e >> 2), uint32_t(uint64_t(e) >> 34), a.step, it.id), a.k0, a.k1);
    const float m_step = scale_step(sw & 0xffu), u_step = scale_step(sw >> 8);
    uint32_t m_top = 0, u_top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = decode<kMBits>((mw >> (8 * i)) & 0xffu, m_step);
      u[i] = decode<kUBits>((uw >> (8 * i)) & 0xffu, u_step);
      float v = __fmul_rn(u[i], u[i]);
      step_elem(p[i], a.scale != nullptr ? __fmul_rn(g[i], scale) : g[i], m[i], v, u[i], a.opt);
      if (e + i >= it.n) m[i] = 0.0f, u[i] = 0.0f;  // (padding's codes are 0)
      m_top = max(m_top, finite_bits(m[i]));
      u_top = max(u_top, finite_bits(u[i]));
    }
    const uint32_t ms = state_scale<kMBits>(__reduce_max_sync(0xffffffffu, m_top)),
                   us = state_scale<kUBits>(__reduce_max_sync(0xffffffffu, u_top));
    const float m_inverse = scale_inverse(ms), u_inverse = scale_inverse(us);
    const uint32_t r[4] = {random.x, random.y, random.z, random.w};
    uint32_t mo = 0, uo = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c = encode<kMBits>(m[i], m_inverse, r[i] & 0xffffu) | ((__float_as_uint(m[i]) >> 24) & 0x80u);
      uint32_t d = encode<kUBits>(u[i], u_inverse, r[i] >> 16);
      if (u[i] > 0.0f) d = max(d, 1u);  // what is not zero stays so: a step divides by it
      mo |= c << (8 * i);
      uo |= d << (8 * i);
    }
    *mc = mo;
    *uc = uo;
    if (lane == 0) *sc = uint16_t(ms | us << 8);
    store4(it.p, e, it.n, p);
    if (it.copy != nullptr) store_half4(it.copy, it.copied == uint8_t(Elem::kFp16), e, it.n, p);
  }
}

// What states in 8 bits stand for.  (Items: p and copy are where m and u go, `grad` their type.)
__global__ void __launch_bounds__(kThreads) roi_adamw_state8_load_kernel(const __grid_constant__ Args a) {
  pdl_begin(a.wait);
  for (Walk w(a); w.tile < w.end; ++w.tile) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * kTile + 4 * threadIdx.x;
    if (e >= it.n) continue;
    const uint32_t mw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(it.a) + e);
    const uint32_t uw = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(it.b) + e);
    const uint32_t sw = reinterpret_cast<const uint16_t*>(it.scales)[e >> 7];
    const float m_step = scale_step(sw & 0xffu), u_step = scale_step(sw >> 8);
    float m[4], u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = decode<kMBits>((mw >> (8 * i)) & 0xffu, m_step);
      u[i] = decode<kUBits>((uw >> (8 * i)) & 0xffu, u_step);
    }
    if (it.grad == uint8_t(Elem::kFp32)) {
      if (it.p != nullptr) store4(it.p, e, it.n, m);
      if (it.copy != nullptr) store4(static_cast<float*>(it.copy), e, it.n, u);
    } else {
      const bool fp16 = it.grad == uint8_t(Elem::kFp16);
      if (it.p != nullptr) store_half4(it.p, fp16, e, it.n, m);
      if (it.copy != nullptr) store_half4(it.copy, fp16, e, it.n, u);
    }
  }
}

}  // namespace

int launch_optim(const OptimCall& c, const OptimItem* items, int count) {
  int launched = 0;
  bool wait = lone_pdl(c.stream);
  Args a;
  a.opt = c.opt;
  a.k0 = uint32_t(c.seed);
  a.k1 = uint32_t(c.seed >> 32);
  a.step = c.step;
  a.scale = c.scale;
  auto kern = c.kind == OptimKind::kStep ? roi_adamw_step_kernel
              : c.kind == OptimKind::kStep8 ? roi_adamw_step8_kernel
                                            : roi_adamw_state8_load_kernel;
  for (int i = 0; i < count;) {
    a.count = 0;
    a.tiles = 0;
    for (; i < count && a.count < kMost; ++i) {
      const OptimItem& x = items[i];
      if (x.n == 0) continue;
      a.it[a.count++] = {x.p, x.g, x.a, x.b, x.scales, x.copy, x.n, a.tiles, x.id, uint8_t(x.grad), uint8_t(x.copied)};
      a.tiles += (x.n + kTile - 1) / kTile;
    }
    if (a.count == 0) break;
    a.wait = wait;
    const int64_t cap = int64_t(sm_count()) * 5;
    if (launch_maybe_pdl(kern, int(a.tiles < cap ? a.tiles : cap), kThreads, 0, c.stream, wait, a) < 0) return -1;
    ++launched;
    wait = true;
  }
  return launched;
}

}  // namespace roi
