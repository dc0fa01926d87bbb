// The AdamW step over many tensors at once (the one of roi_mask_bwd_adamw, on gradients that are there already: after a
// data-parallel reduction, or of norm weights), with moments in 32 bits, or in 8.
//
// Moments in 8 bits: m in e4m3 and u = sqrt(v) without a sign, four bits of exponent and four of mantissa with the same
// bias, in blocks of 128 consecutive elements with a power of two each (2^(s - 127), s - 127 the least exponent that keeps
// the block's largest under the largest code, 448 and 480).  The root halves v's range in octaves, so that 19 octaves under a
// block's largest stay.  Codes are rounded up with the probability of what they would drop.  To the nearest, u would not follow
// a vanishing gradient down: it falls by 1 - sqrt(b2) a step, 2.5 % at b2 = 0.95, and half a code's step is 3.1 % of u at the start of an
// octave and 1.6 % at its end, so that it would fall too fast there and stay for good at 1.1875 times a power of two, or 1.125, or 1.0625.
// The probability is compared in 16 bits, m's in the low and u's in the high half of the element's Philox word (counter
// as the mask's noise: element / 4, step, tensor).  The parameters take the step from the moments before they are rounded.
//
// Bound by memory: 28 bytes an element in 32 bits (fp32 gradients; 7.15 TB/s, where a copy has 6.79), 16 in 8 (6.0).
//
// Tensors are cut into tiles that follow one another over all tensors; a CTA has every gridDim.x-th.  A thread has 8
// consecutive elements of a tile, or 16 where the moments are in 8 bits: whole sectors of each array, and a block in eight
// neighbouring lanes.
#include "roi_launch.h"
#include "roi_rows.cuh"

namespace roi {
namespace {

constexpr int kThreads = 128;
constexpr int kEach32 = 8, kEach8 = 16, kBlock = 128;
constexpr int kCtas32 = 10, kCtas8 = 5, kCtasLoad = 12;  // of an SM
// In 32 bits a launch has a CTA a tile, so that tiles are taken in their order: 912 us for a 7B-shaped block's step, 1019 where the CTAs
// that the SMs hold went over them, 992 and 959 with two and four times as many.  In 8 bits, where a CTA's start counts, four
// times what is held (the block with the states read back: one, two, four, eight times and a CTA a tile 893, 864, 852, 844, 885 us;
// eight 0.5B-shaped blocks 468, 457, 454, 467, 467).
constexpr int kWaves8 = 4;

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
  bool sectors;          // every array starts on a sector
};
// Items a launch: a launch copies its arguments whole, so few have a form of their own (nine tensors, one call on the host:
// 5.2 us with the arguments of 400, 4.3 with those of 24).
constexpr int kMost = 400, kFew = 24;
struct Settings {
  int count;
  bool wait;
  AdamW opt;
  uint32_t keys[2][10];  // of Philox's rounds
  uint32_t step;
  const float* scale;  // nullable: a factor of the gradients
  bool plain;          // (8 bits) settings within quick_pair's range
  float one;           // 1, as a number that the compiler does not know (add2)
  int64_t tiles;
};
template <int N>
struct ArgsOf : Settings {
  Item it[N];
};
static_assert(sizeof(ArgsOf<kMost>) <= 32764, "kernel parameter block");

// Whole sectors (memory that this kernel writes as well).
__device__ __forceinline__ void load_sector(const void* p, uint32_t* w) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
// N elements from the `left` of a row that are left (zeros past them), and back.
template <Elem E, int N>
__device__ __forceinline__ void load_words(const void* p, int64_t left, bool sectors, RowWords<E, N>& r) {
  using T = typename ElemType<E>::T;
  constexpr int W = RowWords<E, N>::kWords;
  if (left >= N && W % 8 == 0 && sectors) {
#pragma unroll
    for (int i = 0; i < W / 8; ++i) load_sector(static_cast<const uint32_t*>(p) + 8 * i, r.u + 8 * i);
  } else if (left >= N) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[i];
      r.u[4 * i] = v.x, r.u[4 * i + 1] = v.y, r.u[4 * i + 2] = v.z, r.u[4 * i + 3] = v.w;
    }
  } else {
    r.zero();
    const T* q = static_cast<const T*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i < left) {
        if constexpr (E == Elem::kFp32) r.u[i] = __float_as_uint(q[i]);
        else r.u[i / 2] |= uint32_t(q[i]) << (16 * (i % 2));
      }
    }
  }
}
template <Elem E, int N>
__device__ __forceinline__ void store_words(void* p, int64_t left, bool sectors, const RowWords<E, N>& r) {
  using T = typename ElemType<E>::T;
  constexpr int W = RowWords<E, N>::kWords;
  if (left >= N && W % 8 == 0 && sectors) {
#pragma unroll
    for (int i = 0; i < W / 8; ++i) store32(static_cast<uint32_t*>(p) + 8 * i, r.u + 8 * i);
  } else if (left >= N) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i)
      reinterpret_cast<uint4*>(p)[i] = make_uint4(r.u[4 * i], r.u[4 * i + 1], r.u[4 * i + 2], r.u[4 * i + 3]);
  } else {
    T* q = static_cast<T*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < left) q[i] = r.at(i);
  }
}
template <Elem E, int N>
__device__ __forceinline__ void load_sectors(const void* p, float (&v)[N]) {
  RowWords<E, N> r;
#pragma unroll
  for (int i = 0; i < RowWords<E, N>::kWords / 8; ++i) load_sector(static_cast<const uint32_t*>(p) + 8 * i, r.u + 8 * i);
  r.get(v);
}
template <int N>
__device__ __forceinline__ void load_floats(const void* p, int64_t left, bool sectors, float (&v)[N]) {
  RowWords<Elem::kFp32, N> r;
  load_words(p, left, sectors, r);
  r.get(v);
}
template <int N>
__device__ __forceinline__ void store_floats(void* p, int64_t left, bool sectors, const float (&v)[N]) {
  RowWords<Elem::kFp32, N> r;
  r.set(v);
  store_words(p, left, sectors, r);
}
// In 16 bits or 32.
template <int N>
__device__ __forceinline__ void load_any(const void* p, uint8_t type, int64_t e, int64_t left, bool sectors, float (&v)[N]) {
  if (type == uint8_t(Elem::kFp32)) {
    load_floats(static_cast<const float*>(p) + e, left, sectors, v);
    return;
  }
  RowWords<Elem::kBf16, N> r;
  load_words(static_cast<const uint16_t*>(p) + e, left, sectors, r);
  if (type == uint8_t(Elem::kBf16)) {
    r.get(v);
  } else {
    RowWords<Elem::kFp16, N> h;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) h.u[i] = r.u[i];
    h.get(v);
  }
}
template <int N>
__device__ __forceinline__ void store_any(void* p, uint8_t type, int64_t e, int64_t left, bool sectors, const float (&v)[N]) {
  if (type == uint8_t(Elem::kFp32)) {
    store_floats(static_cast<float*>(p) + e, left, sectors, v);
    return;
  }
  RowWords<Elem::kBf16, N> r;
  if (type == uint8_t(Elem::kBf16)) {
    r.set(v);
  } else {
    RowWords<Elem::kFp16, N> h;
    h.set(v);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r.u[i] = h.u[i];
  }
  store_words(static_cast<uint16_t*>(p) + e, left, sectors, r);
}

// ---------------------------------------------------------------------------
// moments in 8 bits
// ---------------------------------------------------------------------------
constexpr int kMBits = 3, kUBits = 4;
// Scale bytes that no step writes stand for the nearest that one does.
__device__ __forceinline__ uint32_t state_byte(uint32_t s) { return min(max(s, 1u), 247u); }
__device__ __forceinline__ float power(uint32_t biased) { return __uint_as_float(biased << 23); }
// Up to here 2^(s - 7) and 2^(7 - s) are float32 numbers; above, factors come in two.
constexpr uint32_t kScaleDirect = 133;

// Four codes of m: the instruction gives them in fp16, which holds them, and NaN with them.
__device__ __forceinline__ void decode_m4(uint32_t w, float step, F2* v) {
  uint32_t a, b;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
      : "=r"(a), "=r"(b)
      : "r"(w));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
  v[0] = f2(x.x, x.y) * f2(step), v[1] = f2(y.x, y.y) * f2(step);
}
// Not zero where a byte of w is.
__device__ __forceinline__ uint32_t zero_byte(uint32_t w) { return (w - 0x01010101u) & ~w & 0x80808080u; }
// Four codes of u: a code's bits at the place of a float's are its value times 2^-120, subnormals among them.
__device__ __forceinline__ void decode_u4(uint32_t w, uint32_t s, F2* v) {
  constexpr uint32_t kMask = 0xffu << 19;
  const F2 k = f2(power(s <= kScaleDirect ? s + 120u : 247u));
  v[0] = f2(__uint_as_float((w << 19) & kMask), __uint_as_float((w << 11) & kMask)) * k;
  v[1] = f2(__uint_as_float((w << 3) & kMask), __uint_as_float((w >> 5) & kMask)) * k;
  if (s > kScaleDirect) v[0] = v[0] * f2(power(s)), v[1] = v[1] * f2(power(s));
}
// 16 codes of each: a lane's of a tile.
__device__ __forceinline__ void decode_m(const uint32_t (&w)[4], float step, F2 (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) decode_m4(w[j], step, v + 2 * j);
}
__device__ __forceinline__ void decode_u(const uint32_t (&w)[4], uint32_t s, F2 (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) decode_u4(w[j], s, v + 2 * j);
  if ((zero_byte(~w[0]) | zero_byte(~w[1]) | zero_byte(~w[2]) | zero_byte(~w[3])) != 0u) {
    // the last code, a NaN
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      auto nan = [&](int k, float x) { return ((w[i / 2] >> (8 * k)) & 0xffu) == 0xffu ? __uint_as_float(0x7fc00000u) : x; };
      v[i] = f2(nan(2 * (i & 1), lo(v[i])), nan(2 * (i & 1) + 1, hi(v[i])));
    }
  }
}
// The scale byte from the bits of the largest finite magnitude (largest codes 1.75 2^8 and 1.875 2^8).
template <int BITS>
__device__ __forceinline__ uint32_t state_scale(uint32_t top_bits) {
  constexpr uint32_t kAbove = BITS == kMBits ? 0x1fffffu : 0x0fffffu;
  return uint32_t(max(int((top_bits + kAbove) >> 23) - 8, 1));
}
// The code of a magnitude, in bits 16 to 23: x 2^(127 - s) 2^-120 has the code at the head of a float's bits, behind the sign (products
// towards zero: what is under 2^-149 is dropped), and the 16 bits behind it decide with 16 random ones whether it is rounded up.
template <int BITS>
__device__ __forceinline__ uint32_t encode_bits(float scaled, uint32_t random) {
  return (__float_as_uint(scaled) >> (7 - BITS)) + random;
}
template <int BITS>
__device__ __forceinline__ void encode_pair(F2 x, float k, uint32_t r0, uint32_t r1, uint32_t& c0, uint32_t& c1) {
  F2 t;
  asm("mul.rz.f32x2 %0, %1, %2;" : "=l"(t.v) : "l"(x.v), "l"(f2(k).v));
  c0 = encode_bits<BITS>(lo(t), r0), c1 = encode_bits<BITS>(hi(t), r1);
}
// Any scale, and what is not finite.
template <int BITS>
__device__ __forceinline__ uint32_t encode_any(float x, uint32_t s, uint32_t random) {
  if (abs_bits(x) >= kInfBits) return (BITS == kMBits ? 0x7fu : 0xffu) << 16;
  if (s <= kScaleDirect) return encode_bits<BITS>(__fmul_rz(x, power(134u - s)), random);
  // (2^-100 first: of what that rounds, nothing reaches a code of a block whose largest is over 2^14)
  return encode_bits<BITS>(__fmul_rz(x * power(27u), __uint_as_float(s <= 233u ? (234u - s) << 23 : 1u << (256u - s))), random);
}
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = abs_bits(x);
  return b >= kInfBits ? 0u : b;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Of the lanes of a block.
__device__ __forceinline__ uint32_t block_max(uint32_t v) {
#pragma unroll
  for (int m = 1; m < kBlock / kEach8; m *= 2) v = max(v, __shfl_xor_sync(0xffffffffu, v, m));
  return v;
}
// Byte k of each of four words.
template <int K>
__device__ __forceinline__ uint32_t pack_byte(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  constexpr uint32_t kPick = K | (K + 4) << 4;
  return __byte_perm(__byte_perm(a, b, kPick), __byte_perm(c, d, kPick), 0x5410);
}

// One element's moments, then its parameter from them; u is the root of the new v.  (adamw_elem, operation for operation.)
__device__ __forceinline__ void moments_elem(float g, float& m, float& v, const AdamW& o) {
  m = __fadd_rn(__fmul_rn(o.b1, m), __fmul_rn(o.omb1, g));
  v = __fadd_rn(__fmul_rn(o.b2, v), __fmul_rn(o.omb2, __fmul_rn(g, g)));
}
__device__ __forceinline__ float step_elem(float p, float m, float v, float& u, const AdamW& o) {
  u = __fsqrt_rn(v);
  return __fsub_rn(__fmul_rn(p, o.decay), __fdiv_rn(__fmul_rn(o.step, m), __fadd_rn(__fmul_rn(u, o.r), o.eps)));
}
// The same for two elements side by side in packed instructions.  A packed product that a packed sum follows may be fused with
// it; so the sums are multiplications by 1 and additions, fused by themselves, which round as the addition does.
__device__ __forceinline__ F2 add2(F2 x, F2 y, const Settings& a) { return vfma(x, f2(a.one), y); }
__device__ __forceinline__ void moments_pair(F2 g, F2& m, F2& v, const Settings& a) {
  const AdamW& o = a.opt;
  m = add2(f2(o.b1) * m, f2(o.omb1) * g, a);
  v = add2(f2(o.b2) * v, f2(o.omb2) * (g * g), a);
}
// The parameters, without a branch for what is far out of range.  Root and quotient by Goldschmidt's and Newton's iterations from
// the hardware's reciprocals, each with a last correction by its remainder, which a fused multiply-add gives exactly
// (Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990).  All roots to 2^31
// round as the instruction does, and so did 2^34 quotients of random significands.  For v <= 2^62, |m| <= 2^62, eps from 2^-40 to
// 2^40 (the reciprocal of a divisor over 2^126 would be 0) and steps of at most 2^20 (Settings::plain); v comes from where it may be subnormal by 2^64; a quotient of a step m under 2^-102, whose
// remainder may not be exact, may be a bit off.
constexpr float kQuickMost = 4611686018427387904.0f;  // 2^62
__device__ __forceinline__ F2 quick_pair(F2 p, F2 m, F2 v, F2& u, const Settings& a) {
  const AdamW& o = a.opt;
  const F2 w = v * f2(18446744073709551616.0f), minus = f2(-1.0f);
  float y0, y1;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(lo(w)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(hi(w)));
  F2 x = w * f2(y0, y1), h = f2(y0, y1) * f2(-0.5f);  // (the root, and minus half its reciprocal)
  const F2 e = vfma(h, x, f2(0.5f));
  x = vfma(x, e, x), h = vfma(h, e, h);
  x = vfma(vfma(x, x, w * minus), h, x);
  x = x * f2(2.3283064365386963e-10f);  // 2^-32
  u = f2(lo(v) > 0.0f ? lo(x) : 0.0f, hi(v) > 0.0f ? hi(x) : 0.0f);
  const F2 d = add2(u * f2(o.r), f2(o.eps), a), n = f2(o.step) * m, md = d * minus;
  F2 r = f2(rcp_approx(lo(d)), rcp_approx(hi(d)));
  r = vfma(r, vfma(md, r, f2(1.0f)), r);
  F2 q = n * r;
  q = vfma(vfma(md, q, n), r, q);
  return vfma(q, f2(-a.one), p * f2(o.decay));
}

// The tiles of this CTA, every gridDim.x-th, and the item of its first.
struct Walk {
  int64_t tile;
  int item;
  template <class Args>
  __device__ __forceinline__ explicit Walk(const Args& a) {
    tile = blockIdx.x;
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.it[mid].tile0 <= tile) lo = mid;
      else hi = mid - 1;
    }
    item = lo;
  }
};

template <class Args>
__global__ void __launch_bounds__(kThreads, kCtas32) roi_adamw_step_kernel(const __grid_constant__ Args a) {
  pdl_begin(a.wait);
  const float scale = a.scale != nullptr ? __ldg(a.scale) : 1.0f;
  for (Walk w(a); w.tile < a.tiles; w.tile += gridDim.x) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * (kThreads * kEach32) + kEach32 * threadIdx.x, left = it.n - e;
    if (left <= 0) continue;
    const bool sectors = it.sectors;
    float p[kEach32], g[kEach32], m[kEach32], v[kEach32], u;
    // (without a branch between the loads: where ways meet, the compiler waits for what is on its way)
    if (sectors && left >= kEach32 && it.grad == uint8_t(Elem::kFp32)) {
      load_sectors<Elem::kFp32>(it.p + e, p);
      load_sectors<Elem::kFp32>(static_cast<const float*>(it.a) + e, m);
      load_sectors<Elem::kFp32>(static_cast<const float*>(it.b) + e, v);
      load_sectors<Elem::kFp32>(static_cast<const float*>(it.g) + e, g);
    } else {
      load_floats(it.p + e, left, sectors, p);
      load_floats(static_cast<const float*>(it.a) + e, left, sectors, m);
      load_floats(static_cast<const float*>(it.b) + e, left, sectors, v);
      load_any(it.g, it.grad, e, left, sectors, g);
    }
#pragma unroll
    for (int i = 0; i < kEach32; ++i) {
      moments_elem(a.scale != nullptr ? __fmul_rn(g[i], scale) : g[i], m[i], v[i], a.opt);
      p[i] = step_elem(p[i], m[i], v[i], u, a.opt);
    }
    store_floats(it.p + e, left, sectors, p);
    store_floats(static_cast<float*>(it.a) + e, left, sectors, m);
    store_floats(static_cast<float*>(it.b) + e, left, sectors, v);
    if (it.copy != nullptr) store_any(it.copy, it.copied, e, left, sectors, p);
  }
}

// The words of elements 4 q on.
__device__ __forceinline__ uint4 words_of(const Settings& a, uint64_t q, uint32_t id) {
  uint4 c = make_uint4(uint32_t(q), uint32_t(q >> 32), a.step, id);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = uint64_t(kPhiloxM0) * c.x, p1 = uint64_t(kPhiloxM1) * c.z;
    c = make_uint4(uint32_t(p1 >> 32) ^ c.y ^ a.keys[0][r], uint32_t(p1), uint32_t(p0 >> 32) ^ c.w ^ a.keys[1][r], uint32_t(p0));
  }
  return c;
}

// The step with moments in 8 bits.  64 instructions an element; on the way (a 7B-shaped
// block of 233 million elements, fp32 gradients, the states read back after it, us): element by element, four a thread 1884;
// whole sectors, decoding and encoding by words 1067; roots and quotients without a branch 1001; packed arithmetic 975; a CTA's tiles
// gridDim apart, and loads without a branch between them 896; more CTAs than an SM holds 839.  Registers for four to seven CTAs an
// SM: 878, 839, 846 (spills 80 bytes), 866 (320).  As fast or slower, before the last two: the next tile by bulk copies into shared
// memory, prefetched into L2, or loaded into registers while one is encoded; eight elements a thread; pointers that move
// along a tensor.
template <class Args>
__global__ void __launch_bounds__(kThreads, kCtas8) roi_adamw_step8_kernel(const __grid_constant__ Args a) {
  constexpr int kLanes = kBlock / kEach8, kPairs = kEach8 / 2, kWords = kEach8 / 4;  // lanes of a block; a lane's pairs, words of codes
  pdl_begin(a.wait);
  const float scale = a.scale != nullptr ? __ldg(a.scale) : 1.0f;
  const int lane = threadIdx.x & 31;
  for (Walk w(a); w.tile < a.tiles; w.tile += gridDim.x) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * (kThreads * kEach8) + kEach8 * threadIdx.x, left = it.n - e;
    if (left + kEach8 * lane <= 0) continue;  // (a warp has whole blocks)
    const bool there = left + kEach8 * (lane & (kLanes - 1)) > 0;  // whether its block has elements of the tensor
    float p[kEach8], g[kEach8];
    union {
      uint4 c;
      uint32_t w[kWords];
    } mw, uw;
    mw.c = uw.c = make_uint4(0u, 0u, 0u, 0u);
    uint32_t sw = 0;
    uint4* mc = reinterpret_cast<uint4*>(static_cast<uint8_t*>(it.a) + e);
    uint4* uc = reinterpret_cast<uint4*>(static_cast<uint8_t*>(it.b) + e);
    uint16_t* sc = reinterpret_cast<uint16_t*>(it.scales) + (e >> 7);
    // All loads of a way follow one another without a branch: where ways meet, the compiler waits for what is on its way.
    const bool whole = it.sectors && left + kEach8 * lane >= kEach8 * 32;  // (of the warp)
    if (whole && it.grad == uint8_t(Elem::kFp32)) {
      mw.c = *mc, uw.c = *uc, sw = *sc;
      load_sectors<Elem::kFp32>(it.p + e, p);
      load_sectors<Elem::kFp32>(static_cast<const float*>(it.g) + e, g);
    } else if (whole && it.grad == uint8_t(Elem::kBf16)) {
      mw.c = *mc, uw.c = *uc, sw = *sc;
      load_sectors<Elem::kFp32>(it.p + e, p);
      load_sectors<Elem::kBf16>(static_cast<const uint16_t*>(it.g) + e, g);
    } else {
      if (there) mw.c = *mc, uw.c = *uc, sw = *sc;
      load_floats(it.p + e, left, it.sectors, p);
      load_any(it.g, it.grad, e, left, it.sectors, g);
    }
    const float m_step = power(state_byte(sw & 0xffu));
    const uint32_t u_byte = state_byte(sw >> 8);
    F2 m[kPairs], u[kPairs];
    decode_m(mw.w, m_step, m);
    decode_u(uw.w, u_byte, u);
    // the moments, u for now v
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      u[i] = u[i] * u[i];
      moments_pair(f2(g[2 * i], g[2 * i + 1]) * f2(scale), m[i], u[i], a);  // (1 without a factor: the product is exact)
    }
    if (left < kEach8) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {  // (padding's codes are 0)
        m[i] = f2(2 * i < left ? lo(m[i]) : 0.0f, 2 * i + 1 < left ? hi(m[i]) : 0.0f);
        u[i] = f2(2 * i < left ? lo(u[i]) : 0.0f, 2 * i + 1 < left ? hi(u[i]) : 0.0f);
      }
    }
    float m_top = 0.0f, v_top = 0.0f;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      m_top = max3_nan(m_top, fabsf(lo(m[i])), fabsf(hi(m[i])));
      v_top = max3_nan(v_top, lo(u[i]), hi(u[i]));
    }
    const bool quick = a.plain && m_top <= kQuickMost && v_top <= kQuickMost;
    if (__all_sync(0xffffffffu, quick)) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const F2 x = quick_pair(f2(p[2 * i], p[2 * i + 1]), m[i], u[i], u[i], a);
        p[2 * i] = lo(x), p[2 * i + 1] = hi(x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        float u0, u1;
        p[2 * i] = step_elem(p[2 * i], lo(m[i]), lo(u[i]), u0, a.opt);
        p[2 * i + 1] = step_elem(p[2 * i + 1], hi(m[i]), hi(u[i]), u1, a.opt);
        u[i] = f2(u0, u1);
      }
    }
    store_floats(it.p + e, left, it.sectors, p);
    if (it.copy != nullptr) store_any(it.copy, it.copied, e, left, it.sectors, p);
    // (a NaN's bits are above an infinity's; the largest u is the root of the largest v)
    uint32_t m_bits = block_max(abs_bits(m_top)), u_bits = block_max(abs_bits(__fsqrt_rn(v_top)));
    uint32_t ms = state_scale<kMBits>(m_bits), us = state_scale<kUBits>(u_bits);
    const bool direct = max(m_bits, u_bits) < kInfBits && max(ms, us) <= kScaleDirect;
    if (__all_sync(0xffffffffu, direct)) {
      const float mk = power(134u - ms), uk = power(134u - us);
#pragma unroll
      for (int q = 0; q < kWords; ++q) {
        const uint4 r = words_of(a, (uint64_t(e) >> 2) + q, it.id);
        uint32_t c[4], d[4];
        encode_pair<kMBits>(m[2 * q], mk, r.x & 0xffffu, r.y & 0xffffu, c[0], c[1]);
        encode_pair<kMBits>(m[2 * q + 1], mk, r.z & 0xffffu, r.w & 0xffffu, c[2], c[3]);
        encode_pair<kUBits>(u[2 * q], uk, r.x >> 16, r.y >> 16, d[0], d[1]);
        encode_pair<kUBits>(u[2 * q + 1], uk, r.z >> 16, r.w >> 16, d[2], d[3]);
        mw.w[q] = pack_byte<2>(c[0], c[1], c[2], c[3]);
        uw.w[q] = pack_byte<2>(d[0], d[1], d[2], d[3]);
      }
    } else {
      m_bits = u_bits = 0;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        m_bits = max(m_bits, max(finite_bits(lo(m[i])), finite_bits(hi(m[i]))));
        u_bits = max(u_bits, max(finite_bits(lo(u[i])), finite_bits(hi(u[i]))));
      }
      ms = state_scale<kMBits>(block_max(m_bits)), us = state_scale<kUBits>(block_max(u_bits));
#pragma unroll
      for (int q = 0; q < kWords; ++q) {
        const uint4 r = words_of(a, (uint64_t(e) >> 2) + q, it.id);
        const F2 *x = m + 2 * q, *y = u + 2 * q;
        mw.w[q] = pack_byte<2>(encode_any<kMBits>(lo(x[0]), ms, r.x & 0xffffu), encode_any<kMBits>(hi(x[0]), ms, r.y & 0xffffu),
                               encode_any<kMBits>(lo(x[1]), ms, r.z & 0xffffu), encode_any<kMBits>(hi(x[1]), ms, r.w & 0xffffu));
        uw.w[q] = pack_byte<2>(encode_any<kUBits>(lo(y[0]), us, r.x >> 16), encode_any<kUBits>(hi(y[0]), us, r.y >> 16),
                               encode_any<kUBits>(lo(y[1]), us, r.z >> 16), encode_any<kUBits>(hi(y[1]), us, r.w >> 16));
      }
    }
#pragma unroll
    for (int q = 0; q < kWords; ++q) {
      const F2* x = m + 2 * q;
      mw.w[q] |= pack_byte<3>(__float_as_uint(lo(x[0])), __float_as_uint(hi(x[0])), __float_as_uint(lo(x[1])), __float_as_uint(hi(x[1]))) &
                 0x80808080u;
    }
    if ((zero_byte(uw.w[0]) | zero_byte(uw.w[1]) | zero_byte(uw.w[2]) | zero_byte(uw.w[3])) != 0u) {
      // what is not zero stays so: a step divides by it
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const uint32_t codes = uw.w[i / 2];
        auto least = [&](int k, float v) { return ((codes >> (8 * k)) & 0xffu) == 0u && v > 0.0f ? 1u << (8 * k) : 0u; };
        uw.w[i / 2] |= least(2 * (i & 1), lo(u[i])) | least(2 * (i & 1) + 1, hi(u[i]));
      }
    }
    if (there) {
      *mc = mw.c;
      *uc = uw.c;
      if ((lane & (kLanes - 1)) == 0) *sc = uint16_t(ms | us << 8);
    }
  }
}

// What states in 8 bits stand for.  (Items: p and copy are where m and u go, `grad` their type.)
template <class Args>
__global__ void __launch_bounds__(kThreads, kCtasLoad) roi_adamw_state8_load_kernel(const __grid_constant__ Args a) {
  pdl_begin(a.wait);
  for (Walk w(a); w.tile < a.tiles; w.tile += gridDim.x) {
    while (w.item + 1 < a.count && a.it[w.item + 1].tile0 <= w.tile) ++w.item;
    const Item& it = a.it[w.item];
    const int64_t e = (w.tile - it.tile0) * (kThreads * kEach8) + kEach8 * threadIdx.x, left = it.n - e;
    if (left <= 0) continue;
    const uint4 mq = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(it.a) + e);
    const uint4 uq = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(it.b) + e);
    const uint32_t mw[4] = {mq.x, mq.y, mq.z, mq.w}, uw[4] = {uq.x, uq.y, uq.z, uq.w};
    const uint32_t sw = reinterpret_cast<const uint16_t*>(it.scales)[e >> 7];
    const float m_step = power(state_byte(sw & 0xffu));
    const uint32_t u_byte = state_byte(sw >> 8);
    F2 x[8];
    float v[16];
    auto store = [&](void* to) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[2 * i] = lo(x[i]), v[2 * i + 1] = hi(x[i]);
      store_any(to, it.grad, e, left, it.sectors, v);
    };
    if (it.p != nullptr) {
      decode_m(mw, m_step, x);
      store(it.p);
    }
    if (it.copy != nullptr) {
      decode_u(uw, u_byte, x);
      store(it.copy);
    }
  }
}

template <int N>
int launch(const OptimCall& c, const OptimItem* items, int count) {
  using Args = ArgsOf<N>;
  int launched = 0;
  bool wait = lone_pdl(c.stream);
  Args a;
  a.opt = c.opt;
  for (uint32_t r = 0; r < 10; ++r) {
    a.keys[0][r] = uint32_t(c.seed) + r * kPhiloxW0;
    a.keys[1][r] = uint32_t(c.seed >> 32) + r * kPhiloxW1;
  }
  a.step = c.step;
  a.scale = c.scale;
  a.one = 1.0f;
  a.plain = c.opt.eps >= 9.094947017729282e-13f && c.opt.eps <= 1099511627776.0f && c.opt.step <= 1048576.0f;  // 2^-40, 2^40, 2^20
  const int tile = c.kind == OptimKind::kStep ? kThreads * kEach32 : kThreads * kEach8;
  auto kern = c.kind == OptimKind::kStep ? roi_adamw_step_kernel<Args>
              : c.kind == OptimKind::kStep8 ? roi_adamw_step8_kernel<Args>
                                            : roi_adamw_state8_load_kernel<Args>;
  for (int i = 0; i < count;) {
    a.count = 0;
    a.tiles = 0;
    for (; i < count && a.count < N; ++i) {
      const OptimItem& x = items[i];
      if (x.n == 0) continue;
      // (codes are accessed by 16 bytes)
      uintptr_t starts = reinterpret_cast<uintptr_t>(x.p) | reinterpret_cast<uintptr_t>(x.g) | reinterpret_cast<uintptr_t>(x.copy);
      if (c.kind == OptimKind::kStep) starts |= reinterpret_cast<uintptr_t>(x.a) | reinterpret_cast<uintptr_t>(x.b);
      a.it[a.count++] = {x.p,  x.g,     x.a,  x.b, x.scales,        x.copy,          x.n,
                         a.tiles, x.id, uint8_t(x.grad), uint8_t(x.copied), (starts & 31u) == 0};
      a.tiles += (x.n + tile - 1) / tile;
    }
    if (a.count == 0) break;
    a.wait = wait;
    const int64_t most = c.kind == OptimKind::kStep8 ? int64_t(sm_count()) * kWaves8 * kCtas8 : int64_t(1) << 30;
    if (launch_maybe_pdl(kern, int(a.tiles < most ? a.tiles : most), kThreads, 0, c.stream, wait, a) < 0) return -1;
    ++launched;
    wait = true;
  }
  return launched;
}

}  // namespace

int launch_optim(const OptimCall& c, const OptimItem* items, int count) {
  return count <= kFew ? launch<kFew>(c, items, count) : launch<kMost>(c, items, count);
}

}  // namespace roi
