// Activation checkpoints in 8 bits: blocks of 32 consecutive columns of a row share a power
// of two (the OCP microscaling layout of 8-bit integers).  With a the largest magnitude of a
// block, its scale byte s and its codes q are
//   s = clamp((bits(a) + 0xffff) >> 23, 7, 254), or 255 where a is infinite or NaN
//   q = clamp(round_half_even(x 2^(133 - s)), -127, 127), or 0 where s = 255
// and they stand for q 2^(s - 133), or NaN where s = 255.  s - 133 is the least exponent e
// with a <= 127.5 2^e (bits(a) + 0xffff carries into the exponent exactly where the mantissa
// is past 255/128), at least -126, so that every scale is a normal number, and at most 121, so
// that every value is finite.  The products by a power of two are exact, so the codes are the
// same on every path, and a value has 7 bits and a sign: bf16 holds it exactly.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "roi_common.cuh"

namespace roi {

enum class Elem : int { kBf16 = 0, kFp16 = 1, kFp32 = 2 };

template <Elem E>
struct ElemType;
template <>
struct ElemType<Elem::kBf16> {
  using T = uint16_t;
};
template <>
struct ElemType<Elem::kFp16> {
  using T = uint16_t;
};
template <>
struct ElemType<Elem::kFp32> {
  using T = float;
};
template <Elem E>
constexpr int elem_bytes() {
  return int(sizeof(typename ElemType<E>::T));
}

template <Elem E>
__device__ __forceinline__ float to_f32(typename ElemType<E>::T v) {
  if constexpr (E == Elem::kBf16) return __uint_as_float(uint32_t(v) << 16);
  if constexpr (E == Elem::kFp16) return __half2float(__ushort_as_half(v));
  if constexpr (E == Elem::kFp32) return v;
}
template <Elem E>
__device__ __forceinline__ typename ElemType<E>::T from_f32(float v) {
  if constexpr (E == Elem::kBf16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
  if constexpr (E == Elem::kFp16) return __half_as_ushort(__float2half_rn(v));
  if constexpr (E == Elem::kFp32) return v;
}

// The scale byte of a block from the bits of its largest magnitude (a NaN's bits are above
// an infinity's, so their maximum as integers finds both).
constexpr uint32_t kInfBits = 0x7f800000u;
constexpr uint32_t kScaleNaN = 255u, kScaleMin = 7u, kScaleMax = 254u;
__device__ __forceinline__ uint32_t block8_scale(uint32_t amax_bits) {
  const uint32_t s = (amax_bits + 0xffffu) >> 23;
  return amax_bits >= kInfBits ? kScaleNaN : min(max(s, kScaleMin), kScaleMax);
}
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// 2^(133 - s), what the elements of a block are multiplied by (s <= 254).
__device__ __forceinline__ float block8_inverse(uint32_t s) { return __uint_as_float((260u - s) << 23); }
// 2^(s - 133), NaN for s = 255; bytes below 7, which no call writes, stand for zero.
__device__ __forceinline__ float block8_step(uint32_t s) {
  return s == kScaleNaN ? __uint_as_float(0x7fc00000u) : __uint_as_float((max(s, 6u) - 6u) << 23);
}
// One code in the low byte: the sum with 3 2^22 rounds to the nearest integer, ties to even,
// and leaves it in the low bits.
__device__ __forceinline__ uint32_t block8_code(float x, float inverse) {
  constexpr float kMagic = 12582912.0f;
  const float v = __fmaf_rn(x, inverse, kMagic);
  return __float_as_uint(fminf(fmaxf(v, kMagic - 127.0f), kMagic + 127.0f));
}
// Four codes in a word; `keep` is 0 in a block of codes 0 (s = 255), else all ones.
__device__ __forceinline__ uint32_t block8_codes4(const float* x, float inverse, uint32_t keep) {
  const uint32_t a = __byte_perm(block8_code(x[0], inverse), block8_code(x[1], inverse), 0x0040);
  const uint32_t b = __byte_perm(block8_code(x[2], inverse), block8_code(x[3], inverse), 0x0040);
  return __byte_perm(a, b, 0x5410) & keep;
}
// The values of the four codes of a word, in pairs.  A code's byte, its sign bit turned, in the
// mantissa of 2^23 is 2^23 + 128 + the code; difference and product are exact.
__device__ __forceinline__ void block8_pairs(uint32_t word, float step, F2& a, F2& b) {
  const uint32_t u = word ^ 0x80808080u;
  const F2 minus = f2(-8388736.0f), s = f2(step);
  a = (f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7440)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7441))) + minus) * s;
  b = (f2(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7442)), __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7443))) + minus) * s;
}
// The element type's value: fp16 ends before the largest checkpointed values do.
template <Elem E>
__device__ __forceinline__ float block8_clip(float v) {
  if constexpr (E == Elem::kFp16) return fabsf(v) > 65504.0f ? copysignf(65504.0f, v) : v;
  return v;
}

// Bytes of a row's codes (whole blocks) and of its scales (whole words of four blocks).
__host__ __device__ inline int64_t block8_pitch(int64_t cols) { return (cols + 31) / 32 * 32; }
__host__ __device__ inline int64_t block8_scale_pitch(int64_t cols) { return (cols + 127) / 128 * 4; }

}  // namespace roi
