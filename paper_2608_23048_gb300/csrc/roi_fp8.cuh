// Copies in 8-bit floating point whose blocks of 128 share a power of two, as the block-scaled
// matrix instructions take them (codes in e4m3 or e5m2, a scale byte s for 2^(s - 127)).  With a the largest magnitude of a
// block and F the format's largest number (448 or 57344, both 1.75 times a power of two),
//   s = 127 + the least e with a <= F 2^e, no less than 1, or 255 where a is infinite or NaN
//   q = x 2^(127 - s), rounded to the format, ties to even; 0 where s = 255
// The product by a power of two is exact, so codes are the same on every path.
//
// An activation's blocks are 128 consecutive columns of a row.  A weight's are 128 x 128: the same copy then serves the
// product that sums over its columns and the one that sums over its rows.
#pragma once

#include "roi_rows.cuh"

namespace roi {

enum class Fp8 : int { kE4M3 = 0, kE5M2 = 1 };

constexpr int kFp8Block = 128;
constexpr uint32_t kFp8ScaleNaN = 255u;

// The scale byte from the bits of the largest magnitude: adding what lies between 1.75's mantissa and all ones
// carries into the exponent exactly where the mantissa is past 1.75's.
template <Fp8 F>
__device__ __forceinline__ uint32_t fp8_scale(uint32_t top_bits) {
  constexpr int kTop = F == Fp8::kE4M3 ? 8 : 15;  // F = 1.75 2^kTop
  const int s = int((top_bits + 0x1fffffu) >> 23) - kTop;
  return top_bits >= kInfBits ? kFp8ScaleNaN : uint32_t(max(s, 1));
}
// 2^(127 - s); s is at most 247, or 255 for a block that is not finite: 0 there.
__device__ __forceinline__ float fp8_inverse(uint32_t s) {
  return s == kFp8ScaleNaN ? 0.0f : __uint_as_float((254u - s) << 23);
}
// Four codes in a word.
template <Fp8 F>
__device__ __forceinline__ uint32_t fp8_codes4(const float* x, float inverse) {
  uint16_t a, b;
  const float v0 = x[0] * inverse, v1 = x[1] * inverse, v2 = x[2] * inverse, v3 = x[3] * inverse;
  if constexpr (F == Fp8::kE4M3) {
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(v1), "f"(v0));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(v3), "f"(v2));
  } else {
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(a) : "f"(v1), "f"(v0));
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(b) : "f"(v3), "f"(v2));
  }
  return uint32_t(a) | (uint32_t(b) << 16);
}
// The codes of 16 elements of a block with scale byte s.
template <Fp8 F, Elem E>
__device__ __forceinline__ uint4 fp8_codes16(const RowWords<E, 16>& r, uint32_t s) {
  float v[16];
  r.get(v);
  const float inverse = fp8_inverse(s);
  uint4 q;
  q.x = fp8_codes4<F>(v, inverse);
  q.y = fp8_codes4<F>(v + 4, inverse);
  q.z = fp8_codes4<F>(v + 8, inverse);
  q.w = fp8_codes4<F>(v + 12, inverse);
  // (infinity times 0 is no number, whose code is not 0)
  if (s == kFp8ScaleNaN) q = make_uint4(0u, 0u, 0u, 0u);
  return q;
}

// Bytes of a row's codes (whole blocks) and of its scales (granules of 16 blocks).
__host__ __device__ inline int64_t fp8_pitch(int64_t cols) { return (cols + 127) / 128 * 128; }
__host__ __device__ inline int64_t fp8_scale_pitch(int64_t cols) { return (cols + 2047) / 2048 * 16; }

}  // namespace roi
