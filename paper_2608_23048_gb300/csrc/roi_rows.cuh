// Rows of matrices that start anywhere: 16-byte loads and stores of consecutive elements at
// addresses that need not be multiples of 16.
//
// A lane's W words (16, 32 or 64 bytes) at an address of remainder m = address mod 16:
//  - a load reads the W / 4 + 1 aligned granules around them and shifts (Window): the words
//    stay as they were read until they are used, so that loads can be far ahead;
//  - a store puts together aligned granules from the end of the lane before and its own words
//    (store_words, by the whole warp; the first and last lane write what has no neighbour
//    element by element).
// Nothing outside [row, row + cols) is read or written: what lies at the ends of a row goes
// element by element.
#pragma once

#include "roi_block8.cuh"

namespace roi {

// words[0 .. W) of the stream `w`, from byte `m` (a multiple of 2, 0 .. 14) on.
template <int W>
__device__ __forceinline__ void shift_words(const uint32_t (&w)[W + 4], uint32_t m, uint32_t (&out)[W]) {
  uint32_t a[W + 2], b[W + 1];
#pragma unroll
  for (int i = 0; i < W + 2; ++i) a[i] = (m & 8u) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < W + 1; ++i) b[i] = (m & 4u) ? a[i + 1] : a[i];
  const uint32_t pick = (m & 2u) ? 0x5432u : 0x3210u;
#pragma unroll
  for (int i = 0; i < W; ++i) out[i] = __byte_perm(b[i], b[i + 1], pick);
}

template <Elem E, int N>  // N elements a lane
struct RowWords {
  static constexpr int kWords = N * elem_bytes<E>() / 4;
  uint32_t u[kWords];
  __device__ __forceinline__ void get(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (E == Elem::kFp32) v[i] = __uint_as_float(u[i]);
      if constexpr (E == Elem::kBf16) v[i] = __uint_as_float(i % 2 == 0 ? u[i / 2] << 16 : u[i / 2] & 0xffff0000u);
      if constexpr (E == Elem::kFp16) v[i] = __half2float(__ushort_as_half(uint16_t(i % 2 == 0 ? u[i / 2] : u[i / 2] >> 16)));
    }
  }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (E == Elem::kFp32) u[i] = __float_as_uint(v[i]);
      if constexpr (E == Elem::kBf16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&b);
      }
      if constexpr (E == Elem::kFp16) {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) u[i] = 0;
  }
  __device__ __forceinline__ typename ElemType<E>::T at(int i) const {
    if constexpr (E == Elem::kFp32) return __uint_as_float(u[i]);
    else return uint16_t(i % 2 == 0 ? u[i / 2] : u[i / 2] >> 16);
  }
  // Elements from column c on, those past the last as zeros, one by one.
  __device__ __forceinline__ void load_elements(const typename ElemType<E>::T* row, int64_t c, int64_t cols) {
    zero();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (c + i < cols) {
        if constexpr (E == Elem::kFp32) u[i] = __float_as_uint(__ldg(row + c + i));
        else u[i / 2] |= uint32_t(__ldg(row + c + i)) << (16 * (i % 2));
      }
    }
  }
};

// N elements from column c of a row on, on their way: ALIGNED (rows start on 16-byte boundaries) as
// they are, else the granules around them.
template <Elem E, int N, bool ALIGNED>
struct Window {
  using R = RowWords<E, N>;
  static constexpr int kWords = R::kWords;
  uint32_t w[ALIGNED ? kWords : kWords + 4];
  uint32_t m;  // (not ALIGNED)

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (ALIGNED ? kWords : kWords + 4); ++i) w[i] = 0;
    m = 0;
  }
  __device__ __forceinline__ void load(const typename ElemType<E>::T* row, int64_t c, int64_t cols) {
    const int64_t left = cols - c;
    if (left <= 0) {
      zero();
      return;
    }
    const typename ElemType<E>::T* p = row + c;
    m = ALIGNED ? 0u : uint32_t(reinterpret_cast<uintptr_t>(p) & 15u);
    // whole granules inside the row
    const bool inside = ALIGNED ? left >= N : c * elem_bytes<E>() >= m && left * elem_bytes<E>() + m >= kWords * 4 + 16;
    if (inside) {
      const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) - m);
#pragma unroll
      for (int i = 0; i < (ALIGNED ? kWords / 4 : kWords / 4 + 1); ++i) {
        const uint4 v = __ldg(q + i);
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    } else {
      R r;
      r.load_elements(row, c, cols);
      zero();
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = r.u[i];
    }
  }
  __device__ __forceinline__ void get(R& r) const {
    if constexpr (ALIGNED) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) r.u[i] = w[i];
    } else {
      shift_words<kWords>(w, m, r.u);
    }
  }
};

// All lanes of a warp, in groups of `width` (a power of two) with a row each: lane l of a group
// puts its N elements at columns c = c_0 + N l on.  Lanes may lie past the end (cols < 0: no row).
// A warp that goes along a row piece by piece (width 32) gives the piece before in `prev`, whose
// last lane's end belongs to lane 0's first granule, and says with `more` that another follows.
template <Elem E, int N, bool ALIGNED>
__device__ __forceinline__ void store_row(typename ElemType<E>::T* row, int64_t c, int64_t cols, const RowWords<E, N>& r, int width = 32,
                                          const RowWords<E, N>* prev = nullptr, bool more = false) {
  constexpr int W = RowWords<E, N>::kWords, kPer = 16 / elem_bytes<E>();  // elements of a granule
  const int64_t left = cols - c;
  typename ElemType<E>::T* p = row + c;
  uint32_t s[W + 4];  // the end of the lane before, and this lane's words
  if constexpr (!ALIGNED) {
    const int lane = threadIdx.x & (width - 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t own = r.u[W - 4 + i];
      s[i] = __shfl_sync(0xffffffffu, prev != nullptr && lane == width - 1 ? prev->u[W - 4 + i] : own, (lane + width - 1) & (width - 1), width);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) s[4 + i] = r.u[i];
  }
  const uint32_t m = ALIGNED ? 0u : uint32_t(reinterpret_cast<uintptr_t>(p) & 15u);  // the same in all lanes of a group
  if (m == 0) {
    if (left >= N) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i)
        reinterpret_cast<uint4*>(p)[i] = make_uint4(r.u[4 * i], r.u[4 * i + 1], r.u[4 * i + 2], r.u[4 * i + 3]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < left) p[i] = r.at(i);
    }
  } else if constexpr (!ALIGNED) {
    const int lane = threadIdx.x & (width - 1);
    const bool first = lane == 0 && prev == nullptr;  // nothing comes before
    RowWords<E, N> g;  // the granules from p - m on
    shift_words<W>(s, 16u - m, g.u);
    const int before = int(m) / elem_bytes<E>();  // elements of the lane before
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const int from = i * kPer - before;  // the granule's first column, relative to c
      if ((i > 0 || !first) && left >= from + kPer) {
        reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(p) - m)[i] =
            make_uint4(g.u[4 * i], g.u[4 * i + 1], g.u[4 * i + 2], g.u[4 * i + 3]);
      } else if (left > from) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int k = from + e;
          if ((i > 0 || !first || k >= 0) && k < left) p[k] = g.at(i * kPer + e);
        }
      }
    }
    if (lane == width - 1 && !more) {  // its end has no lane after it
#pragma unroll
      for (int k = N - kPer; k < N; ++k)
        if (k >= N - before && k < left) p[k] = r.at(k);
    }
  }
}

// 32 bytes at a 32-byte boundary.
__device__ __forceinline__ void load32(const void* p, uint32_t* w) {
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
               "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

}  // namespace roi
