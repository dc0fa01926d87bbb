// Rows of matrices that start anywhere: 16-byte loads and stores of consecutive elements at
// addresses that need not be multiples of 16.
//
// A lane's W words (16, 32 or 64 bytes) at an address of remainder m = address mod 16:
//  - a load reads the W / 4 + 1 aligned granules around them and shifts (Window): the words
//    stay as they were read until they are used, so that loads can be far ahead;
//  - a store puts together aligned granules from the end of the lane before and its own words
//    (store_words, by the whole warp; the first and last lane write what has no neighbour
//    element by element).
// Nothing outside a row, [row, row + cols), is written, and load and store_words read nothing outside it either: what lies at
// its ends goes element by element.  load_granules reads whole granules, up to 15 bytes before its words and what follows
// them to the granule's end, and with a row's last words whatever of the next rows or of the gap between they cover;
// get_masked drops it.  in_matrix keeps these reads between the matrix's first byte and its last.
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

// The bits, as float32, of the largest magnitude (a NaN's are above all).
template <Elem E, int N>
__device__ __forceinline__ uint32_t max_bits(const RowWords<E, N>& r) {
  constexpr int W = RowWords<E, N>::kWords;
  if constexpr (E == Elem::kFp32) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) top = max(top, r.u[i] & 0x7fffffffu);
    return top;
  } else {
    // two halves a step; as integers, magnitudes are in the order of their bits
    uint32_t t = r.u[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < W; ++i) t = __vmaxu2(t, r.u[i] & 0x7fff7fffu);
    const uint32_t half = max(t >> 16, t & 0xffffu);
    return abs_bits(to_f32<E>(uint16_t(half)));
  }
}
// The codes of a piece of a block whose largest magnitude has the bits `top` and whose scale byte is s (all lanes).
template <Elem E, int N>
__device__ __forceinline__ void block8_codes(const RowWords<E, N>& r, uint32_t top, uint32_t s, uint32_t (&w)[N / 4]) {
  const float inverse = block8_inverse(min(s, kScaleMax));
  const uint32_t keep = s == kScaleNaN ? 0u : 0xffffffffu;
  float v[N];
  r.get(v);
  // only a magnitude past 127 steps can round past the last code: rare, and the same for the block
  if (__any_sync(0xffffffffu, !(__uint_as_float(top) * inverse <= 127.0f))) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) w[i] = block8_codes4(v + 4 * i, inverse, keep);
  } else {
    const F2 k = f2(inverse), magic = f2(12582912.0f);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const F2 a = vfma(f2(v[4 * i], v[4 * i + 1]), k, magic), b = vfma(f2(v[4 * i + 2], v[4 * i + 3]), k, magic);
      w[i] = __byte_perm(__byte_perm(__float_as_uint(lo(a)), __float_as_uint(hi(a)), 0x0040),
                         __byte_perm(__float_as_uint(lo(b)), __float_as_uint(hi(b)), 0x0040), 0x5410);
    }
  }
}

// N elements from column c of a row on, on their way: the granules around them.
template <Elem E, int N>
struct Window {
  using R = RowWords<E, N>;
  static constexpr int kWords = R::kWords;
  uint32_t w[kWords + 4];
  uint32_t m;

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords + 4; ++i) w[i] = 0;
    m = 0;
  }
  __device__ __forceinline__ void load(const typename ElemType<E>::T* row, int64_t c, int64_t cols) {
    const int64_t left = cols - c;
    if (left <= 0) {
      zero();
      return;
    }
    const typename ElemType<E>::T* p = row + c;
    m = uint32_t(reinterpret_cast<uintptr_t>(p) & 15u);
    // whole granules inside the row
    if (c * elem_bytes<E>() >= m && left * elem_bytes<E>() + m >= kWords * 4 + 16) {
      const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) - m);
#pragma unroll
      for (int i = 0; i < kWords / 4 + 1; ++i) {
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
  // Where the granules around them lie in the matrix, whose first byte and end are given (what is between rows, or the next
  // rows', is read and dropped by get_masked): all lanes but those at the matrix's ends go this way, without a branch at each row's.
  static __device__ __forceinline__ bool in_matrix(const typename ElemType<E>::T* p, const void* begin, const void* end) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p) & ~uintptr_t(15);
    return from >= reinterpret_cast<uintptr_t>(begin) && from + kWords * 4 + 16 <= reinterpret_cast<uintptr_t>(end);
  }
  __device__ __forceinline__ void load_granules(const typename ElemType<E>::T* p) {
    m = uint32_t(reinterpret_cast<uintptr_t>(p) & 15u);
    const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) - m);
#pragma unroll
    for (int i = 0; i < kWords / 4 + 1; ++i) {
      const uint4 v = __ldg(q + i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void get(R& r) const { shift_words<kWords>(w, m, r.u); }
  // ... those from `left` on as zeros.
  __device__ __forceinline__ void get_masked(R& r, int64_t left) const {
    get(r);
    if (left < N) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if constexpr (E == Elem::kFp32) r.u[i] = i < left ? r.u[i] : 0u;
        else r.u[i] &= (2 * i < left ? 0xffffu : 0u) | (2 * i + 1 < left ? 0xffff0000u : 0u);
      }
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
  const int lane = threadIdx.x & (width - 1);
  uint32_t h[4], e[4];  // the group's first and last granule of words, in all its lanes
  if constexpr (!ALIGNED) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t own = r.u[W - 4 + i];
      s[i] = __shfl_sync(0xffffffffu, prev != nullptr && lane == width - 1 ? prev->u[W - 4 + i] : own, (lane + width - 1) & (width - 1), width);
      if (prev == nullptr) h[i] = __shfl_sync(0xffffffffu, r.u[i], 0, width);
      if (!more) e[i] = __shfl_sync(0xffffffffu, own, width - 1, width);
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
    RowWords<E, N> g;  // the granules from p - m on
    shift_words<W>(s, 16u - m, g.u);
    const int before = int(m) / elem_bytes<E>();  // elements of the lane before
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const int from = i * kPer - before;  // the granule's first column, relative to c
      const bool head = i == 0 && lane == 0 && prev == nullptr;
      if (!head && left >= from + kPer) {
        reinterpret_cast<uint4*>(reinterpret_cast<uintptr_t>(p) - m)[i] =
            make_uint4(g.u[4 * i], g.u[4 * i + 1], g.u[4 * i + 2], g.u[4 * i + 3]);
      } else if (!head && left > from) {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
          if (from + k < left) p[from + k] = g.at(i * kPer + k);
      }
    }
    // what has no lane before or after it, an element a lane (groups have eight lanes at least)
    auto element = [&](const uint32_t (&w)[4]) {
      const int at = E == Elem::kFp32 ? lane : lane >> 1;
      const uint32_t v = at == 0 ? w[0] : at == 1 ? w[1] : at == 2 ? w[2] : w[3];
      if constexpr (E == Elem::kFp32) return __uint_as_float(v);
      else return uint16_t(lane & 1 ? v >> 16 : v);
    };
    const int64_t left0 = left + int64_t(lane) * N;  // of lane 0
    if (prev == nullptr && lane < kPer - before && lane < left0) (p - lane * N)[lane] = element(h);
    const int64_t k = int64_t(width) * N - kPer + lane;  // relative to lane 0
    if (!more && lane < kPer && lane >= kPer - before && k < left0) (p - lane * N)[k] = element(e);
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

// Copies of whole matrices, 16 columns a lane.
// Row and place in the row of the `i`-th item of a row-major walk over rows of `per_row`
// items, from the row and the place of the walk's start (one division of 64 bits a tile).
__device__ __forceinline__ void walk(int64_t row0, int64_t rem0, uint32_t i, int64_t per_row, int64_t& row, int64_t& j) {
  j = rem0 + i;
  row = row0;
  if (j >= per_row) {
    if (per_row <= 0x3fffffff) {
      const uint32_t q = uint32_t(j) / uint32_t(per_row);
      row += q;
      j -= int64_t(q) * per_row;
    } else {
      ++row;
      j -= per_row;
    }
  }
}

// Rows anywhere.  A warp's task: 32 / width rows, or one segment of a row.
__device__ __forceinline__ void row_task(int64_t task, int width, int segments, int64_t& row, int64_t& piece) {
  const int lane = threadIdx.x & 31;
  if (segments > 1) {
    row = task / segments;
    piece = (task - row * segments) * 32 + lane;
  } else {
    row = task * (32 / width) + lane / width;
    piece = lane & (width - 1);
  }
}

// Rows that are whole 32-byte sectors apart.
inline bool in_sectors(const void* p, int64_t ld, int64_t rows, int bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 31u) == 0 && (rows <= 1 || ld * bytes % 32 == 0);
}
// Rows anywhere: the lanes of a row, a power of two that holds its pieces, or a whole warp that
// goes over it in segments.  Returns the tiles of the launch.
template <class Args>
int64_t by_rows(Args& a) {
  a.width = 8;
  while (a.width < 32 && a.width < a.pieces) a.width *= 2;
  a.segments = int((a.pieces + 31) / 32);
  const int64_t per = 32 / a.width;
  return (a.rows + per - 1) / per * a.segments;
}

}  // namespace roi
