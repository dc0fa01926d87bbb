// C ABI of libroi (see include/roi.h): host-side validation, then one launch.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <vector>
#include <cstdint>
#include <cstring>

#include "roi.h"
#include "roi_fp8.cuh"
#include "roi_launch.h"

namespace roi {

// The device status record: word 0 the status bits (kStatusTimeout), words 2-3
// the ring-wait limit in ns (2 s).  One per device; the kernels get its address.
__device__ __align__(16) unsigned int g_roi_device_status[4] = {0u, 0u, 2000000000u, 0u};

namespace {

std::atomic<uint64_t> g_launches{0};

unsigned int* status_word() {
  // Device address of this module's status word on the current device.
  void* p = nullptr;
  if (cudaGetSymbolAddress(&p, g_roi_device_status) != cudaSuccess) return nullptr;
  return static_cast<unsigned int*>(p);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Range {
  const void* p;
  uint64_t bytes;
};

bool overlaps(const Range& a, const Range& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}

// Outputs must not overlap inputs or each other.
template <int NI, int NO>
bool any_alias(const Range (&in)[NI], const Range (&out)[NO]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlaps(out[o], in[i])) return true;
    for (int p = o + 1; p < NO; ++p)
      if (overlaps(out[o], out[p])) return true;
  }
  return false;
}

bool finite_positive(float x) { return std::isfinite(x) && x > 0.0f; }

// Across a batch: true if an output range overlaps any other range (input or
// output).  Sort by start; a range overlaps an earlier one iff it starts before
// the largest end seen so far (of outputs, for an input; of all, for an output).
struct Tagged {
  uintptr_t lo, hi;
  bool out;
};
bool batch_alias(std::vector<Tagged>& r) {
  std::sort(r.begin(), r.end(), [](const Tagged& a, const Tagged& b) { return a.lo < b.lo; });
  uintptr_t end_all = 0, end_out = 0;
  for (const Tagged& x : r) {
    if (x.out ? x.lo < end_all : x.lo < end_out) return true;
    end_all = std::max(end_all, x.hi);
    if (x.out) end_out = std::max(end_out, x.hi);
  }
  return false;
}
void add_range(std::vector<Tagged>& r, const void* p, uint64_t bytes, bool out) {
  if (p == nullptr || bytes == 0) return;
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  r.push_back({lo, lo + uintptr_t(bytes), out});
}

roi_status check_common(int N, int M, float tau, int64_t rows, int64_t cols) {
  if (!(N >= 1 && N < M && M <= 32)) return ROI_ERR_NM;
  if (rows < 0 || cols <= 0 || cols % M != 0) return ROI_ERR_SHAPE;
  if (rows > 0 && cols > INT64_MAX / 64 / rows) return ROI_ERR_SHAPE;
  if (!finite_positive(tau)) return ROI_ERR_TAU;
  return ROI_OK;
}

NoiseParams make_noise(const roi_noise_state& st, int64_t cols) {
  NoiseParams np;
  np.k0 = static_cast<uint32_t>(st.seed & 0xffffffffu);
  np.k1 = static_cast<uint32_t>(st.seed >> 32);
  np.step = st.step;
  np.tensor_id = st.tensor_id;
  np.inv_lam = 1.0f / st.lambda;
  np.l2e_inv_lam = static_cast<float>(1.4426950408889634 / static_cast<double>(st.lambda));
  np.e_base = static_cast<uint64_t>(st.row_offset) * static_cast<uint64_t>(cols);
  return np;
}

// A row-major matrix with a row stride, as a place in memory: `pitch` and `width` in bytes.
struct Strided {
  const void* p;
  uint64_t rows, pitch, width;
};
bool overlaps(const Strided& a, const Strided& b) {
  if (a.p == nullptr || b.p == nullptr || a.rows == 0 || b.rows == 0) return false;
  const Range ra = {a.p, (a.rows - 1) * a.pitch + a.width}, rb = {b.p, (b.rows - 1) * b.pitch + b.width};
  if (!overlaps(ra, rb)) return false;
  if (a.pitch != b.pitch) return true;
  // the same stride: apart where neither's columns reach the other's
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  const uint64_t d = pb >= pa ? (pb - pa) % a.pitch : (a.pitch - (pa - pb) % a.pitch) % a.pitch;
  return !(a.width <= d && d + b.width <= a.pitch);
}
Strided flat(const void* p, uint64_t bytes) { return {p, bytes == 0 ? 0u : 1u, bytes, bytes}; }
template <int NI, int NO>
bool any_alias(const Strided (&in)[NI], const Strided (&out)[NO]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (overlaps(out[o], in[i])) return true;
    for (int p = o + 1; p < NO; ++p)
      if (overlaps(out[o], out[p])) return true;
  }
  return false;
}

bool known_type(int dtype) { return dtype == ROI_BF16 || dtype == ROI_FP16 || dtype == ROI_FP32; }
int type_bytes(int dtype) { return dtype == ROI_FP32 ? 4 : 2; }
// A matrix of `rows` rows with stride ld: sizes that fit.
bool good_shape(int64_t rows, int64_t cols, int64_t ld) {
  return rows >= 0 && cols > 0 && cols <= INT64_MAX / 1024 && (rows == 0 || (ld >= cols && ld <= INT64_MAX / 64 / rows));
}
bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % unsigned(bytes) == 0; }
Strided matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int bytes) {
  return {p, uint64_t(rows), uint64_t(ld) * uint64_t(bytes), uint64_t(cols) * uint64_t(bytes)};
}

roi_status finish(int launched) {
  if (launched < 0) return ROI_ERR_CUDA;
  g_launches.fetch_add(static_cast<uint64_t>(launched), std::memory_order_relaxed);
  return ROI_OK;
}

}  // namespace

int sm_count() {
  static int cache[64] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 1;
  if (cache[dev] == 0) {
    int n = 0;
    cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    cache[dev] = n > 0 ? n : 1;
  }
  return cache[dev];
}

}  // namespace roi

using namespace roi;

extern "C" {

static roi_status mask_fwd(const float* logits, const roi_bf16* W, int N, int M, float tau, const roi_noise_state* st,
                           int64_t rows, int64_t cols, roi_bf16* out_Wm, float* out_soft, uint32_t* out_hard,
                           bool straight_through, void* stream) {
  if (st == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, rows, cols);
  if (s != ROI_OK) return s;
  if (st->row_offset < 0) return ROI_ERR_SHAPE;
  if (!finite_positive(st->lambda)) return ROI_ERR_TAU;
  if (rows == 0) return ROI_OK;  // nothing is read or written; pointers may be NULL
  if (logits == nullptr || W == nullptr || out_Wm == nullptr) return ROI_ERR_NULL;
  if (!aligned16(logits) || !aligned16(W) || !aligned16(out_Wm) || !aligned16(out_soft) || !aligned16(out_hard))
    return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  const Range in[2] = {{logits, uint64_t(E) * 4}, {W, uint64_t(E) * 2}};
  const Range out[3] = {{out_Wm, uint64_t(E) * 2}, {out_soft, uint64_t(E) * 4}, {out_hard, uint64_t((E + 31) / 32) * 4}};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  if (E == 0) return ROI_OK;
  FwdCall c;
  c.phi = logits;
  c.W = W;
  c.Wm = out_Wm;
  c.soft = out_soft;
  c.hard = out_hard;
  c.st = straight_through;
  c.E = E;
  c.N = N;
  c.M = M;
  c.tau = tau;
  c.np = make_noise(*st, cols);
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_fwd(c));
}

static roi_status fwd_batch(const roi_fwd_item* items, int count, int N, int M, float tau, bool straight_through,
                            void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, 0, M);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  ranges.reserve(size_t(count) * 5);
  for (int i = 0; i < count; ++i) {
    const roi_fwd_item& it = items[i];
    s = check_common(N, M, tau, it.rows, it.cols);
    if (s != ROI_OK) return s;
    if (it.st.row_offset < 0) return ROI_ERR_SHAPE;
    if (!finite_positive(it.st.lambda)) return ROI_ERR_TAU;
    if (it.rows == 0) continue;
    if (it.logits == nullptr || it.W == nullptr || it.out_Wm == nullptr) return ROI_ERR_NULL;
    if (!aligned16(it.logits) || !aligned16(it.W) || !aligned16(it.out_Wm) || !aligned16(it.out_soft) ||
        !aligned16(it.out_hard))
      return ROI_ERR_ALIGN;
    const int64_t E = it.rows * it.cols;
    add_range(ranges, it.logits, uint64_t(E) * 4, false);
    add_range(ranges, it.W, uint64_t(E) * 2, false);
    add_range(ranges, it.out_Wm, uint64_t(E) * 2, true);
    add_range(ranges, it.out_soft, uint64_t(E) * 4, true);
    add_range(ranges, it.out_hard, uint64_t((E + 31) / 32) * 4, true);
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  if (ranges.empty()) return ROI_OK;  // only empty items: nothing is read or written
  unsigned int* status = status_word();
  if (status == nullptr) return ROI_ERR_CUDA;
  std::vector<FwdCall> calls;
  calls.reserve(size_t(count));
  for (int i = 0; i < count; ++i) {
    const roi_fwd_item& it = items[i];
    if (it.rows == 0) continue;
    FwdCall c;
    c.phi = it.logits;
    c.W = it.W;
    c.Wm = it.out_Wm;
    c.soft = it.out_soft;
    c.hard = it.out_hard;
    c.st = straight_through;
    c.E = it.rows * it.cols;
    c.N = N;
    c.M = M;
    c.tau = tau;
    c.np = make_noise(it.st, it.cols);
    c.status = status;
    c.stream = static_cast<cudaStream_t>(stream);
    calls.push_back(c);
  }
  return finish(launch_fwd_batch(calls.data(), int(calls.size())));
}

roi_status roi_mask_fwd_batch(const roi_fwd_item* items, int count, int N, int M, float tau, void* stream) {
  return fwd_batch(items, count, N, M, tau, false, stream);
}

roi_status roi_mask_fwd_st_batch(const roi_fwd_item* items, int count, int N, int M, float tau, void* stream) {
  return fwd_batch(items, count, N, M, tau, true, stream);
}

roi_status roi_mask_bwd_st_batch(const roi_bwd_st_item* items, int count, int N, int M, float tau, void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, 0, M);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  ranges.reserve(size_t(count) * 6);
  for (int i = 0; i < count; ++i) {
    const roi_bwd_st_item& it = items[i];
    s = check_common(N, M, tau, it.rows, it.cols);
    if (s != ROI_OK) return s;
    if (it.st.row_offset < 0) return ROI_ERR_SHAPE;
    if (!finite_positive(it.st.lambda)) return ROI_ERR_TAU;
    if (it.rows == 0) continue;
    if (it.logits == nullptr || it.W == nullptr || it.dWm == nullptr || it.out_dlogits == nullptr ||
        (it.out_dW != nullptr && it.hard == nullptr))
      return ROI_ERR_NULL;
    if (!aligned16(it.logits) || !aligned16(it.W) || !aligned16(it.dWm) || !aligned16(it.hard) ||
        !aligned16(it.out_dlogits) || !aligned16(it.out_dW))
      return ROI_ERR_ALIGN;
    const int64_t E = it.rows * it.cols;
    add_range(ranges, it.logits, uint64_t(E) * 4, false);
    add_range(ranges, it.W, uint64_t(E) * 2, false);
    add_range(ranges, it.dWm, uint64_t(E) * 2, false);
    add_range(ranges, it.hard, uint64_t((E + 31) / 32) * 4, false);
    add_range(ranges, it.out_dlogits, uint64_t(E) * 4, true);
    add_range(ranges, it.out_dW, uint64_t(E) * 2, true);
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  if (ranges.empty()) return ROI_OK;
  unsigned int* status = status_word();
  if (status == nullptr) return ROI_ERR_CUDA;
  std::vector<BwdCall> calls;
  calls.reserve(size_t(count));
  for (int i = 0; i < count; ++i) {
    const roi_bwd_st_item& it = items[i];
    if (it.rows == 0) continue;
    BwdCall c{};
    c.phi = it.logits;
    c.W = it.W;
    c.dWm = it.dWm;
    c.dphi = it.out_dlogits;
    c.dW = it.out_dW;
    c.hard_in = it.out_dW != nullptr ? it.hard : nullptr;
    c.E = it.rows * it.cols;
    c.N = N;
    c.M = M;
    c.tau = tau;
    c.np = make_noise(it.st, it.cols);
    c.status = status;
    c.stream = static_cast<cudaStream_t>(stream);
    calls.push_back(c);
  }
  return finish(launch_bwd_batch(calls.data(), int(calls.size())));
}

roi_status roi_mask_bwd_batch(const roi_bwd_item* items, int count, int N, int M, float tau, void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, 0, M);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  ranges.reserve(size_t(count) * 5);
  for (int i = 0; i < count; ++i) {
    const roi_bwd_item& it = items[i];
    s = check_common(N, M, tau, it.rows, it.cols);
    if (s != ROI_OK) return s;
    if (it.st.row_offset < 0) return ROI_ERR_SHAPE;
    if (!finite_positive(it.st.lambda)) return ROI_ERR_TAU;
    if (it.rows == 0) continue;
    if (it.logits == nullptr || it.W == nullptr || it.dWm == nullptr || it.out_dlogits == nullptr)
      return ROI_ERR_NULL;
    if (!aligned16(it.logits) || !aligned16(it.W) || !aligned16(it.dWm) || !aligned16(it.out_dlogits) ||
        !aligned16(it.out_dW))
      return ROI_ERR_ALIGN;
    const int64_t E = it.rows * it.cols;
    add_range(ranges, it.logits, uint64_t(E) * 4, false);
    add_range(ranges, it.W, uint64_t(E) * 2, false);
    add_range(ranges, it.dWm, uint64_t(E) * 2, false);
    add_range(ranges, it.out_dlogits, uint64_t(E) * 4, true);
    add_range(ranges, it.out_dW, uint64_t(E) * 2, true);
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  if (ranges.empty()) return ROI_OK;  // only empty items: nothing is read or written
  unsigned int* status = status_word();
  if (status == nullptr) return ROI_ERR_CUDA;
  std::vector<BwdCall> calls;
  calls.reserve(size_t(count));
  for (int i = 0; i < count; ++i) {
    const roi_bwd_item& it = items[i];
    if (it.rows == 0) continue;
    BwdCall c{};
    c.phi = it.logits;
    c.W = it.W;
    c.dWm = it.dWm;
    c.dphi = it.out_dlogits;
    c.dW = it.out_dW;
    c.E = it.rows * it.cols;
    c.N = N;
    c.M = M;
    c.tau = tau;
    c.np = make_noise(it.st, it.cols);
    c.status = status;
    c.stream = static_cast<cudaStream_t>(stream);
    calls.push_back(c);
  }
  return finish(launch_bwd_batch(calls.data(), int(calls.size())));
}

roi_status roi_mask_fwd_ex(const float* logits, const roi_bf16* W, int N, int M, float tau,
                           const roi_noise_state* st, int64_t rows, int64_t cols, roi_bf16* out_Wm,
                           float* out_soft, uint32_t* out_hard, void* stream) {
  return mask_fwd(logits, W, N, M, tau, st, rows, cols, out_Wm, out_soft, out_hard, false, stream);
}

roi_status roi_mask_fwd_st(const float* logits, const roi_bf16* W, int N, int M, float tau,
                           const roi_noise_state* st, int64_t rows, int64_t cols, roi_bf16* out_Wm,
                           float* out_soft, uint32_t* out_hard, void* stream) {
  return mask_fwd(logits, W, N, M, tau, st, rows, cols, out_Wm, out_soft, out_hard, true, stream);
}

roi_status roi_mask_fwd(const float* logits, const roi_bf16* W, int N, int M, float tau, uint64_t seed,
                        uint32_t step, int64_t rows, int64_t cols, roi_bf16* out_Wm, float* out_soft,
                        uint32_t* out_hard, void* stream) {
  roi_noise_state st;
  st.seed = seed;
  st.step = step;
  st.tensor_id = 0;
  st.lambda = 1.0f;
  st.row_offset = 0;
  return roi_mask_fwd_ex(logits, W, N, M, tau, &st, rows, cols, out_Wm, out_soft, out_hard, stream);
}

// The fused optimizer of roi_mask_bwd_adamw: logits updated in place, moments m, v.
struct FusedAdamW {
  float* phi;
  float* m;
  float* v;
  AdamW opt;
};

static roi_status mask_bwd(const float* logits, const roi_bf16* W, const roi_noise_state* st, int N, int M,
                           const roi_bf16* dWm, const uint32_t* hard, float tau, int64_t rows, int64_t cols,
                           float* out_dlogits, roi_bf16* out_dW, const FusedAdamW* fo, void* stream) {
  if (st == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, rows, cols);
  if (s != ROI_OK) return s;
  if (st->row_offset < 0) return ROI_ERR_SHAPE;
  if (!finite_positive(st->lambda)) return ROI_ERR_TAU;
  if (rows == 0) return ROI_OK;
  if (logits == nullptr || W == nullptr || dWm == nullptr || (out_dlogits == nullptr && fo == nullptr))
    return ROI_ERR_NULL;
  if (fo != nullptr && (fo->m == nullptr || fo->v == nullptr)) return ROI_ERR_NULL;
  if (!aligned16(logits) || !aligned16(W) || !aligned16(dWm) || !aligned16(out_dlogits) || !aligned16(out_dW))
    return ROI_ERR_ALIGN;
  if (fo != nullptr && (!aligned16(fo->m) || !aligned16(fo->v))) return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  // with the fused optimizer the logits are updated in place: they count as an
  // output for the overlap check against every other tensor (but not themselves)
  const Range in[4] = {{fo ? nullptr : logits, uint64_t(E) * 4}, {W, uint64_t(E) * 2}, {dWm, uint64_t(E) * 2},
                       {hard, uint64_t((E + 31) / 32) * 4}};
  const Range out[5] = {{out_dlogits, uint64_t(E) * 4}, {out_dW, uint64_t(E) * 2},
                        {fo ? logits : nullptr, uint64_t(E) * 4}, {fo ? fo->m : nullptr, uint64_t(E) * 4},
                        {fo ? fo->v : nullptr, uint64_t(E) * 4}};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  if (E == 0) return ROI_OK;
  BwdCall c;
  c.phi = logits;
  c.W = W;
  c.dWm = dWm;
  c.dphi = out_dlogits;
  c.dW = out_dW;
  c.hard_in = hard;
  c.phi_out = fo ? fo->phi : nullptr;
  c.m = fo ? fo->m : nullptr;
  c.v = fo ? fo->v : nullptr;
  c.opt = fo ? fo->opt : AdamW{};
  c.E = E;
  c.N = N;
  c.M = M;
  c.tau = tau;
  c.np = make_noise(*st, cols);
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_bwd(c));
}

roi_status roi_mask_bwd(const float* logits, const roi_bf16* W, const roi_noise_state* st, int N, int M,
                        const roi_bf16* dWm, float tau, int64_t rows, int64_t cols, float* out_dlogits,
                        roi_bf16* out_dW, void* stream) {
  return mask_bwd(logits, W, st, N, M, dWm, nullptr, tau, rows, cols, out_dlogits, out_dW, nullptr, stream);
}

roi_status roi_mask_bwd_st(const float* logits, const roi_bf16* W, const roi_noise_state* st, int N, int M,
                           const roi_bf16* dWm, const uint32_t* hard, float tau, int64_t rows, int64_t cols,
                           float* out_dlogits, roi_bf16* out_dW, void* stream) {
  if (out_dW != nullptr && hard == nullptr && rows > 0) return ROI_ERR_NULL;
  if (!aligned16(hard)) return ROI_ERR_ALIGN;
  return mask_bwd(logits, W, st, N, M, dWm, out_dW != nullptr ? hard : nullptr, tau, rows, cols, out_dlogits,
                  out_dW, nullptr, stream);
}

// Checks the optimizer settings and forms the step's constants, rounded to float
// as the float32 statement of the step forms them.
static roi_status adamw_constants(const roi_adamw* opt, AdamW* out) {
  if (opt == nullptr) return ROI_ERR_NULL;
  const bool ok = std::isfinite(opt->lr) && opt->lr >= 0.0f && opt->beta1 >= 0.0f && opt->beta1 < 1.0f &&
                  opt->beta2 >= 0.0f && opt->beta2 < 1.0f && finite_positive(opt->eps) &&
                  std::isfinite(opt->weight_decay) && opt->weight_decay >= 0.0f && opt->t >= 1;
  if (!ok) return ROI_ERR_OPT;
  out->b1 = opt->beta1;
  out->omb1 = 1.0f - opt->beta1;
  out->b2 = opt->beta2;
  out->omb2 = 1.0f - opt->beta2;
  out->eps = opt->eps;
  out->decay = 1.0f - opt->lr * opt->weight_decay;
  const double t = static_cast<double>(opt->t);
  out->step = static_cast<float>(static_cast<double>(opt->lr) / (1.0 - std::pow(static_cast<double>(opt->beta1), t)));
  out->r = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(static_cast<double>(opt->beta2), t)));
  return ROI_OK;
}

roi_status roi_mask_bwd_adamw(float* logits, const roi_bf16* W, const roi_noise_state* st, int N, int M,
                              const roi_bf16* dWm, float tau, int64_t rows, int64_t cols, float* m, float* v,
                              const roi_adamw* opt, float* out_dlogits, roi_bf16* out_dW, void* stream) {
  FusedAdamW fo;
  const roi_status s = adamw_constants(opt, &fo.opt);
  if (s != ROI_OK) return s;
  fo.phi = logits;
  fo.m = m;
  fo.v = v;
  return mask_bwd(logits, W, st, N, M, dWm, nullptr, tau, rows, cols, out_dlogits, out_dW, &fo, stream);
}

roi_status roi_mask_bwd_adamw_batch(const roi_adamw_item* items, int count, int N, int M, float tau,
                                    const roi_adamw* opt, void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  AdamW k;
  roi_status s = adamw_constants(opt, &k);
  if (s != ROI_OK) return s;
  s = check_common(N, M, tau, 0, M);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  ranges.reserve(size_t(count) * 7);
  for (int i = 0; i < count; ++i) {
    const roi_adamw_item& it = items[i];
    s = check_common(N, M, tau, it.rows, it.cols);
    if (s != ROI_OK) return s;
    if (it.st.row_offset < 0) return ROI_ERR_SHAPE;
    if (!finite_positive(it.st.lambda)) return ROI_ERR_TAU;
    if (it.rows == 0) continue;
    if (it.logits == nullptr || it.W == nullptr || it.dWm == nullptr || it.m == nullptr || it.v == nullptr)
      return ROI_ERR_NULL;
    if (!aligned16(it.logits) || !aligned16(it.W) || !aligned16(it.dWm) || !aligned16(it.m) || !aligned16(it.v) ||
        !aligned16(it.out_dlogits) || !aligned16(it.out_dW))
      return ROI_ERR_ALIGN;
    const int64_t E = it.rows * it.cols;
    add_range(ranges, it.W, uint64_t(E) * 2, false);
    add_range(ranges, it.dWm, uint64_t(E) * 2, false);
    add_range(ranges, it.logits, uint64_t(E) * 4, true);  // read and written
    add_range(ranges, it.m, uint64_t(E) * 4, true);
    add_range(ranges, it.v, uint64_t(E) * 4, true);
    add_range(ranges, it.out_dlogits, uint64_t(E) * 4, true);
    add_range(ranges, it.out_dW, uint64_t(E) * 2, true);
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  if (ranges.empty()) return ROI_OK;
  unsigned int* status = status_word();
  if (status == nullptr) return ROI_ERR_CUDA;
  std::vector<BwdCall> calls;
  calls.reserve(size_t(count));
  for (int i = 0; i < count; ++i) {
    const roi_adamw_item& it = items[i];
    if (it.rows == 0) continue;
    BwdCall c{};
    c.phi = it.logits;
    c.W = it.W;
    c.dWm = it.dWm;
    c.dphi = it.out_dlogits;
    c.dW = it.out_dW;
    c.phi_out = it.logits;
    c.m = it.m;
    c.v = it.v;
    c.opt = k;
    c.E = it.rows * it.cols;
    c.N = N;
    c.M = M;
    c.tau = tau;
    c.np = make_noise(it.st, it.cols);
    c.status = status;
    c.stream = static_cast<cudaStream_t>(stream);
    calls.push_back(c);
  }
  return finish(launch_bwd_batch(calls.data(), int(calls.size())));
}

float roi_anneal(float init, float end, uint32_t t, uint32_t T_anneal) {
  if (T_anneal == 0) return end;
  const double x = static_cast<double>(init) *
                   std::pow(static_cast<double>(end) / static_cast<double>(init),
                            static_cast<double>(t) / static_cast<double>(T_anneal));
  return static_cast<float>(x > static_cast<double>(end) ? x : static_cast<double>(end));
}

roi_status roi_export_compressed_2of4(const float* logits, const roi_bf16* W, int64_t rows, int64_t cols,
                                      roi_bf16* out_values, uint32_t* out_meta, void* stream) {
  roi_status s = check_common(2, 4, 1.0f, rows, cols);
  if (s != ROI_OK) return s;
  if ((rows * cols) % 32 != 0) return ROI_ERR_SHAPE;
  if (rows == 0) return ROI_OK;
  if (logits == nullptr || W == nullptr || out_values == nullptr || out_meta == nullptr) return ROI_ERR_NULL;
  if (!aligned16(logits) || !aligned16(W) || !aligned16(out_values) || !aligned16(out_meta)) return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  const Range in[2] = {{logits, uint64_t(E) * 4}, {W, uint64_t(E) * 2}};
  const Range out[2] = {{out_values, uint64_t(E)}, {out_meta, uint64_t(E / 32) * 4}};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  CompressCall c;
  c.phi = logits;
  c.W = W;
  c.values = out_values;
  c.meta = out_meta;
  c.E = E;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_export_compressed_2of4(c));
}

roi_status roi_hard_mask_export(const float* logits, int N, int M, int64_t rows, int64_t cols, uint32_t* out_bits,
                                const roi_bf16* W, roi_bf16* out_Wpruned, void* stream) {
  roi_status s = check_common(N, M, 1.0f, rows, cols);
  if (s != ROI_OK) return s;
  if (rows == 0) return ROI_OK;
  if (logits == nullptr || out_bits == nullptr) return ROI_ERR_NULL;
  if ((W == nullptr) != (out_Wpruned == nullptr)) return ROI_ERR_NULL;
  if (!aligned16(logits) || !aligned16(out_bits) || !aligned16(W) || !aligned16(out_Wpruned)) return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  const Range in[2] = {{logits, uint64_t(E) * 4}, {W, uint64_t(E) * 2}};
  const Range out[2] = {{out_bits, uint64_t((E + 31) / 32) * 4}, {out_Wpruned, uint64_t(E) * 2}};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  if (E == 0) return ROI_OK;
  ExportCall c;
  c.phi = logits;
  c.bits = out_bits;
  c.W = W;
  c.Wp = out_Wpruned;
  c.E = E;
  c.N = N;
  c.M = M;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_export(c));
}

size_t roi_masked_linear_workspace_size(int64_t T, int64_t rows, int64_t cols) {
  if (T <= 0 || T > 256 || rows <= 0 || cols <= 0 || cols > INT64_MAX / 64 / rows) return 0;
  return linear_workspace_bytes(T, rows, cols);
}

}  // extern "C"

namespace roi {
namespace {

// Split-K scratch of roi_masked_linear_fwd_noalloc: one static array per device,
// ROI_LINEAR_SCRATCH_BYTES long.
static __device__ __align__(256) unsigned char g_linear_scratch[ROI_LINEAR_SCRATCH_BYTES];

// The array's device address on the current device, looked up once per device
// (nullptr if the lookup fails or the address is not 256-byte aligned).
void* linear_scratch() {
  static std::atomic<void*> cache[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  void* p = cache[dev].load(std::memory_order_acquire);
  if (p == nullptr) {
    if (cudaGetSymbolAddress(&p, g_linear_scratch) != cudaSuccess || p == nullptr ||
        (reinterpret_cast<uintptr_t>(p) & 255u) != 0)
      return nullptr;
    cache[dev].store(p, std::memory_order_release);
  }
  return p;
}

}  // namespace
}  // namespace roi

extern "C" {

roi_status roi_masked_linear_fwd(const roi_bf16* X, const float* logits, const roi_bf16* W, int N, int M, float tau,
                                 const roi_noise_state* st, int64_t T, int64_t rows, int64_t cols, float* out_Y,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (st == nullptr) return ROI_ERR_NULL;
  roi_status s = check_common(N, M, tau, rows, cols);
  if (s != ROI_OK) return s;
  if (!linear_supported(N, M)) return ROI_ERR_NM;
  if (st->row_offset < 0 || T < 0 || T > 256 || cols % 8 != 0) return ROI_ERR_SHAPE;
  if (!finite_positive(st->lambda)) return ROI_ERR_TAU;
  if (rows == 0 || T == 0) return ROI_OK;  // nothing is read or written; pointers may be NULL
  if (X == nullptr || logits == nullptr || W == nullptr || out_Y == nullptr) return ROI_ERR_NULL;
  if (!aligned16(X) || !aligned16(logits) || !aligned16(W) || !aligned16(out_Y) || !aligned16(workspace))
    return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  const Range in[3] = {{X, uint64_t(T * cols) * 2}, {logits, uint64_t(E) * 4}, {W, uint64_t(E) * 2}};
  const Range out[2] = {{out_Y, uint64_t(T * rows) * 4}, {workspace, workspace == nullptr ? 0 : uint64_t(workspace_bytes)}};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  LinearCall c;
  c.X = X;
  c.phi = logits;
  c.W = W;
  c.Y = out_Y;
  c.workspace = workspace;
  c.workspace_bytes = workspace == nullptr ? 0 : workspace_bytes;
  c.T = T;
  c.rows = rows;
  c.cols = cols;
  c.N = N;
  c.M = M;
  c.tau = tau;
  c.np = make_noise(*st, cols);
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_masked_linear(c));
}

roi_status roi_masked_linear_fwd_noalloc(const roi_bf16* X, const float* logits, const roi_bf16* W, int N, int M,
                                         float tau, const roi_noise_state* st, int64_t T, int64_t rows, int64_t cols,
                                         float* out_Y, void* stream) {
  const size_t need = roi_masked_linear_workspace_size(T, rows, cols);
  if (need > size_t(ROI_LINEAR_SCRATCH_BYTES)) return ROI_ERR_SHAPE;
  void* ws = nullptr;
  if (need > 0) {
    ws = linear_scratch();
    if (ws == nullptr) return ROI_ERR_CUDA;
  }
  return roi_masked_linear_fwd(X, logits, W, N, M, tau, st, T, rows, cols, out_Y, ws, need, stream);
}

int64_t roi_checkpoint_pitch(int64_t cols) { return cols <= 0 || cols > INT64_MAX / 1024 ? 0 : block8_pitch(cols); }
int64_t roi_checkpoint_scale_pitch(int64_t cols) {
  return cols <= 0 || cols > INT64_MAX / 1024 ? 0 : block8_scale_pitch(cols);
}

static roi_status checkpoint_call(const void* x_in, void* x_out, int8_t* codes, uint8_t* scales, int dtype, int64_t rows,
                                  int64_t cols, int64_t ld, void* stream) {
  if (!known_type(dtype)) return ROI_ERR_TYPE;
  if (!good_shape(rows, cols, ld)) return ROI_ERR_SHAPE;
  if (rows == 0) return ROI_OK;
  const void* x = x_in != nullptr ? x_in : x_out;
  if (x == nullptr || codes == nullptr || scales == nullptr) return ROI_ERR_NULL;
  const int b = type_bytes(dtype);
  if (!aligned_to(x, b) || !aligned16(codes) || !aligned_to(scales, 4)) return ROI_ERR_ALIGN;
  const Strided m = matrix(x, rows, cols, ld, b), q = flat(codes, uint64_t(rows) * uint64_t(block8_pitch(cols))),
                s = flat(scales, uint64_t(rows) * uint64_t(block8_scale_pitch(cols)));
  if (overlaps(m, q) || overlaps(m, s) || (x_in != nullptr && overlaps(q, s))) return ROI_ERR_ALIAS;
  CheckpointCall c;
  c.x_in = x_in;
  c.x_out = x_out;
  c.codes = codes;
  c.scales = scales;
  c.dtype = static_cast<Elem>(dtype);
  c.rows = rows;
  c.cols = cols;
  c.ld = ld;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(x_in != nullptr ? launch_checkpoint_save(c) : launch_checkpoint_load(c));
}

roi_status roi_checkpoint_save(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t* out_codes,
                               uint8_t* out_scales, void* stream) {
  return checkpoint_call(x, nullptr, out_codes, out_scales, dtype, rows, cols, ldx, stream);
}

roi_status roi_checkpoint_load(const int8_t* codes, const uint8_t* scales, int dtype, int64_t rows, int64_t cols,
                               void* out_x, int64_t ldx, void* stream) {
  // (the codes and scales of a load are only read)
  return checkpoint_call(nullptr, out_x, const_cast<int8_t*>(codes), const_cast<uint8_t*>(scales), dtype, rows, cols, ldx,
                         stream);
}

// The norms count the columns of a row in 32 bits.
static constexpr int64_t kNormCols = int64_t(1) << 30;

roi_status roi_norm_fwd(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int kind, const void* gamma,
                        const void* beta, int param_dtype, float eps, void* out_y, int64_t ldy, float* out_mean,
                        float* out_rstd, int8_t* out_xcodes, uint8_t* out_xscales, int8_t* out_ycodes,
                        uint8_t* out_yscales, void* stream) {
  const bool layer = kind == ROI_LAYER_NORM;
  if (!known_type(dtype) || (param_dtype != dtype && param_dtype != ROI_FP32) || (!layer && kind != ROI_RMS_NORM) ||
      !std::isfinite(eps) || eps < 0.0f || (!layer && (beta != nullptr || out_mean != nullptr)))
    return ROI_ERR_TYPE;
  if (!good_shape(rows, cols, ldx) || !good_shape(rows, cols, ldy) || cols > kNormCols) return ROI_ERR_SHAPE;
  if (rows == 0) return ROI_OK;
  if (x == nullptr || out_y == nullptr || (out_xcodes == nullptr) != (out_xscales == nullptr) ||
      (out_ycodes == nullptr) != (out_yscales == nullptr))
    return ROI_ERR_NULL;
  const int b = type_bytes(dtype), pb = type_bytes(param_dtype);
  if (!aligned_to(x, b) || !aligned_to(out_y, b) || !aligned16(gamma) || !aligned16(beta) || !aligned_to(out_mean, 4) ||
      !aligned_to(out_rstd, 4) || !aligned16(out_xcodes) || !aligned16(out_ycodes) || !aligned_to(out_xscales, 4) ||
      !aligned_to(out_yscales, 4))
    return ROI_ERR_ALIGN;
  const uint64_t q = uint64_t(rows) * uint64_t(block8_pitch(cols)), s = uint64_t(rows) * uint64_t(block8_scale_pitch(cols));
  const Strided in[3] = {matrix(x, rows, cols, ldx, b), flat(gamma, uint64_t(cols) * pb), flat(beta, uint64_t(cols) * pb)};
  const Strided out[7] = {matrix(out_y, rows, cols, ldy, b), flat(out_mean, uint64_t(rows) * 4), flat(out_rstd, uint64_t(rows) * 4),
                          flat(out_xcodes, q), flat(out_xscales, s), flat(out_ycodes, q), flat(out_yscales, s)};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  NormFwdCall c;
  c.x = x;
  c.y = out_y;
  c.gamma = gamma;
  c.beta = beta;
  c.mean = out_mean;
  c.rstd = out_rstd;
  c.xcodes = out_xcodes;
  c.xscales = out_xscales;
  c.ycodes = out_ycodes;
  c.yscales = out_yscales;
  c.dtype = static_cast<Elem>(dtype);
  c.layer = layer;
  c.params32 = param_dtype == ROI_FP32;
  c.eps = eps;
  c.rows = rows;
  c.cols = cols;
  c.ldx = ldx;
  c.ldy = ldy;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_norm_fwd(c));
}

size_t roi_norm_bwd_workspace_size(int64_t rows, int64_t cols) {
  return good_shape(rows, cols, cols) && rows > 0 ? norm_bwd_workspace_bytes(rows, cols) : 0;
}

roi_status roi_norm_bwd(const void* dy, int dtype, int64_t rows, int64_t cols, int64_t lddy, const void* x, int64_t ldx,
                        const int8_t* codes, const uint8_t* scales, int kind, const void* gamma, int param_dtype,
                        const float* mean, const float* rstd, void* out_dx, int64_t lddx, float* out_dgamma,
                        float* out_dbeta, void* workspace, size_t workspace_bytes, void* stream) {
  const bool layer = kind == ROI_LAYER_NORM;
  if (!known_type(dtype) || (param_dtype != dtype && param_dtype != ROI_FP32) || (!layer && kind != ROI_RMS_NORM) ||
      (!layer && (mean != nullptr || out_dbeta != nullptr)))
    return ROI_ERR_TYPE;
  if (!good_shape(rows, cols, lddy) || !good_shape(rows, cols, lddx) || (x != nullptr && !good_shape(rows, cols, ldx)) ||
      cols > kNormCols)
    return ROI_ERR_SHAPE;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (!aligned_to(out_dgamma, 4) || !aligned_to(out_dbeta, 4)) return ROI_ERR_ALIGN;
  if (rows == 0) {  // empty sums
    if ((out_dgamma != nullptr && cudaMemsetAsync(out_dgamma, 0, size_t(cols) * 4, st) != cudaSuccess) ||
        (out_dbeta != nullptr && cudaMemsetAsync(out_dbeta, 0, size_t(cols) * 4, st) != cudaSuccess))
      return ROI_ERR_CUDA;
    return ROI_OK;
  }
  const bool sums = out_dgamma != nullptr || out_dbeta != nullptr;
  if (dy == nullptr || out_dx == nullptr || rstd == nullptr || (layer && mean == nullptr) ||
      (codes == nullptr) != (scales == nullptr) || (x == nullptr) == (codes == nullptr) || (sums && workspace == nullptr))
    return ROI_ERR_NULL;
  const size_t need = sums ? norm_bwd_workspace_bytes(rows, cols) : 0;
  if (workspace_bytes < need) return ROI_ERR_SHAPE;
  const int b = type_bytes(dtype), pb = type_bytes(param_dtype);
  if (!aligned_to(dy, b) || !aligned_to(x, b) || !aligned_to(out_dx, b) || !aligned16(codes) || !aligned_to(scales, 4) ||
      !aligned16(gamma) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) || !aligned16(workspace))
    return ROI_ERR_ALIGN;
  const Strided in[7] = {matrix(dy, rows, cols, lddy, b),
                         matrix(x, rows, cols, ldx, b),
                         flat(codes, uint64_t(rows) * uint64_t(block8_pitch(cols))),
                         flat(scales, uint64_t(rows) * uint64_t(block8_scale_pitch(cols))),
                         flat(gamma, uint64_t(cols) * pb),
                         flat(mean, uint64_t(rows) * 4),
                         flat(rstd, uint64_t(rows) * 4)};
  const Strided out[4] = {matrix(out_dx, rows, cols, lddx, b), flat(out_dgamma, uint64_t(cols) * 4),
                          flat(out_dbeta, uint64_t(cols) * 4), flat(sums ? workspace : nullptr, need)};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  NormBwdCall c;
  c.dy = dy;
  c.x = x;
  c.codes = codes;
  c.scales = scales;
  c.gamma = gamma;
  c.mean = mean;
  c.rstd = rstd;
  c.dx = out_dx;
  c.dgamma = out_dgamma;
  c.dbeta = out_dbeta;
  c.workspace = workspace;
  c.dtype = static_cast<Elem>(dtype);
  c.layer = layer;
  c.params32 = param_dtype == ROI_FP32;
  c.rows = rows;
  c.cols = cols;
  c.lddy = lddy;
  c.ldx = ldx;
  c.lddx = lddx;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = st;
  return finish(launch_norm_bwd(c));
}

// Tensor-map coordinates and tile numbers are 32-bit.
static bool wgrad_shape(int64_t T, int64_t rows, int64_t cols, int64_t lddy) {
  constexpr int64_t kMost = int64_t(1) << 30;
  return good_shape(T, rows, lddy) && good_shape(rows, cols, cols) && rows > 0 && T <= kMost && rows <= kMost && cols <= kMost &&
         (rows / 128 + 1) * (cols / 128 + 1) <= kMost;
}

size_t roi_masked_linear_wgrad_workspace_size(int64_t T, int64_t rows, int64_t cols, int64_t lddy) {
  return T > 0 && wgrad_shape(T, rows, cols, lddy) ? wgrad_workspace_bytes(T, rows, cols, lddy) : 0;
}

roi_status roi_masked_linear_wgrad(const roi_bf16* dY, int64_t lddy, const int8_t* codes, const uint8_t* scales, int64_t T,
                                   int64_t rows, int64_t cols, roi_bf16* out_dWm, float* acc, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (rows == 0 && T >= 0 && cols > 0) return ROI_OK;
  if (!wgrad_shape(T, rows, cols, lddy)) return ROI_ERR_SHAPE;
  const size_t copy = wgrad_copy_bytes(T, rows, lddy);
  if ((out_dWm == nullptr && acc == nullptr) || (T > 0 && (dY == nullptr || codes == nullptr || scales == nullptr)) ||
      (copy > 0 && workspace == nullptr))
    return ROI_ERR_NULL;
  if (copy > 0 && workspace_bytes < copy) return ROI_ERR_SHAPE;
  if (!aligned16(dY) || !aligned16(codes) || !aligned_to(scales, 4) || !aligned16(out_dWm) || !aligned16(acc) ||
      !aligned16(workspace))
    return ROI_ERR_ALIGN;
  const uint64_t E = uint64_t(rows) * uint64_t(cols);
  const size_t need = T > 0 ? wgrad_workspace_bytes(T, rows, cols, lddy) : 0;
  const uint64_t used = workspace == nullptr ? 0 : need < workspace_bytes ? need : workspace_bytes;
  const Strided in[3] = {matrix(dY, T, rows, lddy, 2), flat(codes, uint64_t(T) * uint64_t(block8_pitch(cols))),
                         flat(scales, uint64_t(T) * uint64_t(block8_scale_pitch(cols)))};
  const Strided out[3] = {flat(out_dWm, E * 2), flat(acc, E * 4), flat(workspace, used)};
  if (any_alias(in, out)) return ROI_ERR_ALIAS;
  WgradCall c;
  c.dY = dY;
  c.codes = codes;
  c.scales = scales;
  c.dWm = out_dWm;
  c.acc = acc;
  c.workspace = workspace;
  c.workspace_bytes = workspace == nullptr ? 0 : workspace_bytes;
  c.T = T;
  c.rows = rows;
  c.cols = cols;
  c.lddy = lddy;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_wgrad(c));
}

int64_t roi_fp8_pitch(int64_t cols) { return cols <= 0 || cols > INT64_MAX / 1024 ? 0 : fp8_pitch(cols); }
int64_t roi_fp8_scale_pitch(int64_t cols) { return cols <= 0 || cols > INT64_MAX / 1024 ? 0 : fp8_scale_pitch(cols); }

static bool known_format(int format) { return format == ROI_E4M3 || format == ROI_E5M2; }
// Tensor-map coordinates and tile numbers are 32-bit.
static constexpr int64_t kFp8Most = int64_t(1) << 30;

static roi_status fp8_save(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int format, bool weight,
                           uint8_t* codes, uint8_t* scales, void* stream) {
  if (!known_type(dtype) || !known_format(format)) return ROI_ERR_TYPE;
  if (!good_shape(rows, cols, ld) || rows > kFp8Most || cols > kFp8Most) return ROI_ERR_SHAPE;
  if (rows == 0) return ROI_OK;
  if (x == nullptr || codes == nullptr || scales == nullptr) return ROI_ERR_NULL;
  const int b = type_bytes(dtype);
  if (!aligned_to(x, weight ? 16 : b) || !aligned16(codes) || !aligned16(scales)) return ROI_ERR_ALIGN;
  const Strided m[1] = {matrix(x, rows, cols, ld, b)};
  const Strided out[2] = {flat(codes, uint64_t(rows) * uint64_t(fp8_pitch(cols))),
                          flat(scales, uint64_t(weight ? (rows + 127) / 128 : rows) * uint64_t(fp8_scale_pitch(cols)))};
  if (any_alias(m, out)) return ROI_ERR_ALIAS;
  Fp8SaveCall c;
  c.x = x;
  c.codes = codes;
  c.scales = scales;
  c.dtype = static_cast<Elem>(dtype);
  c.format = static_cast<Fp8>(format);
  c.rows = rows;
  c.cols = cols;
  c.ld = ld;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(weight ? launch_fp8_save_weight(c) : launch_fp8_save(c));
}

roi_status roi_fp8_save(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int format, uint8_t* out_codes,
                        uint8_t* out_scales, void* stream) {
  return fp8_save(x, dtype, rows, cols, ldx, format, false, out_codes, out_scales, stream);
}

roi_status roi_fp8_save_weight(const roi_bf16* W, int64_t rows, int64_t cols, uint8_t* out_codes, uint8_t* out_scales, void* stream) {
  return fp8_save(W, ROI_BF16, rows, cols, cols, ROI_E4M3, true, out_codes, out_scales, stream);
}

static roi_status fp8_linear(bool dgrad, const uint8_t* x_codes, const uint8_t* x_scales, int format, const uint8_t* w_codes,
                             const uint8_t* w_scales, int64_t T, int64_t rows, int64_t cols, void* out, int dtype, int64_t ldo,
                             void* stream) {
  if (!known_type(dtype) || !known_format(format)) return ROI_ERR_TYPE;
  const int64_t outs = dgrad ? cols : rows, width = dgrad ? rows : cols;
  if (T < 0 || rows < 0 || cols <= 0 || T > kFp8Most || rows > kFp8Most || cols > kFp8Most) return ROI_ERR_SHAPE;
  if (T == 0 || outs == 0) return ROI_OK;
  if (!good_shape(T, outs, ldo) || ((outs + 127) / 128) * ((T + 255) / 256) > kFp8Most) return ROI_ERR_SHAPE;
  const int b = type_bytes(dtype);
  if (out == nullptr || (width > 0 && (x_codes == nullptr || x_scales == nullptr || w_codes == nullptr || w_scales == nullptr)))
    return ROI_ERR_NULL;
  if (!aligned_to(out, b) || !aligned16(x_codes) || !aligned16(x_scales) || !aligned16(w_codes) || !aligned16(w_scales))
    return ROI_ERR_ALIGN;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (width == 0)  // empty sums
    return cudaMemset2DAsync(out, size_t(ldo) * b, 0, size_t(outs) * b, size_t(T), st) == cudaSuccess ? ROI_OK : ROI_ERR_CUDA;
  const Strided in[4] = {flat(x_codes, uint64_t(T) * uint64_t(fp8_pitch(width))), flat(x_scales, uint64_t(T) * uint64_t(fp8_scale_pitch(width))),
                         flat(w_codes, uint64_t(rows) * uint64_t(fp8_pitch(cols))),
                         flat(w_scales, uint64_t((rows + 127) / 128) * uint64_t(fp8_scale_pitch(cols)))};
  const Strided o[1] = {matrix(out, T, outs, ldo, b)};
  if (any_alias(in, o)) return ROI_ERR_ALIAS;
  Fp8LinearCall c;
  c.x_codes = x_codes;
  c.x_scales = x_scales;
  c.w_codes = w_codes;
  c.w_scales = w_scales;
  c.out = out;
  c.format = static_cast<Fp8>(format);
  c.dtype = static_cast<Elem>(dtype);
  c.dgrad = dgrad;
  c.T = T;
  c.rows = rows;
  c.cols = cols;
  c.ldo = ldo;
  c.status = status_word();
  if (c.status == nullptr) return ROI_ERR_CUDA;
  c.stream = st;
  return finish(launch_fp8_linear(c));
}

roi_status roi_fp8_linear_fwd(const uint8_t* x_codes, const uint8_t* x_scales, int format, const uint8_t* w_codes,
                              const uint8_t* w_scales, int64_t T, int64_t rows, int64_t cols, void* out_y, int dtype, int64_t ldy,
                              void* stream) {
  return fp8_linear(false, x_codes, x_scales, format, w_codes, w_scales, T, rows, cols, out_y, dtype, ldy, stream);
}

roi_status roi_fp8_linear_dgrad(const uint8_t* dy_codes, const uint8_t* dy_scales, int format, const uint8_t* w_codes,
                                const uint8_t* w_scales, int64_t T, int64_t rows, int64_t cols, void* out_dx, int dtype, int64_t lddx,
                                void* stream) {
  return fp8_linear(true, dy_codes, dy_scales, format, w_codes, w_scales, T, rows, cols, out_dx, dtype, lddx, stream);
}

// Elements of a tensor whose byte counts fit.
static bool good_count(int64_t n) { return n >= 0 && n <= INT64_MAX / 64; }
static uint64_t whole_blocks(int64_t n) { return (uint64_t(n) + 127) / 128 * 128; }

roi_status roi_adamw_step(const roi_adamw_step_item* items, int count, const roi_adamw* opt, const float* grad_scale, void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  OptimCall c{};
  const roi_status s = adamw_constants(opt, &c.opt);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  std::vector<OptimItem> to;
  ranges.reserve(size_t(count) * 5 + 1);
  to.reserve(size_t(count));
  if (!aligned_to(grad_scale, 4)) return ROI_ERR_ALIGN;
  add_range(ranges, grad_scale, 4, false);
  for (int i = 0; i < count; ++i) {
    const roi_adamw_step_item& x = items[i];
    if (!known_type(x.grad_dtype) || (x.out_copy != nullptr && x.copy_dtype != ROI_BF16 && x.copy_dtype != ROI_FP16)) return ROI_ERR_TYPE;
    if (!good_count(x.n)) return ROI_ERR_SHAPE;
    if (x.n == 0) continue;
    if (x.param == nullptr || x.grad == nullptr || x.m == nullptr || x.v == nullptr) return ROI_ERR_NULL;
    if (!aligned16(x.param) || !aligned16(x.grad) || !aligned16(x.m) || !aligned16(x.v) || !aligned16(x.out_copy)) return ROI_ERR_ALIGN;
    const uint64_t n = uint64_t(x.n);
    add_range(ranges, x.grad, n * uint64_t(type_bytes(x.grad_dtype)), false);
    add_range(ranges, x.param, n * 4, true);
    add_range(ranges, x.m, n * 4, true);
    add_range(ranges, x.v, n * 4, true);
    add_range(ranges, x.out_copy, n * 2, true);
    to.push_back({x.param, x.grad, x.m, x.v, nullptr, x.out_copy, x.n, 0u, static_cast<Elem>(x.grad_dtype),
                  x.out_copy != nullptr ? static_cast<Elem>(x.copy_dtype) : Elem::kBf16});
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  c.kind = OptimKind::kStep;
  c.scale = grad_scale;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_optim(c, to.data(), int(to.size())));
}

roi_status roi_adamw_step8(const roi_adamw_step8_item* items, int count, const roi_adamw* opt, uint64_t seed, const float* grad_scale,
                           void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  OptimCall c{};
  const roi_status s = adamw_constants(opt, &c.opt);
  if (s != ROI_OK) return s;
  std::vector<Tagged> ranges;
  std::vector<OptimItem> to;
  ranges.reserve(size_t(count) * 6 + 1);
  to.reserve(size_t(count));
  if (!aligned_to(grad_scale, 4)) return ROI_ERR_ALIGN;
  add_range(ranges, grad_scale, 4, false);
  for (int i = 0; i < count; ++i) {
    const roi_adamw_step8_item& x = items[i];
    if (!known_type(x.grad_dtype) || (x.out_copy != nullptr && x.copy_dtype != ROI_BF16 && x.copy_dtype != ROI_FP16)) return ROI_ERR_TYPE;
    if (!good_count(x.n)) return ROI_ERR_SHAPE;
    if (x.n == 0) continue;
    if (x.param == nullptr || x.grad == nullptr || x.m_codes == nullptr || x.u_codes == nullptr || x.scales == nullptr) return ROI_ERR_NULL;
    if (!aligned16(x.param) || !aligned16(x.grad) || !aligned16(x.m_codes) || !aligned16(x.u_codes) || !aligned_to(x.scales, 2) ||
        !aligned16(x.out_copy))
      return ROI_ERR_ALIGN;
    const uint64_t n = uint64_t(x.n), codes = whole_blocks(x.n);
    add_range(ranges, x.grad, n * uint64_t(type_bytes(x.grad_dtype)), false);
    add_range(ranges, x.param, n * 4, true);
    add_range(ranges, x.m_codes, codes, true);
    add_range(ranges, x.u_codes, codes, true);
    add_range(ranges, x.scales, codes / 64, true);
    add_range(ranges, x.out_copy, n * 2, true);
    to.push_back({x.param, x.grad, x.m_codes, x.u_codes, x.scales, x.out_copy, x.n, x.tensor_id, static_cast<Elem>(x.grad_dtype),
                  x.out_copy != nullptr ? static_cast<Elem>(x.copy_dtype) : Elem::kBf16});
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  c.kind = OptimKind::kStep8;
  c.seed = seed;
  c.step = opt->t;
  c.scale = grad_scale;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_optim(c, to.data(), int(to.size())));
}

roi_status roi_adamw_state8_load(const roi_adamw_state8_item* items, int count, void* stream) {
  if (count < 0) return ROI_ERR_SHAPE;
  if (count > 0 && items == nullptr) return ROI_ERR_NULL;
  OptimCall c{};
  std::vector<Tagged> ranges;
  std::vector<OptimItem> to;
  ranges.reserve(size_t(count) * 5);
  to.reserve(size_t(count));
  for (int i = 0; i < count; ++i) {
    const roi_adamw_state8_item& x = items[i];
    if (!known_type(x.dtype)) return ROI_ERR_TYPE;
    if (!good_count(x.n)) return ROI_ERR_SHAPE;
    if (x.n == 0) continue;
    if (x.m_codes == nullptr || x.u_codes == nullptr || x.scales == nullptr || (x.out_m == nullptr && x.out_u == nullptr)) return ROI_ERR_NULL;
    if (!aligned16(x.m_codes) || !aligned16(x.u_codes) || !aligned_to(x.scales, 2) || !aligned16(x.out_m) || !aligned16(x.out_u))
      return ROI_ERR_ALIGN;
    const uint64_t bytes = uint64_t(x.n) * uint64_t(type_bytes(x.dtype)), codes = whole_blocks(x.n);
    add_range(ranges, x.m_codes, codes, false);
    add_range(ranges, x.u_codes, codes, false);
    add_range(ranges, x.scales, codes / 64, false);
    add_range(ranges, x.out_m, bytes, true);
    add_range(ranges, x.out_u, bytes, true);
    to.push_back({static_cast<float*>(x.out_m), nullptr, const_cast<uint8_t*>(x.m_codes), const_cast<uint8_t*>(x.u_codes),
                  const_cast<uint8_t*>(x.scales), x.out_u, x.n, 0u, static_cast<Elem>(x.dtype), Elem::kBf16});
  }
  if (batch_alias(ranges)) return ROI_ERR_ALIAS;
  c.kind = OptimKind::kLoad8;
  c.stream = static_cast<cudaStream_t>(stream);
  return finish(launch_optim(c, to.data(), int(to.size())));
}

static roi_status noise_call(const roi_noise_state* st, int64_t rows, int64_t cols, uint32_t* words, float* g,
                             void* stream) {
  if (st == nullptr) return ROI_ERR_NULL;
  if (rows < 0 || cols <= 0 || (rows > 0 && cols > INT64_MAX / 64 / rows) || st->row_offset < 0) return ROI_ERR_SHAPE;
  if (rows == 0) return ROI_OK;
  if (words == nullptr && g == nullptr) return ROI_ERR_NULL;
  if (!aligned16(words) || !aligned16(g)) return ROI_ERR_ALIGN;
  const int64_t E = rows * cols;
  return finish(launch_noise(make_noise(*st, cols), E, words, g, static_cast<cudaStream_t>(stream)));
}

roi_status roi_noise_words(const roi_noise_state* st, int64_t rows, int64_t cols, uint32_t* out_words, void* stream) {
  if (out_words == nullptr && rows > 0) return ROI_ERR_NULL;
  return noise_call(st, rows, cols, out_words, nullptr, stream);
}

roi_status roi_gumbel_noise(const roi_noise_state* st, int64_t rows, int64_t cols, float* out_g, void* stream) {
  if (out_g == nullptr && rows > 0) return ROI_ERR_NULL;
  return noise_call(st, rows, cols, nullptr, out_g, stream);
}

roi_status roi_set_ring_wait_limit_ns(uint64_t ns) {
  if (cudaMemcpyToSymbol(g_roi_device_status, &ns, sizeof(ns), kStatusLimitWord * sizeof(unsigned int)) !=
      cudaSuccess)
    return ROI_ERR_CUDA;
  return ROI_OK;
}

roi_status roi_device_status(void* stream) {
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return ROI_ERR_CUDA;
  unsigned int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_roi_device_status, sizeof(v)) != cudaSuccess) return ROI_ERR_CUDA;
  if (v != 0) {
    const unsigned int zero = 0;
    cudaMemcpyToSymbol(g_roi_device_status, &zero, sizeof(zero));
    return ROI_ERR_TIMEOUT;
  }
  return ROI_OK;
}

const char* roi_status_string(roi_status s) {
  switch (s) {
    case ROI_OK: return "ok";
    case ROI_ERR_NULL: return "a required pointer is NULL (or W / out_Wpruned given without the other)";
    case ROI_ERR_SHAPE: return "bad shape: rows < 0, cols <= 0, cols % M != 0, size overflow or row_offset < 0";
    case ROI_ERR_NM: return "need 1 <= N < M <= 32";
    case ROI_ERR_TAU: return "tau and lambda must be finite and > 0";
    case ROI_ERR_ALIGN: return "tensor pointers must be 16-byte aligned";
    case ROI_ERR_ALIAS: return "an output overlaps an input or another output";
    case ROI_ERR_CUDA: return "CUDA error while launching";
    case ROI_ERR_TIMEOUT: return "a kernel gave up waiting on its own copies";
    case ROI_ERR_OPT: return "bad optimizer settings: need lr, weight_decay >= 0 finite, 0 <= beta < 1, eps > 0, t >= 1";
    case ROI_ERR_TYPE:
      return "unknown element type or norm kind, eps not finite and >= 0, or a mean or bias with a norm that has none";
  }
  return "unknown status";
}

uint64_t roi_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

}  // extern "C"
