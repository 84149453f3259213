// What a per-site classifier answers with and learns from: per active site
// the log probability of its label, the entropy of its class distribution and
// the best classes, and the gradient of those numbers at the logits.
//
// Row x of `classes` values, m = max x, t = sum of exp(x_k - m) over all
// classes but one largest, L = log1p(t) (so log sum exp x = m + L):
//   log p_k = (x_k - m) - L,   H = L - sum_k exp(x_k - m) (x_k - m) / (1 + t).
// Leaving the largest (a 1) out of t keeps a sure row's small numbers: its
// log probability is -t, where log(1 + t) would have dropped t's low bits.
// Sums are fp32, over the values as they are stored.
#include <algorithm>

#include "internal.h"
#include "numeric.h"

namespace sscn {

namespace {

constexpr int kMaxTop = 16;  // best classes a call may ask for

// Order of the best classes as one whole number, larger first: by value (NaN
// above everything, -0 equal to 0), ties to the lowest class.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t cls) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = x != x ? 0xfffffffeu : ((int32_t)b < 0 ? ~b : b | 0x80000000u);
  return (uint64_t)o << 32 | (0xffffffffu - cls);
}
__device__ __forceinline__ uint32_t key_class(uint64_t k) { return 0xffffffffu - (uint32_t)k; }

// A row's sums: s over the values below m, eq = how many equal m, a = sum of
// exp(d) d.
struct RowSums {
  float s, a;
  int eq;
};
__device__ __forceinline__ void add_value(RowSums& q, float x, float m, float base) {
  const float d = x - base;
  const float e = expf(d);
  const bool top = x == m;
  q.s += top ? 0.f : e;  // a NaN stays in s
  q.eq += top;
  q.a += e * (d < -200.f ? -200.f : d);  // exp(-200) is 0: no 0 * inf
}
// (L, H) from the sums.  A row of -inf only: 0, 0.  NaN or +inf in the row: NaN.
__device__ __forceinline__ float2 finish(float m, const RowSums& q) {
  if (m == INFINITY || q.s != q.s) return make_float2(NAN, NAN);
  if (m == -INFINITY) return make_float2(0.f, 0.f);
  const float t = q.s + (float)(q.eq - 1);
  const float l = log1pf(t);
  return make_float2(l, l - q.a / (1.f + t));
}

__device__ __forceinline__ uint64_t shfl_xor_u64(uint64_t v, int d) {
  const uint32_t lo = __shfl_xor((uint32_t)v, d, 64), hi = __shfl_xor((uint32_t)(v >> 32), d, 64);
  return (uint64_t)hi << 32 | lo;
}

// One wavefront per row, lanes over the classes; the best classes by one more
// pass over the row for each.
template <typename T>
__global__ __launch_bounds__(256) void k_scores(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                const int32_t* __restrict__ labels, int top_k,
                                                float* __restrict__ logprob, float* __restrict__ entropy,
                                                float* __restrict__ stats, int32_t* __restrict__ top_index,
                                                float* __restrict__ top_logprob) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < n; r += (int64_t)gridDim.x * 4) {
    const T* row = z + r * ldz;
    float m = -INFINITY;
    for (int k = lane; k < classes; k += 64) m = fmaxf(m, ld(row + k));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    const float base = m == -INFINITY ? 0.f : m;
    RowSums q{0.f, 0.f, 0};
    for (int k = lane; k < classes; k += 64) add_value(q, ld(row + k), m, base);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
      q.s += __shfl_xor(q.s, d, 64);
      q.a += __shfl_xor(q.a, d, 64);
      q.eq += __shfl_xor(q.eq, d, 64);
    }
    const float2 lh = finish(m, q);
    uint64_t last = ~0ull;
    for (int j = 0; j < top_k; ++j) {
      uint64_t best = 0;
      for (int k = lane; k < classes; k += 64) {
        const uint64_t key = rank_key(ld(row + k), (uint32_t)k);
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int d = 32; d >= 1; d >>= 1) best = max(best, shfl_xor_u64(best, d));
      last = best;
      if (lane == 0) {
        const uint32_t k = key_class(best);
        top_index[r * top_k + j] = (int32_t)k;
        top_logprob[r * top_k + j] = (ld(row + k) - base) - lh.x;
      }
    }
    if (lane == 0) {
      if (logprob) {
        const int lab = labels[r];
        logprob[r] = lab < 0 ? 0.f : lab >= classes ? NAN : (ld(row + lab) - base) - lh.x;
      }
      entropy[r] = lh.y;
      stats[2 * r] = m;
      stats[2 * r + 1] = lh.x;
    }
  }
}

// The gradient.  With A_k what class k receives directly (g = dlogprob where k
// is the label, dtop_j where k is the j-th best class) and G their sum,
//   dx_k = -A_k expm1(log p_k) - p_k ((G - A_k) + h (log p_k + H)),  h = dentropy,
// which is A_k - p_k (G + h (log p_k + H)) without that form's cancellation
// where p_k is close to 1.  One wavefront per row.
template <typename T>
__global__ __launch_bounds__(256) void k_scores_grad(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                     const int32_t* __restrict__ labels,
                                                     const float* __restrict__ stats,
                                                     const float* __restrict__ entropy, int top_k,
                                                     const int32_t* __restrict__ top_index,
                                                     const float* __restrict__ dlogprob,
                                                     const float* __restrict__ dentropy,
                                                     const float* __restrict__ dtop, T* __restrict__ dz,
                                                     int64_t ldd) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < n; r += (int64_t)gridDim.x * 4) {
    const T* row = z + r * ldz;
    const float m = stats[2 * r], L = stats[2 * r + 1];
    const bool empty = m == -INFINITY && L == 0.f;
    const float h = dentropy ? dentropy[r] : 0.f, H = dentropy ? entropy[r] : 0.f;
    const int lab = dlogprob ? labels[r] : -1;
    const float g = lab < 0 ? 0.f : lab >= classes ? NAN : dlogprob[r];
    float G = g;
    if (dtop)
      for (int j = 0; j < top_k; ++j) G += dtop[r * top_k + j];
    for (int k = lane; k < classes; k += 64) {
      float A = k == lab ? g : 0.f;
      if (dtop)
        for (int j = 0; j < top_k; ++j) A += top_index[r * top_k + j] == k ? dtop[r * top_k + j] : 0.f;
      const float lp = (ld(row + k) - m) - L;
      const float p = expf(lp);
      const float v = -A * expm1f(lp) - p * ((G - A) + (p == 0.f ? 0.f : h * (lp + H)));
      st(dz + r * ldd + k, empty ? 0.f : v);
    }
  }
}

sscn_status check_rows(const void* p, int64_t ld, int64_t n, int classes, sscn_dtype dtype) {
  if (dtype != SSCN_F32 && dtype != SSCN_BF16) return fail(SSCN_ERR_INVALID_ARG, "unknown dtype");
  if (n < 0 || classes < 1) return fail(SSCN_ERR_INVALID_ARG, "scores: n must be >= 0 and classes >= 1");
  if (n > 0 && !p) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL logits or dlogits");
  if (ld < classes) return fail(SSCN_ERR_INVALID_ARG, "scores: row stride below the number of classes");
  if (reinterpret_cast<uintptr_t>(p) % (dtype == SSCN_F32 ? 4 : 2) != 0)
    return fail(SSCN_ERR_INVALID_ARG, "scores: logits or dlogits not aligned to their elements");
  return SSCN_OK;
}
sscn_status check_top(int32_t top_k, int32_t classes) {
  if (top_k < 0 || top_k > std::min<int32_t>(kMaxTop, classes))
    return fail(SSCN_ERR_INVALID_ARG, "scores: top_k must be in [0, min(16, classes)]");
  return SSCN_OK;
}

unsigned wave_grid(int64_t n) { return (unsigned)std::min<int64_t>(ceil_div(n, 4), 1 << 20); }

}  // namespace
}  // namespace sscn

using namespace sscn;

extern "C" sscn_status sscn_label_scores_workspace(int64_t n, int32_t classes, int32_t top_k, int64_t* bytes) {
  if (n < 0 || classes < 1) return fail(SSCN_ERR_INVALID_ARG, "scores: n must be >= 0 and classes >= 1");
  SSCN_TRY(check_top(top_k, classes));
  if (!bytes) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL bytes");
  *bytes = 0;
  return SSCN_OK;
}

extern "C" sscn_status sscn_label_scores(const void* logits, int64_t ldz, int64_t n, int32_t classes,
                                         sscn_dtype dtype, const int32_t* labels, int32_t top_k, float* logprob,
                                         float* entropy, float* stats, int32_t* top_index, float* top_logprob,
                                         void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  SSCN_TRY(check_rows(logits, ldz, n, classes, dtype));
  SSCN_TRY(check_top(top_k, classes));
  if ((labels == nullptr) != (logprob == nullptr) && n > 0)
    return fail(SSCN_ERR_INVALID_ARG, "scores: labels and logprob go together");
  if (n > 0 && (!entropy || !stats)) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL entropy or stats");
  if (n > 0 && top_k > 0 && (!top_index || !top_logprob))
    return fail(SSCN_ERR_INVALID_ARG, "scores: NULL top_index or top_logprob");
  int64_t need = 0;
  SSCN_TRY(sscn_label_scores_workspace(n, classes, top_k, &need));
  if (workspace_bytes < need || (need > 0 && !workspace))
    return fail(SSCN_ERR_INVALID_ARG, "scores: workspace smaller than sscn_label_scores_workspace says");
  if (n == 0) return SSCN_OK;
  if (dtype == SSCN_F32)
    k_scores<float><<<wave_grid(n), 256, 0, stream>>>((const float*)logits, ldz, n, classes, labels, top_k, logprob,
                                                      entropy, stats, top_index, top_logprob);
  else
    k_scores<uint16_t><<<wave_grid(n), 256, 0, stream>>>((const uint16_t*)logits, ldz, n, classes, labels, top_k,
                                                         logprob, entropy, stats, top_index, top_logprob);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

extern "C" sscn_status sscn_label_scores_backward(const void* logits, int64_t ldz, int64_t n, int32_t classes,
                                                  sscn_dtype dtype, const int32_t* labels, const float* stats,
                                                  const float* entropy, int32_t top_k, const int32_t* top_index,
                                                  const float* dlogprob, const float* dentropy, const float* dtop,
                                                  void* dlogits, int64_t ldd, hipStream_t stream) {
  SSCN_TRY(check_rows(logits, ldz, n, classes, dtype));
  SSCN_TRY(check_rows(dlogits, ldd, n, classes, dtype));
  SSCN_TRY(check_top(top_k, classes));
  if (n == 0) return SSCN_OK;
  if (!stats) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL stats");
  if (dlogprob && !labels) return fail(SSCN_ERR_INVALID_ARG, "scores: dlogprob without labels");
  if (dentropy && !entropy) return fail(SSCN_ERR_INVALID_ARG, "scores: dentropy without entropy");
  if (dtop && (top_k == 0 || !top_index)) return fail(SSCN_ERR_INVALID_ARG, "scores: dtop without top_index");
  if (dtype == SSCN_F32)
    k_scores_grad<float><<<wave_grid(n), 256, 0, stream>>>((const float*)logits, ldz, n, classes, labels, stats,
                                                           entropy, top_k, top_index, dlogprob, dentropy, dtop,
                                                           (float*)dlogits, ldd);
  else
    k_scores_grad<uint16_t><<<wave_grid(n), 256, 0, stream>>>((const uint16_t*)logits, ldz, n, classes, labels,
                                                              stats, entropy, top_k, top_index, dlogprob, dentropy,
                                                              dtop, (uint16_t*)dlogits, ldd);
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}
