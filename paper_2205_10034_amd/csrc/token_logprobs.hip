// Log-probabilities of given tokens, entropy and the largest logits of every row (moe_token_logprobs), and the gradient of the first
// two (moe_token_logprobs_backward).  With z = scale x, m = max z, d_j = z_j - m, s = sum exp(d_j):
//   lse = m + log s,  logp_j = d_j - log s,  entropy = log s - sum exp(d_j) d_j / s.
#include "moesys_internal.h"
#include "kv_pages.h"
#include "wave_util.h"
#include <math.h>

namespace moesys {
namespace {

struct RowArgs {
  const char* x;
  int64_t row_stride;  // bytes
  const int32_t* ids;
  float *logp, *lse, *entropy, *top_logp;
  int32_t* top_ids;
  int32_t T, V, K;
  float scale;
};

constexpr int THREADS = 256;

// Order of logits: by value, equal ones by falling index; NaN below all else, the two zeros equal.
__device__ __forceinline__ uint64_t order_of(float x, uint32_t j) {
  uint32_t u = __float_as_uint(x + 0.f);
  u = u >> 31 ? ~u : u | 0x80000000u;
  return ((uint64_t)(x != x ? 0u : u) << 32) | (uint32_t)~j;
}

template <typename F>
__device__ float over_rows(float v, F join) {
  __shared__ float red[THREADS / 64];
  for (int d = 32; d; d >>= 1) v = join(v, __shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
  for (int w = 1; w < THREADS / 64; ++w) v = join(v, red[w]);
  return v;
}

template <typename X>
__global__ __launch_bounds__(THREADS) void rows_kernel(RowArgs a) {
  __shared__ uint64_t best[THREADS];
  const int t = blockIdx.x;
  const X* x = reinterpret_cast<const X*>(a.x + t * a.row_stride);
  float m = -INFINITY;
  bool bad = false;
  for (int j = threadIdx.x; j < a.V; j += THREADS) {
    const float v = (float)x[j];
    bad |= v != v || v == INFINITY;
    m = fmaxf(m, v);
  }
  auto add = [](float p, float q) { return p + q; };
  m = over_rows(m, [](float p, float q) { return fmaxf(p, q); });
  const bool nan = over_rows(bad ? 1.f : 0.f, add) > 0.f, empty = m == -INFINITY;
  float s = 0.f, e = 0.f;
  for (int j = threadIdx.x; j < a.V; j += THREADS) {
    const float d = (empty ? 0.f : (float)x[j] - m) * a.scale, w = empty ? 0.f : expf(d);
    s += w;
    if (w > 0.f) e += w * d;
  }
  s = over_rows(s, add);
  e = over_rows(e, add);
  const float log_s = logf(s);
  auto logp_of = [&](float v) { return nan ? NAN : empty ? -INFINITY : (v - m) * a.scale - log_s; };
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[t] = nan ? NAN : empty ? -INFINITY : m * a.scale + log_s;
    if (a.logp) {
      const int id = a.ids[t];
      a.logp[t] = id >= 0 && id < a.V ? logp_of((float)x[id]) : 0.f;
    }
    if (a.entropy) a.entropy[t] = nan ? NAN : empty ? 0.f : log_s - e / s;
  }
  uint64_t last = ~0ull;
  for (int i = 0; i < a.K; ++i) {
    uint64_t mine = 0;
    for (int j = threadIdx.x; j < a.V; j += THREADS) {
      const uint64_t o = order_of((float)x[j], j);
      if (o < last && o > mine) mine = o;
    }
    __syncthreads();
    best[threadIdx.x] = mine;
    __syncthreads();
    for (int k = 0; k < THREADS; ++k) mine = best[k] > mine ? best[k] : mine;
    last = mine;
    if (threadIdx.x == 0) {
      const uint32_t j = ~(uint32_t)mine;
      a.top_ids[(int64_t)t * a.K + i] = (int)j;
      a.top_logp[(int64_t)t * a.K + i] = logp_of((float)x[j]);
    }
  }
}

struct GradArgs {
  const char* x;
  char* d_x;
  int64_t row_stride, d_row_stride;  // bytes
  const int32_t* ids;
  const float *lse, *d_logp, *entropy, *d_entropy, *d_lse;
  int32_t T, V;
  float scale;
};

template <typename X>
__global__ __launch_bounds__(THREADS) void gradient_kernel(GradArgs a) {
  const int t = blockIdx.x;
  const X* x = reinterpret_cast<const X*>(a.x + t * a.row_stride);
  X* y = reinterpret_cast<X*>(a.d_x + t * a.d_row_stride);
  const int id = a.ids ? a.ids[t] : -1;
  const float lse = a.lse[t], g = a.d_logp && id >= 0 && id < a.V ? a.d_logp[t] : 0.f, ge = a.d_entropy ? a.d_entropy[t] : 0.f, gl = a.d_lse ? a.d_lse[t] : 0.f;
  const bool zero = lse == -INFINITY || (g == 0.f && ge == 0.f && gl == 0.f);
  const float h = ge != 0.f ? a.entropy[t] : 0.f;
  for (int j = threadIdx.x; j < a.V; j += THREADS) {
    float d = 0.f;
    if (!zero) {
      const float lp = (float)x[j] * a.scale - lse, p = expf(lp);
      if (!(p == 0.f)) d = p * (gl - g - ge * (lp + h));
      if (j == id) d += g;
      d *= a.scale;
    }
    y[j] = (X)d;
  }
}

int32_t check_rows(int32_t dtype, int32_t T, int32_t V, float scale, const char* who) {
  if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "%s: dtype=%d unknown", who, dtype);
  if (T < 0 || V < 1) return fail(MOE_ERR_INVALID_ARG, "%s: T=%d must not be negative, V=%d at least 1", who, T, V);
  if (!(scale > 0.f) || !__builtin_isfinite(scale)) return fail(MOE_ERR_INVALID_ARG, "%s: scale must be finite and above 0", who);
  return MOE_OK;
}

}  // namespace
}  // namespace moesys

using namespace moesys;

extern "C" size_t moe_token_logprobs_workspace_bytes(int32_t T, int32_t V, int32_t K) {
  if (T < 0 || V < 1 || K < 0 || K > V || K > MOE_MAX_ALTERNATIVES) {
    fail(MOE_ERR_INVALID_ARG, "T=%d must not be negative, V=%d at least 1, K=%d in 0..min(V, %d)", T, V, K, MOE_MAX_ALTERNATIVES);
    return 0;
  }
  return 256;
}

extern "C" int32_t moe_token_logprobs(int32_t dtype, int32_t T, int32_t V, const void* x, int64_t row_stride, float scale,
                                      const int32_t* ids, float* logp, float* lse, float* entropy, int32_t K, int32_t* top_ids,
                                      float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  const int32_t st = check_rows(dtype, T, V, scale, "moe_token_logprobs");
  if (st != MOE_OK) return st;
  const size_t need = moe_token_logprobs_workspace_bytes(T, V, K);
  if (need == 0) return MOE_ERR_INVALID_ARG;
  const size_t es = elem_size(dtype);
  if (T == 0) return MOE_OK;
  if (!x || ((uintptr_t)x & (es - 1))) return fail(MOE_ERR_INVALID_ARG, "moe_token_logprobs: x is NULL or not aligned to its elements");
  if (row_stride < 0) return fail(MOE_ERR_INVALID_ARG, "moe_token_logprobs: row_stride is negative");
  if (logp && !ids) return fail(MOE_ERR_INVALID_ARG, "moe_token_logprobs: logp without ids");
  if (K > 0 && (!top_ids || !top_logp)) return fail(MOE_ERR_INVALID_ARG, "moe_token_logprobs: top_ids and top_logp must both be given");
  if (!launchable(T, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "moe_token_logprobs: %d rows are too many for one call", T);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_token_logprobs: workspace NULL, misaligned or smaller than %zu bytes", need);
  const RowArgs a{(const char*)x, row_stride * (int64_t)es, ids, logp, lse, entropy, top_logp, top_ids, T, V, K, scale};
  if (dtype == MOE_BF16) hipLaunchKernelGGL(rows_kernel<__bf16>, dim3(T), dim3(THREADS), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(rows_kernel<float>, dim3(T), dim3(THREADS), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "log-probabilities launch");
}

extern "C" int32_t moe_token_logprobs_backward(int32_t dtype, int32_t T, int32_t V, const void* x, int64_t row_stride, float scale,
                                               const int32_t* ids, const float* lse, const float* d_logp, const float* entropy,
                                               const float* d_entropy, const float* d_lse, void* d_x, int64_t d_row_stride,
                                               void* stream) {
  const char* who = "moe_token_logprobs_backward";
  const int32_t st = check_rows(dtype, T, V, scale, who);
  if (st != MOE_OK) return st;
  if (T == 0) return MOE_OK;
  const size_t es = elem_size(dtype);
  if (!x || ((uintptr_t)x & (es - 1)) || !d_x || ((uintptr_t)d_x & (es - 1)) || !lse)
    return fail(MOE_ERR_INVALID_ARG, "%s: x, d_x and lse must be non-NULL, matrices aligned to their elements", who);
  if (d_logp && !ids) return fail(MOE_ERR_INVALID_ARG, "%s: d_logp without ids", who);
  if (d_entropy && !entropy) return fail(MOE_ERR_INVALID_ARG, "%s: d_entropy without entropy", who);
  if (row_stride < 0 || (T > 1 && d_row_stride < V)) return fail(MOE_ERR_INVALID_ARG, "%s: rows of d_x overlap, or row_stride is negative", who);
  if (T > 1 && x == d_x && row_stride != d_row_stride) return fail(MOE_ERR_INVALID_ARG, "%s: in place, d_x must have x's stride", who);
  if (!launchable(T, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows are too many for one call", who, T);
  const GradArgs a{(const char*)x, (char*)d_x, row_stride * (int64_t)es, d_row_stride * (int64_t)es, ids, lse, d_logp, entropy, d_entropy, d_lse, T, V, scale};
  if (dtype == MOE_BF16) hipLaunchKernelGGL(gradient_kernel<__bf16>, dim3(T), dim3(THREADS), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(gradient_kernel<float>, dim3(T), dim3(THREADS), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "log-probabilities gradient launch");
}
