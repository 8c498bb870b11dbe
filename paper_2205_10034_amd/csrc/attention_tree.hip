// Attention of several new tokens per sequence over a paged cache (moe_attention_tree): as for one token,
//   out = sum_j exp(z_j - m) v_j / sum_j exp(z_j - m),  m = max z_j,
// over the places that the token sees: the cache, and of the new tokens those of its word.
#include "attention_internal.h"
#include "draft_tokens.h"
#include "wave_util.h"
#include <float.h>
#include <math.h>

namespace moesys {
namespace {

struct TreeArgs {
  const char *k, *v, *q;
  char* out;
  float* lse;
  const int32_t *table, *lens, *first;
  const uint64_t* words;
  const float* slopes;
  int64_t n_pages, page_stride, token_stride, head_stride, q_token, q_head, o_token, o_head;  // bytes
  PageDivisor page;
  int32_t page_size, table_width, capacity, n_seqs, hq, G, T, max_new, D, window, sinks;
  float scale, cap, inv_cap;
};

template <typename X>
__device__ __forceinline__ float value(const char* p, int d) { return (float)reinterpret_cast<const X*>(p)[d]; }

// A wavefront per token and query head, a place per lane.
template <typename X>
__global__ __launch_bounds__(64) void tree_kernel(TreeArgs a) {
  const int lane = threadIdx.x, t = blockIdx.x / a.hq, h = blockIdx.x % a.hq, hk = h / a.G;
  for (int s = 0; s < a.n_seqs; ++s) {
    const Drafts d = drafts_of(a.first[s], a.first[s + 1], a.T, a.max_new, a.lens[s], a.capacity);
    const int i = t - d.first;
    if (i < 0 || i >= d.n) continue;
    auto sees = [&](int j) { return seen_drafts(a.words, a.words ? a.words[d.first + j] : 0, j, d.n); };
    const uint64_t seen = sees(i);
    const int pos = d.base + draft_depth(seen, i);
    const char* q = a.q + (int64_t)t * a.q_token + (int64_t)h * a.q_head;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < d.len; p0 += 64) {
      const int p = p0 + lane;
      int page = -1, row = 0, pos_p = p;
      bool keep = p < d.len;
      if (keep) {
        const int column = a.page.quotient(p);
        row = p - column * a.page_size;
        page = valid_page(a.table[(int64_t)s * a.table_width + column], a.n_pages);
        if (p >= d.base) {
          const int j = p - d.base;
          keep = (seen >> j) & 1;
          pos_p = d.base + draft_depth(sees(j), j);
        }
        keep = keep && page >= 0 && in_window(pos, pos_p, p, a.window, a.sinks);
      }
      const int64_t at = keep ? (int64_t)page * a.page_stride + (int64_t)row * a.token_stride + (int64_t)hk * a.head_stride : 0;
      float z = -INFINITY;
      if (keep) {
        z = 0.f;
        for (int e = 0; e < a.D; ++e) z += value<X>(q, e) * value<X>(a.k + at, e);
        z *= a.scale;
        if (a.cap > 0.f) z = a.cap * tanhf(z * a.inv_cap);
        if (a.slopes) z -= a.slopes[h] * (float)(pos - pos_p);
      }
      float top = z;
      for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
      if (!__any(keep)) continue;
      const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.f : now, f = m == -INFINITY ? 0.f : expf(m - ref);
      const float w = keep ? expf(z - ref) : 0.f;
      m = now;
      float sum = w;
      for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x, 64);
      l = l * f + sum;
      for (int e = 0; e < 4; ++e) o[e] *= f;
      for (int j = 0; j < 64; ++j) {
        if (!__shfl((int)keep, j, 64)) continue;
        const float wj = __shfl(w, j, 64);
        const int64_t aj = ((int64_t)__shfl((int)(at >> 32), j, 64) << 32) | (uint32_t)__shfl((int)at, j, 64);
        for (int e = 0; e < 4; ++e)
          if (lane + 64 * e < a.D) o[e] += wj * value<X>(a.v + aj, lane + 64 * e);
      }
    }
    char* out = a.out + (int64_t)t * a.o_token + (int64_t)h * a.o_head;
    for (int e = 0; e < 4; ++e)
      if (lane + 64 * e < a.D) reinterpret_cast<X*>(out)[lane + 64 * e] = (X)(l == 0.f ? 0.f : o[e] / l);
    if (a.lse && lane == 0) a.lse[(int64_t)t * a.hq + h] = l == 0.f ? -INFINITY : m + logf(l);
    return;
  }
}

}  // namespace
}  // namespace moesys

using namespace moesys;

extern "C" size_t moe_attention_tree_workspace_bytes(const moe_kv_cache* c, int32_t n_q_heads, int32_t max_new) {
  if (moe_kv_cache_check(c) != MOE_OK) return 0;
  if (n_q_heads < 1 || n_q_heads > MOE_MAX_HEADS || n_q_heads % c->n_kv_heads) {
    fail(MOE_ERR_INVALID_ARG, "n_q_heads=%d must be a multiple of n_kv_heads=%d in 1..%d", n_q_heads, c->n_kv_heads, MOE_MAX_HEADS);
    return 0;
  }
  if (max_new < 1 || max_new > MOE_MAX_DRAFTS) {
    fail(MOE_ERR_INVALID_ARG, "max_new=%d outside 1..%d", max_new, MOE_MAX_DRAFTS);
    return 0;
  }
  return 256;
}

extern "C" int32_t moe_attention_tree(const moe_kv_cache* c, int32_t n_q_heads, int32_t T, int32_t max_new, const moe_head_rows* q,
                                      const int32_t* token_first, const int32_t* seq_lens, const uint64_t* visible,
                                      const moe_tree_options* opt, const moe_head_rows* out, float* lse, void* ws, size_t ws_bytes,
                                      void* stream) {
  int32_t st = moe_kv_cache_check(c);
  if (st != MOE_OK) return st;
  const size_t need = moe_attention_tree_workspace_bytes(c, n_q_heads, max_new);
  if (need == 0) return MOE_ERR_INVALID_ARG;
  if (T < 0) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: T=%d is negative", T);
  if (!opt) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: options are NULL");
  if (!__builtin_isfinite(opt->scale)) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: scale is not finite");
  if (!__builtin_isfinite(opt->softcap) || opt->softcap < 0.f) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: softcap must be finite and not negative");
  if (opt->window < 0 || opt->sinks < 0) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: window=%d and sinks=%d must not be negative", opt->window, opt->sinks);
  if (c->n_seqs == 0 || T == 0) return MOE_OK;
  if (!q || !q->data || !out || !out->data || !token_first || !seq_lens)
    return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: q, out, token_first and seq_lens must be non-NULL");
  if (q->data == out->data) return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: out must not be q");
  const int64_t es = (int64_t)elem_size(c->dtype);
  if (!rows_aligned(q, es) || !rows_aligned(out, es))
    return fail(MOE_ERR_INVALID_ARG, "moe_attention_tree: pointers and strides of q and out must be multiples of 16 bytes");
  if ((int64_t)T * n_q_heads > (1 << 26) - 4) return fail(MOE_ERR_UNSUPPORTED, "moe_attention_tree: %d tokens of %d query heads are too many for one call", T, n_q_heads);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_attention_tree: workspace NULL, misaligned or smaller than %zu bytes", need);
  TreeArgs a{};
  a.k = (const char*)c->k;
  a.v = (const char*)c->v;
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.lse = lse;
  a.table = c->page_table;
  a.lens = seq_lens;
  a.first = token_first;
  a.words = visible;
  a.slopes = opt->slopes;
  a.n_pages = c->n_pages;
  a.page_stride = c->page_stride * es;
  a.token_stride = c->token_stride * es;
  a.head_stride = c->head_stride * es;
  a.q_token = q->token_stride * es;
  a.q_head = q->head_stride * es;
  a.o_token = out->token_stride * es;
  a.o_head = out->head_stride * es;
  a.page = page_divisor(c->page_size);
  a.page_size = c->page_size;
  a.table_width = c->table_width;
  a.capacity = c->table_width * c->page_size;
  a.n_seqs = c->n_seqs;
  a.hq = n_q_heads;
  a.G = n_q_heads / c->n_kv_heads;
  a.T = T;
  a.max_new = max_new;
  a.D = c->head_dim;
  a.window = opt->window;
  a.sinks = opt->sinks;
  a.scale = opt->scale;
  a.cap = opt->softcap;
  // (finite for the smallest caps too: a score of 0 stays 0)
  a.inv_cap = opt->softcap > 0.f ? fminf(1.f / opt->softcap, FLT_MAX) : 0.f;
  if (c->dtype == MOE_BF16) hipLaunchKernelGGL(tree_kernel<__bf16>, dim3(T * n_q_heads), dim3(64), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(tree_kernel<float>, dim3(T * n_q_heads), dim3(64), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "tree attention launch");
}
