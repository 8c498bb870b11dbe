// Attention of one new token per sequence over a paged cache (moe_attention_decode): one pass over the keys and values
// with the running maximum m and sum l of the softmax,
//   m' = max(m, z_j);  l' = l exp(m - m') + exp(z_j - m');  o' = o exp(m - m') + exp(z_j - m') v_j;  out = o / l.
// One wavefront per query head.
#include "attention_internal.h"

namespace moesys {
namespace {

struct DecodeArgs {
  const void *k, *v, *q;
  void* out;
  float* lse;
  const int32_t *table, *lens;
  const float* slopes;
  int64_t n_pages, page_stride, token_stride, head_stride, q_token, q_head, o_token, o_head;
  int32_t page_size, table_width, hq, hkv, D, window;
  float scale, cap;
};

template <typename X> __device__ __forceinline__ float load(const X* p);
template <> __device__ __forceinline__ float load<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load<uint16_t>(const uint16_t* p) { return bf16_to_float(*p); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(uint16_t* p, float v) { *p = (uint16_t)float_to_bf16(v); }

template <typename X>
__global__ __launch_bounds__(64) void decode_kernel(DecodeArgs a) {
  const int b = blockIdx.x, h = blockIdx.y, hk = h / (a.hq / a.hkv), lane = threadIdx.x;
  const int n = kept_length(a.lens[b], a.table_width * a.page_size);
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int i = 0; i < 4; ++i) q[i] = lane + 64 * i < a.D ? load((const X*)a.q + b * a.q_token + h * a.q_head + lane + 64 * i) : 0.f;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  for (int j = first_place(n, a.window); j < n; ++j) {
    const int page = valid_page(a.table[(int64_t)b * a.table_width + j / a.page_size], a.n_pages);
    if (page < 0) continue;
    const int64_t at = page * a.page_stride + (j % a.page_size) * a.token_stride + hk * a.head_stride;
    float z = 0.f;
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.D) z = fmaf(q[i], load((const X*)a.k + at + lane + 64 * i), z);
    for (int s = 32; s; s >>= 1) z += __shfl_xor(z, s, 64);
    z *= a.scale;
    if (a.cap > 0.f) z = a.cap * tanhf(z / a.cap);
    z -= slope * (float)(n - 1 - j);
    const float top = fmaxf(m, z);
    if (top == -INFINITY) continue;
    const float w = expf(z - top), old = expf(m - top);
    m = top;
    l = l * old + w;
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.D) o[i] = o[i] * old + w * load((const X*)a.v + at + lane + 64 * i);
  }
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < a.D) store((X*)a.out + b * a.o_token + h * a.o_head + lane + 64 * i, l > 0.f ? o[i] / l : l == 0.f ? 0.f : l);
  if (a.lse && lane == 0) a.lse[(int64_t)b * a.hq + h] = logf(l) + m;
}

}  // namespace
}  // namespace moesys

using namespace moesys;

extern "C" size_t moe_attention_decode_workspace_bytes(const moe_kv_cache* c, int32_t n_q_heads) {
  if (moe_kv_cache_check(c) != MOE_OK) return 0;
  if (n_q_heads < 1 || n_q_heads > MOE_MAX_HEADS || n_q_heads % c->n_kv_heads) {
    fail(MOE_ERR_INVALID_ARG, "n_q_heads=%d must be a multiple of n_kv_heads=%d in 1..%d", n_q_heads, c->n_kv_heads, MOE_MAX_HEADS);
    return 0;
  }
  return 256;
}

extern "C" int32_t moe_attention_decode(const moe_kv_cache* c, int32_t n_q_heads, const moe_head_rows* q, const int32_t* seq_lens,
                                        const moe_attention_options* opt, const moe_head_rows* out, float* lse, void* ws,
                                        size_t ws_bytes, void* stream) {
  int32_t st = moe_kv_cache_check(c);
  if (st != MOE_OK) return st;
  const size_t need = moe_attention_decode_workspace_bytes(c, n_q_heads);
  if (need == 0) return MOE_ERR_INVALID_ARG;
  if (!opt) return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: options are NULL");
  if (!__builtin_isfinite(opt->scale)) return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: scale is not finite");
  if (!__builtin_isfinite(opt->softcap) || opt->softcap < 0.f) return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: softcap must be finite and not negative");
  if (opt->window < 0) return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: window=%d is negative", opt->window);
  if (c->n_seqs == 0) return MOE_OK;
  if (!q || !q->data || !out || !out->data || !seq_lens) return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: q, out and seq_lens must be non-NULL");
  const size_t es = elem_size(c->dtype);
  if (!rows_aligned(q, es) || !rows_aligned(out, es))
    return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: pointers and strides of q and out must be multiples of 16 bytes");
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_attention_decode: workspace NULL, misaligned or smaller than %zu bytes", need);
  const DecodeArgs a{c->k, c->v, q->data, out->data, lse, c->page_table, seq_lens, opt->slopes, c->n_pages, c->page_stride, c->token_stride,
                     c->head_stride, q->token_stride, q->head_stride, out->token_stride, out->head_stride, c->page_size, c->table_width,
                     n_q_heads, c->n_kv_heads, c->head_dim, opt->window, opt->scale, opt->softcap};
  dim3 grid(c->n_seqs, n_q_heads);
  if (c->dtype == MOE_BF16)
    hipLaunchKernelGGL(decode_kernel<uint16_t>, grid, dim3(64), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(decode_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "attention launch");
}
