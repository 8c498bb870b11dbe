// Rotary positions (moe_rotary) and the append of rotated keys and of values to a paged cache (moe_kv_append).
//
// Pair i of a head's rot_dim/2 pairs turns by position[axis of i] * freqs[i].
#include "attention_internal.h"

namespace moesys {
namespace {

struct Rows {
  void* data;
  int64_t token_stride, head_stride;
};

struct RotaryArgs {
  const double* freqs;
  const int32_t* positions;  // [n_axes, T]
  int32_t T, D, R, first_of_axis1, first_of_axis2;  // pairs from which the second and the third axis count
  float sign;
};

template <typename X> __device__ __forceinline__ float load(const X* p);
template <> __device__ __forceinline__ float load<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load<uint16_t>(const uint16_t* p) { return bf16_to_float(*p); }
__device__ __forceinline__ void store(float* p, float v) { *p = v; }
__device__ __forceinline__ void store(uint16_t* p, float v) { *p = (uint16_t)float_to_bf16(v); }

// Element d of a rotated head.
template <typename X>
__device__ __forceinline__ float rotated(const RotaryArgs& a, const X* x, int t, int d, bool inter) {
  const int half = a.R / 2;
  if (d >= a.R) return load(x + d);
  const int i = inter ? d >> 1 : d < half ? d : d - half;
  const bool second = inter ? (d & 1) : d >= half;
  const int axis = (i >= a.first_of_axis1) + (i >= a.first_of_axis2);
  double turns = (double)a.positions[(size_t)axis * a.T + t] * a.freqs[i] * 0.15915494309189533577;
  turns -= rint(turns);
  float s, c;
  sincospif(2.0f * (float)turns, &s, &c);
  s *= a.sign;
  const float u = load(x + (inter ? 2 * i : i)), v = load(x + (inter ? 2 * i + 1 : i + half));
  return second ? u * s + v * c : u * c - v * s;
}

template <typename X>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, Rows x, Rows out, int heads, bool inter) {
  const int t = blockIdx.x / heads, h = blockIdx.x % heads, d = threadIdx.x;
  float v = 0.f;
  if (d < a.D) v = rotated(a, (const X*)x.data + t * x.token_stride + h * x.head_stride, t, d, inter);
  __syncthreads();  // (out may be x)
  if (d < a.D) store((X*)out.data + t * out.token_stride + h * out.head_stride + d, v);
}

struct CacheArgs {
  void *k, *v;
  const int32_t* table;
  const int32_t *token_seq, *cache_pos;
  int64_t n_pages, page_stride, token_stride, head_stride;
  int32_t page_size, n_seqs, table_width, heads;
};

template <typename X>
__global__ __launch_bounds__(256) void append_kernel(RotaryArgs a, CacheArgs c, Rows k, Rows v, Rows q, Rows q_out, int q_heads, bool rotate,
                                                     bool inter) {
  const int t = blockIdx.x / (2 * c.heads + q_heads), h = blockIdx.x % (2 * c.heads + q_heads), d = threadIdx.x;
  if (h >= 2 * c.heads) {
    const int hq = h - 2 * c.heads;
    float y = 0.f;
    if (d < a.D) y = rotated(a, (const X*)q.data + t * q.token_stride + hq * q.head_stride, t, d, inter);
    __syncthreads();
    if (d < a.D) store((X*)q_out.data + t * q_out.token_stride + hq * q_out.head_stride + d, y);
    return;
  }
  const int s = c.token_seq ? c.token_seq[t] : t, p = c.cache_pos[t];
  if (s < 0 || s >= c.n_seqs || p < 0 || p / c.page_size >= c.table_width || d >= a.D) return;
  const int page = valid_page(c.table[(int64_t)s * c.table_width + p / c.page_size], c.n_pages);
  if (page < 0) return;
  const int64_t at = page * c.page_stride + (p % c.page_size) * c.token_stride + d;
  if (h < c.heads) {
    const X* row = (const X*)k.data + t * k.token_stride + h * k.head_stride;
    store((X*)c.k + at + h * c.head_stride, rotate ? rotated(a, row, t, d, inter) : load(row + d));
  } else {
    const int hv = h - c.heads;
    ((X*)c.v)[at + hv * c.head_stride] = ((const X*)v.data)[t * v.token_stride + hv * v.head_stride + d];
  }
}

int32_t check_rotary(const moe_rotary_spec* r) {
  if (!r) return fail(MOE_ERR_INVALID_ARG, "rotary is NULL");
  if (r->head_dim < 2 || r->head_dim > MOE_MAX_HEAD_DIM)
    return fail(MOE_ERR_INVALID_ARG, "rotary.head_dim=%d outside 2..%d", r->head_dim, MOE_MAX_HEAD_DIM);
  if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2)
    return fail(MOE_ERR_INVALID_ARG, "rotary.rot_dim=%d must be even and in 2..head_dim=%d", r->rot_dim, r->head_dim);
  if (r->interleaved != 0 && r->interleaved != 1) return fail(MOE_ERR_INVALID_ARG, "rotary.interleaved=%d must be 0 or 1", r->interleaved);
  if (r->n_axes < 1 || r->n_axes > MOE_MAX_ROTARY_AXES)
    return fail(MOE_ERR_INVALID_ARG, "rotary.n_axes=%d outside 1..%d", r->n_axes, MOE_MAX_ROTARY_AXES);
  int64_t pairs = 0;
  for (int a = 0; a < r->n_axes; ++a) {
    if (r->axis_pairs[a] < 0) return fail(MOE_ERR_INVALID_ARG, "rotary.axis_pairs[%d]=%d is negative", a, r->axis_pairs[a]);
    pairs += r->axis_pairs[a];
  }
  if (pairs != r->rot_dim / 2) return fail(MOE_ERR_INVALID_ARG, "rotary.axis_pairs add up to %lld, rot_dim/2 is %d", (long long)pairs, r->rot_dim / 2);
  if (!r->freqs) return fail(MOE_ERR_INVALID_ARG, "rotary.freqs is NULL");
  return MOE_OK;
}

RotaryArgs rotary_args(const moe_rotary_spec* r, const int32_t* positions, int32_t T, int D, int inverse) {
  RotaryArgs a{};
  a.T = T;
  a.D = D;
  if (!r) return a;
  a.freqs = r->freqs;
  a.positions = positions;
  a.R = r->rot_dim;
  a.first_of_axis1 = r->n_axes > 1 ? r->axis_pairs[0] : r->rot_dim;
  a.first_of_axis2 = r->n_axes > 2 ? r->axis_pairs[0] + r->axis_pairs[1] : r->rot_dim;
  a.sign = inverse ? -1.f : 1.f;
  return a;
}

Rows rows_of(const moe_head_rows* r) { return r ? Rows{r->data, r->token_stride, r->head_stride} : Rows{nullptr, 0, 0}; }

}  // namespace
}  // namespace moesys

using namespace moesys;

extern "C" int32_t moe_rotary(const moe_rotary_spec* r, int32_t dtype, int32_t T, int32_t n_heads, const moe_head_rows* x,
                              const int32_t* positions, const moe_head_rows* out, int32_t inverse, void* stream) {
  int32_t st = check_rotary(r);
  if (st != MOE_OK) return st;
  if (dtype != MOE_F32 && dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "moe_rotary: dtype=%d unknown", dtype);
  if (T < 0 || n_heads < 1 || n_heads > MOE_MAX_HEADS)
    return fail(MOE_ERR_INVALID_ARG, "moe_rotary: T=%d must not be negative, n_heads=%d in 1..%d", T, n_heads, MOE_MAX_HEADS);
  if (inverse != 0 && inverse != 1) return fail(MOE_ERR_INVALID_ARG, "moe_rotary: inverse=%d must be 0 or 1", inverse);
  if (T == 0) return MOE_OK;
  if (!x || !x->data || !out || !out->data || !positions) return fail(MOE_ERR_INVALID_ARG, "moe_rotary: x, out and positions must be non-NULL");
  if (x->data == out->data && (x->token_stride != out->token_stride || x->head_stride != out->head_stride))
    return fail(MOE_ERR_INVALID_ARG, "moe_rotary: in place, out must have x's strides");
  const RotaryArgs a = rotary_args(r, positions, T, r->head_dim, inverse);
  dim3 grid(T * n_heads);
  if (dtype == MOE_BF16)
    hipLaunchKernelGGL(rotary_kernel<uint16_t>, grid, dim3(256), 0, (hipStream_t)stream, a, rows_of(x), rows_of(out), n_heads, r->interleaved != 0);
  else
    hipLaunchKernelGGL(rotary_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a, rows_of(x), rows_of(out), n_heads, r->interleaved != 0);
  return check_hip(hipGetLastError(), "rotary launch");
}

extern "C" int32_t moe_kv_cache_check(const moe_kv_cache* c) {
  if (!c) return fail(MOE_ERR_INVALID_ARG, "cache is NULL");
  if (c->dtype != MOE_F32 && c->dtype != MOE_BF16) return fail(MOE_ERR_INVALID_ARG, "cache.dtype=%d unknown", c->dtype);
  const int es = (int)elem_size(c->dtype);
  if (c->head_dim < 1 || c->head_dim > MOE_MAX_HEAD_DIM || (c->head_dim * es) % 16)
    return fail(MOE_ERR_INVALID_ARG, "cache.head_dim=%d must be a multiple of %d, at most %d", c->head_dim, 16 / es, MOE_MAX_HEAD_DIM);
  if (c->n_kv_heads < 1 || c->n_kv_heads > MOE_MAX_HEADS) return fail(MOE_ERR_INVALID_ARG, "cache.n_kv_heads=%d outside 1..%d", c->n_kv_heads, MOE_MAX_HEADS);
  if (c->page_size < 1) return fail(MOE_ERR_INVALID_ARG, "cache.page_size=%d must be at least 1", c->page_size);
  if (c->n_seqs < 0 || c->table_width < 0) return fail(MOE_ERR_INVALID_ARG, "cache.n_seqs=%d and table_width=%d must not be negative", c->n_seqs, c->table_width);
  if ((int64_t)c->table_width * c->page_size > INT32_MAX)
    return fail(MOE_ERR_INVALID_ARG, "cache: %lld places per sequence are more than 2^31 - 1", (long long)c->table_width * c->page_size);
  if (c->n_pages < 0 || c->n_pages > INT32_MAX) return fail(MOE_ERR_INVALID_ARG, "cache.n_pages=%lld outside 0..2^31 - 1", (long long)c->n_pages);
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return fail(MOE_ERR_INVALID_ARG, "cache: strides must not be negative");
  if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return fail(MOE_ERR_INVALID_ARG, "cache: k and v must be 16-byte aligned");
  if ((c->page_stride * es) % 16 || (c->token_stride * es) % 16 || (c->head_stride * es) % 16)
    return fail(MOE_ERR_INVALID_ARG, "cache: strides must be multiples of 16 bytes");
  if (c->n_pages > 0 && (!c->k || !c->v)) return fail(MOE_ERR_INVALID_ARG, "cache: k and v must be non-NULL");
  if (c->n_seqs > 0 && c->table_width > 0 && !c->page_table) return fail(MOE_ERR_INVALID_ARG, "cache: page_table is NULL");
  return MOE_OK;
}

extern "C" int32_t moe_kv_append(const moe_kv_cache* c, int32_t T, const moe_head_rows* k, const moe_head_rows* v,
                                 const int32_t* token_seq, const int32_t* cache_pos, const moe_rotary_spec* r,
                                 const int32_t* positions, int32_t n_q_heads, const moe_head_rows* q,
                                 const moe_head_rows* q_out, void* stream) {
  int32_t st = moe_kv_cache_check(c);
  if (st != MOE_OK) return st;
  if (r) {
    st = check_rotary(r);
    if (st != MOE_OK) return st;
    if (r->head_dim != c->head_dim) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: rotary.head_dim=%d, the cache has %d", r->head_dim, c->head_dim);
    if (!positions && r->n_axes != 1) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: %d axes need positions", r->n_axes);
  }
  if (T < 0) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: T=%d is negative", T);
  if (q && !r) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: q without rotary");
  if (q && (n_q_heads < 1 || n_q_heads > MOE_MAX_HEADS)) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: n_q_heads=%d outside 1..%d", n_q_heads, MOE_MAX_HEADS);
  if (T == 0) return MOE_OK;
  if (!k || !k->data || !v || !v->data || !cache_pos) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: k, v and cache_pos must be non-NULL");
  if (!token_seq && T > c->n_seqs) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: %d tokens, %d sequences and no token_seq", T, c->n_seqs);
  if (q && (!q->data || !q_out || !q_out->data)) return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: q and q_out must both be given");
  if (q && q->data == q_out->data && (q->token_stride != q_out->token_stride || q->head_stride != q_out->head_stride))
    return fail(MOE_ERR_INVALID_ARG, "moe_kv_append: in place, q_out must have q's strides");
  const RotaryArgs a = rotary_args(r, positions ? positions : cache_pos, T, c->head_dim, 0);
  const CacheArgs ca{c->k, c->v, c->page_table, token_seq, cache_pos, c->n_pages, c->page_stride, c->token_stride, c->head_stride,
                     c->page_size, c->n_seqs, c->table_width, c->n_kv_heads};
  const int hq = q ? n_q_heads : 0;
  dim3 grid(T * (2 * c->n_kv_heads + hq));
  const bool inter = r && r->interleaved;
  if (c->dtype == MOE_BF16)
    hipLaunchKernelGGL(append_kernel<uint16_t>, grid, dim3(256), 0, (hipStream_t)stream, a, ca, rows_of(k), rows_of(v), rows_of(q), rows_of(q_out), hq, r != nullptr, inter);
  else
    hipLaunchKernelGGL(append_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a, ca, rows_of(k), rows_of(v), rows_of(q), rows_of(q_out), hq, r != nullptr, inter);
  return check_hip(hipGetLastError(), "append launch");
}
