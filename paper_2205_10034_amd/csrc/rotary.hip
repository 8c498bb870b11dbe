// Rotary positions (moe_rotary) and the append of rotated keys and of values to a paged cache (moe_kv_append).
//
// Pair i of a head's rot_dim/2 pairs turns by position[axis of i] * freqs[i]; all heads of a token turn alike.  Bound: HBM, every
// element read and written once (many tokens), or the latency of one launch (few).  One wavefront per token, or several that
// share its heads when there are few tokens: its lanes compute one pair's cosine and sine each, in the shadow of the first
// loads of the rows, and pass them on through LDS; then every lane rotates vectors of 16 bytes (8 or single elements where strides,
// pointers or rot_dim do not allow it), two of them for the halves of a head.
// Measured: append of 16389 tokens with 32 query and 8 kv heads of 128 (403 MB read + written) 85 us, 4.75 TB/s, the rate of a large
// copy; 32768 x 32 heads of 128, half of each rotated, 103 us, 5.2 TB/s; 8192 x 16 heads of 64 on three axes 8.4 us; one token 3 us.
#include "attention_internal.h"

namespace moesys {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4;
constexpr int PAIRS = MOE_MAX_HEAD_DIM / 2;

struct Rows {
  char* data;
  int64_t token_stride, head_stride;  // bytes
};

// What a call does with a token: rows of queries, of keys and of values (moe_rotary has queries only), each head in `units` lanes'
// work.
struct TokenArgs {
  const double* freqs;
  const int32_t* positions;  // [n_axes, T]
  Rows q, q_out, k, v;
  char *cache_k, *cache_v;
  const int32_t *table, *token_seq, *cache_pos;
  int64_t n_pages, page_stride, token_stride, head_stride;  // bytes
  PageDivisor page, per_turned, per_copied;                 // page size, units of a rotated and of a copied head
  int32_t T, D, R, first_of_axis1, first_of_axis2;          // pairs from which the second and the third axis count
  int32_t hq, hkv, turned_units, copied_units, rotated_units, units, splits;
  int32_t page_size, n_seqs, table_width;
  float sign;
};

// A unit's elements: VW of them, loaded and stored as one vector of BYTES, or element by element (BYTES = 0; the first n).
template <typename X, int BYTES, int VW> struct Vector {
  float e[VW];
  __device__ __forceinline__ void load(const char* p, int n) {
    if constexpr (BYTES == 0) {
#pragma unroll
      for (int i = 0; i < VW; ++i) e[i] = i < n ? (float)reinterpret_cast<const X*>(p)[i] : 0.f;
    } else {
      uint32_t w[BYTES / 4];
      if constexpr (BYTES == 16) { const u32x4 v = *reinterpret_cast<const u32x4*>(p); w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3]; }
      else { const u32x2 v = *reinterpret_cast<const u32x2*>(p); w[0] = v[0]; w[1] = v[1]; }
#pragma unroll
      for (int i = 0; i < VW; ++i) {
        if constexpr (sizeof(X) == 2) e[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else e[i] = __uint_as_float(w[i]);
      }
    }
  }
  __device__ __forceinline__ void store(char* p, int n) const {
    if constexpr (BYTES == 0) {
#pragma unroll
      for (int i = 0; i < VW; ++i)
        if (i < n) reinterpret_cast<X*>(p)[i] = (X)e[i];
    } else {
      uint32_t w[BYTES / 4];
#pragma unroll
      for (int i = 0; i < BYTES / 4; ++i) {
        if constexpr (sizeof(X) == 2) { const bf16x2 v = {(__bf16)e[2 * i], (__bf16)e[2 * i + 1]}; w[i] = __builtin_bit_cast(uint32_t, v); }
        else w[i] = __float_as_uint(e[i]);
      }
      if constexpr (BYTES == 16) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
      else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
    }
  }
};

template <typename X, int BYTES, bool INTER>
__global__ __launch_bounds__(64 * WAVES) void token_kernel(TokenArgs a) {
  constexpr int VW = BYTES ? BYTES / (int)sizeof(X) : INTER ? 2 : 1, UNROLL = 4, ES = sizeof(X);
  __shared__ __attribute__((aligned(16))) float cosine[WAVES][PAIRS], sine[WAVES][PAIRS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned job = blockIdx.x * WAVES + wave;
  const int t = (int)(job / (unsigned)a.splits), part = (int)(job % (unsigned)a.splits);
  if (t >= a.T) return;

  // the token's rows in the cache (NULL: its place is not there)
  char *to_k = nullptr, *to_v = nullptr;
  if (a.hkv) {
    const int s = a.token_seq ? a.token_seq[t] : t, p = a.cache_pos[t];
    if (s >= 0 && s < a.n_seqs && p >= 0) {
      const int column = a.page.quotient(p);
      const int page = column < a.table_width ? valid_page(a.table[(int64_t)s * a.table_width + column], a.n_pages) : -1;
      if (page >= 0) {
        const int64_t at = page * a.page_stride + (int64_t)(p - column * a.page_size) * a.token_stride;
        to_k = a.cache_k + at;
        to_v = a.cache_v + at;
      }
    }
  }

  const int q_end = a.hq * a.turned_units, k_end = q_end + a.hkv * a.turned_units, half = a.R / 2;
  bool first = true;
  for (int at = part * 64; at < a.units; at += a.splits * 64 * UNROLL) {
    Vector<X, BYTES, VW> lo[UNROLL], hi[UNROLL];
    char* to[UNROLL];
    int pair[UNROLL], n[UNROLL];  // first pair of a unit, -1: nothing turns; its elements (an odd last one may be alone)
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int unit = at + u * a.splits * 64 + lane;
      to[u] = nullptr;
      pair[u] = -1;
      if (unit >= a.units) continue;
      const bool is_q = unit < q_end, is_v = unit >= k_end;
      const int i = is_q ? unit : is_v ? unit - k_end : unit - q_end;
      const int head = (is_v ? a.per_copied : a.per_turned).quotient(i), j = i - head * (is_v ? a.copied_units : a.turned_units);
      const char* from = is_q ? a.q.data + t * a.q.token_stride + head * a.q.head_stride
                         : is_v ? a.v.data + t * a.v.token_stride + head * a.v.head_stride
                                : a.k.data + t * a.k.token_stride + head * a.k.head_stride;
      char* row = is_q ? a.q_out.data + t * a.q_out.token_stride + head * a.q_out.head_stride : is_v ? to_v : to_k;
      if (!row) continue;
      if (!is_q) row += head * a.head_stride;
      const bool turns = !is_v && j < a.rotated_units;
      const int e = turns || is_v ? j * VW : a.R + (j - a.rotated_units) * VW;
      to[u] = row + e * ES;
      n[u] = a.D - e;
      lo[u].load(from + e * ES, n[u]);
      if (turns) {
        pair[u] = INTER ? e / 2 : e;
        if (!INTER) hi[u].load(from + (e + half) * ES, n[u]);
      }
    }
    if (first) {
      first = false;
      for (int i = lane; i < half; i += 64) {
        const int axis = (i >= a.first_of_axis1) + (i >= a.first_of_axis2);
        // in float64, reduced to one turn: in float32 the angle of position 10^6 would be off by 0.06
        double turns = (double)a.positions[(int64_t)axis * a.T + t] * a.freqs[i] * 0.15915494309189533577;
        turns -= rint(turns);
        // Cosine and sine themselves in float32, as the rotation is: float32 results are off by 4.1e-8 of their size, and by 3.7e-8 with
        // both taken in float64, which costs 8192 tokens' rotation 2 % (9.0 us and 8.8).
        const float near = (float)turns, off = 6.2831853f * (float)(turns - near);  // what rounding to float32 took, in radians
        float s, c;
        sincospif(2.0f * near, &s, &c);
        cosine[wave][i] = c - s * off;
        sine[wave][i] = a.sign * (s + c * off);
      }
      asm volatile("" ::: "memory");  // (a wavefront's LDS operations execute in order)
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      if (!to[u]) continue;
      if (pair[u] >= 0) {
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < VW / 2; ++i) {
            const float c = cosine[wave][pair[u] + i], s = sine[wave][pair[u] + i], x = lo[u].e[2 * i], y = lo[u].e[2 * i + 1];
            lo[u].e[2 * i] = x * c - y * s;
            lo[u].e[2 * i + 1] = x * s + y * c;
          }
        } else {
#pragma unroll
          for (int i = 0; i < VW; ++i) {
            const float c = cosine[wave][pair[u] + i], s = sine[wave][pair[u] + i], x = lo[u].e[i], y = hi[u].e[i];
            lo[u].e[i] = x * c - y * s;
            hi[u].e[i] = x * s + y * c;
          }
          hi[u].store(to[u] + half * ES, n[u]);
        }
      }
      lo[u].store(to[u], n[u]);
    }
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

// Wavefronts that few tokens' heads are dealt out to (16 for each CU): one token's 48 heads 3 us, and many tokens have one each.
constexpr int64_t ENOUGH_WAVES = 4096;

Rows rows_of(const moe_head_rows* r, int64_t es) { return r ? Rows{(char*)r->data, r->token_stride * es, r->head_stride * es} : Rows{nullptr, 0, 0}; }

template <typename X, int BYTES>
void launch_of(const TokenArgs& a, unsigned grid, bool interleaved, hipStream_t s) {
  if (interleaved) hipLaunchKernelGGL((token_kernel<X, BYTES, true>), dim3(grid), dim3(64 * WAVES), 0, s, a);
  else hipLaunchKernelGGL((token_kernel<X, BYTES, false>), dim3(grid), dim3(64 * WAVES), 0, s, a);
}

// a: everything but what follows from the vectors that pointers, strides and rot_dim allow.
int32_t launch_tokens(TokenArgs& a, const moe_rotary_spec* r, int32_t dtype, hipStream_t s) {
  const bool interleaved = r && r->interleaved;
  if (r) {
    a.freqs = r->freqs;
    a.R = r->rot_dim;
    a.first_of_axis1 = r->n_axes > 1 ? r->axis_pairs[0] : r->rot_dim;
    a.first_of_axis2 = r->n_axes > 2 ? r->axis_pairs[0] + r->axis_pairs[1] : r->rot_dim;
  }
  const int es = (int)elem_size(dtype);
  // the lowest bit set in any offset between vectors, in bytes
  uintptr_t bits = 16 | (uintptr_t)(a.D * es) | (uintptr_t)((interleaved ? a.R : a.R / 2) * es);
  for (const Rows* x : {&a.q, &a.q_out, &a.k, &a.v}) bits |= (uintptr_t)x->data | (uintptr_t)x->token_stride | (uintptr_t)x->head_stride;
  const int bytes = bits & 7 ? 0 : bits & 8 ? 8 : 16, vw = bytes ? bytes / es : interleaved ? 2 : 1;
  a.rotated_units = (interleaved ? a.R : a.R / 2) / vw;
  a.turned_units = a.rotated_units + (a.D - a.R + vw - 1) / vw;
  a.copied_units = (a.D + vw - 1) / vw;
  a.per_turned = page_divisor(a.turned_units);
  a.per_copied = page_divisor(a.copied_units);
  a.units = (a.hq + a.hkv) * a.turned_units + a.hkv * a.copied_units;
  const int64_t trips = (a.units + 63) / 64, wanted = (ENOUGH_WAVES + a.T - 1) / a.T;
  a.splits = (int)(wanted < trips ? wanted : trips);
  const int64_t grid = ((int64_t)a.T * a.splits + WAVES - 1) / WAVES;
  if (!launchable(grid, 64 * WAVES)) return fail(MOE_ERR_UNSUPPORTED, "%d tokens are too many for one call", a.T);
  if (dtype == MOE_BF16) {
    if (bytes == 16) launch_of<__bf16, 16>(a, (unsigned)grid, interleaved, s);
    else if (bytes == 8) launch_of<__bf16, 8>(a, (unsigned)grid, interleaved, s);
    else launch_of<__bf16, 0>(a, (unsigned)grid, interleaved, s);
  } else {
    if (bytes == 16) launch_of<float, 16>(a, (unsigned)grid, interleaved, s);
    else if (bytes == 8) launch_of<float, 8>(a, (unsigned)grid, interleaved, s);
    else launch_of<float, 0>(a, (unsigned)grid, interleaved, s);
  }
  return check_hip(hipGetLastError(), "rotary launch");
}

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
  TokenArgs a{};
  const int64_t es = (int64_t)elem_size(dtype);
  a.positions = positions;
  a.q = rows_of(x, es);
  a.q_out = rows_of(out, es);
  a.T = T;
  a.D = r->head_dim;
  a.hq = n_heads;
  a.sign = inverse ? -1.f : 1.f;
  return launch_tokens(a, r, dtype, (hipStream_t)stream);
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
  TokenArgs a{};
  const int64_t es = (int64_t)elem_size(c->dtype);
  a.positions = positions ? positions : cache_pos;
  a.q = rows_of(q, es);
  a.q_out = rows_of(q ? q_out : nullptr, es);
  a.k = rows_of(k, es);
  a.v = rows_of(v, es);
  a.cache_k = (char*)c->k;
  a.cache_v = (char*)c->v;
  a.table = c->page_table;
  a.token_seq = token_seq;
  a.cache_pos = cache_pos;
  a.n_pages = c->n_pages;
  a.page_stride = c->page_stride * es;
  a.token_stride = c->token_stride * es;
  a.head_stride = c->head_stride * es;
  a.page = page_divisor(c->page_size);
  a.page_size = c->page_size;
  a.n_seqs = c->n_seqs;
  a.table_width = c->table_width;
  a.T = T;
  a.D = c->head_dim;
  a.hq = q ? n_q_heads : 0;
  a.hkv = c->n_kv_heads;
  a.sign = 1.f;
  return launch_tokens(a, r, c->dtype, (hipStream_t)stream);
}
