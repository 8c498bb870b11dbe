// Log-probabilities of given tokens, entropy and the largest logits of every row (moe_token_logprobs), and the gradient of the first
// two (moe_token_logprobs_backward).  With z = scale x, m a reference near max z, d_j = z_j - m, s = sum exp(d_j):
//   lse = m + log s,  logp_j = d_j - log s,  entropy = log s - sum exp(d_j) d_j / s,
// in one pass over the logits, lane by lane: s and the entropy's sum follow the lane's own reference, which moves only when a logit
// passes it by a factor of 2^8, and are brought to a common one at the end.  Bound: HBM, with the vector unit close behind.
#include "moesys_internal.h"
#include "kv_pages.h"
#include "wave_util.h"
#include <float.h>
#include <math.h>
#include <type_traits>

namespace moesys {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int PER_LANE = 16, CHUNK = 64 * PER_LANE;  // logits that a lane, a wavefront takes at a time
constexpr int LIST = 128;                            // candidates that a wavefront holds
constexpr int FOUND = 512;                           // groups with candidates that a row's workgroup holds
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LAG_BITS = 8.f;
// lse's rounding is 2^-24 |lse| of every p.  The gradient leaves it there up to 2^-14 of p in bfloat16 (which is rounded to 2^-9), 2^-18 in float32:
template <typename X> constexpr float far_lse = sizeof(X) == 2 ? 1024.f : 64.f;
// ... and, of 1 - p and log p of a token that is nearly certain, up to 2^-11 and 2^-17 of these (8: what s and the power carry, in the same units).
template <typename X> __device__ __forceinline__ float near_certain(float lse) { return (fabsf(lse) + 8.f) * (sizeof(X) == 2 ? 0x1p-13f : 0x1p-7f); }

// 16 bytes of logits at any alignment of their elements
template <typename X> struct __attribute__((packed, aligned(sizeof(X)))) Unaligned {
  u32x4 v;
};
template <typename X> constexpr int per_load = 16 / (int)sizeof(X);
template <typename X> constexpr int loads = PER_LANE / per_load<X>;

// A lane's logits of a chunk: load l holds the elements l*64*per_load + lane*per_load on.
template <typename X>
__device__ __forceinline__ int first_of(int l) { return (l * 64 + (threadIdx.x & 63)) * per_load<X>; }

template <typename X>
__device__ __forceinline__ void load_chunk(const X* x, u32x4 (&v)[loads<X>]) {
#pragma unroll
  for (int l = 0; l < loads<X>; ++l) v[l] = reinterpret_cast<const Unaligned<X>*>(x + first_of<X>(l))->v;
}

__device__ __forceinline__ float element(const __bf16*, const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16); }
__device__ __forceinline__ float element(const float*, const u32x4& v, int e) { return __uint_as_float(v[e]); }
// -infinity, as many as 16 bytes hold
template <typename X> constexpr uint32_t minus_infinities = sizeof(X) == 2 ? 0xff80ff80u : 0xff800000u;

// per_load elements from x[j] on, -infinity in the place of those that are not in 0..V-1
template <typename X>
__device__ __forceinline__ u32x4 load_some(const X* x, int64_t j, int V) {
  if (j >= 0 && j + per_load<X> <= V) return reinterpret_cast<const Unaligned<X>*>(x + j)->v;
  u32x4 v{minus_infinities<X>, minus_infinities<X>, minus_infinities<X>, minus_infinities<X>};
  if (j >= V) return v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (sizeof(X) == 2) {
      const int64_t k = j + 2 * w;
      if (k >= 0 && k < V) v[w] = (v[w] & 0xffff0000u) | reinterpret_cast<const uint16_t*>(x)[k];
      if (k + 1 >= 0 && k + 1 < V) v[w] = (v[w] & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t*>(x)[k + 1] << 16;
    } else if (j + w >= 0 && j + w < V) {
      v[w] = reinterpret_cast<const uint32_t*>(x)[j + w];
    }
  }
  return v;
}

// Order of logits as whole numbers: NaN below all else, the two zeros equal.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }
// ... and among equal ones by falling index
__device__ __forceinline__ uint64_t key_of(uint32_t order, int j) { return ((uint64_t)order << 32) | (uint32_t)~j; }

// What a lane, a wavefront or a part knows of a row: reference m (of x, not of z), s = sum 2^y, e = sum 2^y y, y = (x - m) c.
struct Stats {
  float m, s, e;
};
// The same about another reference.  (Sums that vanish, or are of nothing, add nothing; a NaN stays.)
template <bool ENTROPY>
__device__ __forceinline__ void refer(Stats& a, float m, float c) {
  const float y = (a.m - m) * c, f = a.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(y);
  if (ENTROPY) a.e = f == 0.f ? 0.f : f * (a.e + a.s * y);
  a.s *= f;
  a.m = m;
}

template <typename X, bool ENTROPY>
__device__ __forceinline__ float take_chunk(Stats& a, const u32x4 (&v)[loads<X>], float c, float lag) {
  const X* kind = nullptr;
  float top = element(kind, v[0], 0);
#pragma unroll
  for (int l = 0; l < loads<X>; ++l)
#pragma unroll
    for (int e = 0; e < per_load<X>; ++e) top = fmaxf(top, element(kind, v[l], e));
  if (__any(!(top <= a.m + lag))) {
    const float m = fmaxf(a.m, top);
    if (m != a.m) refer<ENTROPY>(a, m, c);
  }
  const float m = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
  for (int l = 0; l < loads<X>; ++l)
#pragma unroll
    for (int e = 0; e < per_load<X>; ++e) {
      const float y = (element(kind, v[l], e) - m) * c, w = __builtin_amdgcn_exp2f(y);
      a.s += w;
      if (ENTROPY) a.e += w * fmaxf(y, -200.f);  // (a weight of 0, whose logit may be -infinity, adds 0)
    }
  return top;
}

// Joins the wavefront's lanes.
template <bool ENTROPY>
__device__ __forceinline__ void join_lanes(Stats& a, float c) {
  float m = a.m;
#pragma unroll
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
  refer<ENTROPY>(a, m, c);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    a.s += __shfl_xor(a.s, d, 64);
    if (ENTROPY) a.e += __shfl_xor(a.e, d, 64);
  }
}

// What follows from a row's sums.
struct Row {
  float m, log_s, scale;
  bool nan, empty;
  __device__ __forceinline__ Row(const Stats& a, float scale) : m(a.m), log_s(logf(a.s)), scale(scale), nan(a.s != a.s || a.m == INFINITY), empty(a.m == -INFINITY) {}
  __device__ __forceinline__ float logp(float x) const { return nan ? NAN : empty ? -INFINITY : (x - m) * scale - log_s; }
  __device__ __forceinline__ float lse() const { return nan ? NAN : empty ? -INFINITY : m * scale + log_s; }
  __device__ __forceinline__ float entropy(const Stats& a) const { return nan ? NAN : empty ? 0.f : log_s - a.e * LN2 / a.s; }
};

struct RowArgs {
  const char* x;
  int64_t row_stride;  // bytes
  const int32_t* ids;
  float *logp, *lse, *entropy, *top_logp;
  int32_t* top_ids;
  f32x4* part_stats;   // [row][part]: m, s, e
  char* groups;       // [row][chunk][lane]: the largest of a lane's PER_LANE logits (Group)
  int32_t T, V, K, parts, part_chunks, max_chunks;
  float scale, c, lag;
};

// ---- the K largest -------------------------------------------------------------------------------------

// Keys of one wavefront, in LDS, that were above `bound` when they came.
struct TopList {
  uint64_t* keys;  // [LIST]
  int n, K;
  uint64_t bound;

  // The K largest, in falling order; from then on only larger ones come in.
  __device__ __forceinline__ void sort() {
    const int lane = threadIdx.x & 63;
    const uint64_t a = lane < n ? keys[lane] : 0, b = lane + 64 < n ? keys[lane + 64] : 0;
    if (lane < 8 && n + lane < LIST) keys[n + lane] = 0;  // (above none)
    asm volatile("" ::: "memory");                        // (a wavefront's LDS operations execute in order)
    int ra = 0, rb = 0;
    for (int i = 0; i < n; i += 8) {
      uint64_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = keys[i + e];
#pragma unroll
      for (int e = 0; e < 8; ++e) ra += k[e] > a;
      if (n > 64)
#pragma unroll
        for (int e = 0; e < 8; ++e) rb += k[e] > b;
    }
    asm volatile("" ::: "memory");
    if (lane < n && ra < K) keys[ra] = a;
    if (lane + 64 < n && rb < K) keys[rb] = b;
    asm volatile("" ::: "memory");
    if (n >= K) {
      n = K;
      bound = keys[K - 1];
      bound = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(bound >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bound);
    }
  }
};

// A value that K of the lanes' (N each, 0: no value) reach: the K-th largest, cut down to the upper BITS bits; 0 where there are fewer.
template <int BITS, int N>
__device__ __forceinline__ uint32_t reached_by(const uint32_t (&u)[N], int K) {
  uint32_t t = 0;
#pragma unroll
  for (int bit = 31; bit >= 32 - BITS; --bit) {
    const uint32_t more = t | 1u << bit;
    int n = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) n += __popcll(__ballot(u[e] >= more));
    t = n >= K ? more : t;
  }
  return t;
}

// The largest logit of a lane's PER_LANE, as it is kept: a bfloat16's order is told by its upper half.
template <typename X> struct Group;
template <> struct Group<__bf16> {
  typedef uint16_t type;
  static constexpr int BITS = 16;  // of an order that tell groups apart
  static __device__ __forceinline__ uint16_t pack(uint32_t order) { return (uint16_t)(order >> 16); }
  static __device__ __forceinline__ uint32_t order(uint16_t g) { return (uint32_t)g << 16 | (g & 0x8000u ? 0u : 0xffffu); }
  static __device__ __forceinline__ uint32_t order(const u32x4& v, int e) { return order((uint16_t)(v[e / 2] >> (e & 1 ? 16 : 0))); }
};
template <> struct Group<float> {
  typedef uint32_t type;
  static constexpr int BITS = 24;
  static __device__ __forceinline__ uint32_t pack(uint32_t order) { return order; }
  static __device__ __forceinline__ uint32_t order(uint32_t g) { return g; }
  static __device__ __forceinline__ uint32_t order(const u32x4& v, int e) { return v[e]; }
};

// Elements by which a row begins behind a multiple of `line` bytes, on which its chunks lie; and chunks of a row of V elements, at most.
template <typename X>
__device__ __forceinline__ int elements_behind(const X* x, int line) { return (int)((uintptr_t)x & (line - 1)) / (int)sizeof(X); }
int most_chunks(int V, int line, int elem) { return (int)(((int64_t)V + line / elem - 2) / CHUNK) + 1; }

// First element of load l of lane `lane` in chunk c of a row that begins `back` elements behind a chunk's beginning.
template <typename X>
__device__ __forceinline__ int64_t index_of(int c, int l, int lane, int back) { return (int64_t)c * CHUNK + (l * 64 + lane) * per_load<X> - back; }

// A row whose largest logits are wanted.
template <typename X> struct Candidates {
  const X* x;
  const typename Group<X>::type* groups;
  int V, back, chunks;

  // No logit of a group has a larger key than its largest would have in the group's first place.
  __device__ __forceinline__ uint64_t best_key(uint32_t order, int group) const {
    const int64_t j = index_of<X>(group >> 6, 0, group & 63, back);
    return key_of(order, j > 0 ? (int)j : 0);
  }
};

// Lanes' places behind one another, `mine` (up to PER_LANE) to each, and how many there are: a ballot per bit.
__device__ __forceinline__ void places(int mine, int& before, int& all) {
  before = all = 0;
#pragma unroll
  for (int bit = 0; 1 << bit <= PER_LANE; ++bit) {
    const unsigned long long with = __ballot(mine >> bit & 1);
    before += __popcll(with & ((1ull << (threadIdx.x & 63)) - 1)) << bit;
    all += __popcll(with) << bit;
  }
}

// The logits of `count` (up to 64) groups into the list, a group to a lane.
template <typename X>
__device__ __forceinline__ void offer_groups(TopList& top, const uint32_t* found, int count, const Candidates<X>& p) {
  constexpr int N = per_load<X>;
  const int lane = threadIdx.x & 63;
  const bool have = lane < count;
  const uint32_t at = have ? found[lane] : 0;
  const int64_t j0 = index_of<X>(at >> 6, 0, at & 63, p.back);
#pragma unroll 1
  for (int l = 0; l < loads<X>; ++l) {
    const int64_t j = j0 + l * 64 * N;
    const u32x4 v = have ? load_some(p.x, j, p.V) : u32x4{0, 0, 0, 0};
    uint32_t order[N];
#pragma unroll
    for (int e = 0; e < N; ++e) order[e] = order_of(element((const X*)nullptr, v, e));
    // All of them at once, or, where the list cannot hold them even after it was sorted (many equal or rising ones), one of each lane.
    uint32_t left = (1u << N) - 1, now = left;
    while (left) {
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (j + e >= 0 && j + e < p.V && key_of(order[e], (int)(j + e)) > top.bound) mask |= 1u << e;
      mask = have ? mask & now : 0;
      int before, all;
      places(__popc(mask), before, all);
      before += top.n;
      if (top.n + all > LIST) {
        if (top.n > top.K) top.sort();
        else now = left & (0u - left);
        continue;
      }
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (mask >> e & 1) top.keys[before++] = key_of(order[e], (int)(j + e));
      top.n += all;
      asm volatile("" ::: "memory");
      left &= ~now;
      now = left;
    }
  }
}

// The K largest of a row by one wavefront, chunk after chunk, where candidates are many (equal or rising logits, fewer finite ones than K): the
// bound rises on the way.  (20 of 576 rows of 128000 bfloat16 logits of which 5 are finite 72 us, of usual ones 40; one row of 50001 27 for 12.)
template <typename X>
__device__ __forceinline__ void find_in_order(TopList& top, uint32_t* found, const Candidates<X>& p) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  for (int c = 0;;) {
    for (; c < p.chunks; ++c) {
      const bool can = p.best_key(Group<X>::order(p.groups[(int64_t)c * 64 + lane]), c * 64 + lane) > top.bound;
      const unsigned long long all = __ballot(can);
      if (count + __popcll(all) > 64) break;
      if (can) found[count + __popcll(all & ((1ull << lane) - 1))] = c * 64 + lane;
      count += __popcll(all);
    }
    asm volatile("" ::: "memory");
    offer_groups<X>(top, found, count, p);
    if (c >= p.chunks) break;
    count = 0;
  }
  top.sort();
}

// ---- forward -------------------------------------------------------------------------------------------

template <bool ENTROPY>
__device__ __forceinline__ void store_row(const RowArgs& a, int t, const Stats& st, const Row& row, float id_logit, int id) {
  if (a.lse) a.lse[t] = row.lse();
  if (a.logp) a.logp[t] = (unsigned)id < (unsigned)a.V ? row.logp(id_logit) : 0.f;
  if (ENTROPY) a.entropy[t] = row.entropy(st);
}

// TEAM wavefronts to a part of a row, chunk after chunk in turn; their first one ends it.  TOP: groups' maxima are kept for select_kernel,
// which ends the rows.
template <typename X, int TEAM, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void rows_kernel(RowArgs a) {
  using G = Group<X>;
  __shared__ Stats stats[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / TEAM, me = wave % TEAM;
  const unsigned unit = blockIdx.x * (WAVES / TEAM) + team;
  const int t = TEAM == 1 ? (int)unit : (int)(unit / (unsigned)a.parts), part = TEAM == 1 ? 0 : (int)(unit - (unsigned)t * (unsigned)a.parts);
  if (TEAM == 1 && t >= a.T) return;
  const bool ends = !TOP && a.parts == 1;
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  // chunks lie on multiples of 16 bytes (rows of 50001 bfloat16 logits are read at 4.4 TB/s from their own beginnings on, at 5.7 so)
  const int back = elements_behind(x, 16), all_chunks = (int)(((int64_t)a.V + back - 1) / CHUNK) + 1;
  const int c0 = part * a.part_chunks, c1 = c0 + a.part_chunks < all_chunks ? c0 + a.part_chunks : all_chunks;
  const int inside = (int)(((int64_t)a.V + back) / CHUNK), whole = inside < c1 ? inside : c1;  // chunks that end in the row
  typename G::type* groups = reinterpret_cast<typename G::type*>(a.groups) + (int64_t)t * a.max_chunks * 64;

  // the token's own logit, ahead of need
  int id = -1;
  X id_logit{};
  if (ends && a.logp && me == 0) {
    id = a.ids[t];
    id_logit = x[(unsigned)id < (unsigned)a.V ? id : 0];
  }

  Stats st{-INFINITY, 0.f, 0.f};
  auto take = [&](int c, const u32x4 (&v)[loads<X>]) {
    const float top = take_chunk<X, ENTROPY>(st, v, a.c, a.lag);
    if (TOP) groups[(int64_t)c * 64 + lane] = G::pack(order_of(top));
  };
  // (two chunks' loads stay in flight; one that would begin behind the last whole chunk is that one's again)
  auto take_some = [&](int c) {
    u32x4 v[loads<X>];
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) v[l] = load_some(x, index_of<X>(c, l, lane, back), a.V);
    take(c, v);
  };
  int c = c0 + me;
  if (c == 0 && back && whole > 0) {
    take_some(0);
    c += TEAM;
  }
  if (c < whole) {
    u32x4 even[loads<X>], odd[loads<X>];
    const int last = c + (whole - 1 - c) / TEAM * TEAM;
    auto load = [&](int at, u32x4 (&v)[loads<X>]) { load_chunk(x + ((int64_t)(at < last ? at : last) * CHUNK - back), v); };
    load(c, even);
    load(c + TEAM, odd);
    for (; c + TEAM <= last; c += 2 * TEAM) {
      take(c, even);
      load(c + 2 * TEAM, even);
      take(c + TEAM, odd);
      load(c + 3 * TEAM, odd);
    }
    if (c == last) {
      take(c, even);
      c += TEAM;
    }
  }
  if (c < c1) take_some(c);
  join_lanes<ENTROPY>(st, a.c);
  if (TEAM > 1) {
    if (lane == 0) stats[wave] = st;
    lds_barrier();
    if (me != 0) return;
    float m = stats[0].m;
#pragma unroll
    for (int w = 1; w < TEAM; ++w) m = fmaxf(m, stats[w].m);
    refer<ENTROPY>(st, m, a.c);
#pragma unroll
    for (int w = 1; w < TEAM; ++w) {
      Stats other = stats[w];
      refer<ENTROPY>(other, m, a.c);
      st.s += other.s;
      st.e += other.e;
    }
  }
  if (lane != 0) return;
  if (ends) store_row<ENTROPY>(a, t, st, Row(st, a.scale), (float)id_logit, id);
  else a.part_stats[unit] = f32x4{st.m, st.s, st.e, 0.f};
}

// A row's sums from its parts', in order of the lanes that read them; `mine`: those of the lane's first part, read ahead.
__device__ __forceinline__ f32x4 first_part(const RowArgs& a, int t) {
  const int lane = threadIdx.x & 63;
  return lane < a.parts ? a.part_stats[(int64_t)t * a.parts + lane] : f32x4{-INFINITY, 0.f, 0.f, 0.f};
}
template <bool ENTROPY>
__device__ __forceinline__ Stats join_parts(const RowArgs& a, int t, const f32x4& mine) {
  Stats st{mine[0], mine[1], mine[2]};
  for (int p = 64 + (threadIdx.x & 63); p < a.parts; p += 64) {
    const f32x4 v = a.part_stats[(int64_t)t * a.parts + p];
    Stats other{v[0], v[1], v[2]};
    const float m = fmaxf(st.m, other.m);
    refer<ENTROPY>(st, m, a.c);
    refer<ENTROPY>(other, m, a.c);
    st.s += other.s;
    st.e += other.e;
  }
  join_lanes<ENTROPY>(st, a.c);
  return st;
}

// Ends the rows that lay in several parts, a wavefront to a row.
template <typename X, bool ENTROPY>
__global__ __launch_bounds__(64) void join_kernel(RowArgs a) {
  const int t = blockIdx.x;
  int id = -1;
  X id_logit{};
  if (a.logp) {
    id = a.ids[t];
    id_logit = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride)[(unsigned)id < (unsigned)a.V ? id : 0];
  }
  const Stats st = join_parts<ENTROPY>(a, t, first_part(a, t));
  if (threadIdx.x == 0) store_row<ENTROPY>(a, t, st, Row(st, a.scale), (float)id_logit, id);
}

// Ends the rows whose K largest logits are wanted, a workgroup of TEAM wavefronts to a row.  A bound that K of the groups' maxima reach (TEAM 1, rows of
// up to SHORT chunks), or K of the threads' largest, leaves little more than K groups; of their logits, in LDS, those that the K-th largest leaves are
// ranked by counting, a key to a thread.
constexpr int SHORT = 8;
template <typename X, int TEAM, bool ENTROPY>
__global__ __launch_bounds__(64 * TEAM) void select_kernel(RowArgs a) {
  using G = Group<X>;
  constexpr int N = 64 * TEAM, PER = 16 / (int)sizeof(typename G::type), KEYS = TEAM == 1 ? 512 : 1024;
  __shared__ __attribute__((aligned(16))) uint64_t keys[KEYS];
  __shared__ uint32_t found[FOUND], bounds[TEAM][2];
  __shared__ int n_found, n_keys, n_left;
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  const int back = elements_behind(x, 16);
  const Candidates<X> row{x, reinterpret_cast<const typename G::type*>(a.groups) + (int64_t)t * a.max_chunks * 64, a.V, back, (int)(((int64_t)a.V + back - 1) / CHUNK) + 1};
  int id = -1;
  X id_logit{};
  if (a.logp) {
    id = a.ids[t];
    id_logit = x[(unsigned)id < (unsigned)a.V ? id : 0];
  }
  if (threadIdx.x == 0) n_found = n_keys = n_left = 0;
  const f32x4 mine = first_part(a, t);
  // (-infinity and NaN bound nothing)
  auto bounding = [](uint32_t order) { return order <= order_of(-INFINITY) ? 0u : order; };
  auto find = [&](uint32_t order, int group, uint32_t bound) {
    if (order < bound) return;
    const int at = atomicAdd(&n_found, 1);
    if (at < FOUND) found[at] = group;
  };
  const int n_groups = row.chunks * 64;
  uint32_t bound;
  if constexpr (TEAM == 1) {
    uint32_t order[SHORT], u[SHORT];
#pragma unroll
    for (int c = 0; c < SHORT; ++c) order[c] = c < row.chunks ? G::order(row.groups[c * 64 + lane]) : 0;
#pragma unroll
    for (int c = 0; c < SHORT; ++c) u[c] = bounding(order[c]);
    bound = reached_by<G::BITS>(u, a.K);
    int n = 0;
#pragma unroll
    for (int c = 0; c < SHORT; ++c) {
      if (c >= row.chunks) break;
      const unsigned long long all = __ballot(order[c] >= bound);
      if (order[c] >= bound) found[n + __popcll(all & ((1ull << lane) - 1))] = c * 64 + lane;
      n += __popcll(all);
    }
    if (lane == 0) n_found = n;
  } else {
    // 16 bytes of groups to a thread (chunks have 64), or, of shorter rows, single ones, so that every thread has some
    const bool single = row.chunks <= 8 * TEAM;
    uint32_t best[1] = {0};
    if (single) {
#pragma unroll 4
      for (int i = threadIdx.x; i < n_groups; i += N) {
        const uint32_t order = G::order(row.groups[i]);
        best[0] = order > best[0] ? order : best[0];
      }
    } else {
#pragma unroll 2
      for (int i = threadIdx.x * PER; i < n_groups; i += N * PER) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(row.groups + i);
#pragma unroll
        for (int e = 0; e < PER; ++e) best[0] = G::order(v, e) > best[0] ? G::order(v, e) : best[0];
      }
    }
    best[0] = bounding(best[0]);
    uint32_t first = reached_by<G::BITS>(best, a.K), second = reached_by<G::BITS>(best, (a.K - 1) / TEAM + 1);
    if (lane == 0) {
      bounds[wave][0] = first;
      bounds[wave][1] = second;
    }
    lds_barrier();
#pragma unroll
    for (int w = 0; w < TEAM; ++w) {
      first = bounds[w][0] > first ? bounds[w][0] : first;
      second = bounds[w][1] < second ? bounds[w][1] : second;
    }
    // At least K logits reach the larger of these: K threads of one wavefront do, or a TEAM-th of K in each.
    bound = first > second ? first : second;
    if (single) {
#pragma unroll 4
      for (int i = threadIdx.x; i < n_groups; i += N) find(G::order(row.groups[i]), i, bound);
    } else {
#pragma unroll 2
      for (int i = threadIdx.x * PER; i < n_groups; i += N * PER) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(row.groups + i);
#pragma unroll
        for (int e = 0; e < PER; ++e) find(G::order(v, e), i + e, bound);
      }
    }
  }
  const Stats st = join_parts<ENTROPY>(a, t, mine);
  const Row sums(st, a.scale);
  if (threadIdx.x == 0) store_row<ENTROPY>(a, t, st, sums, (float)id_logit, id);
  auto store = [&](int rank, uint64_t key) {
    a.top_ids[(int64_t)t * a.K + rank] = (int)~(uint32_t)key;
    a.top_logp[(int64_t)t * a.K + rank] = sums.logp(of_order((uint32_t)(key >> 32)));
  };
  lds_barrier();
  const int groups = n_found;
  if (groups <= FOUND) {
    for (int i0 = wave * 64; i0 < groups; i0 += N) {
      const bool have = i0 + lane < groups;
      const uint32_t at = have ? found[i0 + lane] : 0;
      const int64_t j0 = index_of<X>(at >> 6, 0, at & 63, back);
      u32x4 v[loads<X>];
      uint32_t mask = 0;
#pragma unroll
      for (int l = 0; l < loads<X>; ++l) v[l] = load_some(x, j0 + l * 64 * per_load<X>, a.V);
#pragma unroll
      for (int l = 0; l < loads<X>; ++l)
#pragma unroll
        for (int e = 0; e < per_load<X>; ++e) {
          const int64_t j = j0 + l * 64 * per_load<X> + e;
          mask |= (uint32_t)((j >= 0) & (j < a.V) & (order_of(element((const X*)nullptr, v[l], e)) >= bound)) << (l * per_load<X> + e);
        }
      int place, all;
      places(have ? __popc(mask) : 0, place, all);
      int begin = lane == 0 ? atomicAdd(&n_keys, all) : 0;
      place += __builtin_amdgcn_readfirstlane(begin);
      if (!have || place + __popc(mask) > KEYS) mask = 0;
#pragma unroll
      for (int l = 0; l < loads<X>; ++l)
#pragma unroll
        for (int e = 0; e < per_load<X>; ++e)
          if (mask >> (l * per_load<X> + e) & 1) keys[place++] = key_of(order_of(element((const X*)nullptr, v[l], e)), (int)(j0 + l * 64 * per_load<X> + e));
    }
    lds_barrier();
    int n = n_keys;
    if (n <= KEYS) {
      // Only those that the K-th largest leaves: 16 or 32 steps over what a lane has of them, where counting takes a step for each of them all.
      auto leave = [&](auto slots) {
        constexpr int SLOTS = decltype(slots)::value, OWN = (SLOTS + TEAM - 1) / TEAM;
        uint32_t order[SLOTS];
#pragma unroll
        for (int e = 0; e < SLOTS; ++e) order[e] = e * 64 + lane < n ? (uint32_t)(keys[e * 64 + lane] >> 32) : 0;
        const uint32_t least = reached_by<8 * (int)sizeof(X)>(order, a.K);
        uint64_t own[OWN];
#pragma unroll
        for (int e = 0; e < OWN; ++e) own[e] = e * N + (int)threadIdx.x < n ? keys[e * N + threadIdx.x] : 0;
        lds_barrier();
#pragma unroll
        for (int e = 0; e < OWN; ++e) {
          const bool stays = e * N + (int)threadIdx.x < n && (uint32_t)(own[e] >> 32) >= least;
          const unsigned long long all = __ballot(stays);
          if (!all) continue;
          int begin = lane == 0 ? atomicAdd(&n_left, __popcll(all)) : 0;
          begin = __builtin_amdgcn_readfirstlane(begin);
          if (stays) keys[begin + __popcll(all & ((1ull << lane) - 1))] = own[e];
        }
        lds_barrier();
        n = n_left;
      };
      if (n > 64 && n > a.K + a.K / 4) {
        if (n <= 128) leave(std::integral_constant<int, 2>());
        else if (n <= 256) leave(std::integral_constant<int, 4>());
        else leave(std::integral_constant<int, KEYS / 64>());
      }
      for (int i = n + threadIdx.x; i < ((n + 7) & ~7); i += N) keys[i] = 0;  // (above none)
      lds_barrier();
      for (int i0 = wave * 64; i0 < n; i0 += N) {
        const uint64_t my_key = i0 + lane < n ? keys[i0 + lane] : ~0ull;
        int rank = 0;
        for (int i = 0; i < n; i += 8)
#pragma unroll
          for (int e = 0; e < 8; ++e) rank += keys[i + e] > my_key;
        if (i0 + lane < n && rank < a.K) store(rank, my_key);
      }
      return;
    }
  }
  if (wave != 0) return;
  TopList top{keys, 0, a.K, (uint64_t)bound << 32};
  find_in_order<X>(top, found, row);
  if (lane < a.K) store(lane, keys[lane]);
}

// How a call's rows are divided; groups' maxima begin `groups` bytes into the workspace.
constexpr int MOST_PARTS = 2048;  // of rows that are split
struct Division {
  int team, parts, part_chunks, max_chunks;
  size_t groups;
};
bool splits(int chunks, int K) { return chunks > (K > 0 ? 16 : 64); }
int most_parts(int chunks) { return (chunks + 7) / 8; }  // of a row
Division division_of(int T, int V, int K) {
  const int chunks = most_chunks(V, 16, 2);
  Division d{chunks <= 2 ? 1 : WAVES, 1, chunks, chunks, 0};
  // Without alternatives, whose kernel joins the parts as well, a split costs a launch: rows of up to 65536 logits, and 256 of
  // any length, are faster whole (us, split / whole: 1 row of 50001 bfloat16 logits 11.8 / 8.2, of 250000 11.0 / 19.0; 200 of 250000 22.5 / 26.9; 300 of 128000
  // 18.1 / 16.8; 1000 float32 rows of 32003 26.8 / 24.0).
  if (splits(chunks, K) && (K > 0 || T < 256)) {
    int parts = T > 0 ? MOST_PARTS / T : 1;
    if (parts > most_parts(chunks)) parts = most_parts(chunks);
    if (parts < 1) parts = 1;
    d.part_chunks = (chunks + parts - 1) / parts;
    d.part_chunks = (d.part_chunks + WAVES - 1) / WAVES * WAVES;
    d.parts = (chunks - 1) / d.part_chunks + 1;
  }
  d.groups = align_up((size_t)T * d.parts * sizeof(f32x4), 256);
  return d;
}

// What division_of wants for T rows and for any fewer: T parts, or as many more as rows are split into.  (The type is not told: groups' maxima
// have float32's four bytes.)
size_t workspace_of(int T, int V, int K) {
  const int chunks = most_chunks(V, 16, 2);
  const int64_t split = (int64_t)T * most_parts(chunks), parts = !splits(chunks, K) ? 0 : split < MOST_PARTS ? split : MOST_PARTS;
  size_t total = align_up((size_t)(K > 0 && T > parts ? T : parts) * sizeof(f32x4), 256);
  if (K > 0) total += (size_t)T * chunks * 64 * sizeof(uint32_t);
  return total < 256 ? 256 : total;
}

template <typename X, bool ENTROPY, bool TOP>
int32_t launch_rows(const RowArgs& a, const Division& d, hipStream_t s) {
  const int64_t units = (int64_t)a.T * d.parts;
  if (d.team == 1) hipLaunchKernelGGL((rows_kernel<X, 1, ENTROPY, TOP>), dim3((unsigned)((units + WAVES - 1) / WAVES)), dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((rows_kernel<X, WAVES, ENTROPY, TOP>), dim3((unsigned)units), dim3(THREADS), 0, s, a);
  int32_t st = check_hip(hipGetLastError(), "log-probabilities launch");
  if (st != MOE_OK || (d.parts == 1 && !TOP)) return st;
  if constexpr (TOP) {
    if (d.max_chunks <= SHORT) hipLaunchKernelGGL((select_kernel<X, 1, ENTROPY>), dim3((unsigned)a.T), dim3(64), 0, s, a);
    else hipLaunchKernelGGL((select_kernel<X, WAVES, ENTROPY>), dim3((unsigned)a.T), dim3(64 * WAVES), 0, s, a);
  } else {
    hipLaunchKernelGGL((join_kernel<X, ENTROPY>), dim3((unsigned)a.T), dim3(64), 0, s, a);
  }
  return check_hip(hipGetLastError(), "log-probabilities join launch");
}

template <typename X>
int32_t launch_rows(const RowArgs& a, const Division& d, hipStream_t s) {
  if (a.K > 0) return a.entropy ? launch_rows<X, true, true>(a, d, s) : launch_rows<X, false, true>(a, d, s);
  return a.entropy ? launch_rows<X, true, false>(a, d, s) : launch_rows<X, false, false>(a, d, s);
}

// ---- backward ------------------------------------------------------------------------------------------

constexpr int LARGE_TEAM = 16;

struct GradArgs {
  const char* x;
  char* d_x;
  int64_t row_stride, d_row_stride;  // bytes
  const int32_t* ids;
  const float *lse, *d_logp, *entropy, *d_entropy, *d_lse;
  int32_t T, V, groups, group_chunks, line, in_place, one_takes_all, owner_shift;
  float scale, c, lag;
};

__device__ __forceinline__ void put(const float (&d)[8], u32x4& v) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const bf16x2 two = {(__bf16)d[2 * w], (__bf16)d[2 * w + 1]};
    v[w] = __builtin_bit_cast(uint32_t, two);
  }
}
__device__ __forceinline__ void put(const float (&d)[4], u32x4& v) {
#pragma unroll
  for (int w = 0; w < 4; ++w) v[w] = __float_as_uint(d[w]);
}

// Past the caches: whole lines go out as they are, and what the next call reads stays.
template <typename X>
__device__ __forceinline__ void store_some(X* x, int64_t j, int V, const u32x4& v) {
  if (j >= 0 && j + per_load<X> <= V) {
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(x + j));
    return;
  }
  if (j >= V) return;  // (most lanes of a short row)
#pragma unroll
  for (int e = 0; e < per_load<X>; ++e) {
    if (j + e < 0 || j + e >= V) continue;
    if constexpr (sizeof(X) == 2) reinterpret_cast<uint16_t*>(x)[j + e] = (uint16_t)(v[e / 2] >> (e & 1 ? 16 : 0));
    else reinterpret_cast<uint32_t*>(x)[j + e] = v[e];
  }
}

// -infinity in the place of element e
__device__ __forceinline__ void forget(const __bf16*, u32x4& v, int e) { v[e / 2] = e & 1 ? (v[e / 2] & 0xffffu) | 0xff800000u : (v[e / 2] & 0xffff0000u) | 0xff80u; }
__device__ __forceinline__ void forget(const float*, u32x4& v, int e) { v[e] = 0xff800000u; }

// Element `at` of a wavefront's chunk, for all its lanes.
template <typename X>
__device__ __forceinline__ float pick(const X* kind, const u32x4 (&v)[loads<X>], int at) {
  constexpr int N = per_load<X>;
  const int l_at = at / (64 * N), w_at = at % N / (N / 4);
  auto choose = [](int which, uint32_t a, uint32_t b) { return (a & ((uint32_t)which - 1u)) | (b & (0u - (uint32_t)which)); };  // 0 or 1
  auto word_of = [&](int w) {
    const uint32_t lower = choose(l_at & 1, v[0][w], v[1][w]);
    if constexpr (loads<X> == 2) return lower;
    else return choose(l_at >> 1 & 1, lower, choose(l_at & 1, v[loads<X> - 2][w], v[loads<X> - 1][w]));
  };
  uint32_t word = choose(w_at >> 1 & 1, choose(w_at & 1, word_of(0), word_of(1)), choose(w_at & 1, word_of(2), word_of(3)));
  word = (uint32_t)__builtin_amdgcn_readlane((int)word, at / N & 63);
  return element(kind, u32x4{word, word, word, word}, at % (N / 4));
}

// TEAM wavefronts to one of a row's `groups`, chunk after chunk in turn, the rows from the last one on (the forward call has read that one last).
//   d_j = scale p_j (gl - g - ge (log p_j + h)),  and scale g more for the token itself, log p_j = scale x_j - lse.
// What lse does not tell well enough is taken from the row again, before anything is written (x may be y):
//  - Of rows far from zero (far_lse), and of the entropy's gradient where nearly all is one token's, the sum.  One group does the whole row; of
//    few rows every group the sum for itself.
//  - Of a token that is nearly certain r = sum_{j != id} p_j, by the group that has it: 1 - p without a difference, and log p = log(1 - r).
// REGISTERS: a row has TEAM chunks or fewer, nothing is read twice.
// Bound: HBM (8192 rows of 50001 bfloat16 logits 265 us, 6.2 TB/s read + written); of rows that are read again also the vector unit, for exp.  us of
// usual rows / rows whose token has all but 1e-4 / rows far from zero:  8192 of 50001 bfloat16 265 / 352 / 434, 1000 of 32003 float32 39 / 54 / 79,
// 1 of 262144 float32 8 / 16 / 19, 16384 of 1000 bfloat16 13 / 19 / 19.  In place: 328, 40, 23, 14 of usual ones, since a row is one group's.
template <typename X, int TEAM, bool REGISTERS>
__global__ __launch_bounds__(TEAM > WAVES ? 64 * TEAM : THREADS) void gradient_kernel(GradArgs a) {
  constexpr int BLOCK = TEAM > WAVES ? TEAM : WAVES;
  __shared__ Stats stats[BLOCK];
  __shared__ float id_lds;
  const X* kind = nullptr;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = wave % TEAM;
  const unsigned units = (unsigned)a.T * (unsigned)a.groups, unit = blockIdx.x * (BLOCK / TEAM) + wave / TEAM;
  if (unit >= units) return;
  const int t = (int)((units - 1 - unit) / (unsigned)a.groups), group = (int)((units - 1 - unit) - (unsigned)t * (unsigned)a.groups);
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  X* y = reinterpret_cast<X*>(a.d_x + (int64_t)t * a.d_row_stride);
  const int back = elements_behind(y, a.line), all_chunks = (int)(((int64_t)a.V + back - 1) / CHUNK) + 1;
  int c0 = group * a.group_chunks, c1 = c0 + a.group_chunks < all_chunks ? c0 + a.group_chunks : all_chunks;
  auto inside = [&](int c) { return !(REGISTERS && TEAM == 1) && (c > 0 || back == 0) && (int64_t)(c + 1) * CHUNK - back <= a.V; };  // the whole chunk is the row's
  auto load = [&](int c, u32x4 (&v)[loads<X>]) {  // (nothing of chunks behind the last)
    if (inside(c)) {
      load_chunk(x + ((int64_t)c * CHUNK - back), v);
    } else {
#pragma unroll
      for (int l = 0; l < loads<X>; ++l) v[l] = load_some(x, index_of<X>(c, l, lane, back), a.V);
    }
  };
  int id = a.ids ? a.ids[t] : -1;
  const float lse = a.lse[t], ge = a.d_entropy ? a.d_entropy[t] : 0.f, gl = a.d_lse ? a.d_lse[t] : 0.f;
  float h = a.d_entropy ? a.entropy[t] : 0.f, g = a.d_logp ? a.d_logp[t] : 0.f;
  if ((unsigned)id >= (unsigned)a.V || !a.d_logp) id = -1;
  if (id < 0) g = 0.f;
  if (ge == 0.f) h = 0.f;
  // the token's own logit, where it is this group's (in place the whole row is)
  const int id_chunk = (int)(((int64_t)id + back) / CHUNK);
  bool has_id = id >= 0 && id_chunk >= c0 && id_chunk < c1;
  float id_logit = 0.f;
  if (lse == -INFINITY || (g == 0.f && ge == 0.f && gl == 0.f)) {
    for (int c = c0 + me; c < c1; c += TEAM)
#pragma unroll
      for (int l = 0; l < loads<X>; ++l) store_some(y, index_of<X>(c, l, lane, back), a.V, u32x4{0, 0, 0, 0});
    return;
  }
  u32x4 v[loads<X>];
  load(c0 + me, v);  // (rows without a gradient are not read)
  if (g == 0.f) {
    id = -1;
    has_id = false;
  }
  if (has_id && id_chunk - c0 < TEAM) {  // a wavefront has it in registers
    if (id_chunk == c0 + me) {
      id_logit = pick(kind, v, (int)((int64_t)id + back - (int64_t)id_chunk * CHUNK));
      if (TEAM > 1 && lane == 0) id_lds = id_logit;
    }
    if (TEAM > 1) {
      lds_barrier();
      id_logit = id_lds;
    }
  } else if (has_id) {
    id_logit = (float)x[id];
    if (a.in_place) {
      asm volatile("" : "+v"(id_logit));  // it has arrived
      lds_barrier();                      // ... everywhere, before its place is written
    }
  }
  const float near = near_certain<X>(lse);
  const bool whole_row = fabsf(lse) > far_lse<X> || (ge != 0.f && fabsf(h) < near);
  if (whole_row && a.one_takes_all) {
    if (group != (t >> a.owner_shift) % a.groups) return;  // (the same of all rows would lie on one die)
    if (c0) load(me, v);
    c0 = 0;
    c1 = all_chunks;
  }
  float m = 0.f, log_s = lse, own = 0.f;
  bool certain = false;  // the token's own element is `own`
  // All of the row but the token's own logit, GULP chunks at a time.
  auto for_others = [&](auto take) {
    constexpr int GULP = REGISTERS ? 1 : 2;
#pragma unroll 1
    for (int c = me; c < all_chunks; c += GULP * TEAM) {
      u32x4 w[GULP][loads<X>];
#pragma unroll
      for (int i = 0; i < GULP; ++i) {
        if constexpr (REGISTERS) {
#pragma unroll
          for (int l = 0; l < loads<X>; ++l) w[i][l] = v[l];
        } else {
          load(c + i * TEAM, w[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < GULP; ++i) {
        if (id >= 0 && id_chunk == c + i * TEAM) {
          const int at = (int)((int64_t)id + back - (int64_t)id_chunk * CHUNK);
#pragma unroll
          for (int l = 0; l < loads<X>; ++l)
#pragma unroll
            for (int e = 0; e < per_load<X>; ++e)
              if (first_of<X>(l) + e == at) forget(kind, w[i][l], e);
        }
        take(w[i]);
      }
    }
  };
  if (__builtin_expect(whole_row, 0)) {
    if (id >= 0 && !has_id) id_logit = (float)x[id];  // (not in place)
    Stats st{-INFINITY, 0.f, 0.f};
    for_others([&](const u32x4 (&w)[loads<X>]) { take_chunk<X, false>(st, w, a.c, a.lag); });
    join_lanes<false>(st, a.c);
    m = st.m;
    if (TEAM > 1) {
      if (lane == 0) stats[wave] = st;
      lds_barrier();  // (the whole row has been read: x may be y)
#pragma unroll
      for (int w = 0; w < TEAM; ++w) m = fmaxf(m, stats[w].m);
      st = Stats{m, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < TEAM; ++w) {
        Stats other = stats[w];
        refer<false>(other, m, a.c);
        st.s += other.s;
      }
    }
    float p = 0.f;
    if (id >= 0) {
      m = fmaxf(m, id_logit);
      refer<false>(st, m, a.c);
      p = __builtin_amdgcn_exp2f((id_logit - m) * a.c);
    }
    const float s = st.s + p, rest = st.s / s;
    log_s = logf(s);
    const float lp = p > st.s ? log1pf(-rest) : (id_logit - m) * a.scale - log_s;
    own = a.scale * (g * rest + (p == 0.f ? 0.f : p / s * (gl - ge * (lp + h))));
    certain = true;
  } else if (has_id && __builtin_fmaf(id_logit, a.scale, -lse) > -near) {
    float rest = 0.f;
    for_others([&](const u32x4 (&w)[loads<X>]) {
#pragma unroll
      for (int l = 0; l < loads<X>; ++l)
#pragma unroll
        for (int e = 0; e < per_load<X>; ++e) rest += __builtin_amdgcn_exp2f(__builtin_fmaf(element(kind, w[l], e), a.scale, -lse) * LOG2E);
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) rest += __shfl_xor(rest, d, 64);
    if (TEAM > 1) {
      if (lane == 0) stats[wave].s = rest;
      lds_barrier();
      rest = 0.f;
#pragma unroll
      for (int w = 0; w < TEAM; ++w) rest += stats[w].s;
    }
    own = a.scale * (g * rest + (1.f - rest) * (gl - ge * (log1pf(-rest) + h)));
    certain = true;
  }
  const float flat = a.scale * (gl - g - ge * h), steep = -a.scale * ge;
  for (int c = c0 + me; c < c1; c += TEAM) {
    const bool all = inside(c);
    X* to = y + ((int64_t)c * CHUNK - back);
    const int id_here = id >= 0 && id_chunk == c ? (int)((int64_t)id + back - (int64_t)c * CHUNK) : -1;
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) {
      const int first = first_of<X>(l);
      float d[per_load<X>];
#pragma unroll
      for (int e = 0; e < per_load<X>; ++e) {
        const float lp = __builtin_fmaf(element(kind, v[l], e) - m, a.scale, -log_s), p = __builtin_amdgcn_exp2f(lp * LOG2E);
        d[e] = p == 0.f ? 0.f : p * __builtin_fmaf(steep, lp, flat);
      }
      if (id_here >= 0)
#pragma unroll
        for (int e = 0; e < per_load<X>; ++e)
          if (first + e == id_here) d[e] = certain ? own : d[e] + a.scale * g;
      u32x4 out;
      put(d, out);
      if (all) __builtin_nontemporal_store(out, reinterpret_cast<u32x4*>(to + first));
      else store_some(y, index_of<X>(c, l, lane, back), a.V, out);
    }
    if (c + TEAM < c1) load(c + TEAM, v);
  }
}

template <typename X, int TEAM>
void launch_gradient(const GradArgs& a, bool registers, unsigned grid, hipStream_t s) {
  const dim3 threads(TEAM > WAVES ? 64 * TEAM : THREADS);
  if (TEAM <= WAVES && registers) hipLaunchKernelGGL((gradient_kernel<X, TEAM, TEAM <= WAVES>), dim3(grid), threads, 0, s, a);
  else hipLaunchKernelGGL((gradient_kernel<X, TEAM, false>), dim3(grid), threads, 0, s, a);
}
template <typename X>
void launch_gradient(const GradArgs& a, int team, bool registers, unsigned grid, hipStream_t s) {
  if (team == 1) launch_gradient<X, 1>(a, registers, grid, s);
  else if (team == WAVES) launch_gradient<X, WAVES>(a, registers, grid, s);
  else launch_gradient<X, LARGE_TEAM>(a, registers, grid, s);
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
  return workspace_of(T, V, K);
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
  const Division d = division_of(T, V, K);
  if (!launchable((int64_t)T * d.parts, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "moe_token_logprobs: %d rows are too many for one call", T);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_token_logprobs: workspace NULL, misaligned or smaller than %zu bytes", need);
  const float c = fminf(scale * LOG2E, FLT_MAX);
  const RowArgs a{(const char*)x, row_stride * (int64_t)es, ids, logp, lse, entropy, top_logp, top_ids, (f32x4*)ws, (char*)ws + d.groups, T, V, K, d.parts, d.part_chunks, d.max_chunks, scale, c, LAG_BITS / c};
  return dtype == MOE_BF16 ? launch_rows<__bf16>(a, d, (hipStream_t)stream) : launch_rows<float>(a, d, (hipStream_t)stream);
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
  // Stores of whole lines: a tenth of the time of 8192 rows of 50001 bfloat16 logits.  Short rows, which a few more elements can cost
  // another chunk, begin on 16 bytes (16384 rows of 1000: a fifth).
  const int line = V > 8 * CHUNK ? 128 : 16, chunks = most_chunks(V, line, (int)es);
  // A chunk to each wavefront of a group, in place the whole row to a group.  Rows of one chunk are a wavefront's own, and so are many rows of up to four
  // (4096 of 3000: 10.3 against 13.7 us); sixteen wavefronts take the rest of a row again sooner than four do, where few rows leave
  // the machine idle behind them (1000 float32 rows of 32003, all of them certain: 55 against 61 us, usual ones 40 for both).
  const bool in_place = x == d_x;
  const int team = chunks == 1 || (chunks <= WAVES && T >= 4096) ? 1 : T < 2048 && chunks > LARGE_TEAM ? LARGE_TEAM : WAVES;
  const int threads = team > WAVES ? 64 * team : THREADS;
  int group_chunks = in_place || team == 1 ? chunks : team, groups = (chunks - 1) / group_chunks + 1;
  while (groups > 1 && !launchable((int64_t)T * groups, threads)) {
    group_chunks *= 2;
    groups = (chunks - 1) / group_chunks + 1;
  }
  // Rows far from zero, one group's alone / every group's: 700 float32 ones of 100003 171 / 355 us, 64 bfloat16 ones of 128000 79 / 34.
  const bool one_takes_all = T >= 128;
  // (workgroups go to the eight dies in turn; the groups that take whole rows are to lie on all of them)
  const int owner_shift = groups % 8 == 0 ? 0 : groups % 4 == 0 ? 1 : groups % 2 == 0 ? 2 : 3;
  const int64_t grid = team == 1 ? ((int64_t)T + WAVES - 1) / WAVES : (int64_t)T * groups;
  if (!launchable(grid, threads)) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows are too many for one call", who, T);
  const float c = fminf(scale * LOG2E, FLT_MAX);
  const GradArgs a{(const char*)x, (char*)d_x, row_stride * (int64_t)es, d_row_stride * (int64_t)es, ids, lse, d_logp, entropy, d_entropy, d_lse, T, V, groups, group_chunks, line, in_place, one_takes_all, owner_shift, scale, c, LAG_BITS / c};
  if (dtype == MOE_BF16) launch_gradient<__bf16>(a, team, chunks <= team, (unsigned)grid, (hipStream_t)stream);
  else launch_gradient<float>(a, team, chunks <= team, (unsigned)grid, (hipStream_t)stream);
  return check_hip(hipGetLastError(), "log-probabilities gradient launch");
}
