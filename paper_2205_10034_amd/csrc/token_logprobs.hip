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

namespace moesys {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int PER_LANE = 16, CHUNK = 64 * PER_LANE;  // logits that a lane, a wavefront takes at a time
constexpr int MAX_CHUNKS = 128;                      // of a part whose largest are wanted (its groups' maxima lie in LDS)
constexpr int LIST = 128;                            // candidates that a wavefront holds
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LAG_BITS = 8.f;

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

// per_load elements from x[j] on, -infinity in the place of those from V on
template <typename X>
__device__ __forceinline__ u32x4 load_some(const X* x, uint32_t j, int V_) {
  const uint32_t V = (uint32_t)V_;
  if (j + per_load<X> <= V) return reinterpret_cast<const Unaligned<X>*>(x + j)->v;
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v[w] = minus_infinities<X>;
    if constexpr (sizeof(X) == 2) {
      if (j + 2 * w < V) v[w] = (v[w] & 0xffff0000u) | reinterpret_cast<const uint16_t*>(x)[j + 2 * w];
      if (j + 2 * w + 1 < V) v[w] = (v[w] & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t*>(x)[j + 2 * w + 1] << 16;
    } else if (j + w < V) {
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
  uint64_t* part_keys;  // [row][part][K], falling, 0: none
  int32_t T, V, K, parts, part_chunks;
  float scale, c, lag;
};

// ---- the K largest -------------------------------------------------------------------------------------

// Keys of one wavefront, in LDS, that are above `bound` when they come.
struct TopList {
  uint64_t* keys;  // [LIST]
  int n, K;
  uint64_t bound;

  // The K largest, in falling order; from then on only larger ones come in.
  __device__ void sort() {
    const int lane = threadIdx.x & 63;
    const uint64_t a = lane < n ? keys[lane] : 0, b = lane + 64 < n ? keys[lane + 64] : 0;
    int ra = 0, rb = 0;
    if (n <= 64) {
      for (int i = 0; i < n; ++i) ra += keys[i] > a;
    } else {
      for (int i = 0; i < n; ++i) {
        const uint64_t k = keys[i];
        ra += k > a;
        rb += k > b;
      }
    }
    asm volatile("" ::: "memory");  // (a wavefront's LDS operations execute in order)
    if (lane < n && ra < K) keys[ra] = a;
    if (lane + 64 < n && rb < K) keys[rb] = b;
    asm volatile("" ::: "memory");
    if (n >= K) {
      n = K;
      bound = keys[K - 1];
    }
  }

  __device__ __forceinline__ void offer(bool have, uint64_t key) {
    unsigned long long all = __ballot(have && key > bound);
    if (!all) return;
    if (n + __popcll(all) > LIST) {
      sort();
      all = __ballot(have && key > bound);
    }
    if (have && key > bound) keys[n + __popcll(all & ((1ull << (threadIdx.x & 63)) - 1))] = key;
    n += __popcll(all);
    asm volatile("" ::: "memory");
  }
};

// The K-th and the K2-th largest of the lanes' values (0: no value), a little less, or 0 where there are fewer.
__device__ __forceinline__ void largest_lanes(uint32_t u, int K, int K2, uint32_t& first, uint32_t& second) {
  const int lane = threadIdx.x & 63;
  const uint32_t mine = (u & ~63u) | (63 - lane);  // all differ
  int rank = 0;
#pragma unroll 16
  for (int i = 0; i < 64; ++i) rank += (uint32_t)__builtin_amdgcn_readlane((int)mine, i) > mine;
  auto of_rank = [&](int r) {
    const unsigned long long who = __ballot(rank == r);
    return (uint32_t)__builtin_amdgcn_readlane((int)mine, (int)__ffsll(who) - 1) & ~63u;
  };
  first = of_rank(K - 1);
  second = of_rank(K2 - 1);
}

// The largest logit of a lane's PER_LANE, as LDS keeps it: a bfloat16's order is told by its upper half.
template <typename X> struct Group;
template <> struct Group<__bf16> {
  typedef uint16_t type;
  static __device__ __forceinline__ uint16_t pack(uint32_t order) { return (uint16_t)(order >> 16); }
  static __device__ __forceinline__ uint32_t order(uint16_t g) { return (uint32_t)g << 16 | (g & 0x8000u ? 0u : 0xffffu); }
};
template <> struct Group<float> {
  typedef uint32_t type;
  static __device__ __forceinline__ uint32_t pack(uint32_t order) { return order; }
  static __device__ __forceinline__ uint32_t order(uint32_t g) { return g; }
};

// The K largest of a part (chunks c0 .. c0+n-1 of the row) into the list, by one wavefront: of the groups whose largest logit can be among them,
// 64 at a time, a group to a lane.
template <typename X>
__device__ void find_largest(TopList& top, const typename Group<X>::type* group_max, uint32_t* found, const X* x, int V, int c0, int n) {
  const int lane = threadIdx.x & 63;
  int count = 0;
  auto flush = [&]() {
    asm volatile("" ::: "memory");
    const bool have = lane < count;
    const uint32_t at = have ? found[lane] : 0, j0 = (at >> 6) * CHUNK + (at & 63) * per_load<X>;
    u32x4 v[loads<X>];
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) v[l] = have ? load_some(x, j0 + l * 64 * per_load<X>, V) : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int l = 0; l < loads<X>; ++l)
#pragma unroll
      for (int e = 0; e < per_load<X>; ++e) {
        const uint32_t j = j0 + l * 64 * per_load<X> + e;
        top.offer(have && j < (uint32_t)V, key_of(order_of(element((const X*)nullptr, v[l], e)), j));
      }
    count = 0;
  };
  for (int c = 0; c < n; ++c) {
    // (no logit of the group has a larger key than its largest would have in the group's first place)
    const uint32_t at = (uint32_t)(c0 + c) * 64 + lane;
    const bool can = key_of(Group<X>::order(group_max[c * 64 + lane]), (at >> 6) * CHUNK + lane * per_load<X>) > top.bound;
    const unsigned long long all = __ballot(can);
    if (!all) continue;
    if (count + __popcll(all) > 64) flush();
    if (can) found[count + __popcll(all & ((1ull << lane) - 1))] = at;
    count += __popcll(all);
  }
  if (count) flush();
  top.sort();
}

// ---- forward -------------------------------------------------------------------------------------------

template <typename X, bool ENTROPY, bool TOP>
__device__ __forceinline__ void finish_row(const RowArgs& a, int t, const Stats& st, X id_logit, int id, const TopList& top) {
  const int lane = threadIdx.x & 63;
  const Row row(st, a.scale);
  if (lane == 0) {
    if (a.lse) a.lse[t] = row.lse();
    if (a.logp) a.logp[t] = (unsigned)id < (unsigned)a.V ? row.logp((float)id_logit) : 0.f;
    if (ENTROPY) a.entropy[t] = row.entropy(st);
  }
  if (TOP && lane < a.K) {
    const uint64_t key = top.keys[lane];
    a.top_ids[(int64_t)t * a.K + lane] = (int)~(uint32_t)key;
    a.top_logp[(int64_t)t * a.K + lane] = row.logp(of_order((uint32_t)(key >> 32)));
  }
}

// TEAM wavefronts to a part of a row, chunk after chunk in turn; their first one ends it.
template <typename X, int TEAM, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(THREADS) void rows_kernel(RowArgs a) {
  using G = Group<X>;
  extern __shared__ __attribute__((aligned(16))) char group_lds[];
  __shared__ uint64_t keys[TOP ? WAVES / TEAM : 1][TOP ? LIST : 1];
  __shared__ uint32_t found[TOP ? WAVES / TEAM : 1][64];
  __shared__ Stats stats[WAVES];
  __shared__ uint32_t bounds[WAVES][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave / TEAM, me = wave % TEAM;
  const unsigned unit = blockIdx.x * (WAVES / TEAM) + team;
  const int t = TEAM == 1 ? (int)unit : (int)(unit / (unsigned)a.parts), part = TEAM == 1 ? 0 : (int)(unit - (unsigned)t * (unsigned)a.parts);
  if (TEAM == 1 && t >= a.T) return;
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  const int c0 = part * a.part_chunks, all_chunks = (a.V - 1) / CHUNK + 1, c1 = c0 + a.part_chunks < all_chunks ? c0 + a.part_chunks : all_chunks;
  const int whole = a.V / CHUNK < c1 ? a.V / CHUNK : c1;  // chunks that end inside the row
  typename G::type* group_max = reinterpret_cast<typename G::type*>(group_lds) + team * a.part_chunks * 64;

  // the token's own logit, ahead of need
  int id = -1;
  X id_logit{};
  if (a.logp && a.parts == 1 && me == 0) {
    id = a.ids[t];
    id_logit = x[(unsigned)id < (unsigned)a.V ? id : 0];
  }

  Stats st{-INFINITY, 0.f, 0.f};
  float lane_top = -INFINITY;
  auto take = [&](int c, const u32x4 (&v)[loads<X>]) {
    const float top = take_chunk<X, ENTROPY>(st, v, a.c, a.lag);
    if (TOP) {
      group_max[(c - c0) * 64 + lane] = G::pack(order_of(top));
      lane_top = fmaxf(lane_top, top);
    }
  };
  int c = c0 + me;
  if (c < whole) {
    u32x4 next[loads<X>];
    load_chunk(x + (int64_t)c * CHUNK, next);
    for (; c + TEAM < whole; c += TEAM) {
      u32x4 v[loads<X>];
#pragma unroll
      for (int l = 0; l < loads<X>; ++l) v[l] = next[l];
      load_chunk(x + (int64_t)(c + TEAM) * CHUNK, next);
      take(c, v);
    }
    take(c, next);
    c += TEAM;
  }
  if (c < c1) {
    u32x4 v[loads<X>];
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) v[l] = load_some(x, c * CHUNK + first_of<X>(l), a.V);
    take(c, v);
  }
  join_lanes<ENTROPY>(st, a.c);
  uint32_t first = 0, second = 0;
  if (TOP) largest_lanes(lane_top == -INFINITY ? 0u : order_of(lane_top), a.K, (a.K - 1) / TEAM + 1, first, second);
  if (TEAM > 1) {
    if (lane == 0) {
      stats[wave] = st;
      bounds[wave][0] = first;
      bounds[wave][1] = second;
    }
    lds_barrier();
    if (me != 0) return;
    float m = stats[0].m;
#pragma unroll
    for (int w = 1; w < TEAM; ++w) {
      m = fmaxf(m, stats[w].m);
      first = bounds[w][0] > first ? bounds[w][0] : first;
      second = bounds[w][1] < second ? bounds[w][1] : second;
    }
    refer<ENTROPY>(st, m, a.c);
#pragma unroll
    for (int w = 1; w < TEAM; ++w) {
      Stats other = stats[w];
      refer<ENTROPY>(other, m, a.c);
      st.s += other.s;
      st.e += other.e;
    }
  }
  // At least K logits of the part reach the larger of these: K lanes of one wavefront do, or a K-th of them in each.
  TopList top{keys[TOP ? team : 0], 0, a.K, (uint64_t)(first > second ? first : second) << 32};
  if (TOP) find_largest<X>(top, group_max, found[team], x, a.V, c0, c1 - c0);
  if (a.parts == 1) {
    finish_row<X, ENTROPY, TOP>(a, t, st, id_logit, id, top);
  } else {
    if (lane == 0) a.part_stats[unit] = f32x4{st.m, st.s, st.e, 0.f};
    if (TOP && lane < a.K) a.part_keys[(int64_t)unit * a.K + lane] = lane < top.n ? top.keys[lane] : 0;
  }
}

// A wavefront to a row: its parts' sums, in order of the lanes that read them, and the largest of their largest.
template <typename X, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(64) void join_kernel(RowArgs a) {
  __shared__ uint64_t keys[TOP ? LIST : 1];
  const int t = blockIdx.x, lane = threadIdx.x;
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  int id = -1;
  X id_logit{};
  if (a.logp) {
    id = a.ids[t];
    id_logit = x[(unsigned)id < (unsigned)a.V ? id : 0];
  }
  const int64_t unit = (int64_t)t * a.parts;
  const uint64_t* part_keys = a.part_keys + unit * a.K;
  Stats st{-INFINITY, 0.f, 0.f};
  uint64_t first = 0, second = ~0ull;
  for (int p = lane; p < a.parts; p += 64) {
    const f32x4 v = a.part_stats[unit + p];
    Stats other{v[0], v[1], v[2]};
    const float m = fmaxf(st.m, other.m);
    refer<ENTROPY>(st, m, a.c);
    refer<ENTROPY>(other, m, a.c);
    st.s += other.s;
    st.e += other.e;
    if (TOP) {
      const uint64_t last = part_keys[(int64_t)p * a.K + a.K - 1], some = part_keys[(int64_t)p * a.K + (a.K - 1) / a.parts];
      first = last > first ? last : first;
      second = some < second ? some : second;
    }
  }
  join_lanes<ENTROPY>(st, a.c);
  TopList top{keys, 0, a.K, 0};
  if (TOP) {
    for (int d = 32; d; d >>= 1) {
      const uint64_t f = __shfl_xor(first, d, 64), s = __shfl_xor(second, d, 64);
      first = f > first ? f : first;
      second = s < second ? s : second;
    }
    const uint64_t reached = first > second ? first : second;
    top.bound = reached ? reached - 1 : 0;
    const int64_t n = (int64_t)a.parts * a.K;
    constexpr int AHEAD = 4;
    for (int64_t i = lane; i - lane < n; i += 64 * AHEAD) {
      uint64_t k[AHEAD];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) k[e] = i + e * 64 < n ? part_keys[i + e * 64] : 0;
#pragma unroll
      for (int e = 0; e < AHEAD; ++e) top.offer(k[e] != 0, k[e]);
    }
    top.sort();
  }
  finish_row<X, ENTROPY, TOP>(a, t, st, id_logit, id, top);
}

// How a call's rows are divided.
struct Division {
  int team, parts, part_chunks;
  size_t keys, total;  // bytes
};
Division division_of(int T, int V, int K) {
  const int chunks = (V - 1) / CHUNK + 1;
  Division d{chunks <= 2 ? 1 : WAVES, 1, chunks, 0, 256};
  if (chunks > 16) {
    int64_t parts = T > 0 ? 2048 / T : 1;
    const int64_t most = (chunks + 7) / 8;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    d.part_chunks = (int)((chunks + parts - 1) / parts);
    d.part_chunks = (d.part_chunks + WAVES - 1) / WAVES * WAVES;
    if (K > 0 && d.part_chunks > MAX_CHUNKS) d.part_chunks = MAX_CHUNKS;
    d.parts = (chunks - 1) / d.part_chunks + 1;
  }
  if (d.parts > 1) {
    d.keys = align_up((size_t)T * d.parts * sizeof(f32x4), 256);
    d.total = d.keys + align_up((size_t)T * d.parts * K * sizeof(uint64_t), 256);
    if (d.total < 256) d.total = 256;
  }
  return d;
}

template <typename X, bool ENTROPY, bool TOP>
int32_t launch_rows(const RowArgs& a, const Division& d, hipStream_t s) {
  const int64_t units = (int64_t)a.T * d.parts;
  const size_t lds = TOP ? (size_t)(WAVES / d.team) * d.part_chunks * 64 * sizeof(typename Group<X>::type) : 0;
  if (d.team == 1) hipLaunchKernelGGL((rows_kernel<X, 1, ENTROPY, TOP>), dim3((unsigned)((units + WAVES - 1) / WAVES)), dim3(THREADS), lds, s, a);
  else hipLaunchKernelGGL((rows_kernel<X, WAVES, ENTROPY, TOP>), dim3((unsigned)units), dim3(THREADS), lds, s, a);
  int32_t st = check_hip(hipGetLastError(), "log-probabilities launch");
  if (st != MOE_OK || d.parts == 1) return st;
  hipLaunchKernelGGL((join_kernel<X, ENTROPY, TOP>), dim3((unsigned)a.T), dim3(64), 0, s, a);
  return check_hip(hipGetLastError(), "log-probabilities join launch");
}

template <typename X>
int32_t launch_rows(const RowArgs& a, const Division& d, hipStream_t s) {
  if (a.K > 0) return a.entropy ? launch_rows<X, true, true>(a, d, s) : launch_rows<X, false, true>(a, d, s);
  return a.entropy ? launch_rows<X, true, false>(a, d, s) : launch_rows<X, false, false>(a, d, s);
}

// ---- backward ------------------------------------------------------------------------------------------

struct GradArgs {
  const char* x;
  char* d_x;
  int64_t row_stride, d_row_stride;  // bytes
  const int32_t* ids;
  const float *lse, *d_logp, *entropy, *d_entropy, *d_lse;
  int32_t T, V, parts, part_chunks;
  float scale;
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

template <typename X>
__device__ __forceinline__ void store_some(X* x, uint32_t j, int V, const u32x4& v) {
  if (j + per_load<X> <= (uint32_t)V) {
    reinterpret_cast<Unaligned<X>*>(x + j)->v = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < per_load<X>; ++e) {
    if (j + e >= (uint32_t)V) continue;
    if constexpr (sizeof(X) == 2) reinterpret_cast<uint16_t*>(x)[j + e] = (uint16_t)(v[e / 2] >> (e & 1 ? 16 : 0));
    else reinterpret_cast<uint32_t*>(x)[j + e] = v[e];
  }
}

// A wavefront to a part of a row, the rows from the last one on (the forward call has read that one last).
template <typename X>
__global__ __launch_bounds__(THREADS) void gradient_kernel(GradArgs a) {
  const unsigned units = (unsigned)a.T * (unsigned)a.parts, unit = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (unit >= units) return;
  const int t = (int)((units - 1 - unit) / (unsigned)a.parts), part = (int)((units - 1 - unit) - (unsigned)t * (unsigned)a.parts);
  const X* x = reinterpret_cast<const X*>(a.x + (int64_t)t * a.row_stride);
  X* y = reinterpret_cast<X*>(a.d_x + (int64_t)t * a.d_row_stride);
  const int all_chunks = (a.V - 1) / CHUNK + 1, c0 = part * a.part_chunks, c1 = c0 + a.part_chunks < all_chunks ? c0 + a.part_chunks : all_chunks;
  const int id = a.ids ? a.ids[t] : -1;
  const float lse = a.lse[t], g = a.d_logp && (unsigned)id < (unsigned)a.V ? a.d_logp[t] : 0.f, ge = a.d_entropy ? a.d_entropy[t] : 0.f, gl = a.d_lse ? a.d_lse[t] : 0.f;
  if (lse == -INFINITY || (g == 0.f && ge == 0.f && gl == 0.f)) {
    for (int c = c0; c < c1; ++c)
#pragma unroll
      for (int l = 0; l < loads<X>; ++l) store_some(y, c * CHUNK + first_of<X>(l), a.V, u32x4{0, 0, 0, 0});
    return;
  }
  const float h = ge != 0.f ? a.entropy[t] : 0.f;
  // p_j (gl - g - ge (log p_j + h)), and g for the token itself
  const float flat = a.scale * (gl - g - ge * h), steep = -a.scale * ge, own = a.scale * g;
  auto take = [&](int c, const u32x4 (&v)[loads<X>]) {
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) {
      const uint32_t j = (uint32_t)c * CHUNK + first_of<X>(l);
      float d[per_load<X>];
#pragma unroll
      for (int e = 0; e < per_load<X>; ++e) {
        const float lp = __builtin_fmaf(element((const X*)nullptr, v[l], e), a.scale, -lse), p = __builtin_amdgcn_exp2f(lp * LOG2E);
        d[e] = p == 0.f ? 0.f : p * __builtin_fmaf(steep, lp, flat);
        if (j + e == (uint32_t)id) d[e] += own;
      }
      u32x4 out;
      put(d, out);
      store_some(y, j, a.V, out);
    }
  };
  for (int c = c0; c < c1; ++c) {
    u32x4 v[loads<X>];
#pragma unroll
    for (int l = 0; l < loads<X>; ++l) v[l] = load_some(x, c * CHUNK + first_of<X>(l), a.V);
    take(c, v);
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
  return division_of(T, V, K).total;
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
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_token_logprobs: workspace NULL, misaligned or smaller than %zu bytes", need);
  const Division d = division_of(T, V, K);
  if (!launchable((int64_t)T * d.parts, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "moe_token_logprobs: %d rows are too many for one call", T);
  const float c = fminf(scale * LOG2E, FLT_MAX);
  const RowArgs a{(const char*)x, row_stride * (int64_t)es, ids, logp, lse, entropy, top_logp, top_ids, (f32x4*)ws, (uint64_t*)((char*)ws + d.keys), T, V, K, d.parts, d.part_chunks, scale, c, LAG_BITS / c};
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
  const int chunks = (V - 1) / CHUNK + 1;
  int per = chunks < 4 ? chunks : 4;
  if ((int64_t)T * ((chunks - 1) / per + 1) < 4096) per = 1;
  const int parts = (chunks - 1) / per + 1;
  const int64_t grid = ((int64_t)T * parts + WAVES - 1) / WAVES;
  if (!launchable(grid, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "%s: %d rows are too many for one call", who, T);
  const GradArgs a{(const char*)x, (char*)d_x, row_stride * (int64_t)es, d_row_stride * (int64_t)es, ids, lse, d_logp, entropy, d_entropy, d_lse, T, V, parts, per, scale};
  if (dtype == MOE_BF16) hipLaunchKernelGGL(gradient_kernel<__bf16>, dim3((unsigned)grid), dim3(THREADS), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(gradient_kernel<float>, dim3((unsigned)grid), dim3(THREADS), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "log-probabilities gradient launch");
}
