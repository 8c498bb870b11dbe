// Places and pages of a paged cache: accepted drafts to their places (moe_kv_compact), pages given back (moe_kv_release), shared
// (moe_kv_fork) and handed out (moe_kv_reserve).  Pages are counted, not listed: refs[p] entries of the table name page p, a free
// one has count 0, and the free pages in rising order are the ones that are given.  So the calls' results do not depend on the order of
// their atomic operations: counts are whole numbers, and nobody looks at one while it changes.
#include "moesys_internal.h"
#include "kv_pages.h"
#include "wave_util.h"

namespace moesys {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PoolArgs {
  char *k, *v;
  int32_t *table, *refs, *lens, *missing, *counts, *list;
  const int32_t *src, *dst;
  int64_t n_pages, page_stride, token_stride, head_stride;  // bytes
  PageDivisor page, unit;                                   // places of a page, 16-byte units of a head's row
  int32_t page_size, table_width, capacity, n_seqs, hkv, units, n, more, blocks;
};

__device__ __forceinline__ int pages_of(const PoolArgs& a, int len) {
  // (a length can reach the largest int32: the last place decides)
  return len > 0 ? a.page.quotient(len - 1) + 1 : 0;
}

// ---- accepted drafts -----------------------------------------------------------------------------------

constexpr int COMPACT_THREADS = 256;
constexpr int COMPACT_UNITS = MOE_MAX_DRAFTS * (MOE_MAX_HEAD_DIM * 4 / 16) / COMPACT_THREADS;  // 16-byte units of a thread, at most

struct CompactArgs {
  PoolArgs pool;
  const int32_t *base, *keep;
  int32_t* new_lens;
  int32_t width;
};

// A workgroup per sequence, kv head and keys or values: all its rows into registers, then out of them.
__global__ __launch_bounds__(COMPACT_THREADS) void compact_kernel(CompactArgs c) {
  const PoolArgs& a = c.pool;
  __shared__ int64_t from[MOE_MAX_DRAFTS], to[MOE_MAX_DRAFTS];  // offset of a row, -1: it is not there
  __shared__ int moved;
  const int s = blockIdx.x / (2 * a.hkv), head = blockIdx.x / 2 % a.hkv;
  char* pool = blockIdx.x & 1 ? a.v : a.k;
  if (threadIdx.x < 64) {
    const int i = threadIdx.x, base = c.base[s], mine = i < c.width ? c.keep[(int64_t)s * c.width + i] : -1;
    const unsigned long long ends = __ballot(mine < 0);
    const int n = ends ? __ffsll(ends) - 1 : 64;
    auto row = [&](int64_t place) {
      if (place < 0 || place >= a.capacity) return (int64_t)-1;
      const int column = a.page.quotient((int)place), page = valid_page(a.table[(int64_t)s * a.table_width + column], a.n_pages);
      return page < 0 ? -1 : page * a.page_stride + (place - (int64_t)column * a.page_size) * a.token_stride + head * a.head_stride;
    };
    // a row that stays where it is is not moved
    const bool moves = i < n && mine != i;
    from[i] = moves ? row((int64_t)base + mine) : -1;
    to[i] = moves ? row((int64_t)base + i) : -1;
    if (i == 0) {
      moved = n;
      if (c.new_lens && head == 0 && !(blockIdx.x & 1)) c.new_lens[s] = base + n;
    }
  }
  __syncthreads();
  u32x4 r[COMPACT_UNITS];
  const int total = moved * a.units;
#pragma unroll
  for (int u = 0; u < COMPACT_UNITS; ++u) {
    const int x = threadIdx.x + u * COMPACT_THREADS;
    if (x < total) {
      const int i = a.unit.quotient(x);
      if (from[i] >= 0 && to[i] >= 0) r[u] = *reinterpret_cast<const u32x4*>(pool + from[i] + (x - i * a.units) * 16);
    }
    asm volatile("" : "+v"(r[u]));  // it has arrived
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < COMPACT_UNITS; ++u) {
    const int x = threadIdx.x + u * COMPACT_THREADS;
    if (x >= total) continue;
    const int i = a.unit.quotient(x);
    if (from[i] >= 0 && to[i] >= 0) *reinterpret_cast<u32x4*>(pool + to[i] + (x - i * a.units) * 16) = r[u];
  }
}

// ---- pages ---------------------------------------------------------------------------------------------

constexpr int THREADS = 256, GIVE_THREADS = 1024;

__global__ __launch_bounds__(THREADS) void release_kernel(PoolArgs a) {
  const int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (x >= (int64_t)a.n_seqs * a.table_width) return;
  const int s = (int)(x / a.table_width), column = (int)(x - (int64_t)s * a.table_width);
  if (column < pages_of(a, a.lens[s])) return;
  const int page = valid_page(a.table[x], a.n_pages);
  if (page >= 0) atomicSub(a.refs + page, 1);
  a.table[x] = -1;
}

struct Pair {
  int src, dst, whole, begun;  // src < 0: left out; whole pages, places of the one behind them
};
__device__ __forceinline__ Pair pair_of(const PoolArgs& a, int i) {
  Pair p{a.src[i], a.dst[i], 0, 0};
  if (p.src < 0 || p.src >= a.n_seqs || p.dst < 0 || p.dst >= a.n_seqs || p.src == p.dst) {
    p.src = -1;
    return p;
  }
  const int len = kept_length(a.lens[p.src], a.capacity);
  p.whole = a.page.quotient(len);
  p.begun = len - p.whole * a.page_size;
  return p;
}

// dst's pages back, src's whole ones shared
__global__ __launch_bounds__(THREADS) void share_kernel(PoolArgs a) {
  const int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (x >= (int64_t)a.n * a.table_width) return;
  const int i = (int)(x / a.table_width), column = (int)(x - (int64_t)i * a.table_width);
  const Pair p = pair_of(a, i);
  if (p.src < 0) return;
  int32_t* entry = a.table + (int64_t)p.dst * a.table_width + column;
  const int had = *entry, gets = column < p.whole ? a.table[(int64_t)p.src * a.table_width + column] : -1;
  if (had != gets) {
    const int out = valid_page(had, a.n_pages), in = valid_page(gets, a.n_pages);
    if (out >= 0) atomicSub(a.refs + out, 1);
    if (in >= 0) atomicAdd(a.refs + in, 1);
    *entry = gets;
  }
}

// This thread's part of a sum in front of it, and the sum of all (GIVE_THREADS threads).
__device__ __forceinline__ int sum_before(int mine, int& all) {
  __shared__ int waves[GIVE_THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(upto, d, 64);
    if (lane >= d) upto += other;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  int before = upto - mine;
  all = 0;
  for (int w = 0; w < GIVE_THREADS / 64; ++w) {
    if (w < wave) before += waves[w];
    all += waves[w];
  }
  return before;
}

// The `wanted` lowest free pages into list, counted as in use; how many there were.
__device__ int take_pages(const PoolArgs& a, int wanted) {
  int found = 0;
  for (int64_t p0 = 0; p0 < a.n_pages && found < wanted; p0 += GIVE_THREADS * 4) {
    const int64_t p = p0 + threadIdx.x * 4;
    bool free[4];
    int mine = 0, all;
    for (int e = 0; e < 4; ++e) mine += free[e] = p + e < a.n_pages && a.refs[p + e] == 0;
    int rank = found + sum_before(mine, all);
    for (int e = 0; e < 4; ++e)
      if (free[e]) {
        if (rank < wanted) {
          a.list[rank] = (int)(p + e);
          a.refs[p + e] = 1;
        }
        ++rank;
      }
    found += all;
  }
  __syncthreads();
  return found < wanted ? found : wanted;
}

// One workgroup: a page for every fork whose source has begun one
__global__ __launch_bounds__(GIVE_THREADS) void fork_pages_kernel(PoolArgs a) {
  int wanted = 0;
  for (int i0 = 0; i0 < a.n; i0 += GIVE_THREADS) {
    const int i = i0 + threadIdx.x;
    int wants = 0, all;
    if (i < a.n) {
      const Pair p = pair_of(a, i);
      wants = p.src >= 0 && p.begun && valid_page(a.table[(int64_t)p.src * a.table_width + p.whole], a.n_pages) >= 0;
    }
    const int rank = wanted + sum_before(wants, all);
    if (i < a.n) a.counts[i] = wants ? rank : -1;
    wanted += all;
  }
  const int had = take_pages(a, wanted);
  if (a.missing && threadIdx.x == 0) *a.missing = wanted - had;
  for (int i = threadIdx.x; i < a.n; i += GIVE_THREADS) {
    const int rank = a.counts[i], page = rank >= 0 && rank < had ? a.list[rank] : -1;
    a.counts[i] = page;
    const Pair p = pair_of(a, i);
    if (page >= 0) a.table[(int64_t)p.dst * a.table_width + p.whole] = page;
  }
}

// The begun pages' places, `blocks` workgroups to a fork; then dst has src's length
__global__ __launch_bounds__(THREADS) void copy_kernel(PoolArgs a) {
  const int i = blockIdx.x / a.blocks;
  const Pair p = pair_of(a, i);
  if (p.src < 0) return;
  if (blockIdx.x % a.blocks == 0 && threadIdx.x == 0) a.lens[p.dst] = a.lens[p.src];
  const int to = a.counts[i];
  if (to < 0) return;
  const int64_t from = a.table[(int64_t)p.src * a.table_width + p.whole];
  const int64_t rows = (int64_t)p.begun * a.hkv, total = 2 * rows * a.units;
  for (int64_t x = (int64_t)(blockIdx.x % a.blocks) * THREADS + threadIdx.x; x < total; x += (int64_t)a.blocks * THREADS) {
    const int64_t row = x / a.units, r = row % rows;
    char* pool = row >= rows ? a.v : a.k;
    const int64_t at = r / a.hkv * a.token_stride + r % a.hkv * a.head_stride + (x - row * a.units) * 16;
    *reinterpret_cast<u32x4*>(pool + to * a.page_stride + at) = *reinterpret_cast<const u32x4*>(pool + from * a.page_stride + at);
  }
}

__device__ __forceinline__ int columns_wanted(const PoolArgs& a, int s) {
  const int len = a.lens[s];
  const int64_t places = (int64_t)len + a.more;
  return len < 0 ? 0 : pages_of(a, places > a.capacity ? a.capacity : (int)places);
}

// Entries that lack a page, a wavefront per sequence
__global__ __launch_bounds__(THREADS) void lacking_kernel(PoolArgs a) {
  const int s = blockIdx.x * (THREADS / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (s >= a.n_seqs) return;
  const int columns = columns_wanted(a, s);
  int n = 0;
  for (int c0 = 0; c0 < columns; c0 += 64) {
    const int c = c0 + lane;
    n += __popcll(__ballot(c < columns && valid_page(a.table[(int64_t)s * a.table_width + c], a.n_pages) < 0));
  }
  if (lane == 0) a.counts[s] = n;
}

// One workgroup: where every sequence's pages begin in the list, and the list
__global__ __launch_bounds__(GIVE_THREADS) void reserve_pages_kernel(PoolArgs a) {
  int64_t wanted = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += GIVE_THREADS) {
    const int s = s0 + threadIdx.x;
    int all;
    const int mine = s < a.n_seqs ? a.counts[s] : 0;
    const int64_t rank = wanted + sum_before(mine, all);
    if (s < a.n_seqs) a.counts[s] = (int)(rank < a.n_pages ? rank : a.n_pages);
    wanted += all;
  }
  const int asked = (int)(wanted < a.n_pages ? wanted : a.n_pages), had = take_pages(a, asked);
  if (threadIdx.x == 0) {
    a.counts[a.n_seqs] = had;
    if (a.missing) *a.missing = (int)(wanted - had);
  }
}

__global__ __launch_bounds__(THREADS) void fill_kernel(PoolArgs a) {
  const int s = blockIdx.x * (THREADS / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (s >= a.n_seqs) return;
  const int columns = columns_wanted(a, s), had = a.counts[a.n_seqs];
  int rank = a.counts[s];
  for (int c0 = 0; c0 < columns; c0 += 64) {
    const int c = c0 + lane;
    int32_t* entry = a.table + (int64_t)s * a.table_width + c;
    const bool lacks = c < columns && valid_page(*entry, a.n_pages) < 0;
    const unsigned long long all = __ballot(lacks);
    const int at = rank + __popcll(all & ((1ull << lane) - 1));
    if (lacks) *entry = at < had ? a.list[at] : -1;
    rank += __popcll(all);
  }
}

PoolArgs pool_of(const moe_kv_cache* c, int32_t* refs, void* ws) {
  PoolArgs a{};
  const int64_t es = (int64_t)elem_size(c->dtype);
  a.k = (char*)c->k;
  a.v = (char*)c->v;
  a.table = const_cast<int32_t*>(c->page_table);
  a.refs = refs;
  a.counts = (int32_t*)ws;
  if (ws) a.list = (int32_t*)((char*)ws + align_up(((size_t)c->n_seqs + 1) * sizeof(int32_t), 256));
  a.n_pages = c->n_pages;
  a.page_stride = c->page_stride * es;
  a.token_stride = c->token_stride * es;
  a.head_stride = c->head_stride * es;
  a.page = page_divisor(c->page_size);
  a.units = (int)(c->head_dim * es / 16);
  a.unit = page_divisor(a.units);
  a.page_size = c->page_size;
  a.table_width = c->table_width;
  a.capacity = c->table_width * c->page_size;
  a.n_seqs = c->n_seqs;
  a.hkv = c->n_kv_heads;
  return a;
}

int32_t check_pool(const moe_kv_cache* c, const int32_t* refs, const char* who) {
  const int32_t st = moe_kv_cache_check(c);
  if (st != MOE_OK) return st;
  if (c->n_pages > 0 && !refs) return fail(MOE_ERR_INVALID_ARG, "%s: refs is NULL", who);
  return MOE_OK;
}

int32_t check_pool_ws(const moe_kv_cache* c, void* ws, size_t ws_bytes, const char* who) {
  const size_t need = moe_kv_pages_workspace_bytes(c);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "%s: workspace NULL, misaligned or smaller than %zu bytes", who, need);
  return MOE_OK;
}

int64_t grid_of(int64_t work, int threads) { return (work + threads - 1) / threads; }

}  // namespace
}  // namespace moesys

using namespace moesys;

extern "C" int32_t moe_kv_compact(const moe_kv_cache* c, const int32_t* base, int32_t width, const int32_t* keep, int32_t* new_lens,
                                  void* stream) {
  const int32_t st = moe_kv_cache_check(c);
  if (st != MOE_OK) return st;
  if (width < 1 || width > MOE_MAX_DRAFTS) return fail(MOE_ERR_INVALID_ARG, "moe_kv_compact: width=%d outside 1..%d", width, MOE_MAX_DRAFTS);
  if (c->n_seqs == 0) return MOE_OK;
  if (!base || !keep) return fail(MOE_ERR_INVALID_ARG, "moe_kv_compact: base and keep must be non-NULL");
  if (new_lens == base) return fail(MOE_ERR_INVALID_ARG, "moe_kv_compact: new_lens must not be base");
  const int64_t grid = (int64_t)c->n_seqs * c->n_kv_heads * 2;
  if (!launchable(grid, COMPACT_THREADS))
    return fail(MOE_ERR_UNSUPPORTED, "moe_kv_compact: %d sequences of %d kv heads are too many for one call", c->n_seqs, c->n_kv_heads);
  const CompactArgs a{pool_of(c, nullptr, nullptr), base, keep, new_lens, width};
  hipLaunchKernelGGL(compact_kernel, dim3((unsigned)grid), dim3(COMPACT_THREADS), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "compact launch");
}

extern "C" int32_t moe_kv_release(const moe_kv_cache* c, int32_t* refs, const int32_t* lens, void* stream) {
  const int32_t st = check_pool(c, refs, "moe_kv_release");
  if (st != MOE_OK) return st;
  const int64_t entries = (int64_t)c->n_seqs * c->table_width;
  if (entries == 0) return MOE_OK;
  if (!lens) return fail(MOE_ERR_INVALID_ARG, "moe_kv_release: lens is NULL");
  if (!launchable(grid_of(entries, THREADS), THREADS)) return fail(MOE_ERR_UNSUPPORTED, "moe_kv_release: a table of %lld entries is too large for one call", (long long)entries);
  PoolArgs a = pool_of(c, refs, nullptr);
  a.lens = const_cast<int32_t*>(lens);
  hipLaunchKernelGGL(release_kernel, dim3((unsigned)grid_of(entries, THREADS)), dim3(THREADS), 0, (hipStream_t)stream, a);
  return check_hip(hipGetLastError(), "release launch");
}

extern "C" size_t moe_kv_pages_workspace_bytes(const moe_kv_cache* c) {
  if (moe_kv_cache_check(c) != MOE_OK) return 0;
  return align_up(((size_t)c->n_seqs + 1) * sizeof(int32_t), 256) + align_up((size_t)c->n_pages * sizeof(int32_t), 256);
}

extern "C" int32_t moe_kv_fork(const moe_kv_cache* c, int32_t* refs, int32_t n, const int32_t* src, const int32_t* dst, int32_t* lens,
                               int32_t* missing, void* ws, size_t ws_bytes, void* stream) {
  int32_t st = check_pool(c, refs, "moe_kv_fork");
  if (st != MOE_OK) return st;
  if (n < 0 || n > c->n_seqs) return fail(MOE_ERR_INVALID_ARG, "moe_kv_fork: n=%d outside 0..%d", n, c->n_seqs);
  if (n > 0 && (!src || !dst || !lens)) return fail(MOE_ERR_INVALID_ARG, "moe_kv_fork: src, dst and lens must be non-NULL");
  st = check_pool_ws(c, ws, ws_bytes, "moe_kv_fork");
  if (st != MOE_OK) return st;
  PoolArgs a = pool_of(c, refs, ws);
  a.lens = lens;
  a.missing = missing;
  a.src = src;
  a.dst = dst;
  a.n = n;
  const int64_t entries = (int64_t)n * c->table_width, units = (int64_t)c->page_size * c->n_kv_heads * a.units * 2;
  const int64_t blocks = grid_of(units, THREADS * 4);
  a.blocks = (int)(blocks < 64 ? blocks : 64);
  if (!launchable(grid_of(entries, THREADS), THREADS) || !launchable((int64_t)n * a.blocks, THREADS))
    return fail(MOE_ERR_UNSUPPORTED, "moe_kv_fork: %d forks are too many for one call", n);
  hipStream_t s = (hipStream_t)stream;
  if (entries > 0) {
    hipLaunchKernelGGL(share_kernel, dim3((unsigned)grid_of(entries, THREADS)), dim3(THREADS), 0, s, a);
    st = check_hip(hipGetLastError(), "fork launch");
    if (st != MOE_OK) return st;
  }
  if (n == 0 && !missing) return MOE_OK;
  hipLaunchKernelGGL(fork_pages_kernel, dim3(1), dim3(GIVE_THREADS), 0, s, a);
  st = check_hip(hipGetLastError(), "fork launch");
  if (st != MOE_OK || n == 0) return st;
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)(n * a.blocks)), dim3(THREADS), 0, s, a);
  return check_hip(hipGetLastError(), "fork launch");
}

extern "C" int32_t moe_kv_reserve(const moe_kv_cache* c, int32_t* refs, const int32_t* lens, int32_t more, int32_t* missing, void* ws,
                                  size_t ws_bytes, void* stream) {
  int32_t st = check_pool(c, refs, "moe_kv_reserve");
  if (st != MOE_OK) return st;
  if (more < 0) return fail(MOE_ERR_INVALID_ARG, "moe_kv_reserve: more=%d is negative", more);
  if (c->n_seqs > 0 && !lens) return fail(MOE_ERR_INVALID_ARG, "moe_kv_reserve: lens is NULL");
  st = check_pool_ws(c, ws, ws_bytes, "moe_kv_reserve");
  if (st != MOE_OK) return st;
  PoolArgs a = pool_of(c, refs, ws);
  a.lens = const_cast<int32_t*>(lens);
  a.missing = missing;
  a.more = more;
  const int64_t grid = grid_of(c->n_seqs, THREADS / 64);
  if (!launchable(grid, THREADS)) return fail(MOE_ERR_UNSUPPORTED, "moe_kv_reserve: %d sequences are too many for one call", c->n_seqs);
  hipStream_t s = (hipStream_t)stream;
  if (c->n_seqs > 0) {
    hipLaunchKernelGGL(lacking_kernel, dim3((unsigned)grid), dim3(THREADS), 0, s, a);
    st = check_hip(hipGetLastError(), "reserve launch");
    if (st != MOE_OK) return st;
  }
  hipLaunchKernelGGL(reserve_pages_kernel, dim3(1), dim3(GIVE_THREADS), 0, s, a);
  st = check_hip(hipGetLastError(), "reserve launch");
  if (st != MOE_OK || c->n_seqs == 0) return st;
  hipLaunchKernelGGL(fill_kernel, dim3((unsigned)grid), dim3(THREADS), 0, s, a);
  return check_hip(hipGetLastError(), "reserve launch");
}
