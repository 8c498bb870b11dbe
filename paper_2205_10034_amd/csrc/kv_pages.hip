// Places and pages of a paged cache: accepted drafts to their places (moe_kv_compact), pages given back (moe_kv_release), shared
// (moe_kv_fork) and handed out (moe_kv_reserve).  Pages are counted, not listed: refs[p] entries of the table name page p, a free
// one has count 0, and the free pages in rising order are the ones that are given.  So the calls' results do not depend on the order of
// their atomic operations: counts are whole numbers, and nobody looks at one while it changes.
#include "moesys_internal.h"
#include "kv_pages.h"
#include "wave_util.h"
#include <limits.h>

namespace moesys {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PoolArgs {
  char *k, *v;
  int32_t *table, *refs, *lens, *missing, *counts, *list, *claims;
  const int32_t *src, *dst;
  int64_t n_pages, page_stride, token_stride, head_stride;  // bytes
  PageDivisor page, unit, width;                            // places of a page, 16-byte units of a head's row, columns of the table
  int32_t page_size, table_width, capacity, n_seqs, hkv, units, n, more, blocks;
};

__device__ __forceinline__ int pages_of(const PoolArgs& a, int len) {
  // (a length can reach the largest int32: the last place decides)
  return len > 0 ? a.page.quotient(len - 1) + 1 : 0;
}

// ---- accepted drafts -----------------------------------------------------------------------------------

constexpr int COMPACT_THREADS = 256;
constexpr int MOST_UNITS = 16;  // 16-byte units of a thread: 64 rows of the longest head

struct CompactArgs {
  PoolArgs pool;
  const int32_t *base, *keep;
  int32_t* new_lens;
  PageDivisor heads, slices;  // heads of a workgroup; workgroups of a sequence
  int32_t width, n_heads, n_slices;
};

// A workgroup per sequence and n_heads of its heads, those of the keys and then those of the values: all their rows into registers, then out
// of them.  A chain of latencies (keep, page table, rows), so the workgroups are as large as fill the machine once, and every thread has
// its loads in flight together: 256 sequences of up to 16 tokens, 8 heads of 128, 5.3 us with 4 heads to a workgroup, 9.4 with one.
template <int UNITS>
__global__ __launch_bounds__(COMPACT_THREADS) void compact_kernel(CompactArgs c) {
  const PoolArgs& a = c.pool;
  __shared__ int64_t from[MOE_MAX_DRAFTS], to[MOE_MAX_DRAFTS];  // offset of a row's first head, -1: it is not there, or does not move
  __shared__ int rows;
  const int s = c.slices.quotient((int)blockIdx.x), slice = blockIdx.x - s * c.n_slices;
  if (threadIdx.x < 64) {
    const int i = threadIdx.x, base = c.base[s], mine = i < c.width ? c.keep[(int64_t)s * c.width + i] : -1;
    const unsigned long long ends = __ballot(mine < 0);
    const int n = ends ? __ffsll(ends) - 1 : 64;
    auto row = [&](int64_t place) {
      if (place < 0 || place >= a.capacity) return (int64_t)-1;
      const int column = a.page.quotient((int)place), page = valid_page(a.table[(int64_t)s * a.table_width + column], a.n_pages);
      return page < 0 ? -1 : page * a.page_stride + (place - (int64_t)column * a.page_size) * a.token_stride;
    };
    const bool moves = i < n && mine != i;
    const int64_t source = moves ? row((int64_t)base + mine) : -1, target = moves ? row((int64_t)base + i) : -1;
    from[i] = target < 0 ? -1 : source;
    to[i] = target;
    if (i == 0) {
      rows = n;
      if (c.new_lens && slice == 0) c.new_lens[s] = base + n;
    }
  }
  __syncthreads();
  u32x4 r[UNITS];
  const int total = rows * c.n_heads * a.units;
  // unit x of the workgroup: which one of its head's, head and row
  auto place_of = [&](int x, int& i) {
    const int hr = a.unit.quotient(x);
    i = c.heads.quotient(hr);
    const int head = slice * c.n_heads + hr - i * c.n_heads;
    if (head >= 2 * a.hkv) i = -1;
    return (head >= a.hkv ? a.v + (head - a.hkv) * a.head_stride : a.k + head * a.head_stride) + (x - hr * a.units) * 16;
  };
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int x = threadIdx.x + u * COMPACT_THREADS;
    if (x < total) {
      int i;
      const char* p = place_of(x, i);
      if (i >= 0 && from[i] >= 0) r[u] = *reinterpret_cast<const u32x4*>(p + from[i]);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int u = 0; u < UNITS; ++u) asm volatile("" : "+v"(r[u]));  // they have arrived
  __syncthreads();
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    const int x = threadIdx.x + u * COMPACT_THREADS;
    if (x >= total) continue;
    int i;
    char* p = place_of(x, i);
    if (i >= 0 && from[i] >= 0) *reinterpret_cast<u32x4*>(p + to[i]) = r[u];
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
__device__ __forceinline__ bool proper(const PoolArgs& a, int src, int dst) { return src >= 0 && src < a.n_seqs && dst >= 0 && dst < a.n_seqs && src != dst; }

// Who may write a sequence: claims[s] becomes the first pair whose dst it is, or -1 if it is some pair's src.
__device__ __forceinline__ void claim(int32_t* claims, int src, int dst, int i) {
  atomicMin(claims + dst, i);
  atomicMin(claims + src, -1);
}
__device__ __forceinline__ Pair whole_pair(const PoolArgs& a, int src, int dst) {
  const int len = kept_length(a.lens[src], a.capacity), whole = a.page.quotient(len);
  return Pair{src, dst, whole, len - whole * a.page_size};
}
__device__ __forceinline__ Pair pair_of(const PoolArgs& a, int i) {
  const int src = a.src[i], dst = a.dst[i];
  return proper(a, src, dst) && a.claims[dst] == i ? whole_pair(a, src, dst) : Pair{-1, -1, 0, 0};
}

// An entry of the table: dst's page back, src's whole one shared
__device__ __forceinline__ void share(const PoolArgs& a, const Pair& p, int column) {
  int32_t* entry = a.table + (int64_t)p.dst * a.table_width + column;
  const int had = *entry, gets = column < p.whole ? a.table[(int64_t)p.src * a.table_width + column] : -1;
  if (had == gets) return;
  const int out = valid_page(had, a.n_pages), in = valid_page(gets, a.n_pages);
  if (out >= 0) atomicSub(a.refs + out, 1);
  if (in >= 0) atomicAdd(a.refs + in, 1);
  *entry = gets;
}

__global__ __launch_bounds__(THREADS) void unclaimed_kernel(PoolArgs a) {
  const int s = blockIdx.x * THREADS + threadIdx.x;
  if (s < a.n_seqs) a.claims[s] = INT_MAX;
}
__global__ __launch_bounds__(THREADS) void claim_kernel(PoolArgs a) {
  const int i = blockIdx.x * THREADS + threadIdx.x;
  if (i < a.n && proper(a, a.src[i], a.dst[i])) claim(a.claims, a.src[i], a.dst[i], i);
}
__global__ __launch_bounds__(THREADS) void share_kernel(PoolArgs a) {
  const int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (x >= (int64_t)a.n * a.table_width) return;
  const int i = (int)(x / a.table_width);
  const Pair p = pair_of(a, i);
  if (p.src >= 0) share(a, p, (int)(x - (int64_t)i * a.table_width));
}

// This thread's part of a sum in front of it, and the sum of all (GIVE_THREADS threads).
template <typename N>
__device__ __forceinline__ N sum_before(N mine, N& all) {
  __shared__ N waves[GIVE_THREADS / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  N upto = mine;
  for (int d = 1; d < 64; d <<= 1) {
    const N other = __shfl_up(upto, d, 64);
    if (lane >= d) upto += other;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  N before = upto - mine;
  all = 0;
  for (int w = 0; w < GIVE_THREADS / 64; ++w) {
    if (w < wave) before += waves[w];
    all += waves[w];
  }
  return before;
}

// Which of a thread's run of pages are free, a bit to each, from page p on.
constexpr int PER = 16;
__device__ __forceinline__ uint32_t free_pages(const PoolArgs& a, int64_t p) {
  struct __attribute__((packed, aligned(4))) Run {
    int32_t v[PER];
  };
  uint32_t free = 0;
  if (p + PER <= a.n_pages) {
    const Run run = *reinterpret_cast<const Run*>(a.refs + p);
#pragma unroll
    for (int e = 0; e < PER; ++e) free |= (uint32_t)(run.v[e] == 0) << e;
  } else {
    for (int e = 0; e < PER; ++e)
      if (p + e < a.n_pages) free |= (uint32_t)(a.refs[p + e] == 0) << e;
  }
  return free;
}

// The `wanted` lowest free pages into list (the first LIST of them also into list_lds), counted as in use; how many there were.
// free: those of the thread's first run, where they have been read already.
constexpr int LIST = 1024;
__device__ __forceinline__ int take_pages(const PoolArgs& a, int wanted, uint32_t free, int32_t* list_lds) {
  int found = 0;
  for (int64_t p0 = 0; p0 < a.n_pages && found < wanted; p0 += GIVE_THREADS * PER) {
    const int64_t p = p0 + threadIdx.x * PER;
    if (p0) free = free_pages(a, p);
    int all;
    int rank = found + sum_before<int>(__popc(free), all);
    for (; free && rank < wanted; free &= free - 1, ++rank) {
      const int page = (int)(p + __ffs(free) - 1);
      if (rank < LIST) list_lds[rank] = page;
      else a.list[rank] = page;
      a.refs[page] = 1;
    }
    found += all;
  }
  if (found > LIST && wanted > LIST) __syncthreads();
  else lds_barrier();
  return found < wanted ? found : wanted;
}

// One workgroup: a page for every fork whose source has begun one (counts[i]: the page, -1 for none, -2 for a pair that is left out).
// ALL, for small tables: it also finds who is written and shares the whole pages, a chain of six trips to the memory where kernels of
// their own take eleven (256 sequences of 67 entries, 64 forks: 8.7 us, with two kernels that look for no double dst 3.2 + 5.2 and a gap).
constexpr int WHOLE_ENTRIES = 32 * GIVE_THREADS, WHOLE_SEQS = 2048;
template <bool ALL>
__global__ __launch_bounds__(GIVE_THREADS) void fork_pages_kernel(PoolArgs a) {
  __shared__ int32_t claims[ALL ? WHOLE_SEQS : 1];
  __shared__ Pair pairs[ALL ? WHOLE_SEQS : 1];
  __shared__ int32_t list[LIST];
  if constexpr (ALL) {
    for (int s = threadIdx.x; s < a.n_seqs; s += GIVE_THREADS) claims[s] = INT_MAX;
    lds_barrier();
    for (int i = threadIdx.x; i < a.n; i += GIVE_THREADS) {
      const int src = a.src[i], dst = a.dst[i];
      const bool is = proper(a, src, dst);
      if (is) claim(claims, src, dst, i);
      pairs[i] = is ? whole_pair(a, src, dst) : Pair{-1, -1, 0, 0};
    }
    lds_barrier();
    for (int i = threadIdx.x; i < a.n; i += GIVE_THREADS)
      if (pairs[i].src >= 0 && claims[pairs[i].dst] != i) pairs[i].src = -1;
    lds_barrier();
    const int entries = a.n * a.table_width;
#pragma unroll 4
    for (int x = threadIdx.x; x < entries; x += GIVE_THREADS) {
      const int i = a.width.quotient(x);
      if (pairs[i].src >= 0) share(a, pairs[i], x - i * a.table_width);
    }
    __syncthreads();
  }
  auto pair = [&](int i) {
    if constexpr (ALL) return pairs[i];
    else return pair_of(a, i);
  };
  const uint32_t free = free_pages(a, threadIdx.x * PER);
  int wanted = 0;
  for (int i0 = 0; i0 < a.n; i0 += GIVE_THREADS) {
    const int i = i0 + threadIdx.x;
    int wants = 0, all;
    Pair p{-1, -1, 0, 0};
    if (i < a.n) {
      p = pair(i);
      wants = p.src >= 0 && p.begun && valid_page(a.table[(int64_t)p.src * a.table_width + p.whole], a.n_pages) >= 0;
    }
    const int rank = wanted + sum_before<int>(wants, all);
    if (i < a.n) a.counts[i] = wants ? rank : p.src < 0 ? -2 : -1;
    wanted += all;
  }
  const int had = take_pages(a, wanted, free, list);
  if (a.missing && threadIdx.x == 0) *a.missing = wanted - had;
  for (int i = threadIdx.x; i < a.n; i += GIVE_THREADS) {  // (a thread's own counts)
    const int rank = a.counts[i];
    if (rank < 0) continue;
    const int page = rank >= had ? -1 : rank < LIST ? list[rank] : a.list[rank];
    a.counts[i] = page;
    const Pair p = pair(i);
    if (page >= 0) a.table[(int64_t)p.dst * a.table_width + p.whole] = page;
  }
}

// The begun pages' places, `blocks` workgroups to a fork; then dst has src's length
__global__ __launch_bounds__(THREADS) void copy_kernel(PoolArgs a) {
  const int i = blockIdx.x / a.blocks, to = a.counts[i], src = a.src[i], dst = a.dst[i];
  if (to == -2) return;
  if (blockIdx.x % a.blocks == 0 && threadIdx.x == 0) a.lens[dst] = a.lens[src];
  if (to < 0) return;
  const Pair p = whole_pair(a, src, dst);
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

// One workgroup: where every sequence's pages begin in the list, and the list.  (The counts 16384 at a time: 1024 sequences of 128 entries over
// 140000 pages 23 us in all three kernels, 4096 of 64 over 300000 48.)
__global__ __launch_bounds__(GIVE_THREADS) void reserve_pages_kernel(PoolArgs a) {
  __shared__ int32_t list[LIST];
  const uint32_t free = free_pages(a, threadIdx.x * PER);
  int64_t wanted = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += GIVE_THREADS) {
    const int s = s0 + threadIdx.x;
    int64_t all;  // (of a thousand tables of two million entries each: beyond int32)
    const int64_t rank = wanted + sum_before<int64_t>(s < a.n_seqs ? a.counts[s] : 0, all);
    if (s < a.n_seqs) a.counts[s] = (int)(rank < a.n_pages ? rank : a.n_pages);
    wanted += all;
  }
  const int asked = (int)(wanted < a.n_pages ? wanted : a.n_pages), had = take_pages(a, asked, free, list);
  for (int i = threadIdx.x; i < (had < LIST ? had : LIST); i += GIVE_THREADS) a.list[i] = list[i];
  if (threadIdx.x == 0) {
    a.counts[a.n_seqs] = had;
    if (a.missing) *a.missing = (int)(wanted - had < INT_MAX ? wanted - had : INT_MAX);
  }
}

__global__ __launch_bounds__(THREADS) void fill_kernel(PoolArgs a) {
  const int s = blockIdx.x * (THREADS / 64) + threadIdx.x / 64, lane = threadIdx.x & 63;
  if (s >= a.n_seqs) return;
  const int columns = columns_wanted(a, s), had = a.counts[a.n_seqs];
  int64_t rank = a.counts[s];
  for (int c0 = 0; c0 < columns; c0 += 64) {
    const int c = c0 + lane;
    int32_t* entry = a.table + (int64_t)s * a.table_width + c;
    const bool lacks = c < columns && valid_page(*entry, a.n_pages) < 0;
    const unsigned long long all = __ballot(lacks);
    const int64_t at = rank + __popcll(all & ((1ull << lane) - 1));
    if (lacks) *entry = at < had ? a.list[at] : -1;
    rank += __popcll(all);
  }
}

// The three kernels above in one, of small tables: a run of entries to a wavefront, 64 at a time, AHEAD of these in flight, in the order in
// which pages are given (256 sequences of 67 entries: 9.8 us, the three 3.0 + 4.1 + 3.4 and two gaps).
__global__ __launch_bounds__(GIVE_THREADS) void reserve_kernel(PoolArgs a) {
  constexpr int WAVES = GIVE_THREADS / 64, TURNS = WHOLE_ENTRIES / GIVE_THREADS, AHEAD = 8;
  __shared__ int columns[WHOLE_SEQS + 1];
  __shared__ int32_t list[LIST];
  __shared__ int lacking[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int entries = a.n_seqs * a.table_width, turns = (entries + GIVE_THREADS - 1) / GIVE_THREADS, begin = wave * turns * 64;
  const unsigned n_pages = a.n_pages < INT_MAX ? (unsigned)a.n_pages : (unsigned)INT_MAX;
  const uint32_t free = free_pages(a, threadIdx.x * PER);
  int entry[AHEAD];
  auto load = [&](int u0) {
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const int x = begin + (u0 + e) * 64 + lane;
      entry[e] = a.table[x < entries ? x : entries - 1];
    }
  };
  if (turns > 0) load(0);
  for (int s = threadIdx.x; s <= a.n_seqs; s += GIVE_THREADS) columns[s] = s < a.n_seqs ? columns_wanted(a, s) : 0;
  lds_barrier();
  // (a turn later an entry's sequence and column are these further on; those beyond the last entry are of no sequence)
  const int seqs = a.width.quotient(64), rest = 64 - seqs * a.table_width;
  int s = a.width.quotient(begin + lane), column = begin + lane - s * a.table_width, n = 0;
  uint32_t lacks = 0;
  for (int u0 = 0; u0 < turns; u0 += AHEAD) {
    if (u0) load(u0);
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
      const bool lack = u0 + e < turns && column < columns[s < a.n_seqs ? s : a.n_seqs] && (unsigned)entry[e] >= n_pages;
      lacks |= (uint32_t)lack << (u0 + e);
      n += __popcll(__ballot(lack));
      s += seqs;
      column += rest;
      const bool next = column >= a.table_width;
      s += next;
      column -= next ? a.table_width : 0;
    }
  }
  if (lane == 0) lacking[wave] = n;
  lds_barrier();
  int rank = 0, wanted = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    rank += w < wave ? lacking[w] : 0;
    wanted += lacking[w];
  }
  const int asked = wanted < a.n_pages ? wanted : (int)a.n_pages, had = take_pages(a, asked, free, list);
  if (a.missing && threadIdx.x == 0) *a.missing = wanted - had;
  for (int u = 0; n && u < turns; ++u) {
    const unsigned long long all = __ballot(lacks >> u & 1);
    const int mine = rank + __popcll(all & ((1ull << lane) - 1));
    if (lacks >> u & 1) a.table[begin + u * 64 + lane] = mine >= had ? -1 : mine < LIST ? list[mine] : a.list[mine];
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
  if (ws) {
    const size_t seqs = align_up(((size_t)c->n_seqs + 1) * sizeof(int32_t), 256);
    a.claims = (int32_t*)((char*)ws + seqs);
    a.list = (int32_t*)((char*)ws + 2 * seqs);
  }
  a.n_pages = c->n_pages;
  a.page_stride = c->page_stride * es;
  a.token_stride = c->token_stride * es;
  a.head_stride = c->head_stride * es;
  a.page = page_divisor(c->page_size);
  a.units = (int)(c->head_dim * es / 16);
  a.unit = page_divisor(a.units);
  a.width = page_divisor(c->table_width > 0 ? c->table_width : 1);
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
  // (a workgroup writes a sequence's new length while others read the next ones' base)
  if (new_lens && new_lens < base + c->n_seqs && base < new_lens + c->n_seqs)
    return fail(MOE_ERR_INVALID_ARG, "moe_kv_compact: new_lens must not overlap base");
  CompactArgs a{};
  a.pool = pool_of(c, nullptr, nullptr);
  a.base = base;
  a.keep = keep;
  a.new_lens = new_lens;
  a.width = width;
  // heads of a workgroup: what its threads' registers hold, unless that leaves the machine idle
  const int per_head = width * a.pool.units, both = 2 * c->n_kv_heads;
  int heads = MOST_UNITS * COMPACT_THREADS / per_head;
  while (heads > 1 && (int64_t)c->n_seqs * ((both + heads - 1) / heads) < 1024) heads = (heads + 1) / 2;
  a.n_heads = heads < both ? heads : both;
  a.n_slices = (both + a.n_heads - 1) / a.n_heads;
  a.heads = page_divisor(a.n_heads);
  a.slices = page_divisor(a.n_slices);
  const int64_t grid = (int64_t)c->n_seqs * a.n_slices;
  if (!launchable(grid, COMPACT_THREADS))
    return fail(MOE_ERR_UNSUPPORTED, "moe_kv_compact: %d sequences of %d kv heads are too many for one call", c->n_seqs, c->n_kv_heads);
  const int units = (per_head * a.n_heads + COMPACT_THREADS - 1) / COMPACT_THREADS;
  hipStream_t st_ = (hipStream_t)stream;
  if (units <= 1) hipLaunchKernelGGL(compact_kernel<1>, dim3((unsigned)grid), dim3(COMPACT_THREADS), 0, st_, a);
  else if (units <= 4) hipLaunchKernelGGL(compact_kernel<4>, dim3((unsigned)grid), dim3(COMPACT_THREADS), 0, st_, a);
  else hipLaunchKernelGGL(compact_kernel<MOST_UNITS>, dim3((unsigned)grid), dim3(COMPACT_THREADS), 0, st_, a);
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
  return 2 * align_up(((size_t)c->n_seqs + 1) * sizeof(int32_t), 256) + align_up((size_t)c->n_pages * sizeof(int32_t), 256);
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
  if (n == 0 && !missing) return MOE_OK;
  if (entries <= WHOLE_ENTRIES && c->n_seqs <= WHOLE_SEQS) {
    hipLaunchKernelGGL(fork_pages_kernel<true>, dim3(1), dim3(GIVE_THREADS), 0, s, a);
  } else {
    hipLaunchKernelGGL(unclaimed_kernel, dim3((unsigned)grid_of(c->n_seqs, THREADS)), dim3(THREADS), 0, s, a);
    st = check_hip(hipGetLastError(), "fork launch");
    if (st != MOE_OK) return st;
    if (n > 0) {
      hipLaunchKernelGGL(claim_kernel, dim3((unsigned)grid_of(n, THREADS)), dim3(THREADS), 0, s, a);
      st = check_hip(hipGetLastError(), "fork launch");
      if (st != MOE_OK) return st;
    }
    if (entries > 0) {
      hipLaunchKernelGGL(share_kernel, dim3((unsigned)grid_of(entries, THREADS)), dim3(THREADS), 0, s, a);
      st = check_hip(hipGetLastError(), "fork launch");
      if (st != MOE_OK) return st;
    }
    hipLaunchKernelGGL(fork_pages_kernel<false>, dim3(1), dim3(GIVE_THREADS), 0, s, a);
  }
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
  if (c->n_seqs <= WHOLE_SEQS && (int64_t)c->n_seqs * c->table_width <= WHOLE_ENTRIES) {
    hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(GIVE_THREADS), 0, s, a);
    return check_hip(hipGetLastError(), "reserve launch");
  }
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
