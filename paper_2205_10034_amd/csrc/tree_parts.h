// What the kernels of the attention of drafted tokens share: their arguments, how a batch is dealt out to workgroups, and how a row ends.
#pragma once
#include "attention_internal.h"
#include "draft_tokens.h"
#include "wave_util.h"
#include <float.h>
#include <math.h>
#include <type_traits>

namespace moesys {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct TreeArgs {
  const char *k, *v, *q;
  char* out;
  float* lse;
  const int32_t *table, *lens, *first;
  const uint64_t* words;
  const float* slopes;
  float* part_o;   // [slot][items][rows][D]
  f32x2* part_ml;  // [slot][items][rows]: maximum and sum
  int2* plan;      // [row tile][sequence]: slot of the first piece, pieces
  int64_t n_pages, page_stride, token_stride, head_stride, q_token, q_head, o_token, o_head;  // bytes
  PageDivisor page, kv_heads, group;  // places of a page, kv heads, query heads of a kv head
  double inverse_parts;
  int32_t last_column;  // of the table; 0 also of one without columns, where `table` is some other memory whose entries nobody uses
  int32_t page_size, table_width, capacity, n_seqs, hq, hkv, G, T, max_new, D, window, sinks, rows, items, row_tiles, parts, may_split, small;  // small: sequences up to this length are not split where there is a workgroup for each
  float scale, cap, inv_cap;
};

namespace {

constexpr int WAVES = 4;
// How far a score may pass the running maximum before the maximum moves (a little less than 8 log 2); weights are scaled down by 2^8.
constexpr int LAG_BITS = 8;
constexpr float LAG = 5.5f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Rows of places that are not there and dimensions beyond head_dim are read from here.
__device__ const u32x4 ZEROS[MOE_MAX_HEAD_DIM * 4 / 16] = {};

__device__ __forceinline__ Drafts drafts(const TreeArgs& a, int s) { return drafts_of(a.first[s], a.first[s + 1], a.T, a.max_new, a.lens[s], a.capacity); }

// A value that all lanes hold, for the scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// How the workgroups of an item share the batch: its sequences' tiles stand in one row, of which part w has w*share .. (w+1)*share - 1.
struct Deal {
  int64_t share, total, begin;  // of a part, of the row; where in the row sequence b begins
  int b;                        // the part's first sequence
  bool one_each;                // the row counts sequences, none is split
};

// Places in the row of sequence s, whose row tile rt may have no rows.
template <int TILE>
__device__ __forceinline__ int places_in_row(const TreeArgs& a, int s, int rt, int& tiles) {
  const Drafts d = drafts(a, s);
  tiles = span_of(d, a.window, a.sinks, TILE).tiles;
  return rt * a.rows < d.n * a.G ? (int)row_tiles(tiles) : 0;
}

// LEAST: tiles of a part, at least.
template <int TILE, int LEAST>
__device__ __forceinline__ Deal deal(const TreeArgs& a, int rt, int w) {
  const int lane = threadIdx.x & 63;
  Deal p{};
  if (!a.may_split) {
    p.one_each = true;
    p.share = share_of_row(a.n_seqs, a.inverse_parts, 1);
    p.total = a.n_seqs;
    p.begin = w * p.share;
    p.b = (int)p.begin;
    return p;
  }
  int longest = 0, tiles = 0;
  int64_t total = 0, mine0 = 0;
  for (int s = lane; s < a.n_seqs; s += 64) {
    const int mine = places_in_row<TILE>(a, s, rt, tiles);
    if (s == lane) mine0 = mine;
    total += mine;
    longest = tiles > longest ? tiles : longest;
  }
  if (a.n_seqs <= a.parts && !__any(longest > a.small / TILE)) {
    p.one_each = true;
    p.share = 1;
    p.total = a.n_seqs;
    p.begin = p.b = w;
    return p;
  }
  for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d, 64);
  p.total = uniform(total, 0);
  p.share = uniform(share_of_row(p.total, a.inverse_parts, LEAST), 0);
  const int64_t at = w * p.share;
  int64_t mine = mine0;
  for (int s = 0; s < a.n_seqs; s += 64) {
    if (s) mine = s + lane < a.n_seqs ? places_in_row<TILE>(a, s + lane, rt, tiles) : 0;
    int64_t upto = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t other = __shfl_up(upto, d, 64);
      if (lane >= d) upto += other;
    }
    const unsigned long long beyond = __ballot(p.begin + upto > at);
    if (beyond) {
      const int who = __ffsll(beyond) - 1;
      p.b = s + who;
      p.begin += uniform(upto - mine, who);
      return p;
    }
    p.begin += uniform(upto, 63);
  }
  p.total = 0;  // nothing is left for this part
  return p;
}

// exp(x), the last step a power of two
__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

// Of a pair of bfloat16 numbers, those that are infinite or NaN: 1.0 in their place, 0 elsewhere.
__device__ __forceinline__ uint32_t not_finite(uint32_t v) {
  return ((v & 0x7f80u) == 0x7f80u ? 0x3f80u : 0u) | ((v & 0x7f800000u) == 0x7f800000u ? 0x3f800000u : 0u);
}
__device__ __forceinline__ float not_finite(float v) { return fabsf(v) < INFINITY ? 0.f : 1.f; }

// Four finished elements of a row; the first four bring the row's lse along.
template <typename X>
__device__ __forceinline__ void store_row(const TreeArgs& a, int t, int h, int d, f32x4 y, float sum, float top) {
  if (sum == 0.f) y = f32x4{0.f, 0.f, 0.f, 0.f};
  else y *= 1.f / sum;
  char* p = a.out + (int64_t)t * a.o_token + (int64_t)h * a.o_head + d * sizeof(X);
  if constexpr (sizeof(X) == 2) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(p) = y;
  if (a.lse && d == 0) a.lse[(int64_t)t * a.hq + h] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum * (1 << LAG_BITS)) * LN2;
}

}  // namespace

// Calls of bfloat16 with more than SHARED_FROM rows of tokens and query heads to a kv head: keys and values reach the wavefronts through LDS
// (attention_tree_shared.hip).
constexpr int SHARED_FROM = 32;
constexpr int shared_blocks(int rows, int dims) { return rows > 64 && dims <= 128 ? 2 : 1; }  // 16 rows each of a wavefront
constexpr int shared_tile(int dims, int blocks) { return dims * blocks <= 64 ? 64 : 32; }    // places that a workgroup takes at a time
constexpr int shared_least(int dims, int blocks) { return 256 / shared_tile(dims, blocks); }  // tiles of a part, at least
int32_t launch_tree_shared(const TreeArgs& a, int blocks, unsigned grid, bool nt, hipStream_t s);

}  // namespace moesys
