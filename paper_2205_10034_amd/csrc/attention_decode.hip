// Attention of one new token per sequence over a paged cache (moe_attention_decode): one pass over the keys and values
// with the running maximum m and sum l of the softmax,
//   m' = max(m, z_j);  l' = l exp(m - m') + exp(z_j - m');  o' = o exp(m - m') + exp(z_j - m') v_j;  out = o / l,
// split over the length into pieces whose (m, l, o) are joined at the end with the weights exp(m_i - max m).
//
// Bound: HBM, every key and value once; the arithmetic is G = query heads per kv head multiply-adds per element.  So the kernel
// is built around loads that go from memory into the registers that the matrix instructions read:
//  - A wavefront takes tiles of 32 places (16 in float32, and beyond 128 dimensions, where registers are short) and the up to 16
//    query heads of one kv head.
//  - Scores: S^T[place, head] = K Q^T, keys as the first operand.  The contraction index of an instruction may be any permutation
//    of the dimensions as long as both operands use it.  A load brings eight keys' whole 128-byte lines: rows 0-7 of the operand
//    are those keys' first half lines and rows 8-15 their second ones, so each operand is multiplied with both halves of the
//    queries and half of each product is used.  (16 half lines per load, which need no second product, read 1.3 GB in 250 us;
//    whole ones in 232, and only they gain from loads past the caches.)
//  - Output: O^T[dim, head] += V^T P^T.  A lane of S^T holds four places of one head, which is how the second operand wants P^T
//    when the places of an instruction are taken in that order: no data moves between lanes.  The first operand has to hold eight
//    places of one dimension: a lane loads the same EPL dimensions of those places and pairs the halves with one v_perm per four
//    bytes, row m of the instruction standing for dimension m*EPL + j in the j-th of EPL products.
//  - Keys of the next tile are requested when this tile's scores are formed, values when its output is: one kind of loads is in
//    flight while the other is used, and the other wavefronts of the CU hide the rest.
//  - All sequences' tiles stand in one row that the resident workgroups share evenly (Deal): no last round, no long sequence that
//    the others wait for.
// Measured: 256 sequences of 2048 to 14336 places, 64 query and 8 kv heads of 128 (8.5 GB of keys and values) 1262 us, 6.7 TB/s; 64 of
// 100 to 8192 (1.3 GB) 201 us, 6.5 TB/s; one of 131071 (0.54 GB) 88 us, of which the join takes 5; one of 173, 16 heads of 64: 7 us,
// four dependent trips to memory, and 10 with a page table of 1000 more columns, which alone decide whether the join is launched.
#include "attention_internal.h"
#include "wave_util.h"
#include <float.h>
#include <math.h>

namespace moesys {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4;
constexpr int HEADS = 16;  // query heads of a tile
// Tiles of a part for each of its wavefronts, at least: 8 sequences of 100 to 1500 places take 15.9 us with 2 or 1 and 16.8 with 4, 150 of
// up to 300 31.6, 31.7 and 33.9 (fewer CUs at work).
constexpr int LEAST_PER_WAVE = 2;
// Joins of so many rows take a wavefront each: of 16384 rows, with the attention before them, 1261 us, 1269 with a workgroup each; of 8192
// 172 and 178.
constexpr int MANY_ROWS = 1024;
// Sequences that are not split.  None longer than TINY_PLACES: a piece's four trips to memory are all there is, so the fewest rounds
// of workgroups count (292 sequences of one place, 16 heads of 192: 19 us; shared evenly, 9 pieces one after the other per
// workgroup, 36).  None longer than SMALL_PLACES, and a workgroup for each: the join would cost more than it saves (one of 173
// places 7.7 us and 12.2, 16 of up to 1000 places 15.5 and 18.3, 512 of up to 700 128 and 144; 256 of up to 2000 are better shared,
// 172 against 197).
constexpr int TINY_PLACES = 128, SMALL_PLACES = 1024;
// How far a score may pass the running maximum before the maximum moves (a little less than 8 log 2); weights are scaled down by 2^8.
constexpr int LAG_BITS = 8;
constexpr float LAG = 5.5f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Rows of places that are not there and dimensions beyond head_dim are read from here: no load leaves the caller's rows, and what
// lies in places that are not kept reaches no product.
__device__ const u32x4 ZEROS[MOE_MAX_HEAD_DIM * 4 / 16] = {};

// Workgroups of the decode kernel that a CU holds: two need up to 256 registers a lane, which keys and values on their way leave room
// for; a third or a fourth costs registers for what is in flight (64 sequences, 1.3 GB: 210 us with two, 237 with three).  256 dimensions
// of float32 need more than 256 (0.5 GB: 100 us with one, 163 with two, which spill); of bfloat16, in tiles of 16 places, they do not
// (96 sequences with a window 44.3 us with two, 44.7 with one).
constexpr int resident_workgroups(int dims, int elem) { return dims <= 128 || elem == 2 ? 2 : 1; }

struct DecodeArgs {
  const char *k, *v, *q;
  char* out;
  float* lse;
  const int32_t *table, *lens;
  const float* slopes;
  float* part_o;   // [slot][items][rows][D]
  f32x2* part_ml;  // [slot][items][rows]
  int2* plan;      // [sequence]: slot of the first piece, pieces
  int64_t n_pages, page_stride, token_stride, head_stride, q_token, q_head, o_token, o_head;  // bytes
  PageDivisor page, per_kv_head, per_rows;  // places of a page, items of a kv head, rows of an item
  struct {
    PageDivisor per_part;  // workgroups of a part
    int32_t parts;
    double inverse_parts;
  } share_of_grid[3];  // with 1, 2 and 4 items a workgroup
  int32_t page_size, table_width, capacity, n_seqs, hq, G, rows, items, hts, log_heads, parts, may_split, D, window, least;
  float scale, cap, inv_cap;
};

template <typename X, int DP> struct Shape;
template <int DP> struct Shape<__bf16, DP> {
  static constexpr int SUB = DP <= 128 ? 2 : 1, EPL = DP < 128 ? 4 : 8, KSTEPS = DP / 32;
};
template <int DP> struct Shape<float, DP> {
  static constexpr int SUB = 1, EPL = 4, KSTEPS = DP / 16;
};

template <int BYTES> struct Words;
template <> struct Words<8> { typedef u32x2 type; };
template <> struct Words<16> { typedef u32x4 type; };

// How many of the neighbouring items, 2 to the power of what comes back, one workgroup takes so that the `rows` fit `grid`
// workgroups, if they can.
__device__ __forceinline__ int side_by_side(int items, int64_t rows, int64_t grid) {
  return rows <= grid || items % 2 ? 0 : rows <= 2 * grid || items % 4 ? 1 : 2;
}

// A value that all lanes hold, for the scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = __builtin_amdgcn_readlane((int)(v >> 32), lane);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}

// How the workgroups share the batch, from its lengths, and this one's part of it.  Every wavefront finds it by itself.
struct Deal {
  int log_heads, first_item, w;  // items of a workgroup (their logarithm), the first of them, the part
  bool one_each;              // the row counts sequences, not tiles: no sequence is split
  bool aligned;               // every sequence begins a part
  int64_t share, total;       // of a part, of the row
  int64_t begin;              // where in the row sequence b begins
  int b, len;                 // the part's first sequence, its length
};

__device__ __forceinline__ Deal deal(const DecodeArgs& a, int tile) {
  const int lane = threadIdx.x & 63, id = blockIdx.x;
  auto tiles_in = [&](int len) {
    const int n = kept_length(len, a.capacity);
    return kept_tiles(n, first_place(n, a.window), tile);
  };
  const int64_t rows = (int64_t)a.n_seqs * a.items, grid = gridDim.x;
  Deal p{};
  auto take = [&](int log_heads) {
    p.log_heads = log_heads;
    p.w = a.share_of_grid[log_heads].per_part.quotient(id);
    p.first_item = (id - p.w * (a.items >> log_heads)) << log_heads;
  };
  auto whole = [&] {
    take(side_by_side(a.items, rows, grid));
    const auto& g = a.share_of_grid[p.log_heads];
    p.one_each = true;
    p.share = share_of_row(a.n_seqs, g.inverse_parts, 1);
    p.total = a.n_seqs;
    p.begin = p.w * p.share;
    p.b = (int)p.begin;
    if (p.begin < p.total) p.len = a.lens[p.b];
    return p;
  };
  if (!a.may_split) return whole();
  int len = lane < a.n_seqs ? a.lens[lane] : 0, longest = tiles_in(len);
  int64_t mine = lane < a.n_seqs ? row_tiles(longest) : 0, total = mine;
  for (int s = lane + 64; s < a.n_seqs; s += 64) {
    const int t = tiles_in(a.lens[s]);
    longest = t > longest ? t : longest;
    total += row_tiles(t);
  }
  const bool tiny = !__any(longest > TINY_PLACES / tile), small = !__any(longest > SMALL_PLACES / tile);
  if (tiny || (small && rows <= grid)) return whole();
  for (int d = 1; d < 64 && d < a.n_seqs; d <<= 1) total += __shfl_xor(total, d, 64);
  p.total = uniform(total, 0);
  take(a.log_heads);
  p.share = uniform(share_of_row(p.total, a.share_of_grid[p.log_heads].inverse_parts, a.least >> p.log_heads), 0);
  // A piece costs its trips to memory, about what a tile of every wavefront costs where all of them read: for up to that much a
  // part, sequences begin parts of their own and no part holds two pieces.
  if (a.n_seqs > 1 && a.n_seqs < a.share_of_grid[p.log_heads].parts) {
    const int64_t wider = uniform(share_of_row(p.total, 1.0 / (a.share_of_grid[p.log_heads].parts - a.n_seqs), a.least >> p.log_heads), 0);
    p.aligned = wider - p.share <= (WAVES >> p.log_heads);
    if (p.aligned) p.share = wider;
  }
  const int64_t at = p.w * p.share;
  for (int s = 0; s < a.n_seqs;) {
    if (p.aligned) mine = aligned_tiles(mine, p.share);
    int64_t upto = mine;
    for (int d = 1; d < 64 && d < a.n_seqs; d <<= 1) {
      const int64_t other = __shfl_up(upto, d, 64);
      if (lane >= d) upto += other;
    }
    const unsigned long long beyond = __ballot(p.begin + upto > at);
    if (beyond) {
      const int who = __ffsll(beyond) - 1;
      p.b = s + who;
      p.len = __builtin_amdgcn_readlane(len, who);
      p.begin += uniform(upto - mine, who);
      if (p.aligned) p.total = at + p.share;  // (this part's end will do)
      return p;
    }
    p.begin += uniform(upto, 63);
    s += 64;
    len = s + lane < a.n_seqs ? a.lens[s + lane] : 0;
    mine = s + lane < a.n_seqs ? row_tiles(tiles_in(len)) : 0;
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

// Addresses that come out of LDS are global ones: told so, the compiler reads them with loads that the waits for LDS do not wait for.
template <bool NT, typename W>
__device__ __forceinline__ W read(const char* p) {
  const auto* at = (const __attribute__((address_space(1))) W*)(uintptr_t)p;
  if constexpr (NT) return __builtin_nontemporal_load(at);
  else return *at;
}

// acc + a b for 16 bytes of contraction index per lane and operand
template <bool BF16>
__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, f32x4 acc) {
  if constexpr (BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), acc, 0, 0, 0);
    return acc;
  }
}

// acc + a b over the places of a tile, 8 (two subtiles) or 4 of them per lane as pairs of bfloat16
template <int SUB>
__device__ __forceinline__ f32x4 weighted(const uint32_t (&a)[2 * SUB], const uint32_t (&b)[2 * SUB], f32x4 acc) {
  if constexpr (SUB == 2)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, (u32x4{a[0], a[1], a[2], a[3]})), __builtin_bit_cast(bf16x8, (u32x4{b[0], b[1], b[2], b[3]})), acc, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(i16x4, (u32x2{a[0], a[1]})), __builtin_bit_cast(i16x4, (u32x2{b[0], b[1]})), acc, 0, 0, 0);
}

// What the lane 32 away holds.
__device__ __forceinline__ float other_half(float x, int lane) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(lane < 32 ? both[1] : both[0]);
}

// Four finished elements of a head; the first four bring the head's lse along.
template <typename X>
__device__ __forceinline__ void store_row(const DecodeArgs& a, int b, int h, int d, f32x4 y, float sum, float top) {
  if (sum == 0.f) y = f32x4{0.f, 0.f, 0.f, 0.f};
  else y *= 1.f / sum;
  char* p = a.out + (int64_t)b * a.o_token + (int64_t)h * a.o_head + d * sizeof(X);
  if constexpr (sizeof(X) == 2) *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
  else *reinterpret_cast<f32x4*>(p) = y;
  if (a.lse && d == 0) a.lse[(int64_t)b * a.hq + h] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum * (1 << LAG_BITS)) * LN2;
}

// A part of the batch per workgroup, piece after piece; its wavefronts take an item's tiles in turn.  An item is a kv head and up to 16
// of its query heads.
// FULL: head_dim is DP, no lane's dimensions lie beyond it.
template <typename X, int DP, bool FULL, bool NT>
__global__ __launch_bounds__(64 * WAVES, resident_workgroups(DP, sizeof(X))) void decode_kernel(DecodeArgs a) {
  using S = Shape<X, DP>;
  constexpr bool BF16 = sizeof(X) == 2;
  constexpr int SUB = S::SUB, TILE = 16 * SUB, EPL = S::EPL, KSTEPS = S::KSTEPS, LINES = KSTEPS / 2, NV = 4 * SUB, BD = 16 * EPL, NBLK = DP / BD, PITCH = BD + 4;
  constexpr uint32_t EVERY = (uint32_t)((1ull << TILE) - 1);
  using VWord = typename Words<EPL * sizeof(X)>::type;
  extern __shared__ __attribute__((aligned(16))) float o_lds[];  // [WAVES][rows][PITCH]
  __shared__ uint64_t row_at[WAVES][2][TILE];
  __shared__ f32x2 ml_lds[WAVES][HEADS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m16 = lane & 15, g = lane >> 4, line_at = (g + 4 * (m16 >> 3)) * 16;
  // wavefronts of a workgroup: wave_heads neighbouring items, `step` of them on the tiles of each in turn
  Deal at = deal(a, TILE);
  const int wave_heads = 1 << at.log_heads, w = at.w, step = WAVES >> at.log_heads;
  int64_t x = w * at.share;
  const int64_t x_end = x + at.share < at.total ? x + at.share : at.total;
  if (x >= x_end) return;
  const int item = at.first_item + (wave & (wave_heads - 1)), hk = a.per_kv_head.quotient(item), ht = item - hk * a.hts;
  auto heads_of = [&](int tile_of_heads) { return a.G - tile_of_heads * HEADS < HEADS ? a.G - tile_of_heads * HEADS : HEADS; };
  const int my_heads = heads_of(ht);
  const char* zeros = reinterpret_cast<const char*>(ZEROS);
  const char* base = (lane < 32 ? a.k : a.v) + hk * a.head_stride;  // lanes 0-31 place the keys' rows, the others the values'
  const int tp = lane & (TILE - 1);
  const bool plain = a.cap == 0.f && !a.slopes;
  const float slope = a.slopes && m16 < my_heads ? a.slopes[hk * a.G + ht * HEADS + m16] : 0.f;

  for (int piece_no = 0; x < x_end; ++piece_no) {
    // the piece of sequence b that lies in this part
    const int b = at.b;
    const int32_t* table = a.table + (int64_t)b * a.table_width;
    // the table's entry for this lane's place of tile tt; an entry of the table in any case
    auto entry_of = [&](int tt) {
      const unsigned column = (unsigned)a.page.quotient((int)((unsigned)tt * TILE + tp)), last = (unsigned)a.table_width - 1u;
      return table[column < last ? column : last];
    };
    const int from = (int)(x - at.begin), mine = from + (wave >> at.log_heads);
    // without a window the first tiles are known before the length is
    const bool early = a.window == 0 && a.table_width > 0;
    int now = -1, entry = -1;
    if (early) {
      now = entry_of(mine);
      entry = entry_of(mine + step);
    }
    const int n = kept_length(at.len, a.capacity), first = first_place(n, a.window), tile0 = first / TILE, tiles = kept_tiles(n, first, TILE);
    const int64_t b_end = at.begin + (at.one_each ? 1 : at.aligned ? aligned_tiles(row_tiles(tiles), at.share) : row_tiles(tiles));
    const int upto = b_end <= x_end ? tiles : (int)(x_end - at.begin);
    const bool whole = from == 0 && b_end <= x_end;
    const int slot = 2 * w + (piece_no > 0);
    if (from == 0 && threadIdx.x == 0 && item == 0) a.plan[b] = make_int2(slot, whole ? 1 : part_of(b_end - 1, at.share) - w + 1);
    const int t_end = tiles ? tile0 + upto : 0;
    int t = tile0 + mine;

    // Nothing in the loop that loads is conditional: what a tile beyond the last one would load is ZEROS.  (Behind a branch the
    // compiler waits for every load in flight before it uses the first.)
    auto is_kept = [&](int tt) {
      const int p = (int)((unsigned)tt * TILE + tp);
      return tt < t_end && p >= first && p < n;
    };
    // rows of tile tt into LDS; returns which places are kept
    auto place_rows = [&](int tt, int entry) {
      const int p = (int)((unsigned)tt * TILE + tp), page = is_kept(tt) ? valid_page(entry, a.n_pages) : -1;
      const int in_page = p - a.page.quotient(p) * a.page_size;
      const char* row = page >= 0 ? base + page * a.page_stride + in_page * a.token_stride : zeros;
      if (TILE == 32 || (lane & 16) == 0) row_at[wave][lane >> 5][tp] = reinterpret_cast<uint64_t>(row);
      const uint32_t kept = (uint32_t)__ballot(page >= 0) & EVERY;
      asm volatile("" ::: "memory");  // (a wavefront's LDS operations execute in order)
      return kept;
    };

    u32x4 kr[SUB][2][LINES];
    VWord vr[NV][NBLK];
    // 8 keys' whole 128-byte lines per instruction: lane (m16, g) has the g + 4 (m16 / 8)-th 16 bytes of key m16 % 8's
    auto load_keys = [&]() {
#pragma unroll
      for (int st = 0; st < SUB; ++st)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const char* row = reinterpret_cast<const char*>(row_at[wave][0][st * 16 + e * 8 + (m16 & 7)]) + line_at;
#pragma unroll
          for (int c = 0; c < LINES; ++c) {
            const char* p = row + c * 128;
            if (!FULL && c * 128 + line_at >= a.D * (int)sizeof(X)) p = zeros;
            kr[st][e][c] = read<NT, u32x4>(p);
          }
        }
    };
    auto load_values = [&]() {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const char* row = reinterpret_cast<const char*>(row_at[wave][1][u / 4 * 16 + g * 4 + u % 4]) + m16 * (EPL * sizeof(X));
#pragma unroll
        for (int blk = 0; blk < NBLK; ++blk) {
          const char* p = row + blk * (BD * sizeof(X));
          if (!FULL && (blk * 16 + m16) * EPL >= a.D) p = zeros;
          vr[u][blk] = read<NT, VWord>(p);
        }
      }
    };

    float m = -INFINITY, mref = 0.f, l = 0.f;
    f32x4 o[NBLK][EPL];
#pragma unroll
    for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
      for (int j = 0; j < EPL; ++j) o[blk][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (t < t_end) {
      u32x4 qr[KSTEPS];
      const bool have = m16 < my_heads;
      const char* q_row = a.q + (int64_t)b * a.q_token + (int64_t)(hk * a.G + ht * HEADS + m16) * a.q_head + g * 16;
#pragma unroll
      for (int s = 0; s < KSTEPS; ++s) qr[s] = read<false, u32x4>(have && (s * 64 + g * 16) < a.D * (int)sizeof(X) ? q_row + s * 64 : zeros);
      if (!early) {
        now = entry_of(t);
        entry = entry_of(t + step);
      }
      uint32_t kept = place_rows(t, now);
      __builtin_amdgcn_sched_barrier(0);  // (the loop counts on the keys being requested first)
      load_keys();
      __builtin_amdgcn_sched_barrier(0);
      load_values();
      do {
        const uint32_t here = kept;
        const int entry_next = entry_of(t + 2 * step);
        f32x4 z[SUB];
#pragma unroll
        for (int st = 0; st < SUB; ++st) {
          // [e][h]: keys e*8.. by the halves h of their lines; rows 8h..8h+7 of the product are the ones that mean something
          f32x4 part[2][2];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              part[e][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int c = 0; c < LINES; ++c) part[e][h] = product<BF16>(kr[st][e][c], qr[2 * c + h], part[e][h]);
            }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // a place's other half lies 32 lanes away
            const float mine = lane < 32 ? part[0][0][i] : part[1][1][i], other = lane < 32 ? part[1][0][i] : part[0][1][i];
            z[st][i] = mine + other_half(other, lane);
          }
        }
        kept = place_rows(t + step, entry);
        entry = entry_next;
        load_keys();
        // Scores stay in their own units until the maximum is taken off: in powers of two those beyond 2.4e38 would be infinite.
        if (plain) {
#pragma unroll
          for (int st = 0; st < SUB; ++st) z[st] *= a.scale;
        } else {
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float s = z[st][i] * a.scale;
              if (a.cap > 0.f) s = a.cap * tanhf(s * a.inv_cap);
              s -= slope * (float)(n - 1 - (t * TILE + st * 16 + g * 4 + i));
              z[st][i] = s;
            }
        }
        if (here != EVERY) {
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!((here >> (st * 16 + g * 4 + i)) & 1)) z[st][i] = -INFINITY;
        }
        float top = z[0][0];
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, z[st][i]);
        // The maximum moves only when some score passes it by a factor of nearly 2^8, so that the four lanes of a head need not exchange
        // theirs.  All weights are 2^-8 of what they would be (sums, and so lse, with them): none is above 1, and no product with a
        // finite value overflows.
        if (__any(top > m + LAG)) {
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float now = fmaxf(m, top), f = now == -INFINITY ? 1.f : power(m - now);
          m = now;
          mref = now == -INFINITY ? 0.f : now;
          l *= f;
#pragma unroll
          for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
            for (int j = 0; j < EPL; ++j) o[blk][j] *= f;
        }
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            z[st][i] = power(z[st][i] - mref) * (1.f / (1 << LAG_BITS));
            l += z[st][i];
          }
        if constexpr (BF16) {
          // A weight enters as the sum of three bfloat16 numbers, each the leading 8 bits of what the ones before leave: all of its 24.
          // (With two, 16 to 17 bits, outputs whose values cancel over a long cache carried three times the error of a 32-bit sum.)
          uint32_t weight[3][2 * SUB];
#pragma unroll
          for (int i = 0; i < 2 * SUB; ++i) {
            float p0 = z[i / 2][i % 2 * 2], p1 = z[i / 2][i % 2 * 2 + 1];
#pragma unroll
            for (int s = 0; s < 3; ++s) {
              const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
              weight[s][i] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
              p0 -= __uint_as_float(u0 & 0xffff0000u);
              p1 -= __uint_as_float(u1 & 0xffff0000u);
            }
          }
#pragma unroll
          for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
            for (int j = 0; j < EPL; ++j) {
              uint32_t vt[2 * SUB];
#pragma unroll
              for (int i = 0; i < 2 * SUB; ++i)
                vt[i] = __builtin_amdgcn_perm(vr[2 * i + 1][blk][j / 2], vr[2 * i][blk][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
              for (int s = 0; s < 3; ++s) o[blk][j] = weighted<SUB>(vt, weight[s], o[blk][j]);
            }
        } else {
#pragma unroll
          for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < EPL; ++j)
                o[blk][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr[i][blk][j]), z[0][i], o[blk][j], 0, 0, 0);
        }
        load_values();
        t += step;
      } while (t < t_end);
    }

    // the wavefronts' parts: common maximum, then the sum through LDS
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    lds_barrier();  // (the piece before has been read)
    if (g == 0) ml_lds[wave][m16] = f32x2{m, l};
    lds_barrier();
    // (wavefront w and those a multiple of wave_heads away have the same kv head)
    auto joined_max = [&](int w, int row) {
      float top = -INFINITY;
      for (w &= wave_heads - 1; w < WAVES; w += wave_heads) top = fmaxf(top, ml_lds[w][row][0]);
      return top;
    };
    auto part_weight = [&](int w, int row, float top) { return top == -INFINITY ? 1.f : power(ml_lds[w][row][0] - top); };
    const float f = m16 < my_heads ? part_weight(wave, m16, joined_max(wave, m16)) : 0.f;
    const int d = threadIdx.x % (BD / 4) * 4;
#pragma unroll
    for (int blk = 0; blk < NBLK; ++blk) {
      if (blk) lds_barrier();
      if (m16 < my_heads) {
        float* row = o_lds + (wave * a.rows + m16) * PITCH;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < EPL; j += 4)
            *reinterpret_cast<f32x4*>(row + (g * 4 + i) * EPL + j) =
                f32x4{o[blk][j][i] * f, o[blk][j + 1][i] * f, o[blk][j + 2][i] * f, o[blk][j + 3][i] * f};
      }
      lds_barrier();
      const int dim = blk * BD + d;
      for (int i = threadIdx.x / (BD / 4); i < a.rows * wave_heads; i += 64 * WAVES / (BD / 4)) {
        const int wh = a.per_rows.quotient(i), r = i - wh * a.rows, its = at.first_item + wh;  // the row's item
        const int its_hk = a.per_kv_head.quotient(its), its_ht = its - its_hk * a.hts;
        if (r >= heads_of(its_ht)) continue;
        const float top = joined_max(wh, r);
        float sum = 0.f;
        f32x4 y{0.f, 0.f, 0.f, 0.f};
        for (int w = wh; w < WAVES; w += wave_heads) {
          sum += ml_lds[w][r][1] * part_weight(w, r, top);
          y += *reinterpret_cast<const f32x4*>(o_lds + (w * a.rows + r) * PITCH + d);
        }
        if (!FULL && dim >= a.D) continue;
        if (whole) {
          store_row<X>(a, b, its_hk * a.G + its_ht * HEADS + r, dim, y, sum, top);
        } else {
          const int64_t part = ((int64_t)slot * a.items + its) * a.rows + r;
          *reinterpret_cast<f32x4*>(a.part_o + part * a.D + dim) = y;
          if (dim == 0) a.part_ml[part] = f32x2{top, sum};
        }
      }
    }
    x = b_end;
    at.begin = b_end;
    if (x < x_end) at.len = a.lens[++at.b];
  }
}

// Joins the pieces of (sequence, query head) rows in their order; sequences of one piece are complete already.  ROW threads work on a
// row: a wavefront where there are many rows, of few pieces each, a whole workgroup where there are few.
constexpr int JOIN_THREADS = 256;
template <typename X, int ROW>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(DecodeArgs a) {
  constexpr int AHEAD = 8, WIDE = ROW / 64;
  extern __shared__ __attribute__((aligned(16))) float weights[];  // one per piece and row
  __shared__ float red[2][WIDE];
  __shared__ f32x4 sums[JOIN_THREADS];
  auto barrier = [] {
    if (WIDE > 1) lds_barrier();
    else asm volatile("" ::: "memory");  // (a wavefront's LDS operations execute in order)
  };
  const int id = blockIdx.x * (JOIN_THREADS / ROW) + threadIdx.x / ROW;
  if (id >= a.n_seqs * a.hq) return;
  const int b = id / a.hq, h = id % a.hq;
  const int2 plan = a.plan[b];
  if (plan.y <= 1) return;
  const int hk = h / a.G, r = h % a.G % HEADS, item = hk * a.hts + h % a.G / HEADS;
  auto row = [&](int j) { return ((int64_t)piece_slot(plan.x, j) * a.items + item) * a.rows + r; };
  const int tid = threadIdx.x % ROW, lane = tid & 63, wave = tid >> 6;
  float* weight = weights + threadIdx.x / ROW * a.parts;
  const int across = a.D <= 64 ? 16 : a.D <= 128 ? 32 : 64, d = tid % across * 4, groups = ROW / across, first = tid / across;
  f32x4 part[AHEAD];
  // the first rows are requested before their weights are known
  auto request = [&](int j0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int j = j0 + u * groups;
      part[u] = j < plan.y && d < a.D ? *reinterpret_cast<const f32x4*>(a.part_o + row(j) * a.D + d) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  auto over_row = [&](float v, int which, auto join) {
#pragma unroll
    for (int s = 32; s; s >>= 1) v = join(v, __shfl_xor(v, s, 64));
    if (WIDE == 1) return v;
    if (lane == 0) red[which][wave] = v;
    lds_barrier();
    v = red[which][0];
#pragma unroll
    for (int w = 1; w < WIDE; ++w) v = join(v, red[which][w]);
    return v;
  };
  float top = -INFINITY;
  for (int j = tid; j < plan.y; j += ROW) top = fmaxf(top, a.part_ml[row(j)][0]);
  request(first);
  top = over_row(top, 0, [](float x, float y) { return fmaxf(x, y); });
  float sum = 0.f;
  for (int j = tid; j < plan.y; j += ROW) {
    const f32x2 ml = a.part_ml[row(j)];
    const float f = top == -INFINITY ? 1.f : power(ml[0] - top);
    weight[j] = f;
    sum += f * ml[1];
  }
  sum = over_row(sum, 1, [](float x, float y) { return x + y; });
  barrier();
  f32x4 y{0.f, 0.f, 0.f, 0.f};
  for (int j0 = first;;) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (j0 + u * groups < plan.y) y += weight[j0 + u * groups] * part[u];
    j0 += AHEAD * groups;
    if (j0 >= plan.y) break;
    request(j0);
  }
  f32x4* mine = sums + threadIdx.x / ROW * ROW;
  mine[tid] = y;
  barrier();
  if (tid >= across || d >= a.D) return;
  for (int i = 1; i < groups; ++i) y += mine[tid + i * across];
  store_row<X>(a, b, h, d, y, sum, top);
}

// The split of a call: what its grid, its workspace and its kernels agree on.
struct Split {
  int rows, items, wave_heads, least, parts;
  int64_t grid;  // workgroups of the decode kernel
  bool nt, join;
  size_t ml, o, total;  // bytes: offsets of the pieces (the plan lies in front)
};

Split split_of(const moe_kv_cache* c, int32_t n_q_heads, int32_t window) {
  Split s;
  const int G = n_q_heads / c->n_kv_heads, es = (int)elem_size(c->dtype), tile = es == 2 && c->head_dim <= 128 ? 32 : 16;
  s.rows = G < HEADS ? G : HEADS;
  s.items = c->n_kv_heads * ((G + HEADS - 1) / HEADS);
  // Neighbouring items by one workgroup: tiles of query heads that read the same keys and values (64 heads on one kv head 97 us
  // apart, 73 together), and kv heads whose rows are neighbours in memory, 512 bytes of them (256-byte rows, 8.5 GB: 1333 us one by
  // one, 1261 by twos, 1308 by fours; 128-byte rows: 108, 96 and 90).
  const bool several = s.items > c->n_kv_heads, neighbours = c->head_stride < c->token_stride;
  const int wanted = several ? 4 : !neighbours ? 1 : c->head_dim * es <= 128 ? 4 : 2;
  s.wave_heads = s.items % wanted == 0 ? wanted : s.items % 2 == 0 && wanted > 1 ? 2 : 1;
  s.least = LEAST_PER_WAVE * WAVES;
  const int64_t capacity = (int64_t)c->table_width * c->page_size, tiles = (capacity + tile - 1) / tile;
  const int64_t resident = 256 * resident_workgroups(c->head_dim, es), pieces = (tiles + s.least - 1) / s.least;
  // one round of workgroups, and at least one for every item; no more than there can be pieces of work
  int64_t grid = (int64_t)c->n_seqs * s.items * (pieces > 1 ? pieces : 1);
  if (grid > resident) grid = resident;
  if (grid < s.items) grid = s.items;
  s.grid = grid;
  s.parts = (int)(grid * (s.items % 4 == 0 ? 4 : s.items % 2 == 0 ? 2 : 1) / s.items);  // the most there can be
  // sequences that no deal splits: no second launch, and no look at all the lengths
  const int64_t kept = window > 0 && window + tile < capacity ? window + tile : capacity;
  const int64_t work = (int64_t)c->n_seqs * s.items;
  s.join = kept > SMALL_PLACES;
  if (!s.join && work > grid) {
    // more short sequences than one round holds: a workgroup for each, so that the long ones among them do not meet
    const int wave_heads = kept > TINY_PLACES ? s.wave_heads : s.items % 4 == 0 ? 4 : s.items % 2 == 0 ? 2 : 1;
    s.grid = work / wave_heads;
  }
  // Pools that the last-level cache (256 MB) cannot keep for the next call are read past it: 537 MB 89 us, 101 through the caches; of
  // 79 MB that it keeps 25.9 and 25.2.  The pool's size counts and not what a call reads of it: of a pool of 3 GB, other places in each call,
  // 135 MB 33.6 us and 37.5, 25 MB 15.3 and 16.1, 0.7 MB 7.4 and 7.5 (the same places again and again 32.0 and 30.3, 14.5 and 14.3, 7.4 and
  // 7.5).  Not where tiles of query heads read the same keys and values one beside the other: 64 heads on one kv head, 153 MB, 78 us
  // and 70, 32 on each of four, 307 MB, 93 and 86.
  s.nt = !several && (double)c->n_pages * c->page_size * c->n_kv_heads * c->head_dim * 2 * es > (double)(300 << 20);
  s.ml = align_up((size_t)c->n_seqs * sizeof(int2), 256);
  s.o = s.ml + align_up((size_t)s.parts * 2 * s.items * s.rows * sizeof(f32x2), 256);
  s.total = s.o + align_up((size_t)s.parts * 2 * s.items * s.rows * c->head_dim * sizeof(float), 256);
  return s;
}

// Workgroups of the join of so many rows: four rows each where there are many.
int64_t join_grid(int64_t rows) { return rows >= MANY_ROWS ? (rows * 64 + JOIN_THREADS - 1) / JOIN_THREADS : rows; }

template <typename X, int DP, bool NT>
void launch(const DecodeArgs& a, unsigned grid, hipStream_t s) {
  const size_t lds = (size_t)WAVES * a.rows * (16 * Shape<X, DP>::EPL + 4) * sizeof(float);
  if (a.D == DP) hipLaunchKernelGGL((decode_kernel<X, DP, true, NT>), dim3(grid), dim3(64 * WAVES), lds, s, a);
  else hipLaunchKernelGGL((decode_kernel<X, DP, false, NT>), dim3(grid), dim3(64 * WAVES), lds, s, a);
}

template <typename X, int DP>
void launch(const DecodeArgs& a, unsigned grid, bool nt, hipStream_t s) {
  if (nt) launch<X, DP, true>(a, grid, s);
  else launch<X, DP, false>(a, grid, s);
}

template <typename X>
int32_t launch_decode(const DecodeArgs& a, const Split& sp, hipStream_t s) {
  const unsigned grid = (unsigned)sp.grid;
  if (a.D <= 64) launch<X, 64>(a, grid, sp.nt, s);
  else if (a.D <= 128) launch<X, 128>(a, grid, sp.nt, s);
  else launch<X, 256>(a, grid, sp.nt, s);
  int32_t st = check_hip(hipGetLastError(), "attention launch");
  if (st != MOE_OK || !sp.join) return st;
  const int64_t rows = (int64_t)a.n_seqs * a.hq;
  const unsigned join = (unsigned)join_grid(rows);
  // (a row has about parts / sequences pieces; the weights of four rows' take LDS)
  if (rows >= MANY_ROWS) {
    const size_t lds = (size_t)sp.parts * (JOIN_THREADS / 64) * sizeof(float);
    hipLaunchKernelGGL((join_kernel<X, 64>), dim3(join), dim3(JOIN_THREADS), lds, s, a);
  } else {
    hipLaunchKernelGGL((join_kernel<X, JOIN_THREADS>), dim3(join), dim3(JOIN_THREADS), (size_t)sp.parts * sizeof(float), s, a);
  }
  return check_hip(hipGetLastError(), "attention join launch");
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
  return split_of(c, n_q_heads, 0).total;
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
  const int64_t es = (int64_t)elem_size(c->dtype);
  if (!rows_aligned(q, es) || !rows_aligned(out, es))
    return fail(MOE_ERR_INVALID_ARG, "moe_attention_decode: pointers and strides of q and out must be multiples of 16 bytes");
  const Split sp = split_of(c, n_q_heads, opt->window);
  // (a sequence has at most 64 query heads per workgroup: their product stays below 2^31)
  if (!launchable(sp.grid, 64 * WAVES) || (sp.join && !launchable(join_grid((int64_t)c->n_seqs * n_q_heads), JOIN_THREADS)))
    return fail(MOE_ERR_UNSUPPORTED, "moe_attention_decode: %d sequences of %d query heads are too many for one call", c->n_seqs, n_q_heads);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_attention_decode: workspace NULL, misaligned or smaller than %zu bytes", need);
  DecodeArgs a{};
  a.k = (const char*)c->k;
  a.v = (const char*)c->v;
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.lse = lse;
  a.table = c->page_table;
  a.lens = seq_lens;
  a.slopes = opt->slopes;
  a.plan = (int2*)ws;
  a.part_ml = (f32x2*)((char*)ws + sp.ml);
  a.part_o = (float*)((char*)ws + sp.o);
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
  a.n_seqs = c->n_seqs;
  a.hq = n_q_heads;
  a.G = n_q_heads / c->n_kv_heads;
  a.rows = sp.rows;
  a.items = sp.items;
  a.log_heads = sp.wave_heads >> 1;
  for (int k = 0; k < 3; ++k) {
    const int groups = sp.items >> k;
    if (groups == 0) continue;  // (never taken)
    a.share_of_grid[k].per_part = page_divisor(groups);
    a.share_of_grid[k].parts = (int)(sp.grid / groups);
    a.share_of_grid[k].inverse_parts = 1.0 / a.share_of_grid[k].parts;
  }
  a.hts = sp.items / c->n_kv_heads;
  a.per_kv_head = page_divisor(a.hts);
  a.per_rows = page_divisor(sp.rows);
  a.capacity = c->table_width * c->page_size;
  a.D = c->head_dim;
  a.window = opt->window;
  a.least = sp.least;
  a.parts = sp.parts;
  a.may_split = sp.join;
  a.scale = opt->scale;
  a.cap = opt->softcap;
  // (finite for the smallest caps too: a score of 0 stays 0)
  a.inv_cap = opt->softcap > 0.f ? fminf(1.f / opt->softcap, FLT_MAX) : 0.f;
  return c->dtype == MOE_BF16 ? launch_decode<__bf16>(a, sp, (hipStream_t)stream) : launch_decode<float>(a, sp, (hipStream_t)stream);
}
