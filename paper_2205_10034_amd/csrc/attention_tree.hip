// Attention of several new tokens per sequence over a paged cache (moe_attention_tree): as for one token,
//   m' = max(m, z_j);  l' = l exp(m - m') + exp(z_j - m');  o' = o exp(m - m') + exp(z_j - m') v_j;  out = o / l,
// in one pass over the places that some token of the sequence sees, split over the length into pieces that are joined at the end.
//
// The rows of a kv head are its new tokens times the G query heads that share it, 16 to a block of the matrix instructions, one or two
// blocks to a workgroup, so that keys and values are read once for up to 32 rows; bfloat16 calls with more take attention_tree_shared.hip
// (32 sequences of 3000 to 5000 places, 4 kv heads of 128: 32 rows 71 us here and as many there, of 64 40 and 46, of 256 105 and 127; 64 rows
// 104 here, with four blocks, and 78 there).  Bound: HBM, and for short or windowed calls the trips to memory at the start of a piece
// (length, table entry, keys) and of every tile.  A tile in each wavefront's registers, the next one's loads behind the products that use it:
//  - Scores: S^T[place, row] = K Q^T, keys as the first operand, from memory into the registers that the instruction reads.  A load
//    brings eight keys' whole 128-byte lines; the operand wants half lines of sixteen, which is an exchange of lanes 8 apart.
//  - Output: O^T[dim, row] += V^T P^T.  A lane of S^T holds four places of one row, which is how the second operand wants P^T when the
//    places of an instruction are taken in that order.  The first operand pairs the halves of the values of two places.
//  - The queries of all rows lie in LDS, 16 bytes of padding to a row: every wavefront reads all of them for each tile.
//  - Who sees what is looked up only in tiles that hold new tokens, a window's edge or places that are not there.
#include "tree_parts.h"

namespace moesys {
namespace {

constexpr int LEAST = 2 * WAVES;  // tiles of a part, at least

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

// Workgroups that a CU holds.
constexpr int resident_workgroups(int dims, int elem, int blocks) { return blocks * dims <= 256 && dims * elem < 1024 ? 2 : 1; }

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

// Two registers of eight keys' whole lines each become the sixteen keys' first and second half lines: lanes 8-15 of every 16 in
// the first change places with lanes 0-7 in the second.
__device__ __forceinline__ void half_lines(u32x4& a, u32x4& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int x = (int)a[e], y = (int)b[e];
    a[e] = (uint32_t)__builtin_amdgcn_update_dpp(x, y, 0x128 /* row_ror:8 */, 0xf, 0xc, false);
    b[e] = (uint32_t)__builtin_amdgcn_update_dpp(y, x, 0x128, 0xf, 0x3, false);
  }
}

// A part of the batch per workgroup, piece after piece; its wavefronts take an item's tiles in turn.  An item is a kv head and up
// to 16 RB of the rows that its tokens and query heads make.
// FULL: head_dim is DP, no lane's dimensions lie beyond it.
template <typename X, int DP, int RB, bool FULL, bool NT>
__global__ __launch_bounds__(64 * WAVES, resident_workgroups(DP, sizeof(X), RB)) void tree_kernel(TreeArgs a) {
  using S = Shape<X, DP>;
  constexpr bool BF16 = sizeof(X) == 2;
  constexpr int SUB = S::SUB, TILE = 16 * SUB, EPL = S::EPL, LINES = S::KSTEPS / 2, NV = 4 * SUB, BD = 16 * EPL, NBLK = DP / BD, PITCH = BD + 4;
  constexpr int ROWS = 16 * RB, QPITCH = DP * (int)sizeof(X) + 16;
  constexpr uint32_t EVERY = (uint32_t)((1ull << TILE) - 1);
  using VWord = typename Words<EPL * sizeof(X)>::type;
  __shared__ __attribute__((aligned(16))) char q_lds[ROWS * QPITCH];
  __shared__ __attribute__((aligned(16))) float o_lds[WAVES * 16 * PITCH];
  __shared__ uint64_t row_at[WAVES][2][TILE];
  __shared__ f32x2 ml_lds[WAVES][ROWS];
  __shared__ uint64_t seen_lds[ROWS];     // what a row's token sees of the new ones
  __shared__ int depth_lds[MOE_MAX_DRAFTS];  // of the sequence's new tokens
  __shared__ int token_lds[ROWS];         // a row's token

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m16 = lane & 15, g = lane >> 4, line_at = (g + 4 * (m16 >> 3)) * 16;
  const int w = blockIdx.x / a.items, item = blockIdx.x - w * a.items, rt = a.kv_heads.quotient(item), hk = item - rt * a.hkv;
  Deal at = deal<TILE, LEAST>(a, rt, w);
  int64_t x = w * at.share;
  const int64_t x_end = x + at.share < at.total ? x + at.share : at.total;
  if (x >= x_end) return;
  const char* zeros = reinterpret_cast<const char*>(ZEROS);
  const char* base_row = (lane < 32 ? a.k : a.v) + hk * a.head_stride;  // lanes 0-31 place the keys' rows, the others the values'
  const int tp = lane & (TILE - 1);
  const bool plain = a.cap == 0.f && !a.slopes;

  for (int piece_no = 0; x < x_end; ++piece_no) {
    // the piece of sequence b that lies in this part
    const int b = at.b;
    const Drafts d = drafts(a, b);
    const int my_rows = d.n * a.G - rt * ROWS < ROWS ? d.n * a.G - rt * ROWS : ROWS;
    const Span span = span_of(d, a.window, a.sinks, TILE);
    const int in_row = at.one_each ? 1 : my_rows > 0 ? (int)row_tiles(span.tiles) : 0;
    const int64_t b_end = at.begin + in_row;
    if (b_end <= x || my_rows <= 0) {  // no rows here
      x = b_end > x ? b_end : x;
      at.begin = b_end;
      if (++at.b >= a.n_seqs) break;
      continue;
    }
    const int from = (int)(x - at.begin), upto = b_end <= x_end ? span.tiles : (int)(x_end - at.begin);
    const bool whole = from == 0 && b_end <= x_end;
    const int slot = 2 * w + (piece_no > 0);
    if (from == 0 && threadIdx.x == 0 && hk == 0) a.plan[(int64_t)rt * a.n_seqs + b] = make_int2(slot, whole ? 1 : part_of(b_end - 1, at.share) - w + 1);
    const int32_t* table = a.table + (int64_t)b * a.table_width;

    // queries, and what the rows see
    lds_barrier();  // (the piece before has been read)
    for (int i = threadIdx.x; i < ROWS * (QPITCH / 16 - 1); i += 64 * WAVES) {
      const int r = i / (QPITCH / 16 - 1), c = i - r * (QPITCH / 16 - 1), token = a.group.quotient(rt * ROWS + r), head = rt * ROWS + r - token * a.G;
      const bool have = r < my_rows && c * 16 < a.D * (int)sizeof(X);
      const char* from_q = a.q + (int64_t)(d.first + token) * a.q_token + (int64_t)(hk * a.G + head) * a.q_head + c * 16;
      *reinterpret_cast<u32x4*>(q_lds + r * QPITCH + c * 16) = read<false, u32x4>(have ? from_q : zeros);
    }
    auto sees = [&](int i) { return seen_drafts(a.words, a.words ? a.words[d.first + i] : 0, i, d.n); };
    if ((int)threadIdx.x < d.n) depth_lds[threadIdx.x] = draft_depth(sees(threadIdx.x), threadIdx.x);
    if (threadIdx.x >= 64 && threadIdx.x < 64 + ROWS) {
      const int r = threadIdx.x - 64, token = a.group.quotient(rt * ROWS + r);
      seen_lds[r] = r < my_rows ? sees(token) : 0;
      token_lds[r] = r < my_rows ? token : 0;
    }
    lds_barrier();
    int pos[RB];  // of this lane's rows
    float slope[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = rb * 16 + m16;
      pos[rb] = d.base + depth_lds[token_lds[r]];
      slope[rb] = a.slopes && r < my_rows ? a.slopes[hk * a.G + (rt * ROWS + r - token_lds[r] * a.G)] : 0.f;
    }
    const int last_pos = d.base + d.n - 1;  // no position is beyond it

    // Nothing in the loop that loads is conditional: what a tile beyond the last one would load is ZEROS.  (Behind a branch the
    // compiler waits for every load in flight before it uses the first.)
    auto entry_of = [&](int u) {  // the table's entry for this lane's place of the u-th tile; an entry of the table in any case
      const unsigned column = (unsigned)a.page.quotient((int)((unsigned)span.tile(u) * TILE + tp)), last = (unsigned)a.last_column;
      return table[column < last ? column : last];
    };
    // rows of the u-th tile into LDS; returns which places are there
    auto place_rows = [&](int u, int entry) {
      const int p = (int)((unsigned)span.tile(u) * TILE + tp), page = u < upto && p < d.len ? valid_page(entry, a.n_pages) : -1;
      const int in_page = p - a.page.quotient(p) * a.page_size;
      const char* row = page >= 0 ? base_row + page * a.page_stride + in_page * a.token_stride : zeros;
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

    float m[RB], mref[RB], l[RB];
    f32x4 o[RB][NBLK][EPL];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY;
      mref[rb] = l[rb] = 0.f;
#pragma unroll
      for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
        for (int j = 0; j < EPL; ++j) o[rb][blk][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int u = from + wave;
    if (u < upto) {
      int entry = entry_of(u + WAVES);
      uint32_t kept = place_rows(u, entry_of(u));
      __builtin_amdgcn_sched_barrier(0);  // (the loop counts on the keys being requested first)
      load_keys();
      __builtin_amdgcn_sched_barrier(0);
      load_values();
      do {
        const uint32_t here = kept;
        const int p0 = span.tile(u) * TILE;
        const int entry_next = entry_of(u + 2 * WAVES);
        f32x4 z[RB][SUB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int st = 0; st < SUB; ++st) z[rb][st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < LINES; ++c) {
#pragma unroll
          for (int st = 0; st < SUB; ++st) half_lines(kr[st][0][c], kr[st][1][c]);
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
              const u32x4 q = *reinterpret_cast<const u32x4*>(q_lds + (rb * 16 + m16) * QPITCH + (2 * c + e) * 64 + g * 16);
#pragma unroll
              for (int st = 0; st < SUB; ++st) z[rb][st] = product<BF16>(kr[st][e][c], q, z[rb][st]);
            }
        }
        kept = place_rows(u + WAVES, entry);
        entry = entry_next;
        load_keys();
        // Scores stay in their own units until the maximum is taken off: in powers of two those beyond 2.4e38 would be infinite.
        const bool with_drafts = p0 > d.base - TILE;
        if (plain) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int st = 0; st < SUB; ++st) z[rb][st] *= a.scale;
        } else {
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int p = p0 + st * 16 + g * 4 + i;
              int pos_p = p;
              if (with_drafts && p >= d.base) pos_p = d.base + depth_lds[p - d.base < MOE_MAX_DRAFTS ? p - d.base : 0];
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) {
                float s = z[rb][st][i] * a.scale;
                if (a.cap > 0.f) s = a.cap * tanhf(s * a.inv_cap);
                z[rb][st][i] = s - slope[rb] * (float)(pos[rb] - pos_p);
              }
            }
        }
        // Everyone sees everything of a tile that is all there, before the new tokens, and in the window of the last position or among
        // the sinks.
        const bool masked = here != EVERY || with_drafts || (a.window > 0 && last_pos - p0 >= a.window && p0 > a.sinks - TILE);
        uint32_t seen_here = 0;  // places that this lane's rows see, 4 SUB bits to a row
        if (__builtin_expect(masked, 0)) {
          uint64_t seen[RB];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) seen[rb] = seen_lds[rb * 16 + m16];
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int p = p0 + st * 16 + g * 4 + i, j = p - d.base, jj = j & (MOE_MAX_DRAFTS - 1);  // (places that are there have j < n)
              const uint32_t there = (here >> (st * 16 + g * 4 + i)) & 1, cached = j < 0;
              const int pos_p = cached ? p : d.base + depth_lds[jj];
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) {
                const uint32_t ok = there & (cached | (uint32_t)(seen[rb] >> jj)) & (uint32_t)in_window(pos[rb], pos_p, p, a.window, a.sinks);
                z[rb][st][i] = ok ? z[rb][st][i] : -INFINITY;
                seen_here |= ok << ((rb * SUB + st) * 4 + i);
              }
            }
        }
        // The maximum moves only when some score passes it by a factor of nearly 2^8, so that the four lanes of a row need not exchange
        // theirs.  All weights are 2^-8 of what they would be (sums, and so lse, with them): none is above 1, and no product with a
        // finite value overflows.  (The difference is compared: from 2^24 on a sum with LAG would be rounded up.)
        float top[RB];
        bool moves = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          top[rb] = z[rb][0][0];
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[rb] = fmaxf(top[rb], z[rb][st][i]);
          moves |= top[rb] - m[rb] > LAG;
        }
        if (__builtin_expect(__any(moves), 0)) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            float t = fmaxf(top[rb], __shfl_xor(top[rb], 16, 64));
            t = fmaxf(t, __shfl_xor(t, 32, 64));
            const float now = fmaxf(m[rb], t), f = now == -INFINITY ? 1.f : power(m[rb] - now);
            m[rb] = now;
            mref[rb] = now == -INFINITY ? 0.f : now;
            l[rb] *= f;
#pragma unroll
            for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
              for (int j = 0; j < EPL; ++j) o[rb][blk][j] *= f;
          }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              z[rb][st][i] = power(z[rb][st][i] - mref[rb]) * (1.f / (1 << LAG_BITS));
              l[rb] += z[rb][st][i];
            }
        // A value that is not finite and that only some rows see would reach the others as 0 times it: its element of the rows that see it
        // becomes NaN, and it leaves the tile.
        bool odd = false;
        if (__builtin_expect(masked, 0)) {
#pragma unroll
          for (int u = 0; u < NV; ++u)
#pragma unroll
            for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
              for (int e = 0; e < (int)(sizeof(VWord) / 4); ++e) {
                if constexpr (BF16) odd |= not_finite(vr[u][blk][e]) != 0;
                else odd |= not_finite(__uint_as_float(vr[u][blk][e])) != 0.f;
              }
          odd = __any(odd);
        }
        if (__builtin_expect(odd, 0)) {
          if constexpr (BF16) {
#pragma unroll
            for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
              for (int j = 0; j < EPL; ++j) {
                uint32_t bad[2 * SUB];
#pragma unroll
                for (int i = 0; i < 2 * SUB; ++i)
                  bad[i] = not_finite(__builtin_amdgcn_perm(vr[2 * i + 1][blk][j / 2], vr[2 * i][blk][j / 2], j & 1 ? 0x07060302u : 0x05040100u));
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                  uint32_t see[2 * SUB];
#pragma unroll
                  for (int i = 0; i < 2 * SUB; ++i) {
                    const uint32_t bits = seen_here >> ((rb * SUB + i / 2) * 4 + i % 2 * 2);
                    see[i] = (bits & 1 ? 0x3f80u : 0u) | (bits & 2 ? 0x3f800000u : 0u);
                  }
                  const f32x4 hit = weighted<SUB>(bad, see, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                  for (int i = 0; i < 4; ++i)
                    if (hit[i] > 0.f) o[rb][blk][j][i] = NAN;
                }
                __builtin_amdgcn_sched_barrier(0);
              }
#pragma unroll
            for (int u = 0; u < NV; ++u)
#pragma unroll
              for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
                for (int e = 0; e < (int)(sizeof(VWord) / 4); ++e) {
                  const uint32_t bad = not_finite(vr[u][blk][e]);
                  vr[u][blk][e] &= ~((bad & 0xffffu ? 0xffffu : 0u) | (bad >> 16 ? 0xffff0000u : 0u));
                }
          } else {
#pragma unroll
            for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < EPL; ++j) {
                  const float bad = not_finite(__uint_as_float(vr[i][blk][j]));
                  if (bad != 0.f) vr[i][blk][j] = 0u;
#pragma unroll
                  for (int rb = 0; rb < RB; ++rb) {
                    const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x4f32(bad, (seen_here >> (rb * SUB * 4 + i)) & 1 ? 1.f : 0.f, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                      if (hit[e] > 0.f) o[rb][blk][j][e] = NAN;
                  }
                  __builtin_amdgcn_sched_barrier(0);
                }
          }
        }
        if constexpr (BF16) {
          // A weight enters as the sum of two bfloat16 numbers, each rounded to nearest: 17 bits of it, an error that half a step of the
          // output covers unless 2^8 values cancel.  (A third one, all 24 bits, would be another third of all the matrix work.)
          uint32_t weight[RB][2][2 * SUB];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int i = 0; i < 2 * SUB; ++i) {
              const float p0 = z[rb][i / 2][i % 2 * 2], p1 = z[rb][i / 2][i % 2 * 2 + 1];
              const uint32_t head = pack_bf16(p0, p1);
              weight[rb][0][i] = head;
              weight[rb][1][i] = pack_bf16(p0 - __uint_as_float(head << 16), p1 - __uint_as_float(head & 0xffff0000u));
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
              for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int s = 0; s < 2; ++s) o[rb][blk][j] = weighted<SUB>(vt, weight[rb][s], o[rb][blk][j]);
            }
        } else {
#pragma unroll
          for (int blk = 0; blk < NBLK; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < EPL; ++j) {
                const float v = __uint_as_float(vr[i][blk][j]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][blk][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, z[rb][0][i], o[rb][blk][j], 0, 0, 0);
              }
        }
        load_values();
        u += WAVES;
      } while (u < upto);
    }

    // the wavefronts' parts: common maximum, then the sum through LDS, 16 rows and BD dimensions at a time
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      l[rb] += __shfl_xor(l[rb], 16, 64);
      l[rb] += __shfl_xor(l[rb], 32, 64);
      if (g == 0) ml_lds[wave][rb * 16 + m16] = f32x2{m[rb], l[rb]};
    }
    lds_barrier();
    auto joined_max = [&](int r) {
      float top = ml_lds[0][r][0];
#pragma unroll
      for (int v = 1; v < WAVES; ++v) top = fmaxf(top, ml_lds[v][r][0]);
      return top;
    };
    auto part_weight = [&](int v, int r, float top) { return top == -INFINITY ? 1.f : power(ml_lds[v][r][0] - top); };
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if (rb * 16 >= my_rows) break;
      const float f = part_weight(wave, rb * 16 + m16, joined_max(rb * 16 + m16));
#pragma unroll
      for (int blk = 0; blk < NBLK; ++blk) {
        if (rb + blk) lds_barrier();
        float* row = o_lds + (wave * 16 + m16) * PITCH;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < EPL; j += 4)
            *reinterpret_cast<f32x4*>(row + (g * 4 + i) * EPL + j) =
                f32x4{o[rb][blk][j][i] * f, o[rb][blk][j + 1][i] * f, o[rb][blk][j + 2][i] * f, o[rb][blk][j + 3][i] * f};
        lds_barrier();
        const int dd = threadIdx.x % (BD / 4) * 4, dim = blk * BD + dd;
        for (int r16 = threadIdx.x / (BD / 4); r16 < 16; r16 += 64 * WAVES / (BD / 4)) {
          const int r = rb * 16 + r16;
          if (r >= my_rows || (!FULL && dim >= a.D)) continue;
          const float top = joined_max(r);
          float sum = 0.f;
          f32x4 y{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int v = 0; v < WAVES; ++v) {
            sum += ml_lds[v][r][1] * part_weight(v, r, top);
            y += *reinterpret_cast<const f32x4*>(o_lds + (v * 16 + r16) * PITCH + dd);
          }
          if (whole) {
            const int token = token_lds[r];
            store_row<X>(a, d.first + token, hk * a.G + (rt * ROWS + r - token * a.G), dim, y, sum, top);
          } else {
            const int64_t part = ((int64_t)slot * a.items + item) * ROWS + r;
            *reinterpret_cast<f32x4*>(a.part_o + part * a.D + dim) = y;
            if (dim == 0) a.part_ml[part] = f32x2{top, sum};
          }
        }
      }
    }
    x = b_end;
    at.begin = b_end;
    if (++at.b >= a.n_seqs) break;
  }
}

// Joins the pieces of (token, query head) rows in their order, LANES lanes to a row (four dims each); sequences of one piece are complete already.
constexpr int JOIN_THREADS = 256;
template <typename X, int LANES>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(TreeArgs a) {
  constexpr int AHEAD = 8;
  const int64_t id = (int64_t)blockIdx.x * (JOIN_THREADS / LANES) + threadIdx.x / LANES;
  const int lane = threadIdx.x % LANES, s = (int)(id / (a.max_new * a.hq)), rest = (int)(id - (int64_t)s * a.max_new * a.hq), i = rest / a.hq, h = rest - i * a.hq;
  if (s >= a.n_seqs) return;
  const Drafts d = drafts(a, s);
  if (i >= d.n) return;
  const int hk = a.group.quotient(h), rr = i * a.G + h - hk * a.G, rt = rr / a.rows, r = rr - rt * a.rows, item = rt * a.hkv + hk;
  const int2 plan = a.plan[(int64_t)rt * a.n_seqs + s];
  if (plan.y <= 1) return;
  auto row = [&](int j) { return ((int64_t)piece_slot(plan.x, j) * a.items + item) * a.rows + r; };
  float top = -INFINITY, sum = 0.f;
  for (int j = lane; j < plan.y; j += LANES) top = fmaxf(top, a.part_ml[row(j)][0]);
#pragma unroll
  for (int x = LANES / 2; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
  const int dim = lane * 4;
  f32x4 y{0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < plan.y; j0 += LANES) {
    float f = 0.f;
    if (j0 + lane < plan.y) {
      const f32x2 ml = a.part_ml[row(j0 + lane)];
      f = top == -INFINITY ? 1.f : power(ml[0] - top);
      sum += f * ml[1];
    }
    const int n = plan.y - j0 < LANES ? plan.y - j0 : LANES;
    for (int j = 0; j < n; j += AHEAD) {
      f32x4 part[AHEAD];
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        part[e] = j + e < n && dim < a.D ? *reinterpret_cast<const f32x4*>(a.part_o + row(j0 + j + e) * a.D + dim) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < AHEAD; ++e)
        if (j + e < n) y += __shfl(f, j + e, LANES) * part[e];
    }
  }
#pragma unroll
  for (int x = LANES / 2; x; x >>= 1) sum += __shfl_xor(sum, x, 64);
  if (dim < a.D) store_row<X>(a, d.first + i, h, dim, y, sum, top);
}

// The split of a call: what its grid, its workspace and its kernels agree on.
struct Split {
  int blocks, rows, row_tiles, items, parts, small;
  bool shared, nt, may_split;
  size_t ml, o, total;  // bytes: offsets of the pieces (the plan lies in front); enough for fewer new tokens too, as far as `rows` is the same
};

Split split_of(const moe_kv_cache* c, int32_t n_q_heads, int32_t max_new, int32_t window, int32_t sinks) {
  Split s;
  const int es = (int)elem_size(c->dtype), rows = max_new * (n_q_heads / c->n_kv_heads), dims = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
  s.shared = es == 2 && rows > SHARED_FROM;
  s.blocks = s.shared ? shared_blocks(rows, dims) : rows <= 16 ? 1 : 2;
  s.rows = 16 * s.blocks * (s.shared ? WAVES : 1);
  s.row_tiles = (rows + s.rows - 1) / s.rows;
  s.items = c->n_kv_heads * s.row_tiles;
  const int64_t capacity = (int64_t)c->table_width * c->page_size, reach = (int64_t)window + sinks + MOE_MAX_DRAFTS + 64;
  const int64_t kept = window > 0 && reach < capacity ? reach : capacity;
  // A workgroup takes 128 or 64 places at a time where wavefronts have tiles of their own, 64 or 32 where they share them: 8 steps are
  // about the time of the launch that joins pieces.
  s.small = s.shared ? 256 : 1024;
  s.may_split = kept > s.small;
  const int64_t resident = 256 * (s.shared ? 2 : resident_workgroups(dims, es, s.blocks));
  int64_t parts = resident / s.items > 1 ? resident / s.items : 1;
  const int least = s.shared ? 256 : (es == 2 && dims <= 128 ? 32 : 16) * LEAST;  // places of a part
  const int64_t most = (int64_t)c->n_seqs * ((capacity + least - 1) / least);  // pieces of work there can be
  if (parts > most) parts = most > 1 ? most : 1;
  int64_t most_slots = 2 * s.rows * (resident > s.items ? resident : s.items);  // of this call or one of fewer items
  if (most_slots > 2 * s.rows * most * s.items) most_slots = 2 * s.rows * most * s.items;
  if (!s.may_split) parts = c->n_seqs;
  s.parts = (int)parts;
  // Pools that the last-level cache (256 MB) cannot keep for the next call are read past it, where one workgroup reads them.
  s.nt = s.row_tiles == 1 && (double)c->n_pages * c->page_size * c->n_kv_heads * c->head_dim * 2 * es > (double)(300 << 20);
  const int64_t slots = s.may_split ? 2 * parts * s.items * s.rows : 0;
  s.ml = align_up((size_t)c->n_seqs * s.row_tiles * sizeof(int2), 256);
  s.o = s.ml + align_up((size_t)slots * sizeof(f32x2), 256);
  if (!s.may_split || most_slots < slots) most_slots = slots;
  s.total = s.ml + align_up((size_t)most_slots * sizeof(f32x2), 256) + align_up((size_t)most_slots * c->head_dim * sizeof(float), 256);
  if (s.total < 256) s.total = 256;
  return s;
}

template <typename X, int DP, int RB, bool FULL>
void launch(const TreeArgs& a, unsigned grid, bool nt, hipStream_t s) {
  if (nt) hipLaunchKernelGGL((tree_kernel<X, DP, RB, FULL, true>), dim3(grid), dim3(64 * WAVES), 0, s, a);
  else hipLaunchKernelGGL((tree_kernel<X, DP, RB, FULL, false>), dim3(grid), dim3(64 * WAVES), 0, s, a);
}

template <typename X, int DP>
void launch(const TreeArgs& a, int blocks, unsigned grid, bool nt, hipStream_t s) {
  auto of = [&](auto rb) {
    if (a.D == DP) launch<X, DP, decltype(rb)::value, true>(a, grid, nt, s);
    else launch<X, DP, decltype(rb)::value, false>(a, grid, nt, s);
  };
  if (blocks == 1) of(std::integral_constant<int, 1>());
  else of(std::integral_constant<int, 2>());
}

template <typename X>
int32_t launch_tree(const TreeArgs& a, const Split& sp, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)sp.parts * sp.items);
  if (sp.shared) {
    const int32_t st = launch_tree_shared(a, sp.blocks, grid, sp.nt, s);
    if (st != MOE_OK) return st;
  } else if (a.D <= 64) launch<X, 64>(a, sp.blocks, grid, sp.nt, s);
  else if (a.D <= 128) launch<X, 128>(a, sp.blocks, grid, sp.nt, s);
  else launch<X, 256>(a, sp.blocks, grid, sp.nt, s);
  const int32_t st = check_hip(hipGetLastError(), "tree attention launch");
  if (st != MOE_OK || !sp.may_split) return st;
  const int64_t rows = (int64_t)a.n_seqs * a.max_new * a.hq;
  auto join = [&](auto lanes) {
    constexpr int LANES = decltype(lanes)::value, PER = JOIN_THREADS / LANES;
    hipLaunchKernelGGL((join_kernel<X, LANES>), dim3((unsigned)((rows + PER - 1) / PER)), dim3(JOIN_THREADS), 0, s, a);
  };
  if (a.D <= 64) join(std::integral_constant<int, 16>());
  else if (a.D <= 128) join(std::integral_constant<int, 32>());
  else join(std::integral_constant<int, 64>());
  return check_hip(hipGetLastError(), "tree attention join launch");
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
  // a larger call's workspace serves a smaller one: the most that any number of new tokens up to max_new wants
  size_t total = split_of(c, n_q_heads, max_new, 0, 0).total;
  for (int rows = 16; rows <= 64; rows *= 2) {  // (up to which the rows of a workgroup are the same)
    const int fewer = rows / (n_q_heads / c->n_kv_heads);
    if (fewer < 1 || fewer >= max_new) continue;
    const size_t less = split_of(c, n_q_heads, fewer, 0, 0).total;
    total = less > total ? less : total;
  }
  return total;
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
  const Split sp = split_of(c, n_q_heads, max_new, opt->window, opt->sinks);
  if ((int64_t)T * n_q_heads > (1 << 26) - 4 || !launchable((int64_t)sp.parts * sp.items, 64 * WAVES) ||
      (sp.may_split && !launchable((int64_t)c->n_seqs * max_new * n_q_heads / (JOIN_THREADS / 64) + 1, JOIN_THREADS)))
    return fail(MOE_ERR_UNSUPPORTED, "moe_attention_tree: %d tokens, %d sequences of up to %d, of %d query heads are too many for one call", T, c->n_seqs, max_new, n_q_heads);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < need)
    return fail(MOE_ERR_WORKSPACE, "moe_attention_tree: workspace NULL, misaligned or smaller than %zu bytes", need);
  TreeArgs a{};
  a.k = (const char*)c->k;
  a.v = (const char*)c->v;
  a.q = (const char*)q->data;
  a.out = (char*)out->data;
  a.lse = lse;
  a.table = c->table_width > 0 ? c->page_table : (const int32_t*)ws;
  a.last_column = c->table_width > 0 ? c->table_width - 1 : 0;
  a.lens = seq_lens;
  a.first = token_first;
  a.words = visible;
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
  a.capacity = c->table_width * c->page_size;
  a.n_seqs = c->n_seqs;
  a.hq = n_q_heads;
  a.G = n_q_heads / c->n_kv_heads;
  a.group = page_divisor(a.G);
  a.T = T;
  a.max_new = max_new;
  a.D = c->head_dim;
  a.window = opt->window;
  a.sinks = opt->sinks;
  a.rows = sp.rows;
  a.row_tiles = sp.row_tiles;
  a.kv_heads = page_divisor(c->n_kv_heads);
  a.hkv = c->n_kv_heads;
  a.items = sp.items;
  a.parts = sp.parts;
  a.inverse_parts = 1.0 / sp.parts;
  a.may_split = sp.may_split;
  a.small = sp.small;
  a.scale = opt->scale;
  a.cap = opt->softcap;
  // (finite for the smallest caps too: a score of 0 stays 0)
  a.inv_cap = opt->softcap > 0.f ? fminf(1.f / opt->softcap, FLT_MAX) : 0.f;
  return c->dtype == MOE_BF16 ? launch_tree<__bf16>(a, sp, (hipStream_t)stream) : launch_tree<float>(a, sp, (hipStream_t)stream);
}
