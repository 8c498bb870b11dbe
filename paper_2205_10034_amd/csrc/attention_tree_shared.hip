// Attention of drafted tokens, many rows to a kv head (see attention_tree.hip): every wavefront of a workgroup has rows of its own and reads
// the same tile of keys and values from LDS.
//
// Up to 64 rows the memory binds: tiles of 16 KB go through registers, up to two ahead, into the other one of two tiles in LDS, two workgroups
// to a CU.  64 sequences of up to 8192 places, 16 tokens, 32 heads on 8 of 128: 187 us in this kernel, 5.3 TB/s; some 30 of them are the
// starts and ends of pieces, the tiles themselves come at 6.5 TB/s.  (A tile in every wavefront's own registers, one wavefront per SIMD: 280.)
// From 128 rows on, 32 to a wavefront, a tile takes it 2000 clocks of which 770 are matrix instructions and about as many exponentials,
// packing and addresses; two wavefronts per SIMD overlap some of that: 64 tokens on 131071 places, 251 us, 550 TFLOP/s (820 with the
// weights' second halves).  Registers decide: 60 spilled ones cost a third of the time, since their way back waits for the tiles.
//  - A tile's rows lie in LDS as in memory, their 16-byte chunks exchanged by key(row), so that neither the keys (16 rows, one chunk
//    each) nor the values (8 rows, two neighbouring chunks) nor the stores meet in a bank.
//  - Scores: S^T[place, row] = K Q^T, the queries in registers.  Output: O^T[dim, row] += V^T P^T, the values read by the transposing
//    LDS read: the places of an instruction in the order in which a lane of S^T holds them.
#include "tree_parts.h"

namespace moesys {
namespace {

// Places in LDS of the 16-byte chunks of a row that lies CHUNKS of them long.
template <int CHUNKS>
__device__ __forceinline__ int key_of(int row) {
  if constexpr (CHUNKS >= 16) return (row & 7) << 1 | (row >> 3 & 1);
  else return (row >> 1 & 3) << 1 | (row >> 3 & 1);  // (two rows to 256 bytes)
}

__device__ __forceinline__ bf16x8 values_of(const char* p, int stride) {
  using Part = __attribute__((address_space(3))) i16x4;
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Part*)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Part*)(p + stride));
  typedef short i16x8 __attribute__((ext_vector_type(8)));
  return __builtin_bit_cast(bf16x8, (__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)));
}

template <bool NT>
__device__ __forceinline__ u32x4 read16(const char* p) {
  const auto* at = (const __attribute__((address_space(1))) u32x4*)(uintptr_t)p;
  if constexpr (NT) return __builtin_nontemporal_load(at);
  else return *at;
}

// FULL: head_dim is DP.  PLAIN: no cap, no slopes.  A wavefront has 16 RB rows of the workgroup's.
template <int DP, int RB, bool FULL, bool NT, bool PLAIN>
__global__ __launch_bounds__(64 * WAVES, 2) void shared_kernel(TreeArgs a) {
  constexpr int TILE = shared_tile(DP, RB), SUB = TILE / 16, PAIRS = SUB / 2, KSTEPS = DP / 32, NDB = DP / 16, PITCH = 2 * DP;
  constexpr int CHUNKS = DP / 8, ROWS = 16 * RB * WAVES, MINE = TILE / WAVES, PER = 64 / CHUNKS, LOADS = MINE / PER;
  constexpr int SETS = RB == 1 && DP <= 128 ? 2 : 1;  // of registers for tiles on their way
  constexpr uint64_t EVERY = TILE == 64 ? ~0ull : (1ull << TILE) - 1;
  // Plain scores are taken as powers of two while the maximum, in these units, is below 2^18.  It is rounded by itself there, and so are a score that is
  // compared with it and its sum with LAG_BITS: by 3 2^-7 in all, which LAG2 makes room for (no weight above 1); beyond 2^32 it would be off by more
  // than all exponents of float32.
  constexpr float LAG2 = LAG_BITS - 0.05f, FAST_BELOW = 0x1p18f;
  __shared__ __attribute__((aligned(1024))) char tiles[2][2][TILE * PITCH];  // [buffer][keys, values]
  __shared__ uint16_t there[2][WAVES];
  __shared__ uint64_t seen_lds[ROWS];
  __shared__ int depth_lds[MOE_MAX_DRAFTS], token_lds[ROWS];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m16 = lane & 15, g = lane >> 4;
  const int w = blockIdx.x / a.items, item = blockIdx.x - w * a.items, rt = a.kv_heads.quotient(item), hk = item - rt * a.hkv;
  Deal at = deal<TILE, shared_least(DP, RB)>(a, rt, w);
  int64_t x = w * at.share;
  const int64_t x_end = x + at.share < at.total ? x + at.share : at.total;
  if (x >= x_end) return;
  const char* zeros = reinterpret_cast<const char*>(ZEROS);

  // this lane's part of a tile: of its wavefront's rows MINE, row PER*i + lane / CHUNKS, one chunk
  const int my_row = lane / CHUNKS, my_chunk = lane % CHUNKS;
  const bool chunk_there = FULL || my_chunk * 8 < a.D;
  const char *k_chunk = a.k + hk * a.head_stride + my_chunk * 16, *v_chunk = a.v + hk * a.head_stride + my_chunk * 16;
  int store_at[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int row = wave * MINE + i * PER + my_row;
    store_at[i] = row * PITCH + (my_chunk ^ key_of<CHUNKS>(row)) * 16;
  }
  // where it reads: keys of row m16 of 16, chunk 4 kstep + g; values of row 4 g + m16 / 4, 4 dims from 4 (m16 % 4) on of 16
  const int key_at = m16 * PITCH + ((g ^ key_of<CHUNKS>(m16)) << 4);
  const int v_row = g * 4 + (m16 >> 2), value_at = v_row * PITCH + (((m16 >> 1 & 1) ^ key_of<CHUNKS>(v_row)) << 4) + (m16 & 1) * 8;

  const float c2 = a.scale * LOG2E;

  for (int piece_no = 0; x < x_end; ++piece_no) {
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

    // The place of lane % MINE of this wavefront's rows of the u-th tile: its table entry, and where its row lies (-1: it is not there).
    auto entry_of = [&](int u) {
      const unsigned column = (unsigned)a.page.quotient((int)((unsigned)span.tile(u) * TILE + wave * MINE + (lane & (MINE - 1)))), last = (unsigned)a.last_column;
      return table[column < last ? column : last];
    };
    auto row_of = [&](int u, int entry) {
      const int p = (int)((unsigned)span.tile(u) * TILE + wave * MINE + (lane & (MINE - 1))), page = u < upto && p < d.len ? valid_page(entry, a.n_pages) : -1;
      return page >= 0 ? page * a.page_stride + (p - a.page.quotient(p) * a.page_size) * a.token_stride : (int64_t)-1;
    };
    // Where this lane's rows of the tile that is loaded next lie, worked out a tile before: what the lanes tell one another takes as long as
    // many products.
    int64_t next[LOADS];
    uint32_t next_there = 0, coming[SETS];  // which of the wavefront's rows are there; of those on their way
    auto place = [&](int64_t row) {
      next_there = (uint32_t)__ballot(row >= 0) & ((1u << MINE) - 1);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int lo = __shfl((int)(uint32_t)row, i * PER + my_row, 64), hi = __shfl((int)(row >> 32), i * PER + my_row, 64);
        next[i] = (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
      }
    };
    u32x4 kr[SETS][LOADS], vr[SETS][LOADS];
    auto load = [&](int set) {
      coming[set] = next_there;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const bool have = next[i] >= 0 && chunk_there;
        kr[set][i] = read16<NT>(have ? k_chunk + next[i] : zeros);
        vr[set][i] = read16<NT>(have ? v_chunk + next[i] : zeros);
      }
    };
    auto put = [&](int set, int buffer) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        *reinterpret_cast<u32x4*>(tiles[buffer][0] + store_at[i]) = kr[set][i];
        *reinterpret_cast<u32x4*>(tiles[buffer][1] + store_at[i]) = vr[set][i];
      }
      if (lane == 0) there[buffer][wave] = (uint16_t)coming[set];
    };

    lds_barrier();  // (the piece before has been read)
    int entry = entry_of(from + 1);
    place(row_of(from, entry_of(from)));
    load(0);
    place(row_of(from + 1, entry));
    entry = entry_of(from + 2);
    if constexpr (SETS == 2) {
      load(1);
      place(row_of(from + 2, entry));
      entry = entry_of(from + 3);
    }
    auto sees = [&](int i) { return seen_drafts(a.words, a.words ? a.words[d.first + i] : 0, i, d.n); };
    if ((int)threadIdx.x < d.n) depth_lds[threadIdx.x] = draft_depth(sees(threadIdx.x), threadIdx.x);
    if ((int)threadIdx.x < ROWS) {
      const int r = threadIdx.x, token = a.group.quotient(rt * ROWS + r);
      seen_lds[r] = r < my_rows ? sees(token) : 0;
      token_lds[r] = r < my_rows ? token : 0;
    }
    const bool active = wave * 16 * RB < my_rows;
    u32x4 q[RB][KSTEPS];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = (wave * RB + rb) * 16 + m16, token = a.group.quotient(rt * ROWS + r), head = rt * ROWS + r - token * a.G;
      const char* from_q = a.q + (int64_t)(d.first + token) * a.q_token + (int64_t)(hk * a.G + head) * a.q_head + g * 16;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) q[rb][ks] = read16<false>(r < my_rows && (FULL || ks * 32 + g * 8 < a.D) ? from_q + ks * 64 : zeros);
    }
    put(0, 0);
    lds_barrier();
    int pos[RB];
    float slope[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = (wave * RB + rb) * 16 + m16;
      pos[rb] = d.base + depth_lds[token_lds[r]];
      slope[rb] = a.slopes && r < my_rows ? a.slopes[hk * a.G + (rt * ROWS + r - token_lds[r] * a.G)] : 0.f;
    }
    const int last_pos = d.base + d.n - 1;  // no position is beyond it

    // Plain scores (no cap, no slopes) are taken as powers of two at once, exp2(c2 z - m), and m is in those units too; others, and those whose
    // maximum is not below FAST_BELOW, keep their own units until the maximum is taken off.
    bool fast = PLAIN && a.scale > 0.f && c2 < 1e30f;
    float m[RB], l[RB];
    f32x4 o[RB][NDB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY;
      l[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Keys of two steps of the contraction index, values of AHEAD instructions are read before they are wanted: a read takes as long as four to eight
    // of the matrix instructions that wait for it, and the compiler by itself keeps none of them ahead.
    constexpr int AHEAD = RB == 1 ? 6 : 4, VALUES = PAIRS * NDB;
    auto read_keys = [&](bf16x8 (&key)[2][SUB], int buffer, int ks) {
#pragma unroll
      for (int st = 0; st < SUB; ++st) key[ks & 1][st] = *reinterpret_cast<const bf16x8*>(tiles[buffer][0] + ((key_at ^ ks << 6) + st * 16 * PITCH));
    };
    auto read_values = [&](int buffer, int n) { return values_of(tiles[buffer][1] + ((value_at ^ (n % NDB) << 5) + n / NDB * 32 * PITCH), 16 * PITCH); };
    // Which places of a tile this lane's rows see, 4 SUB bits to a row.
    auto seen_of = [&](int p0, uint64_t here, uint32_t (&bits)[RB]) {
      uint64_t seen[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        seen[rb] = seen_lds[(wave * RB + rb) * 16 + m16];
        bits[rb] = 0;
      }
#pragma unroll
      for (int st = 0; st < SUB; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int p = p0 + st * 16 + g * 4 + i, j = p - d.base, jj = j & (MOE_MAX_DRAFTS - 1);  // (places that are there have j < n)
          const uint32_t is_there = (uint32_t)(here >> (st * 16 + g * 4 + i)) & 1, cached = j < 0;
          const int pos_p = cached ? p : d.base + depth_lds[jj];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            bits[rb] |= (is_there & (cached | (uint32_t)(seen[rb] >> jj)) & (uint32_t)in_window(pos[rb], pos_p, p, a.window, a.sinks)) << (st * 4 + i);
        }
    };
    auto compute = [&](int p0, int buffer, uint64_t here, bool masked, bf16x8 (&key)[2][SUB]) {
      f32x4 z[RB][SUB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int st = 0; st < SUB; ++st) z[rb][st] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) z[rb][st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[ks & 1][st], __builtin_bit_cast(bf16x8, q[rb][ks]), z[rb][st], 0, 0, 0);
        if (ks + 2 < KSTEPS) read_keys(key, buffer, ks + 2);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!PLAIN) {
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int p = p0 + st * 16 + g * 4 + i;
            int pos_p = p;
            if (p0 > d.base - TILE && p >= d.base) pos_p = d.base + depth_lds[p - d.base < MOE_MAX_DRAFTS ? p - d.base : 0];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
              float s = z[rb][st][i] * a.scale;
              if (a.cap > 0.f) s = a.cap * tanhf(s * a.inv_cap);
              z[rb][st][i] = s - slope[rb] * (float)(pos[rb] - pos_p);
            }
          }
      } else if (__builtin_expect(!fast, 0)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int st = 0; st < SUB; ++st) z[rb][st] *= a.scale;
      }
      if (__builtin_expect(masked, 0)) {
        uint32_t bits[RB];
        seen_of(p0, here, bits);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[rb][st][i] = bits[rb] >> (st * 4 + i) & 1 ? z[rb][st][i] : -INFINITY;
      }
      // The maximum moves only when some score passes it by a factor of nearly 2^8, so that the four lanes of a row need not exchange
      // theirs.  All weights are 2^-8 of what they would be (sums, and so lse, with them): none is above 1, and no product with a
      // finite value overflows.
      float top[RB];
      bool moves = false;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        top[rb] = z[rb][0][0];
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[rb] = fmaxf(top[rb], z[rb][st][i]);
        // (the difference, since a sum can be rounded up; a first score is always one, also where its power is beyond float32)
        moves |= (fast ? top[rb] * c2 : top[rb]) - m[rb] > (fast ? LAG2 : LAG) || (m[rb] == -INFINITY && top[rb] > -INFINITY);
      }
      if (__builtin_expect(__any(moves), 0)) {
        bool far = false;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 16, 64));
          top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 32, 64));
          const float now = fmaxf(m[rb], top[rb] * c2);
          far |= (fabsf(now) >= FAST_BELOW && now != -INFINITY) || (m[rb] == -INFINITY && top[rb] > -INFINITY && now == -INFINITY);
        }
        if (__builtin_expect(fast && __any(far), 0)) {  // (the conversion rounds a maximum as a score of its size is rounded)
          fast = false;
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            m[rb] *= LN2;
            top[rb] = -INFINITY;
#pragma unroll
            for (int st = 0; st < SUB; ++st) {
              z[rb][st] *= a.scale;
#pragma unroll
              for (int i = 0; i < 4; ++i) top[rb] = fmaxf(top[rb], z[rb][st][i]);
            }
            top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 16, 64));
            top[rb] = fmaxf(top[rb], __shfl_xor(top[rb], 32, 64));
          }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const float now = fmaxf(m[rb], fast ? top[rb] * c2 : top[rb]), less = m[rb] - now, f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(fast ? less : less * LOG2E);
          m[rb] = now;
          l[rb] *= f;
#pragma unroll
          for (int db = 0; db < NDB; ++db) o[rb][db] *= f;
        }
      }
      bf16x8 value[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) value[n] = read_values(buffer, n);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float ref = m[rb] == -INFINITY ? 0.f : m[rb];
        if (__builtin_expect(fast, 1)) {
          const float shift = -(ref + LAG_BITS);
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[rb][st][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[rb][st][i], c2, shift));
        } else {
#pragma unroll
          for (int st = 0; st < SUB; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) z[rb][st][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[rb][st][i] - ref, LOG2E, (float)-LAG_BITS));
        }
#pragma unroll
        for (int st = 0; st < SUB; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) l[rb] += z[rb][st][i];
      }
      // A weight enters as the sum of two bfloat16 numbers, each rounded to nearest: 17 bits of it, an error that half a step of the
      // output covers unless 2^8 values cancel.
      u32x4 head[RB][PAIRS], rest[RB][PAIRS];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int pr = 0; pr < PAIRS; ++pr)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w0 = z[rb][2 * pr + i / 2][i % 2 * 2], w1 = z[rb][2 * pr + i / 2][i % 2 * 2 + 1];
            uint32_t h = pack_bf16(w0, w1);
            asm("" : "+v"(h));  // (or each half is rounded once more by itself)
            head[rb][pr][i] = h;
            rest[rb][pr][i] = pack_bf16(w0 - __uint_as_float(h << 16), w1 - __uint_as_float(h & 0xffff0000u));
          }
      // two blocks of dims at a time: four or more products between two of the same sum
#pragma unroll
      for (int n0 = 0; n0 < VALUES; n0 += 2) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int n = n0; n < n0 + 2; ++n)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              o[rb][n % NDB] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value[n % AHEAD], __builtin_bit_cast(bf16x8, part == 0 ? head[rb][n / NDB] : rest[rb][n / NDB]), o[rb][n % NDB], 0, 0, 0);
#pragma unroll
        for (int n = n0; n < n0 + 2; ++n)
          if (n + AHEAD < VALUES) value[n % AHEAD] = read_values(buffer, n + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    // A value that is not finite and that only some rows see would reach the others as 0 times it: its element of the rows that see it becomes
    // NaN, and it leaves the tile.  (All wavefronts find the same.  Nothing of this is in the way of other tiles: a jump over it beside every
    // product, or a second loop of products, costs more than the products.)
    auto without_odd_values = [&](int p0, int buffer, uint64_t here) __attribute__((always_inline)) {
      uint32_t any = 0;
#pragma unroll 1
      for (int n = 0; n < VALUES; ++n) {
        const u32x4 bits = __builtin_bit_cast(u32x4, read_values(buffer, n));
#pragma unroll
        for (int i = 0; i < 4; ++i) any |= not_finite(bits[i]);
      }
      if (__builtin_expect(!__any(any != 0), 1)) return;
      if (active) {
        uint32_t seen[RB];
        seen_of(p0, here, seen);
#pragma unroll
        for (int n = 0; n < VALUES; ++n) {
          u32x4 bad = __builtin_bit_cast(u32x4, read_values(buffer, n));
#pragma unroll
          for (int i = 0; i < 4; ++i) bad[i] = not_finite(bad[i]);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            u32x4 see;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t s = seen[rb] >> ((2 * (n / NDB) + i / 2) * 4 + i % 2 * 2);
              see[i] = (s & 1 ? 0x3f80u : 0u) | (s & 2 ? 0x3f800000u : 0u);
            }
            const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, bad), __builtin_bit_cast(bf16x8, see), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (hit[i] > 0.f) o[rb][n % NDB][i] = NAN;
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      lds_barrier();  // (all have looked)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        u32x4* at = reinterpret_cast<u32x4*>(tiles[buffer][1] + store_at[i]);
        u32x4 bits = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bad = not_finite(bits[e]);
          bits[e] &= ~((bad & 0xffffu ? 0xffffu : 0u) | (bad >> 16 ? 0xffff0000u : 0u));
        }
        *at = bits;
      }
      lds_barrier();
    };
    auto step = [&](int u, auto parity) __attribute__((always_inline)) {
      constexpr int BUFFER = decltype(parity)::value;
      bf16x8 key[2][SUB];
      read_keys(key, BUFFER, 0);
      read_keys(key, BUFFER, 1);
      uint64_t here = 0;
#pragma unroll
      for (int v = 0; v < WAVES; ++v) here |= (uint64_t)there[BUFFER][v] << (v * MINE);
      load(SETS == 2 ? BUFFER : 0);  // tile u + SETS (one behind the last one: zeros)
      place(row_of(u + SETS + 1, entry));
      entry = entry_of(u + SETS + 2);
      __builtin_amdgcn_sched_barrier(0);  // (they are on their way while the tile is worked on)
      const int p0 = span.tile(u) * TILE;
      // Everyone sees everything of a tile that is all there, before the new tokens, and in the window of the last position or among
      // the sinks.
      const bool masked = here != EVERY || p0 > d.base - TILE || (a.window > 0 && last_pos - p0 >= a.window && p0 > a.sinks - TILE);
      if (__builtin_expect(masked, 0)) without_odd_values(p0, BUFFER, here);
      if (active) compute(p0, BUFFER, here, masked, key);
      __builtin_amdgcn_sched_barrier(0);
      put(SETS == 2 ? BUFFER ^ 1 : 0, BUFFER ^ 1);
      lds_barrier();
    };
    for (int u = from; u < upto; u += 2) {
      step(u, std::integral_constant<int, 0>());
      if (u + 1 >= upto) break;
      step(u + 1, std::integral_constant<int, 1>());
    }

#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      l[rb] += __shfl_xor(l[rb], 16, 64);
      l[rb] += __shfl_xor(l[rb], 32, 64);
      const int r = (wave * RB + rb) * 16 + m16;
      if (r >= my_rows) continue;
      const float top = fast ? m[rb] * LN2 : m[rb];
      const int token = token_lds[r], head = rt * ROWS + r - token * a.G;
      const int64_t part = ((int64_t)slot * a.items + item) * ROWS + r;
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const int dim = db * 16 + g * 4;
        if (!FULL && dim >= a.D) continue;
        if (whole) store_row<__bf16>(a, d.first + token, hk * a.G + head, dim, o[rb][db], l[rb], top);
        else *reinterpret_cast<f32x4*>(a.part_o + part * a.D + dim) = o[rb][db];
      }
      if (!whole && g == 0) a.part_ml[part] = f32x2{top, l[rb]};
    }
    x = b_end;
    at.begin = b_end;
    if (++at.b >= a.n_seqs) break;
  }
}

template <int DP, int RB>
void launch(const TreeArgs& a, unsigned grid, bool nt, hipStream_t s) {
  auto of = [&](auto full, auto past, auto plain) {
    hipLaunchKernelGGL((shared_kernel<DP, RB, decltype(full)::value, decltype(past)::value, decltype(plain)::value>), dim3(grid), dim3(64 * WAVES), 0, s, a);
  };
  const std::true_type yes;
  const std::false_type no;
  auto with = [&](auto plain) {
    if (a.D == DP) nt ? of(yes, yes, plain) : of(yes, no, plain);
    else nt ? of(no, yes, plain) : of(no, no, plain);
  };
  if (a.cap == 0.f && !a.slopes) with(yes);
  else with(no);
}

}  // namespace

int32_t launch_tree_shared(const TreeArgs& a, int blocks, unsigned grid, bool nt, hipStream_t s) {
  if (a.D > 128) launch<256, 1>(a, grid, nt, s);
  else if (a.D > 64) blocks == 1 ? launch<128, 1>(a, grid, nt, s) : launch<128, 2>(a, grid, nt, s);
  else blocks == 1 ? launch<64, 1>(a, grid, nt, s) : launch<64, 2>(a, grid, nt, s);
  return check_hip(hipGetLastError(), "tree attention launch");
}

}  // namespace moesys
