// Places of a paged cache and which of them a new token attends to.  Plain C++ for the host as well: the CPU tests run it.
#pragma once
#include <stdint.h>

#ifdef __HIPCC__
#define MOESYS_HD __host__ __device__ __forceinline__
#else
#define MOESYS_HD inline
#endif

namespace moesys {

// Places of a sequence as attention takes them: a length outside what the table can hold is clamped to it.
MOESYS_HD int kept_length(int len, int capacity) { return len < 0 ? 0 : len > capacity ? capacity : len; }

// First place that a window leaves (0: no window).
MOESYS_HD int first_place(int len, int window) { return window > 0 && len > window ? len - window : 0; }

// Tiles (of `tile` places, aligned to multiples of it) that hold the kept places first .. n-1.
MOESYS_HD int kept_tiles(int n, int first, int tile) { return n > 0 ? (n - 1) / tile - first / tile + 1 : 0; }

// Page that a table entry names, or -1: a page that is not there.
MOESYS_HD int valid_page(int entry, int64_t n_pages) { return entry >= 0 && entry < n_pages ? entry : -1; }

// Division of 0..2^31-1 by a page size: with 2^(s-1) < d <= 2^s and mul = ceil(2^(31+s) / d), mul*d exceeds 2^(31+s) by less
// than d <= 2^s, so p*mul >> (31+s) is the quotient for every p < 2^31.
struct PageDivisor {
  uint32_t mul, shift;
  MOESYS_HD int quotient(int p) const { return (int)(((uint64_t)(uint32_t)p * mul) >> shift); }
};
inline PageDivisor page_divisor(int d) {
  uint32_t s = 0;
  while ((1ull << s) < (uint64_t)d) ++s;
  return PageDivisor{(uint32_t)(((1ull << (31 + s)) + (uint64_t)d - 1) / (uint64_t)d), 31 + s};
}

// How attention splits over the length.  A sequence's kept places lie in tiles; `items` workgroups (key-value heads times tiles
// of query heads) each work on every tile.  One size c of chunks for the whole batch, from the lengths alone: about `target`
// workgroups in all, at least `least` tiles a chunk.  With c >= total*items/target the sum over the sequences of ceil(tiles/c)
// is at most target/items + sequences, which is what the grid and the workspace are made for.
MOESYS_HD int chunk_tiles(int64_t total_tiles, int items, int target, int least) {
  const int64_t c = (total_tiles * items + target - 1) / target;
  return c < least ? least : (int)c;
}
// Chunks of a sequence (an empty one has one, which writes its zeros).
MOESYS_HD int chunk_count(int tiles, int c) { return tiles <= c ? 1 : (tiles - 1) / c + 1; }
// First tile of chunk j of n: even shares, the first ones one longer.
MOESYS_HD int chunk_begin(int tiles, int n, int j) {
  const int share = tiles / n, rest = tiles % n;
  return j * share + (j < rest ? j : rest);
}
// The most chunks a batch can have, whatever its lengths.
inline int64_t most_chunks(int64_t sequences, int items, int target, int least, int64_t tiles_per_sequence) {
  const int64_t each = tiles_per_sequence <= least ? 1 : (tiles_per_sequence - 1) / least + 1;
  const int64_t split = target / items + sequences;
  return each * sequences < split ? each * sequences : split;
}

}  // namespace moesys
