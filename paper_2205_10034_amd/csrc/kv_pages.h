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

// A launch holds fewer than 2^32 work-items: more are refused before anything of the call runs.
inline bool launchable(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }

// How attention deals the batch out.  The sequences' tiles stand in one row, sequence after sequence, an empty one as one tile
// (somebody has to write its zeros); part w of the row is the tiles w*share .. (w+1)*share - 1.  A part holds pieces of one or more
// sequences; a sequence that lies in one part is finished there, the pieces of the others are joined.
MOESYS_HD int64_t row_tiles(int tiles) { return tiles > 0 ? tiles : 1; }
// Tiles of a part: total / parts rounded up, which `parts` of them hold the row with, at least `least`.  inverse = 1.0 / parts; half a
// tile below, the product is further from a whole number than its rounding reaches.
MOESYS_HD int64_t share_of_row(int64_t total, double inverse, int least) {
  const int64_t share = (int64_t)(((double)total - 0.5) * inverse) + 1;
  return share < least ? least : share;
}
// A sequence's place in a row where sequences begin parts: whole shares.  (Tiles and shares are below 2^31.)
MOESYS_HD int64_t aligned_tiles(int64_t tiles, int64_t share) { return (int64_t)(((uint32_t)tiles + (uint32_t)share - 1u) / (uint32_t)share) * share; }
// Part that tile `at` of the row lies in; the quotient in float64 is off by one at most.
MOESYS_HD int part_of(int64_t at, int64_t share) {
  int64_t w = (int64_t)((double)at / (double)share);
  if (w * share > at) --w;
  if ((w + 1) * share <= at) ++w;
  return (int)w;
}
// Pieces that can be unfinished are a part's first and its last: two slots for each part, 2w for the first piece.  Slot of piece j of
// a sequence whose first piece has slot `first`: it goes on as the first piece of the parts that follow.
MOESYS_HD int piece_slot(int first, int j) { return j == 0 ? first : (first / 2 + j) * 2; }

}  // namespace moesys
