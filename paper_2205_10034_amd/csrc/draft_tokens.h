// The new tokens of a sequence: which rows are theirs, where they stand and what they see.  Plain C++ for the host as well: the CPU
// tests run it.
#pragma once
#include "kv_pages.h"

namespace moesys {

// Rows of a sequence's new tokens, and its places: base cached ones, then the tokens' own, len in all.
struct Drafts {
  int first, n, base, len;
};
MOESYS_HD Drafts drafts_of(int from, int to, int T, int max_new, int len, int capacity) {
  Drafts d;
  d.first = from < 0 ? 0 : from > T ? T : from;
  const int end = to < d.first ? d.first : to > T ? T : to;
  d.n = end - d.first < max_new ? end - d.first : max_new;
  d.len = kept_length(len, capacity);
  d.base = d.len > d.n ? d.len - d.n : 0;
  return d;
}

MOESYS_HD int bits_set(uint64_t v) { return __builtin_popcountll(v); }
// Words of n tokens: bits 0 .. n-1 mean something.
MOESYS_HD uint64_t drafts_mask(int n) { return n >= 64 ? ~0ull : (1ull << n) - 1; }
// What token i of n sees of the new tokens; word: its own, or without words itself and those before it.
MOESYS_HD uint64_t seen_drafts(bool words, uint64_t word, int i, int n) { return (words ? word : i >= 63 ? ~0ull : (2ull << i) - 1) & drafts_mask(n); }
// How far behind the cache token i stands.
MOESYS_HD int draft_depth(uint64_t seen, int i) { return bits_set(seen & ~(1ull << i)); }

// Whether a window shows place p, at position pos_p, to a token at position pos.  (Distances are below 2^31.)
MOESYS_HD bool in_window(int pos, int pos_p, int p, int window, int sinks) { return (window <= 0) | (pos - pos_p < window) | (p < sinks); }

// Tiles of places that some new token can see: `sinks` of them from the first place on, then those from `from` on, `tiles` in all.
struct Span {
  int sinks, from, tiles;
  MOESYS_HD int tile(int u) const { return u < sinks ? u : u - sinks + from; }
};
MOESYS_HD Span span_of(const Drafts& d, int window, int sinks, int tile) {
  Span s{0, 0, 0};
  if (d.len <= 0) return s;
  const int upto = (d.len - 1) / tile + 1;
  if (window > 0 && d.base >= window) {  // (no token stands before the base: what lies window or more behind it is seen by none)
    const int from = (d.base - window + 1) / tile, shown = sinks < d.len ? sinks : d.len, front = shown > 0 ? (shown - 1) / tile + 1 : 0;
    if (front < from) {
      s.sinks = front;
      s.from = from;
    }
  }
  s.tiles = s.sinks + upto - s.from;
  return s;
}

}  // namespace moesys
