// How the attention of several new tokens per request shares out its work: items (256 or 128 rows of one key head of a request) and their tiles of cached
// rows.  Plain functions, so that they can be run on the host as well.
#pragma once
#include <stdint.h>

#include "paged_tiles.h"

namespace pact {

// sum of floor((a i + b) / m) over i = 0 .. n - 1: whole multiples of m leave a and b, what is left counts lattice points below a line, and counting them
// along the other axis gives a shorter sum of the same kind (the steps of Euclid's algorithm).
// (In 32 bits where they are enough: a division in 64 takes as long as the rest of the set-up of a call with few requests.)
template <typename I> PAGED_HD unsigned long long floor_sum_in(I n, I m, I a, I b) {
  unsigned long long sum = 0;
  while (n) {
    if (a >= m) {
      sum += (unsigned long long)(n & 1 ? (unsigned long long)n * ((n - 1) / 2) : (unsigned long long)(n / 2) * (n - 1)) * (a / m);
      a %= m;
    }
    if (b >= m) {
      sum += (unsigned long long)n * (b / m);
      b %= m;
    }
    const I top = a * n + b;
    if (top < m) break;
    n = top / m;
    b = top % m;
    const I t = m;
    m = a;
    a = t;
  }
  return sum;
}
PAGED_HD unsigned long long floor_sum(unsigned long long n, unsigned long long m, unsigned long long a, unsigned long long b) {
  // (a and b fall below m in the first step and m never grows, so a n + b stays below m (n + 1))
  if (n < (1u << 31) && m < (1u << 31) && a < (1u << 31) && b < (1ull << 32) && m * (n + 1) < (1ull << 32)) return floor_sum_in<unsigned>((unsigned)n, (unsigned)m, (unsigned)a, (unsigned)b);
  return floor_sum_in<unsigned long long>(n, m, a, b);
}

// Requests whose rows overlap may be served more rows in all than there are, and their items and tiles go beyond the 32 bits that the host has checked for n_rows of them.  (`rows` of at most
// PACT_MAX_REQUESTS requests, each below 2^31.)
PAGED_HD bool chunk_rows_fit(unsigned long long rows, long long n_rows) { return rows <= (unsigned long long)n_rows; }

// One request of a chunk: `n` new tokens that are served out of `want`, the last of `len` cached rows.
struct ChunkLengths {
  int n, want, len;
};
PAGED_HD int chunk_before(const ChunkLengths &q) { return q.len > q.want ? q.len - q.want : 0; }   // rows cached before the new ones
// Rows that a token sees: none where there are more new tokens than rows and it comes before the first (by up to 2^31 - 2 rows, so that nothing could be taken from a negative number).
PAGED_HD int chunk_seen(const ChunkLengths &q, int token, bool causal) {
  const int seen = causal ? q.len - q.want + token + 1 : q.len;
  return seen < 0 ? 0 : seen < q.len ? seen : q.len;
}
// Whether a tile from row0 on has rows beyond `seen` (which is not negative: row0 + tile may be 2^31).
PAGED_HD bool chunk_edge(int row0, int tile, int seen) { return seen - row0 < tile; }
PAGED_HD int chunk_items(const ChunkLengths &q, int group, int rows) { return (int)(((unsigned)q.n * (unsigned)group + (unsigned)rows - 1u) / (unsigned)rows); }   // (n g < 2^31)
// Tiles of `tile` rows that item i of a key head meets.  Its last row is of token ceil(min(n g, (i + 1) rows) / g) - 1.
PAGED_HD int chunk_tiles(const ChunkLengths &q, int i, int group, int rows, int tile, bool causal) {
  if (!causal) return q.len > tile ? (int)(((unsigned)q.len + tile - 1u) / (unsigned)tile) : 1;
  const unsigned all = (unsigned)q.n * (unsigned)group, end = (unsigned)(i + 1) * (unsigned)rows;
  const int tokens = end < all ? (int)((end + (unsigned)group - 1u) / (unsigned)group) : q.n;
  return (int)(((unsigned)chunk_before(q) + (unsigned)tokens + tile - 1u) / (unsigned)tile);
}
// The same over all items of a key head (a division by g and one by the tile in turn round up like one by their product).
PAGED_HD unsigned long long chunk_tiles_of_head(const ChunkLengths &q, int group, int rows, int tile, bool causal) {
  const int items = chunk_items(q, group, rows);
  if (items == 0) return 0;
  const int last = chunk_tiles(q, items - 1, group, rows, tile, causal);
  if (!causal) return (unsigned long long)items * last;
  if (items <= 8) {                        // (fewer steps than those of the sum)
    unsigned long long sum = last;
    for (int i = 0; i + 1 < items; ++i) sum += chunk_tiles(q, i, group, rows, tile, true);
    return sum;
  }
  const unsigned long long m = (unsigned long long)group * tile;
  return floor_sum((unsigned long long)items - 1, m, rows, (unsigned long long)chunk_before(q) * group + rows + m - 1) + last;
}

}  // namespace pact
