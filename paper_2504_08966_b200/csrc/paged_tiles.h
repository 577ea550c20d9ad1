// How the attention over a paged cache shares out its work: which tiles a CTA has, and where the rows of a tile lie.  Plain functions, so that
// they can be run on the host as well.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define PAGED_HD __host__ __device__ __forceinline__
#else
#define PAGED_HD inline
#endif

namespace pact {

constexpr int kTile = 64;                  // rows of a tile
constexpr int kRowsOfWarp = 16;

// Tiles of one key head of a request with `rows` cached rows: of all its rows, or of the first n_select entries of its list of pages (but no more entries
// than it has pages).
PAGED_HD int tiles_of_request(int rows, int page, bool selected, int n_select) {
  if (!selected) return (int)(((unsigned)rows + kTile - 1u) / kTile);
  const long long have = (long long)(((unsigned)rows + (unsigned)page - 1u) / (unsigned)page), pages = have < n_select ? have : n_select;
  return (int)((pages * page + kTile - 1) / kTile);
}

// T tiles in G shares of floor(T / G) or one more, G <= T: the first tile of share i, and the share that tile t is in.
PAGED_HD long long share_begin(long long i, long long G, long long T) { return i * T / G; }
PAGED_HD long long share_of(long long t, long long G, long long T) { return ((t + 1) * G - 1) / T; }

// u / n and the rest for 0 <= u < 256 n, 1 <= n < 2^26: the quotient in fp32, a few units in its last place off, is off by one at most.
template <typename I> PAGED_HD int divide_small(I u, int n, int *rest) {
#ifdef __CUDA_ARCH__
  int h = (int)__fdividef((float)u, (float)n);
#else
  int h = (int)((float)u / (float)n);
#endif
  I r = u - (I)h * n;
  if (r < 0) {
    --h;
    r += n;
  } else if (r >= n) {
    ++h;
    r -= n;
  }
  *rest = (int)r;
  return h;
}

// Page and place of every 16 rows of tile j, and how many of them count (a byte each).  A page id outside the cache makes its rows count for nothing and
// sets `bad`.  per_box: 16 rows times this always lie in one page.
struct TileRows {
  int id[4], off[4];
  uint32_t rows;
  bool bad;
};
PAGED_HD TileRows locate_rows(int j, int len, int page, int per_box, const int32_t *table, int n_pages, const int32_t *selected, int n_select) {
  TileRows t;
  t.rows = 0;
  t.bad = false;
  const int pages = (int)(((unsigned)len + (unsigned)page - 1u) / (unsigned)page), listed = selected && n_select < pages ? n_select : pages;
  const unsigned r = (unsigned)j * kTile, first = r / (unsigned)page;   // (below 2^31 + 64 * 1024)
  int place[4], at = (int)first, off = (int)(r - first * (unsigned)page);
#define PAGED_EACH(g) for (int g = 0; g < 4; ++g)
#ifdef __CUDACC__
#define PAGED_UNROLL _Pragma("unroll")
#else
#define PAGED_UNROLL
#endif
  PAGED_UNROLL PAGED_EACH(g) {
    t.off[g] = off;
    place[g] = at < listed ? at : -1;
    off += kRowsOfWarp;
    if (off >= page) {                     // (a page is a multiple of 16 rows)
      off = 0;
      ++at;
    }
  }
  // first all places, then all pages: a trip to memory each
  if (selected) PAGED_UNROLL PAGED_EACH(g) if (g % per_box == 0 && place[g] >= 0) place[g] = selected[place[g]];
  PAGED_UNROLL PAGED_EACH(g) {
    const bool there = g % per_box == 0 && place[g] >= 0 && place[g] < pages && len - (int)((unsigned)place[g] * (unsigned)page + (unsigned)t.off[g]) > 0;
    t.id[g] = there ? table[place[g]] : -1;
    if (!there) place[g] = -1;
  }
  int left = 0;
  PAGED_UNROLL PAGED_EACH(g) {
    if (g % per_box == 0) {                // a box lies in one page
      left = place[g] < 0 ? 0 : len - (int)((unsigned)place[g] * (unsigned)page + (unsigned)t.off[g]);
      if (left > 0 && (t.id[g] < 0 || t.id[g] >= n_pages)) {
        t.bad = true;
        left = 0;
      }
    } else {
      left -= kRowsOfWarp;
    }
    if (left > 0) t.rows |= (uint32_t)(left < kRowsOfWarp ? left : kRowsOfWarp) << (8 * g);
  }
#undef PAGED_EACH
#undef PAGED_UNROLL
  return t;
}

}  // namespace pact
