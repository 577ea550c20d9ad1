"""Attention of several new tokens, on the host: sizes at which the arithmetic of csrc/chunk_tiles.h could leave 32 bits."""
from tests.test_paged_cpu import CSRC, _run


def test_requests_that_fit_their_rows_fit_into_32_bits(tmp_path):
    """Whatever row starts and counts the device finds: either the rows that all requests are served are no more than there are, and then items and tiles stay within what the host has
    checked for as many rows, or the call serves none."""
    _run(tmp_path, r"""
#include <stdio.h>
#include <stdlib.h>
#include "chunk_tiles.h"
using namespace pact;
static long long below(long long n) { return (((long long)rand() << 31) ^ rand()) % n; }
int main() {
  srand(2);
  int accepted = 0, refused = 0, too_many = 0;
  for (int trial = 0; trial < 6000; ++trial) {
    const int rows = 64 << trial % 3, tile = trial % 2 ? 64 : 128, group = 1 + rand() % (trial % 5 ? 8 : 300), heads = 1 + rand() % 16;
    const int B = trial % 4 ? 1 + rand() % 40 : 4096;
    const long long n_rows = 1 + below(1ll << (1 + rand() % 31)), width = 1 + below(1ll << (1 + rand() % 31));
    // as pact_chunk_attention checks
    const long long most_items = (n_rows * group / rows + B) * heads, most_tiles = (width + n_rows) / tile + 1;
    if (n_rows > INT32_MAX / group || most_items > INT32_MAX / 2 || most_items > INT32_MAX / most_tiles) continue;
    unsigned long long served = 0, items = 0, tiles = 0;
    for (int b = 0; b < B; ++b) {
      const long long start = trial % 3 == 0 ? 0 : below(n_rows + 1), want = trial % 3 == 1 ? below(n_rows / B + 1) : below(INT32_MAX), len = below(width + 1);
      ChunkLengths q;
      q.want = (int)want;
      q.n = (int)(want < n_rows - start ? want : n_rows - start);
      q.len = (int)(len < INT32_MAX ? len : INT32_MAX);
      served += q.n;
      items += (unsigned long long)chunk_items(q, group, rows) * heads;
      tiles += chunk_tiles_of_head(q, group, rows, tile, trial & 1) * heads;
    }
    if (!chunk_rows_fit(served, n_rows)) {
      ++refused;
      too_many += items > INT32_MAX || tiles > INT32_MAX;
      continue;
    }
    ++accepted;
    if (items > (unsigned long long)most_items || tiles > INT32_MAX) { printf("%llu items of %lld, %llu tiles\n", items, most_items, tiles); return 1; }
  }
  if (accepted < 300 || refused < 300 || too_many < 30) { printf("%d accepted, %d refused, %d of them too many\n", accepted, refused, too_many); return 1; }
  if (!chunk_rows_fit(0, 0) || chunk_rows_fit(1, 0) || !chunk_rows_fit(INT32_MAX, INT32_MAX) || chunk_rows_fit(4096ull * INT32_MAX, INT32_MAX)) return 1;
  return 0;
}""", ["g++", "-O2", "-std=c++17", "-I", CSRC])


def test_edges_at_the_largest_lengths(tmp_path):
    """Whether a tile has rows that some token does not see, against 64 bits: lengths up to 2^31 - 1."""
    _run(tmp_path, r"""
#include <stdio.h>
#include <initializer_list>
#include "chunk_tiles.h"
using namespace pact;
int main() {
  const int ends[] = {0, 1, 2, 63, 64, 127, 128, 129, 1000, 1 << 30, INT32_MAX - 200, INT32_MAX - 128, INT32_MAX - 127, INT32_MAX - 126, INT32_MAX - 64, INT32_MAX - 15, INT32_MAX - 1, INT32_MAX};
  int past = 0;
  for (int seen : ends)
    for (int tile : {64, 128})
      for (int at : ends)
        for (int back = 0; back < 3; ++back) {
          const long long row0 = ((long long)at / tile - back) * tile;
          if (row0 < 0) continue;
          const bool edge = row0 + tile > seen;
          past += row0 + tile > INT32_MAX;
          if (chunk_edge((int)row0, tile, seen) != edge) { printf("row %lld, tile %d, seen %d\n", row0, tile, seen); return 1; }
        }
  return past > 100 ? 0 : 1;
}""", ["g++", "-O2", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC])


def test_what_a_token_sees_beside_the_largest_counts(tmp_path):
    """Against 64 bits: lengths up to 2^31 - 1, and up to as many more new tokens than rows."""
    _run(tmp_path, r"""
#include <stdio.h>
#include "chunk_tiles.h"
using namespace pact;
int main() {
  const int ends[] = {0, 1, 2, 63, 64, 127, 128, 129, 1000, 1 << 30, INT32_MAX - 200, INT32_MAX - 128, INT32_MAX - 127, INT32_MAX - 126, INT32_MAX - 64, INT32_MAX - 15, INT32_MAX - 1, INT32_MAX};
  int none = 0;
  for (int len : ends)
    for (int want : ends)
      for (int token : ends)
        for (int causal = 0; causal < 2; ++causal) {
          if (token >= want) continue;
          const ChunkLengths q = {want, want, len};
          long long sees = causal ? (long long)len - want + token + 1 : len;
          sees = sees < 0 ? 0 : sees > len ? len : sees;
          none += sees == 0 && len > 0;
          if (chunk_seen(q, token, causal) != sees) { printf("%d rows, %d new, token %d: %d instead of %lld\n", len, want, token, chunk_seen(q, token, causal), sees); return 1; }
        }
  return none > 100 ? 0 : 1;
}""", ["g++", "-O2", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC])
