// Pages that several requests hold: kernel arguments and launchers.
#pragma once
#include "kernels.cuh"

namespace pact {

constexpr int kShareCtas = 16;             // of the one cluster that a call is
constexpr int kShareThreads = 1024;
constexpr int kShareChunk = 64;            // entries of a block table that a warp looks at

struct alignas(16) SharePage {             // (one access of 16 bytes)
  int32_t held, full, tail, first;         // holders in the old tables; in the new ones with all rows; the first request that ends in it; the first place that named it
};
struct alignas(16) ShareSum {              // of a CTA: entries of two kinds, and its status
  int32_t a, b, bad, unused;
};
struct ShareArgs {
  const int32_t *table, *length, *source, *rows, *shared, *free_pages, *n_free;
  int32_t *table_out, *length_out, *shared_out, *free_out, *n_free_out, *moved_to, *copies, *n_copies, *status;
  int B, width, page, n_pages, n_list;     // n_list: entries of `copies`
  // workspace of a fork: what is known of each page; pages that go back, in order; of each chunk of entries how many go back in those before it, and a bit for each that is the
  // first place of its page, and for each whose page goes back
  SharePage *pages;
  int32_t *freed, *chunk_freed;
  uint64_t *chunk_first, *chunk_gone;
  ShareSum *sums;                          // [kShareCtas] what one CTA tells the others
  // workspace of a compaction: a bit for each free page, free ids among the first and used ids beyond them in order
  uint32_t *free_bits;
  int32_t *holes, *strays;
  uint64_t page_mul;                       // ceil(2^33 / (page / 16))
};
// n / page for n below 2^31 + 1024, by a multiplication: with n' = n / 16, p = page / 16 <= 64 and 2^33 <= p page_mul < 2^33 + 64, n' page_mul / 2^33 is above n' / p by less than 1 / p.
__host__ __device__ inline int page_of(uint64_t page_mul, unsigned n) { return (int)((n >> 4) * page_mul >> 33); }
size_t fork_scratch(int requests, int max_pages, int n_pages, ShareArgs *a, char *base);
size_t compact_scratch(int n_pages, ShareArgs *a, char *base);
bool share_fits();                         // whether the device can launch that cluster; before the first launch
cudaError_t launch_cache_fork(const ShareArgs &a, cudaStream_t st);
cudaError_t launch_cache_compact(const ShareArgs &a, cudaStream_t st);

struct PageCopyArgs {
  void *K, *V;
  long long k_page, k_head, k_row, v_page, v_head, v_row;
  float *logw;
  void *bounds;
  float *w_max;
  const int32_t *copies, *n_copies;
  int32_t *status;
  int n_list, n_pages, page, n_kvh, d_h, elt;
};
cudaError_t launch_page_copy(const PageCopyArgs &a, int sm_count, cudaStream_t st);

}  // namespace pact
