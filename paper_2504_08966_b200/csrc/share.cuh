// Pages that several requests hold: kernel arguments and launchers.
#pragma once
#include "kernels.cuh"

namespace pact {

constexpr int kShareCtas = 8;              // of the one cluster that a call is
constexpr int kShareThreads = 1024;
constexpr int kShareChunk = 64;            // entries of a block table that a warp looks at

struct ShareArgs {
  const int32_t *table, *length, *source, *rows, *shared, *free_pages, *n_free;
  int32_t *table_out, *length_out, *shared_out, *free_out, *n_free_out, *moved_to, *copies, *n_copies, *status;
  int B, width, page, n_pages, n_list;     // n_list: entries of `copies`
  // workspace of a fork: of each page the holders in the old tables, those in the new ones that have it full, the first request that ends in it and the first place that
  // named it; pages that go back, in order; of each chunk of entries how many do; of each request whether it copies; what one CTA tells the others
  int32_t *held, *full, *tail, *first, *freed, *chunk_freed, *copies_tail;
  int32_t *totals;                         // [8]
  int32_t *bad;                            // [kShareCtas] a status of each CTA
  // workspace of a compaction: a bit for each free page, free ids among the first and used ids beyond them in order, how many of each CTA
  uint32_t *free_bits;
  int32_t *holes, *strays, *counts;
};
size_t fork_scratch(int requests, int max_pages, int n_pages, ShareArgs *a, char *base);
size_t compact_scratch(int n_pages, ShareArgs *a, char *base);
cudaError_t share_configure();
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
