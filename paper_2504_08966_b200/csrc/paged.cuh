// The paged cache and the attention of one new token over it: kernel arguments and launchers.
#pragma once
#include <cuda.h>

#include "kernels.cuh"

namespace pact {

// ---- cache_plan.cu -------------------------------------------------------------------------------------

struct PlanArgs {
  int32_t *table;
  const int32_t *length, *n_new;
  long long n_new_stride;
  int32_t *free_pages;
  const int32_t *n_free;
  int32_t *length_out, *n_free_out, *row_start;
  int64_t *slot;
  long long n_rows;
  int32_t *status;
  int B, width, page, n_pages, row_stride;
  bool rows;             // this launch writes pages and slots
  bool commit;           // this launch writes lengths, the number of free pages and the row starts
};
cudaError_t launch_cache_plan(PlanArgs a, int sm_count, cudaStream_t st, int *launches);
cudaError_t plan_configure();

// ---- cache_write.cu ------------------------------------------------------------------------------------

struct WriteArgs {
  const void *Kn, *Vn;
  long long ld_row, ld_head;
  const float *logw_new;
  const int64_t *slot;
  long long n_rows;
  void *K, *V;
  long long k_page, k_head, k_row, v_page, v_head, v_row;
  float *logw;
  void *bounds;
  float *w_max;
  int32_t *status;
  int n_pages, page, n_kvh, d_h;
};
cudaError_t launch_cache_write(const WriteArgs &a, bool bf16, int sm_count, cudaStream_t st);

// ---- page_select.cu ------------------------------------------------------------------------------------

constexpr int kMaxSelectPages = 65536;
constexpr int kPickKeys = 8192;            // scores of a request and head that are kept in shared memory
struct SelectArgs {
  const void *Q;
  long long ldQ, ldQh;
  const void *bounds;
  const float *w_max;
  const int32_t *table, *length;
  int32_t *selected, *status;
  unsigned long long *keys;   // [B][n_kvh][width] scores in double, where many are in doubt, as integers that order like them
  uint32_t *approx;           // [B][n_kvh][width] scores in fp32, where they are too many for shared memory
  float scale;
  int B, width, page, n_pages, n_kvh, group, d_h;
  int n_first, n_last, n_select;
};
cudaError_t launch_page_select(const SelectArgs &a, bool bf16, int most_ctas, int sm_count, cudaStream_t st);   // most_ctas: of a cluster
cudaError_t select_pages_configure(int d_h, bool bf16);

// ---- paged_attention.cu --------------------------------------------------------------------------------

struct AttendArgs {
  const void *Q;
  long long ldQ, ldQh;
  const float *logw;
  const int32_t *table, *length, *selected;
  void *out;
  long long ldO, ldOh;
  float *lse;
  int32_t *status;
  float *part_o;         // [2 CTAs][heads of a tile][columns] sums of the parts of a request that several CTAs share
  float2 *part_ml;       // [2 CTAs][heads of a tile] their running maximum and sum
  int4 *desc;            // [CTAs] what was cut at the beginning of a CTA's share
  float scale;
  int B, width, page, n_pages, n_select;
  int n_kvh, group, d_h, head_tiles;
  int box_rows;          // rows of one copy: the largest of 64, 32, 16 that divides the page
  int stages;
  int polls;             // of a wait for copies, or for a free stage
  bool whole_blocks;     // a row is a whole number of 128-byte blocks
  bool out_bf16;
};

// What a context knows about the attention kernels for its heads; filled by paged_configure.
struct PagedCfg {
  void *encode_tiled = nullptr;   // cuTensorMapEncodeTiled
  int blocks = 0;                 // 128-byte blocks of a row; 0: no kernel for this head width
  int tile_heads = 0;             // query heads of a key head that a CTA takes at once
  int head_tiles = 0;
  int cluster = 1;                // largest cluster of CTAs that can be launched
  int clusters[4] = {};           // clusters of 2, 4, 8 and 16 that fit the device at once
};
cudaError_t paged_configure(PagedCfg *cfg, const DeviceCfg &dev, int n_qh, int n_kvh, int d_h, bool bf16);
// bytes of workspace of a call; with `a` its slices are set too
size_t attend_scratch(const PagedCfg &cfg, const DeviceCfg &dev, bool bf16, AttendArgs *a, char *base);
cudaError_t launch_attend(AttendArgs a, const pact_paged_cache &cache, const PagedCfg &cfg, const DeviceCfg &dev, bool bf16, cudaStream_t st,
                          int *launches);

}  // namespace pact
