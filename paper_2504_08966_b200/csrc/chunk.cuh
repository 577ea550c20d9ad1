// Attention of several new tokens per request over the paged cache: kernel arguments and launchers.
#pragma once
#include <cuda.h>

#include "paged.cuh"

namespace pact {

constexpr int kChunkMaxSms = 176;          // most CTAs of a call
constexpr int kChunkPoison = 8;            // segments whose columns with infinite values are remembered at a time
constexpr int kChunkMaxWidth = 256;

// What the join finds about an item of the last round: whether it was cut; whether a CTA began it; the first and the last of the CTAs that share the rest; its
// key head, rows, first row among those of its request, and the request's first row of out.
struct ChunkCut {
  int cut, head, first, last;
  int kv, rows, first_row, reserved;
  long long row0;
};

struct ChunkArgs {
  const void *Q;
  long long ldQ, ldQh;
  const float *logw;
  const int32_t *table, *length, *n_new, *row_start;
  long long n_new_stride, n_rows;
  void *out;
  long long ldO, ldOh;
  float *lse;
  int32_t *status;
  // workspace
  float *part_o;         // [4 CTAs][width / 4][rows of an item][4] sums of the parts of items that several CTAs share, and sums of earlier tiles while a part (or a whole item) is worked on
  float2 *part_ml;       // [4 CTAs][rows of an item] their reference logit and sum
  ChunkCut *cut;         // [2 CTAs]
  int *tail;             // [CTAs] tiles that each CTA has of the line of rests
  int *head;             // [CTAs][CTAs] tiles at the beginning of an item that its CTA takes; a copy for each CTA
  int *pre;              // [CTAs][requests + 1] items of a key head before each request, where they do not fit into shared memory
  int *poison;           // [CTAs][kChunkPoison][kChunkMaxWidth] first row of a segment with an infinity or a NaN in each column of its values
  float scale;
  int B, width, page, n_pages, row_stride;
  int n_kvh, group, d_h;
  int box_rows;          // rows of one copy: the largest of 128, 64, 32, 16 that divides the page and is at most a tile
  int polls;             // of a wait
  int store_bytes;       // rows of out lie at multiples of: 8 (bf16), 16 or 32
  bool causal, out_bf16;
};

// What a context knows about these kernels for its heads; filled by chunk_configure.
struct ChunkCfg {
  void *encode_tiled = nullptr;   // cuTensorMapEncodeTiled
  int blocks = 0;                 // 128-byte blocks of a row; 0: no kernel for this head width
  bool bf16 = false, wide = false;   // wide: fp32 results of bf16 rows
  int rows = 0, tile = 0;         // rows of an item, cached rows of a tile
  int width = 0;                  // columns of a part
  int ctas = 0;
};
cudaError_t chunk_configure(ChunkCfg *cfg, const DeviceCfg &dev, int d_h, bool bf16, bool out_bf16);
// bytes of workspace of a call; with `a` its slices are set too
size_t chunk_scratch(const ChunkCfg &cfg, int requests, ChunkArgs *a, char *base);
// chunk_f32.cu: caches of fp32 rows
struct ChunkFormF32 {
  int rows, tile, width;
};
ChunkFormF32 chunk_form_f32();
cudaError_t chunk_configure_f32(const ChunkCfg &cfg, int d_h);
cudaError_t launch_chunk_f32(const ChunkArgs &a, const pact_paged_cache &cache, const ChunkCfg &cfg, cudaStream_t st);
// chunk_join.cu
cudaError_t launch_chunk_join(const ChunkArgs &a, const ChunkCfg &cfg, cudaStream_t st);
// all of a call
cudaError_t launch_chunk(ChunkArgs a, const pact_paged_cache &cache, const ChunkCfg &cfg, cudaStream_t st, int *launches);

}  // namespace pact
