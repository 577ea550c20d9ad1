// Host side of the calls for pages that several requests hold: argument checks and launches.
#include <string.h>

#include "context.h"
#include "paged_checks.h"
#include "share.cuh"

using namespace pact;

namespace {

pact_status check_share(const pact_ctx *ctx, int page_rows, int n_pages, int n_requests, int max_pages, const int32_t *table, const int32_t *length) {
  const pact_status s = check_requests(ctx, page_rows, n_pages, n_requests, max_pages, table, length);
  if (s != PACT_OK) return s;
  return (int64_t)n_requests * max_pages > INT32_MAX ? PACT_ERR_UNSUPPORTED : PACT_OK;   // (places are counted in 32 bits)
}

uint64_t page_mul_of(int page) { return ((1ull << 33) + page / 16 - 1) / (page / 16); }

}  // namespace

extern "C" {

size_t pact_share_workspace_bytes(const pact_ctx *ctx, int max_requests, int max_pages, int n_pages) {
  if (!ctx || max_requests < 1 || max_requests > PACT_MAX_REQUESTS || max_pages < 1 || n_pages < 1) return 0;
  const size_t x = fork_scratch(max_requests, max_pages, n_pages, nullptr, nullptr), y = compact_scratch(n_pages, nullptr, nullptr);
  return x > y ? x : y;
}

pact_status pact_cache_fork(pact_ctx *ctx, const pact_fork *f, void *stream) {
  if (!ctx || !f) return PACT_ERR_INVALID_ARG;
  pact_status s = check_share(ctx, f->page_rows, f->n_pages, f->n_requests, f->max_pages, f->block_table, f->length);
  if (s != PACT_OK) return s;
  if (!f->source || !f->shared || !f->free_pages || !f->n_free || !f->block_table_out || !f->length_out || !f->shared_out || !f->free_out || !f->n_free_out || !f->copies || !f->n_copies)
    return PACT_ERR_INVALID_ARG;
  if (f->block_table_out == f->block_table || f->length_out == f->length) return PACT_ERR_INVALID_ARG;
  if (ctx->no_share) return PACT_ERR_UNSUPPORTED;
  s = check_ws(f->ws, f->ws_bytes, fork_scratch(f->n_requests, f->max_pages, f->n_pages, nullptr, nullptr));
  if (s != PACT_OK) return s;
  ShareArgs a;
  memset(&a, 0, sizeof(a));
  fork_scratch(f->n_requests, f->max_pages, f->n_pages, &a, (char *)f->ws);
  a.table = f->block_table; a.length = f->length; a.source = f->source; a.rows = f->rows; a.shared = f->shared; a.free_pages = f->free_pages; a.n_free = f->n_free;
  a.table_out = f->block_table_out; a.length_out = f->length_out; a.shared_out = f->shared_out; a.free_out = f->free_out; a.n_free_out = f->n_free_out;
  a.copies = f->copies; a.n_copies = f->n_copies; a.status = f->status;
  a.B = f->n_requests; a.width = f->max_pages; a.page = f->page_rows; a.n_pages = f->n_pages; a.n_list = f->n_requests; a.page_mul = page_mul_of(a.page);
  CK(launch_cache_fork(a, (cudaStream_t)stream));
  ctx->launches += 1;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_cache_compact(pact_ctx *ctx, const pact_compact *c, void *stream) {
  if (!ctx || !c) return PACT_ERR_INVALID_ARG;
  pact_status s = check_share(ctx, c->page_rows, c->n_pages, c->n_requests, c->max_pages, c->block_table, c->length);
  if (s != PACT_OK) return s;
  if (!c->shared || !c->free_pages || !c->n_free || !c->block_table_out || !c->shared_out || !c->free_out || !c->moved_to || !c->copies || !c->n_copies || c->n_list < c->n_pages / 2)
    return PACT_ERR_INVALID_ARG;
  if (ctx->no_share) return PACT_ERR_UNSUPPORTED;
  s = check_ws(c->ws, c->ws_bytes, compact_scratch(c->n_pages, nullptr, nullptr));
  if (s != PACT_OK) return s;
  ShareArgs a;
  memset(&a, 0, sizeof(a));
  compact_scratch(c->n_pages, &a, (char *)c->ws);
  a.table = c->block_table; a.length = c->length; a.shared = c->shared; a.free_pages = c->free_pages; a.n_free = c->n_free;
  a.table_out = c->block_table_out; a.shared_out = c->shared_out; a.free_out = c->free_out; a.moved_to = c->moved_to; a.copies = c->copies; a.n_copies = c->n_copies; a.status = c->status;
  a.B = c->n_requests; a.width = c->max_pages; a.page = c->page_rows; a.n_pages = c->n_pages; a.n_list = c->n_list; a.page_mul = page_mul_of(a.page);
  CK(launch_cache_compact(a, (cudaStream_t)stream));
  ctx->launches += 1;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_page_copy(pact_ctx *ctx, const pact_paged_cache *cache, const pact_copies *c, void *stream) {
  if (!ctx || !c || !on_device(ctx) || c->n_list < 0) return PACT_ERR_INVALID_ARG;
  const pact_status s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  if (c->n_list == 0) return PACT_OK;
  if (!c->copies) return PACT_ERR_INVALID_ARG;
  if (!ctx->paged.blocks) return PACT_ERR_UNSUPPORTED;
  const PageCopyArgs a = {cache->K, cache->V, cache->k_page, cache->k_head, cache->k_row, cache->v_page, cache->v_head, cache->v_row, cache->logw, cache->bounds, cache->w_max,
                          c->copies, c->n_copies, c->status, c->n_list, cache->n_pages, cache->page_rows, ctx->n_kvh, ctx->d_h, ctx->elt};
  CK(launch_page_copy(a, ctx->dev.sm_count, (cudaStream_t)stream));
  ctx->launches += 1;
  CK(cudaGetLastError());
  return PACT_OK;
}

}  // extern "C"
