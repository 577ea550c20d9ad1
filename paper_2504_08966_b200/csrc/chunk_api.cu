// Host side of the calls for several new tokens per request: argument checks and launches.
#include <math.h>
#include <string.h>

#include "context.h"
#include "paged_checks.h"

using namespace pact;

extern "C" {

size_t pact_chunk_workspace_bytes(const pact_ctx *ctx, int max_requests) {
  if (!ctx || max_requests < 1 || max_requests > PACT_MAX_REQUESTS) return 0;
  return chunk_scratch(ctx->chunk, max_requests, nullptr, nullptr);
}

pact_status pact_chunk_attention(pact_ctx *ctx, const pact_paged_cache *cache, const pact_chunk *c, void *stream) {
  if (!ctx || !cache || !c) return PACT_ERR_INVALID_ARG;
  pact_status s = check_requests(ctx, cache->page_rows, cache->n_pages, c->n_requests, c->max_pages, c->block_table, c->length);
  if (s == PACT_OK) s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  const size_t oe = ctx->out == PACT_BF16 ? 2 : 4;
  if ((!c->Q && c->n_rows) || !aligned16(c->Q) || !stride_ok(ctx, c->ldQ) || !stride_ok(ctx, c->ldQh) || !isfinite(c->scale)) return PACT_ERR_INVALID_ARG;
  if ((!c->out && c->n_rows) || reinterpret_cast<uintptr_t>(c->out) % (4 * oe) != 0) return PACT_ERR_INVALID_ARG;
  if (c->ldO < ctx->d_h || c->ldOh < ctx->d_h || c->ldO % 4 != 0 || c->ldOh % 4 != 0) return PACT_ERR_INVALID_ARG;
  if (!c->n_new || c->n_new_stride < 1 || c->n_rows < 0 || c->row_stride < 0 || (c->causal != 0 && c->causal != 1)) return PACT_ERR_INVALID_ARG;
  if (c->row_stride ? c->row_start || c->n_rows != (int64_t)c->n_requests * c->row_stride : !c->row_start) return PACT_ERR_INVALID_ARG;
  if (!ctx->chunk.blocks) return PACT_ERR_UNSUPPORTED;
  const int group = ctx->n_qh / ctx->n_kvh;
  // items and tiles are counted in 32 bits
  const int64_t items = (c->n_rows * group / ctx->chunk.rows + c->n_requests) * ctx->n_kvh;
  const int64_t tiles = ((int64_t)c->max_pages * cache->page_rows + c->n_rows) / ctx->chunk.tile + 1;
  if (c->n_rows > INT32_MAX / group || items > INT32_MAX / 2 || items > INT32_MAX / tiles) return PACT_ERR_UNSUPPORTED;
  s = check_ws(c->ws, c->ws_bytes, chunk_scratch(ctx->chunk, c->n_requests, nullptr, nullptr));
  if (s != PACT_OK) return s;
  ChunkArgs a;
  memset(&a, 0, sizeof(a));
  chunk_scratch(ctx->chunk, c->n_requests, &a, (char *)c->ws);
  a.Q = c->Q; a.ldQ = c->ldQ; a.ldQh = c->ldQh; a.logw = cache->logw; a.table = c->block_table; a.length = c->length; a.n_new = c->n_new; a.row_start = c->row_start;
  a.n_new_stride = c->n_new_stride; a.n_rows = c->n_rows; a.row_stride = c->row_stride;
  a.out = c->out; a.ldO = c->ldO; a.ldOh = c->ldOh; a.lse = c->lse; a.status = c->status; a.scale = c->scale;
  a.B = c->n_requests; a.width = c->max_pages; a.page = cache->page_rows; a.n_pages = cache->n_pages;
  a.n_kvh = ctx->n_kvh; a.group = group; a.d_h = ctx->d_h; a.causal = c->causal != 0; a.out_bf16 = ctx->out == PACT_BF16;
  const uint64_t at = reinterpret_cast<uintptr_t>(c->out) | (uint64_t)c->ldO * oe | (uint64_t)c->ldOh * oe;
  a.store_bytes = at % 32 == 0 ? 32 : at % 16 == 0 ? 16 : 8;
  a.polls = ctx->copy_polls;
  int launches = 0;
  CK(launch_chunk(a, *cache, ctx->chunk, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

}  // extern "C"
