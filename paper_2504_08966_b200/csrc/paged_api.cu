// Host side of the paged cache's calls: argument checks and launches.
#include <math.h>
#include <string.h>

#include "context.h"
#include "paged_checks.h"

using namespace pact;

namespace {

size_t select_scores(const pact_ctx *c, int requests, int pages) { return (size_t)requests * c->n_kvh * pages; }
size_t select_bytes(const pact_ctx *c, int requests, int pages) {
  const size_t of_score = sizeof(unsigned long long) + (pages > kPickKeys ? sizeof(uint32_t) : 0);
  return (select_scores(c, requests, pages) * of_score + kAlign - 1) / kAlign * kAlign;
}

}  // namespace

extern "C" {

pact_status pact_cache_plan(pact_ctx *ctx, const pact_plan *p, void *stream) {
  if (!ctx || !p) return PACT_ERR_INVALID_ARG;
  const pact_status s = check_requests(ctx, p->page_rows, p->n_pages, p->n_requests, p->max_pages, p->block_table, p->length);
  if (s != PACT_OK) return s;
  if (!p->n_new || p->n_new_stride < 1 || !p->free_pages || !p->n_free || !p->length_out || !p->n_free_out) return PACT_ERR_INVALID_ARG;
  if (p->n_rows < 0 || p->row_stride < 0 || (p->row_stride && p->n_rows != (int64_t)p->n_requests * p->row_stride)) return PACT_ERR_INVALID_ARG;
  if (p->n_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  PlanArgs a;
  memset(&a, 0, sizeof(a));
  a.table = p->block_table; a.length = p->length; a.n_new = p->n_new; a.n_new_stride = p->n_new_stride;
  a.free_pages = p->free_pages; a.n_free = p->n_free; a.length_out = p->length_out; a.n_free_out = p->n_free_out;
  a.row_start = p->row_start; a.slot = p->slot; a.n_rows = p->n_rows; a.status = p->status;
  a.B = p->n_requests; a.width = p->max_pages; a.page = p->page_rows; a.n_pages = p->n_pages; a.row_stride = p->row_stride;
  int launches = 0;
  CK(launch_cache_plan(a, ctx->dev.sm_count, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_cache_write(pact_ctx *ctx, const pact_paged_cache *cache, const pact_new_rows *r, void *stream) {
  if (!ctx || !r || !on_device(ctx) || r->n_rows < 0) return PACT_ERR_INVALID_ARG;
  const pact_status s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  if (r->n_rows == 0) return PACT_OK;
  if (!r->K || !r->V || !r->slot || !aligned16(r->K) || !aligned16(r->V) || !stride_ok(ctx, r->ld_row) || !stride_ok(ctx, r->ld_head)) return PACT_ERR_INVALID_ARG;
  if (r->n_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  if (!ctx->paged.blocks) return PACT_ERR_UNSUPPORTED;
  WriteArgs a;
  a.Kn = r->K; a.Vn = r->V; a.ld_row = r->ld_row; a.ld_head = r->ld_head; a.logw_new = cache->logw ? r->logw : nullptr; a.slot = r->slot; a.n_rows = r->n_rows;
  a.K = cache->K; a.V = cache->V; a.k_page = cache->k_page; a.k_head = cache->k_head; a.k_row = cache->k_row;
  a.v_page = cache->v_page; a.v_head = cache->v_head; a.v_row = cache->v_row;
  a.logw = cache->logw; a.bounds = cache->bounds; a.w_max = cache->w_max; a.status = r->status;
  a.n_pages = cache->n_pages; a.page = cache->page_rows; a.n_kvh = ctx->n_kvh; a.d_h = ctx->d_h;
  CK(launch_cache_write(a, ctx->in == PACT_BF16, ctx->dev.sm_count, (cudaStream_t)stream));
  ctx->launches += 1;
  CK(cudaGetLastError());
  return PACT_OK;
}

size_t pact_paged_workspace_bytes(const pact_ctx *ctx, int max_requests, int max_pages) {
  if (!ctx || max_requests < 1 || max_pages < 1) return 0;
  const size_t x = attend_scratch(ctx->paged, ctx->dev, ctx->in == PACT_BF16, nullptr, nullptr), y = select_bytes(ctx, max_requests, max_pages);
  return x > y ? x : y;
}

static pact_status check_query(const pact_ctx *ctx, const pact_paged_cache *cache, const pact_query *q) {
  if (!ctx || !cache || !q) return PACT_ERR_INVALID_ARG;
  pact_status s = check_requests(ctx, cache->page_rows, cache->n_pages, q->n_requests, q->max_pages, q->block_table, q->length);
  if (s == PACT_OK) s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  if (!q->Q || !aligned16(q->Q) || !stride_ok(ctx, q->ldQ) || !stride_ok(ctx, q->ldQh) || !isfinite(q->scale)) return PACT_ERR_INVALID_ARG;
  if (q->selected && q->n_select < 1) return PACT_ERR_INVALID_ARG;
  return ctx->paged.blocks ? PACT_OK : PACT_ERR_UNSUPPORTED;
}

pact_status pact_page_select(pact_ctx *ctx, const pact_paged_cache *cache, const pact_query *q, void *stream) {
  pact_status s = check_query(ctx, cache, q);
  if (s != PACT_OK) return s;
  if (!cache->bounds || !q->selected || q->n_first < 0 || q->n_last < 0 || q->n_first > q->n_select || q->n_last > q->n_select - q->n_first)
    return PACT_ERR_INVALID_ARG;
  if (q->max_pages > kMaxSelectPages) return PACT_ERR_UNSUPPORTED;
  s = check_ws(q->ws, q->ws_bytes, select_bytes(ctx, q->n_requests, q->max_pages));
  if (s != PACT_OK) return s;
  SelectArgs a;
  a.Q = q->Q; a.ldQ = q->ldQ; a.ldQh = q->ldQh; a.bounds = cache->bounds; a.w_max = cache->w_max; a.table = q->block_table; a.length = q->length;
  a.selected = q->selected; a.status = q->status; a.scale = q->scale;
  a.keys = (unsigned long long *)q->ws; a.approx = (uint32_t *)(a.keys + select_scores(ctx, q->n_requests, q->max_pages));
  a.B = q->n_requests; a.width = q->max_pages; a.page = cache->page_rows; a.n_pages = cache->n_pages;
  a.n_kvh = ctx->n_kvh; a.group = ctx->n_qh / ctx->n_kvh; a.d_h = ctx->d_h;
  a.n_first = q->n_first; a.n_last = q->n_last; a.n_select = q->n_select;
  CK(launch_page_select(a, ctx->in == PACT_BF16, ctx->paged.cluster, ctx->dev.sm_count, (cudaStream_t)stream));
  ctx->launches += 1;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_paged_attention(pact_ctx *ctx, const pact_paged_cache *cache, const pact_query *q, void *stream) {
  pact_status s = check_query(ctx, cache, q);
  if (s != PACT_OK) return s;
  const size_t oe = ctx->out == PACT_BF16 ? 2 : 4;
  if (!q->out || reinterpret_cast<uintptr_t>(q->out) % (4 * oe) != 0) return PACT_ERR_INVALID_ARG;
  if (q->ldO < ctx->d_h || q->ldOh < ctx->d_h || q->ldO % 4 != 0 || q->ldOh % 4 != 0) return PACT_ERR_INVALID_ARG;
  const int64_t rows = (int64_t)(q->selected && q->n_select < q->max_pages ? q->n_select : q->max_pages) * cache->page_rows;
  if (q->n_requests * ((rows + 63) / 64) > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  AttendArgs a;
  memset(&a, 0, sizeof(a));
  s = check_ws(q->ws, q->ws_bytes, attend_scratch(ctx->paged, ctx->dev, ctx->in == PACT_BF16, &a, (char *)q->ws));
  if (s != PACT_OK) return s;
  a.Q = q->Q; a.ldQ = q->ldQ; a.ldQh = q->ldQh; a.logw = cache->logw; a.table = q->block_table; a.length = q->length; a.selected = q->selected;
  a.out = q->out; a.ldO = q->ldO; a.ldOh = q->ldOh; a.lse = q->lse; a.status = q->status; a.scale = q->scale;
  a.B = q->n_requests; a.width = q->max_pages; a.page = cache->page_rows; a.n_pages = cache->n_pages; a.n_select = q->selected ? q->n_select : 0;
  a.n_kvh = ctx->n_kvh; a.group = ctx->n_qh / ctx->n_kvh; a.d_h = ctx->d_h; a.out_bf16 = ctx->out == PACT_BF16;
  a.polls = ctx->copy_polls;
  int launches = 0;
  CK(launch_attend(a, *cache, ctx->paged, ctx->dev, ctx->in == PACT_BF16, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

}  // extern "C"
