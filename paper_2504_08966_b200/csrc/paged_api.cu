// Host side of the paged cache's calls: argument checks and launches.
#include <math.h>
#include <string.h>

#include "context.h"

using namespace pact;

namespace {

constexpr size_t kAlign = 256;

bool on_device(const pact_ctx *c) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == c->device;
}

pact_status check_requests(const pact_ctx *c, int page_rows, int n_pages, int n_requests, int max_pages, const int32_t *table, const int32_t *length) {
  if (!c || !table || !length || !on_device(c)) return PACT_ERR_INVALID_ARG;
  if (page_rows < 16 || page_rows > 1024 || page_rows % 16 != 0 || n_pages < 1) return PACT_ERR_INVALID_ARG;
  if (n_requests < 1 || max_pages < 1) return PACT_ERR_INVALID_ARG;
  if (n_requests > PACT_MAX_REQUESTS || (int64_t)max_pages * page_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  return PACT_OK;
}

bool stride_ok(const pact_ctx *c, int64_t ld) { return ld >= c->d_h && ((uint64_t)ld * c->elt) % 16 == 0; }

pact_status check_cache(const pact_ctx *c, const pact_paged_cache *p) {
  if (!p || !p->K || !p->V || !aligned16(p->K) || !aligned16(p->V)) return PACT_ERR_INVALID_ARG;
  if (p->n_pages < 1 || p->page_rows < 16 || p->page_rows > 1024 || p->page_rows % 16 != 0) return PACT_ERR_INVALID_ARG;
  for (int64_t ld : {p->k_page, p->k_head, p->k_row, p->v_page, p->v_head, p->v_row})
    if (!stride_ok(c, ld)) return PACT_ERR_INVALID_ARG;
  if ((p->logw && !aligned16(p->logw)) || (p->bounds && !aligned16(p->bounds)) || !p->bounds != !p->w_max) return PACT_ERR_INVALID_ARG;
  for (int64_t ld : {p->k_page, p->k_head, p->k_row, p->v_page, p->v_head, p->v_row})
    if ((uint64_t)ld * c->elt >= (1ull << 40)) return PACT_ERR_UNSUPPORTED;
  return PACT_OK;
}

pact_status check_ws(void *ws, size_t have, size_t need) {
  return ws && reinterpret_cast<uintptr_t>(ws) % kAlign == 0 && have >= need ? PACT_OK : PACT_ERR_WORKSPACE;
}

size_t select_scores(const pact_ctx *c, int requests, int pages) { return (size_t)requests * c->n_kvh * pages; }
size_t select_bytes(const pact_ctx *c, int requests, int pages) {
  return (select_scores(c, requests, pages) * (sizeof(uint2) + sizeof(unsigned long long)) + kAlign - 1) / kAlign * kAlign;
}

}  // namespace

extern "C" {

pact_status pact_cache_plan(pact_ctx *ctx, int page_rows, int n_pages, int n_requests, int max_pages, int32_t *block_table, const int32_t *length,
                            const int32_t *n_new, int64_t n_new_stride, int32_t *free_pages, const int32_t *n_free, int32_t *length_out,
                            int32_t *n_free_out, int32_t *row_start, int64_t *slot, int64_t n_rows, int row_stride, int32_t *status, void *stream) {
  const pact_status s = check_requests(ctx, page_rows, n_pages, n_requests, max_pages, block_table, length);
  if (s != PACT_OK) return s;
  if (!n_new || n_new_stride < 1 || !free_pages || !n_free || !length_out || !n_free_out) return PACT_ERR_INVALID_ARG;
  if (n_rows < 0 || row_stride < 0 || (row_stride && n_rows != (int64_t)n_requests * row_stride)) return PACT_ERR_INVALID_ARG;
  if (n_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  PlanArgs a;
  memset(&a, 0, sizeof(a));
  a.table = block_table; a.length = length; a.n_new = n_new; a.n_new_stride = n_new_stride;
  a.free_pages = free_pages; a.n_free = n_free; a.length_out = length_out; a.n_free_out = n_free_out;
  a.row_start = row_start; a.slot = slot; a.n_rows = n_rows; a.status = status;
  a.B = n_requests; a.width = max_pages; a.page = page_rows; a.n_pages = n_pages; a.row_stride = row_stride;
  int launches = 0;
  CK(launch_cache_plan(a, ctx->dev.sm_count, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_cache_write(pact_ctx *ctx, const pact_paged_cache *cache, const void *K_new, const void *V_new, int64_t ld_row, int64_t ld_head,
                             const float *logw_new, const int64_t *slot, int64_t n_rows, int32_t *status, void *stream) {
  if (!ctx || !on_device(ctx) || n_rows < 0) return PACT_ERR_INVALID_ARG;
  const pact_status s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  if (n_rows == 0) return PACT_OK;
  if (!K_new || !V_new || !slot || !aligned16(K_new) || !aligned16(V_new) || !stride_ok(ctx, ld_row) || !stride_ok(ctx, ld_head)) return PACT_ERR_INVALID_ARG;
  if (n_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  if (ctx->d_h * ctx->elt > 4096) return PACT_ERR_UNSUPPORTED;   // (a CTA's threads have to hold a row)
  WriteArgs a;
  a.Kn = K_new; a.Vn = V_new; a.ld_row = ld_row; a.ld_head = ld_head; a.logw_new = logw_new; a.slot = slot; a.n_rows = n_rows;
  a.K = cache->K; a.V = cache->V; a.k_page = cache->k_page; a.k_head = cache->k_head; a.k_row = cache->k_row;
  a.v_page = cache->v_page; a.v_head = cache->v_head; a.v_row = cache->v_row;
  a.logw = cache->logw; a.bounds = cache->bounds; a.w_max = cache->w_max; a.status = status;
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

pact_status pact_page_select(pact_ctx *ctx, const pact_paged_cache *cache, const void *Q, int64_t ldQ, int64_t ldQh, int n_requests,
                             const int32_t *block_table, int max_pages, const int32_t *length, float scale, int n_first, int n_last, int n_select,
                             int32_t *selected, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
  if (!ctx || !cache) return PACT_ERR_INVALID_ARG;
  pact_status s = check_requests(ctx, cache->page_rows, cache->n_pages, n_requests, max_pages, block_table, length);
  if (s == PACT_OK) s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  if (!cache->bounds || !Q || !selected || !aligned16(Q) || !stride_ok(ctx, ldQ) || !stride_ok(ctx, ldQh)) return PACT_ERR_INVALID_ARG;
  if (!isfinite(scale) || n_first < 0 || n_last < 0 || n_select < 1 || n_first > n_select || n_last > n_select - n_first) return PACT_ERR_INVALID_ARG;
  if (max_pages > kMaxSelectPages || !ctx->paged.blocks) return PACT_ERR_UNSUPPORTED;
  s = check_ws(ws, ws_bytes, select_bytes(ctx, n_requests, max_pages));
  if (s != PACT_OK) return s;
  SelectArgs a;
  a.Q = Q; a.ldQ = ldQ; a.ldQh = ldQh; a.bounds = cache->bounds; a.w_max = cache->w_max; a.table = block_table; a.length = length;
  a.selected = selected; a.status = status; a.approx = (uint2 *)ws; a.keys = (unsigned long long *)ws + select_scores(ctx, n_requests, max_pages); a.scale = scale;
  a.B = n_requests; a.width = max_pages; a.page = cache->page_rows; a.n_pages = cache->n_pages;
  a.n_kvh = ctx->n_kvh; a.group = ctx->n_qh / ctx->n_kvh; a.d_h = ctx->d_h;
  a.n_first = n_first; a.n_last = n_last; a.n_select = n_select;
  int launches = 0;
  CK(launch_page_select(a, ctx->in == PACT_BF16, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

pact_status pact_paged_attention(pact_ctx *ctx, const pact_paged_cache *cache, const void *Q, int64_t ldQ, int64_t ldQh, int n_requests,
                                 const int32_t *block_table, int max_pages, const int32_t *length, const int32_t *selected, int n_select, float scale,
                                 void *out, int64_t ldO, int64_t ldOh, float *lse, int32_t *status, void *ws, size_t ws_bytes, void *stream) {
  if (!ctx || !cache) return PACT_ERR_INVALID_ARG;
  pact_status s = check_requests(ctx, cache->page_rows, cache->n_pages, n_requests, max_pages, block_table, length);
  if (s == PACT_OK) s = check_cache(ctx, cache);
  if (s != PACT_OK) return s;
  const size_t oe = ctx->out == PACT_BF16 ? 2 : 4;
  if (!Q || !out || !aligned16(Q) || reinterpret_cast<uintptr_t>(out) % (4 * oe) != 0 || !stride_ok(ctx, ldQ) || !stride_ok(ctx, ldQh)) return PACT_ERR_INVALID_ARG;
  if (ldO < ctx->d_h || ldOh < ctx->d_h || ldO % 4 != 0 || ldOh % 4 != 0) return PACT_ERR_INVALID_ARG;
  if (!isfinite(scale) || (selected && n_select < 1)) return PACT_ERR_INVALID_ARG;
  if (!ctx->paged.blocks) return PACT_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)(selected && n_select < max_pages ? n_select : max_pages) * cache->page_rows;
  if (n_requests * ((rows + 63) / 64) > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  AttendArgs a;
  memset(&a, 0, sizeof(a));
  s = check_ws(ws, ws_bytes, attend_scratch(ctx->paged, ctx->dev, ctx->in == PACT_BF16, &a, (char *)ws));
  if (s != PACT_OK) return s;
  a.Q = Q; a.ldQ = ldQ; a.ldQh = ldQh; a.logw = cache->logw; a.table = block_table; a.length = length; a.selected = selected;
  a.out = out; a.ldO = ldO; a.ldOh = ldOh; a.lse = lse; a.status = status;
  a.scale = scale;
  a.B = n_requests; a.width = max_pages; a.page = cache->page_rows; a.n_pages = cache->n_pages; a.n_select = selected ? n_select : 0;
  a.n_kvh = ctx->n_kvh; a.group = ctx->n_qh / ctx->n_kvh; a.d_h = ctx->d_h; a.out_bf16 = ctx->out == PACT_BF16;
  int launches = 0;
  CK(launch_attend(a, *cache, ctx->paged, ctx->dev, ctx->in == PACT_BF16, (cudaStream_t)stream, &launches));
  ctx->launches += launches;
  CK(cudaGetLastError());
  return PACT_OK;
}

}  // extern "C"
