// Checks of arguments that the calls of the paged cache share.
#pragma once
#include "context.h"

namespace pact {

constexpr size_t kAlign = 256;

inline bool on_device(const pact_ctx *c) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == c->device;
}

inline pact_status check_requests(const pact_ctx *c, int page_rows, int n_pages, int n_requests, int max_pages, const int32_t *table, const int32_t *length) {
  if (!c || !table || !length || !on_device(c)) return PACT_ERR_INVALID_ARG;
  if (page_rows < 16 || page_rows > 1024 || page_rows % 16 != 0 || n_pages < 1) return PACT_ERR_INVALID_ARG;
  if (n_requests < 1 || max_pages < 1) return PACT_ERR_INVALID_ARG;
  if (n_requests > PACT_MAX_REQUESTS || (int64_t)max_pages * page_rows > INT32_MAX) return PACT_ERR_UNSUPPORTED;
  return PACT_OK;
}

inline bool stride_ok(const pact_ctx *c, int64_t ld) { return ld >= c->d_h && ((uint64_t)ld * c->elt) % 16 == 0; }

inline pact_status check_cache(const pact_ctx *c, const pact_paged_cache *p) {
  if (!p || !p->K || !p->V || !aligned16(p->K) || !aligned16(p->V)) return PACT_ERR_INVALID_ARG;
  if (p->n_pages < 1 || p->page_rows < 16 || p->page_rows > 1024 || p->page_rows % 16 != 0) return PACT_ERR_INVALID_ARG;
  for (int64_t ld : {p->k_page, p->k_head, p->k_row, p->v_page, p->v_head, p->v_row})
    if (!stride_ok(c, ld)) return PACT_ERR_INVALID_ARG;
  if ((p->logw && !aligned16(p->logw)) || (p->bounds && !aligned16(p->bounds)) || !p->bounds != !p->w_max) return PACT_ERR_INVALID_ARG;
  for (int64_t ld : {p->k_page, p->k_head, p->k_row, p->v_page, p->v_head, p->v_row})
    if ((uint64_t)ld * c->elt >= (1ull << 40)) return PACT_ERR_UNSUPPORTED;
  return PACT_OK;
}

inline pact_status check_ws(void *ws, size_t have, size_t need) {
  return ws && reinterpret_cast<uintptr_t>(ws) % kAlign == 0 && have >= need ? PACT_OK : PACT_ERR_WORKSPACE;
}

}  // namespace pact
