// What the host side of the C ABI shares: the context and how a failed CUDA call is reported.
#pragma once
#include <stdio.h>

#include <atomic>

#include "kernels.cuh"
#include "paged.cuh"

constexpr int kProfStages = 9;

struct pact_ctx {
  int d, n_qh, n_kvh, d_h, d_k, n_qcols;
  pact_dtype in, out;
  int elt;                 // bytes per input element
  pact::DeviceCfg dev;     // of the device the context was created on
  bool umma;               // bf16 keys of a width the tcgen05 tile kernels take
  pact::PagedCfg paged;    // the paged cache's kernels for these heads
  int device;
  char err[256];
  long long launches;      // kernels launched by this context so far
  int spin_limit;          // polls the barrier of the member-list kernel makes before it raises PACT_ERR_TIMEOUT
  int sweep_limit;         // sweeps the centre selection makes before it raises PACT_ERR_TIMEOUT
  int copy_polls;          // polls that a wait of the paged attention makes before it raises PACT_ERR_TIMEOUT, if a second has not passed before
  int prof_on;             // record an event after every stage of pact_reduce
  int prof_n;              // stages recorded by the last profiled call
  cudaEvent_t ev[kProfStages + 1];
  // pact_reduce_host: a stream for the copies in, used by one call at a time (another thread's call does without)
  std::atomic_flag feed_busy = ATOMIC_FLAG_INIT;
  bool fed_before = false;                             // there has been a call large enough for it
  cudaStream_t feed_stream = nullptr;
  cudaEvent_t feed_start = nullptr, feed_keys = nullptr, feed_part[pact::kFeedParts] = {};
};

inline pact_status fail_cuda(pact_ctx *c, cudaError_t e, const char *where) {
  snprintf(c->err, sizeof(c->err), "%s: %s", where, cudaGetErrorString(e));
  return PACT_ERR_CUDA;
}

#define CK(call)                                                     \
  do {                                                               \
    cudaError_t e_ = (call);                                         \
    if (e_ != cudaSuccess) return fail_cuda(ctx, e_, #call);         \
  } while (0)

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
