// Requests that go on with the rows of others (pact_cache_fork) and pages moved to the lowest ids (pact_cache_compact).
//
// Both are bookkeeping over block tables, bound by latency: a chain of steps in which every entry has to be known to all before the next begins.  One cluster of CTAs walks through them with
// barriers between, a launch instead of six; counts go to global memory by integer atomics, whose order does not show.  A warp looks at 64 entries of a table at a time.
#include "share.cuh"

namespace pact {
namespace {

// ---- what both have -------------------------------------------------------------------------------------

__device__ __forceinline__ int cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return (int)r;
}

// Exclusive sums of a value per thread over the CTA, and the total; the shared memory is free again when it returns.
__device__ __forceinline__ int share_scan(int v, int *warp_sums, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  const int before = (warp ? warp_sums[warp - 1] : 0) + x - v;
  *total = warp_sums[31];
  __syncthreads();
  return before;
}

// chunk[b] = chunks of the requests before b, n(b) entries each; chunk[B] all of them
template <typename F> __device__ __forceinline__ void chunk_starts(int B, int *chunk, int *warp_sums, F n) {
  const int per = (B + kShareThreads - 1) / kShareThreads, b0 = min(B, (int)threadIdx.x * per), b1 = min(B, b0 + per);
  int mine = 0, all;
  for (int b = b0; b < b1; ++b) mine += (n(b) + kShareChunk - 1) / kShareChunk;
  int at = share_scan(mine, warp_sums, &all);
  for (int b = b0; b < b1; ++b) {
    chunk[b] = at;
    at += (n(b) + kShareChunk - 1) / kShareChunk;
  }
  if (threadIdx.x == 0) chunk[B] = all;
  __syncthreads();
}
__device__ __forceinline__ int request_of(const int *chunk, int B, int c) {   // (some requests have no chunks)
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (chunk[mid] <= c) lo = mid;
    else hi = mid;
  }
  return lo;
}

constexpr int kMyWarps = kShareThreads / 32;

// f(request, first place, entries) for every chunk of this warp
template <typename F> __device__ __forceinline__ void each_chunk(const int *chunk, int B, int rank, F f) {
  for (int c = rank * kMyWarps + (threadIdx.x >> 5); c < chunk[B]; c += kShareCtas * kMyWarps) {
    const int b = request_of(chunk, B, c);
    f(b, (c - chunk[b]) * kShareChunk, c);
  }
}

struct ShareSmem {
  int warp[32], bad;
  int old_chunk[PACT_MAX_REQUESTS + 1], new_chunk[PACT_MAX_REQUESTS + 1];
};

// ---- fork -------------------------------------------------------------------------------------------------

struct ForkPlan {
  const ShareArgs &a;
  int room;                                // rows of a block table
  __device__ __forceinline__ int length(int b) const { return min(max(a.length[b], 0), room); }
  __device__ __forceinline__ int pages(int b) const { return (length(b) + a.page - 1) / a.page; }
  __device__ __forceinline__ bool has_source(int b) const { return a.source[b] >= 0 && a.source[b] < a.B; }
  __device__ __forceinline__ int rows(int b) const {     // of the new request, within what its source has
    if (!has_source(b)) return 0;
    const int have = length(a.source[b]);
    return a.rows ? min(max(a.rows[b], 0), have) : have;
  }
  __device__ __forceinline__ int tail_page(int b) const {  // the page that its last rows share with what follows them in the source; -1: the rows end with a page
    const int n = rows(b);
    return n % a.page ? a.table[(long long)a.source[b] * a.width + n / a.page] : -1;
  }
  // of a page, once all entries are counted
  __device__ __forceinline__ int outside(int p) const { return a.shared[p] + 1 - a.held[p]; }
  __device__ __forceinline__ bool kept_by_tail(int p) const { return a.tail[p] < a.B && a.full[p] == 0 && outside(p) == 0; }
  __device__ __forceinline__ int now(int p) const { return outside(p) + a.full[p] + (kept_by_tail(p) ? 1 : 0); }
};

__global__ void __launch_bounds__(kShareThreads) k_cache_fork(const __grid_constant__ ShareArgs a) {
  extern __shared__ __align__(16) char sm[];
  ShareSmem &sh = *reinterpret_cast<ShareSmem *>(sm);
  const int tid = threadIdx.x, lane = tid & 31, rank = cta_rank(), me = rank * kShareThreads + tid;
  constexpr int kAll = kShareCtas * kShareThreads;
  if (tid == 0) sh.bad = 0;
  pdl_wait();
  pdl_trigger();
  const ForkPlan plan = {a, a.width * a.page};
  const auto old_at = [&](int b, int j) { return a.table[(long long)b * a.width + j]; };
  const auto is_page = [&](int p) { return p >= 0 && p < a.n_pages; };
  // 1: what is asked for, checked; the words of all pages named cleared
  chunk_starts(a.B, sh.old_chunk, sh.warp, [&](int b) { return plan.pages(b); });
  chunk_starts(a.B, sh.new_chunk, sh.warp, [&](int b) { return plan.rows(b) / a.page; });
  for (int b = me; b < a.B; b += kAll) {
    const int s = a.source[b];
    bool bad = a.length[b] < 0 || a.length[b] > plan.room || s < -1 || s >= a.B;
    if (s >= 0 && s < a.B && a.rows) bad = bad || a.rows[b] < 0 || a.rows[b] > plan.length(s);
    if (bad) sh.bad = PACT_ERR_INVALID_ARG;
  }
  if (me == 0 && (*a.n_free < 0 || *a.n_free > a.n_pages)) sh.bad = PACT_ERR_INVALID_ARG;
  each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int) {
    for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) {
      const int p = old_at(b, j);
      if (is_page(p)) {
        a.held[p] = a.full[p] = 0;
        a.tail[p] = a.first[p] = INT32_MAX;
      } else {
        sh.bad = PACT_ERR_INVALID_ARG;
      }
    }
  });
  if (a.shared_out != a.shared)
    for (int p = me; p < a.n_pages; p += kAll) a.shared_out[p] = a.shared[p];
  cluster_sync();
  // 2: holders before and after
  each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int) {
    for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) {
      const int p = old_at(b, j);
      if (is_page(p)) {
        atomicAdd(a.held + p, 1);
        atomicMin(a.first + p, b * a.width + j);
      }
    }
  });
  each_chunk(sh.new_chunk, a.B, rank, [&](int b, int j0, int) {
    for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.rows(b) / a.page); j += 32) {
      const int p = old_at(a.source[b], j);
      if (is_page(p)) atomicAdd(a.full + p, 1);
    }
  });
  for (int b = me; b < a.B; b += kAll) {
    const int p = plan.tail_page(b);
    if (is_page(p)) atomicMin(a.tail + p, b);
  }
  cluster_sync();
  // 3: pages that go back, by chunks; requests that copy
  each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int c) {
    int n = 0;
    for (int j = j0; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) {
      bool gone = false;
      if (j + lane < plan.pages(b)) {
        const int p = old_at(b, j + lane);
        if (is_page(p)) {
          gone = a.first[p] == b * a.width + j + lane && plan.now(p) == 0;
          if (a.shared[p] < 0 || plan.outside(p) < 0) sh.bad = PACT_ERR_INVALID_ARG;
        }
      }
      n += __popc(__ballot_sync(0xffffffffu, gone));
    }
    if (lane == 0) a.chunk_freed[c] = n;
  });
  for (int b = me; b < a.B; b += kAll) {
    const int p = plan.tail_page(b);
    a.copies_tail[b] = is_page(p) && !(plan.kept_by_tail(p) && a.tail[p] == b);
  }
  __syncthreads();
  if (tid == 0) a.bad[rank] = sh.bad;
  cluster_sync();
  // 4: one CTA sums them up
  if (rank == 0) {
    int freed = 0, copied = 0, all;
    const int chunks = sh.old_chunk[a.B];
    for (int c0 = 0; c0 < chunks; c0 += kShareThreads) {
      const int c = c0 + tid, n = c < chunks ? a.chunk_freed[c] : 0, before = share_scan(n, sh.warp, &all);
      if (c < chunks) a.chunk_freed[c] = freed + before;
      freed += all;
    }
    for (int b0 = 0; b0 < a.B; b0 += kShareThreads) {
      const int b = b0 + tid, n = b < a.B ? a.copies_tail[b] : 0, before = share_scan(n, sh.warp, &all);
      if (b < a.B) a.copies_tail[b] = n ? copied + before : -1;
      copied += all;
    }
    if (tid == 0) {
      int bad = 0;
      for (int c = 0; c < kShareCtas; ++c) bad = min(bad, a.bad[c]);
      const int have = *a.n_free;
      if (!bad && freed > a.n_pages - have) bad = PACT_ERR_INVALID_ARG;
      if (!bad && copied > have + freed) bad = PACT_ERR_NO_PAGES;
      a.totals[0] = bad;
      a.totals[1] = freed;
      a.totals[2] = copied;
      a.totals[3] = have;
      if (bad && a.status) atomicMin(a.status, bad);
    }
  }
  cluster_sync();
  const int bad = a.totals[0], freed = a.totals[1], copied = a.totals[2], have = a.totals[3];
  // 5: pages that go back, in the order of their first places
  if (!bad)
    each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int c) {
      int at = a.chunk_freed[c];
      for (int j = j0; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) {
        const int p = j + lane < plan.pages(b) ? old_at(b, j + lane) : -1;
        const bool gone = p >= 0 && a.first[p] == b * a.width + j + lane && plan.now(p) == 0;
        const uint32_t who = __ballot_sync(0xffffffffu, gone);
        if (gone) a.freed[at + __popc(who & ((1u << lane) - 1u))] = p;
        at += __popc(who);
      }
    });
  cluster_sync();
  // 6: all of it, or nothing
  if (bad) {
    each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int) {
      for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) a.table_out[(long long)b * a.width + j] = old_at(b, j);
    });
    for (int b = me; b < a.B; b += kAll) a.length_out[b] = a.length[b];
    if (a.free_out != a.free_pages)
      for (int i = me; i < min(max(have, 0), a.n_pages); i += kAll) a.free_out[i] = a.free_pages[i];
  } else {
    each_chunk(sh.new_chunk, a.B, rank, [&](int b, int j0, int) {
      for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.rows(b) / a.page); j += 32) a.table_out[(long long)b * a.width + j] = old_at(a.source[b], j);
    });
    const int left = have + freed - copied;
    for (int b = me; b < a.B; b += kAll) {
      const int n = plan.rows(b), p = plan.tail_page(b), k = a.copies_tail[b];
      a.length_out[b] = n;
      if (p >= 0) {
        int mine = p;
        if (k >= 0) {                                                // the k-th page off the top of the stack, on which the freed ones lie
          const int at = have + freed - 1 - k;
          mine = at >= have ? a.freed[at - have] : a.free_pages[at];
          a.copies[3 * k] = p;
          a.copies[3 * k + 1] = mine;
          a.copies[3 * k + 2] = n % a.page;
        }
        a.table_out[(long long)b * a.width + n / a.page] = mine;
      }
    }
    // each page that was named is settled at its first place
    each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int) {
      for (int j = j0 + lane; j < min(j0 + kShareChunk, plan.pages(b)); j += 32) {
        const int p = old_at(b, j);
        if (a.first[p] == b * a.width + j) a.shared_out[p] = max(plan.now(p) - 1, 0);
      }
    });
    for (int i = me; i < left; i += kAll)
      if (i >= have) a.free_out[i] = a.freed[i - have];
      else if (a.free_out != a.free_pages) a.free_out[i] = a.free_pages[i];
  }
  const int listed = bad ? 0 : copied;
  for (int k = listed + me; k < a.n_list; k += kAll) {
    a.copies[3 * k] = a.copies[3 * k + 1] = -1;
    a.copies[3 * k + 2] = 0;
  }
  if (me == 0) {
    *a.n_copies = listed;
    *a.n_free_out = bad ? have : have + freed - copied;
  }
}

// ---- compaction ---------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(kShareThreads) k_cache_compact(const __grid_constant__ ShareArgs a) {
  extern __shared__ __align__(16) char sm[];
  ShareSmem &sh = *reinterpret_cast<ShareSmem *>(sm);
  const int tid = threadIdx.x, lane = tid & 31, rank = cta_rank(), me = rank * kShareThreads + tid;
  constexpr int kAll = kShareCtas * kShareThreads;
  if (tid == 0) sh.bad = 0;
  pdl_wait();
  pdl_trigger();
  const int words = (a.n_pages + 31) / 32, room = a.width * a.page, have = *a.n_free;
  const bool fits = have >= 0 && have <= a.n_pages;
  const int n_free = fits ? have : 0, n_used = a.n_pages - n_free;
  const auto pages = [&](int b) { return (min(max(a.length[b], 0), room) + a.page - 1) / a.page; };
  // 1
  chunk_starts(a.B, sh.old_chunk, sh.warp, pages);
  for (int b = me; b < a.B; b += kAll)
    if ((a.length[b] < 0 || a.length[b] > room) && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
  for (int w = me; w < words; w += kAll) a.free_bits[w] = 0;
  if (me == 0 && !fits) sh.bad = PACT_ERR_INVALID_ARG;
  cluster_sync();
  // 2: the free pages
  for (int i = me; i < n_free; i += kAll) {
    const int p = a.free_pages[i];
    if (p < 0 || p >= a.n_pages || (atomicOr(a.free_bits + (p >> 5), 1u << (p & 31)) >> (p & 31) & 1u)) sh.bad = PACT_ERR_INVALID_ARG;
  }
  __syncthreads();
  if (tid == 0) a.bad[rank] = sh.bad;
  cluster_sync();
  int bad = 0;
  for (int c = 0; c < kShareCtas; ++c) bad = min(bad, a.bad[c]);
  // 3: free ids below n_used and used ones from there on, of this CTA's words; a thread has neighbouring ones
  const int w0 = (int)((long long)words * rank / kShareCtas), w1 = (int)((long long)words * (rank + 1) / kShareCtas);
  const int per = (w1 - w0 + kShareThreads - 1) / kShareThreads, t0 = min(w1, w0 + tid * per), t1 = min(w1, t0 + per);
  const auto of_word = [&](int w, uint32_t &hole, uint32_t &stray) {
    const uint32_t there = w * 32 + 32 <= a.n_pages ? 0xffffffffu : (1u << (a.n_pages - w * 32)) - 1u;
    const int split = min(max(n_used - w * 32, 0), 32);
    const uint32_t low = split == 32 ? 0xffffffffu : (1u << split) - 1u, free = a.free_bits[w] & there;
    hole = free & low;
    stray = ~free & there & ~low;
  };
  int holes = 0, strays = 0, all_holes, all_strays;
  for (int w = t0; w < t1; ++w) {
    uint32_t h, s;
    of_word(w, h, s);
    holes += __popc(h);
    strays += __popc(s);
  }
  int hole_at = share_scan(holes, sh.warp, &all_holes), stray_at = share_scan(strays, sh.warp, &all_strays);
  if (tid == 0) {
    a.counts[2 * rank] = all_holes;
    a.counts[2 * rank + 1] = all_strays;
  }
  cluster_sync();
  // 4: their ids in order (there are as many of the one as of the other)
  int moves = 0;
  for (int c = 0; c < kShareCtas; ++c) {
    if (c < rank) {
      hole_at += a.counts[2 * c];
      stray_at += a.counts[2 * c + 1];
    }
    moves += a.counts[2 * c];
  }
  if (bad) moves = 0;
  if (!bad)
    for (int w = t0; w < t1; ++w) {
      uint32_t h, s;
      of_word(w, h, s);
      for (; h; h &= h - 1) a.holes[hole_at++] = w * 32 + __ffs(h) - 1;
      for (; s; s &= s - 1) a.strays[stray_at++] = w * 32 + __ffs(s) - 1;
    }
  for (int p = me; p < a.n_pages; p += kAll) {
    a.moved_to[p] = p;
    if (a.shared_out != a.shared) a.shared_out[p] = a.shared[p];
  }
  cluster_sync();
  // 5: where they go
  for (int k = me; k < a.n_list; k += kAll) {
    int from = -1, to = -1;
    if (k < moves) {
      from = a.strays[k];
      to = a.holes[k];
      a.moved_to[from] = to;
      const int n = a.shared[from];
      a.shared_out[to] = n;
      a.shared_out[from] = 0;
    }
    a.copies[3 * k] = from;
    a.copies[3 * k + 1] = to;
    a.copies[3 * k + 2] = k < moves ? a.page : 0;
  }
  if (!bad)
    for (int i = me; i < n_free; i += kAll) a.free_out[i] = a.n_pages - 1 - i;
  else if (a.free_out != a.free_pages)
    for (int i = me; i < n_free; i += kAll) a.free_out[i] = a.free_pages[i];
  if (me == 0) {
    *a.n_copies = moves;
    if (bad && a.status) atomicMin(a.status, bad);
  }
  cluster_sync();
  // 6: the tables
  each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int) {
    for (int j = j0 + lane; j < min(j0 + kShareChunk, pages(b)); j += 32) {
      const long long at = (long long)b * a.width + j;
      const int p = a.table[at];
      const bool there = p >= 0 && p < a.n_pages;
      if (!there && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      a.table_out[at] = there ? a.moved_to[p] : p;
    }
  });
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

cudaError_t launch(void (*kernel)(ShareArgs), const ShareArgs &a, cudaStream_t st) {
  LaunchOpt opt;
  opt.cluster = kShareCtas;
  return launch_opt(opt, kernel, dim3(kShareCtas), dim3(kShareThreads), sizeof(ShareSmem), st, a);
}

}  // namespace

size_t fork_scratch(int requests, int max_pages, int n_pages, ShareArgs *a, char *base) {
  size_t at = 0;
  const auto take = [&](size_t n) {
    int32_t *p = reinterpret_cast<int32_t *>(base + at);
    at += round256(n * sizeof(int32_t));
    return p;
  };
  const size_t P = n_pages, chunks = (size_t)requests * ((max_pages + kShareChunk - 1) / kShareChunk);
  int32_t *held = take(P), *full = take(P), *tail = take(P), *first = take(P), *freed = take(P), *chunk_freed = take(chunks), *copies_tail = take(requests), *totals = take(8),
          *bad = take(kShareCtas);
  if (a) {
    a->held = held; a->full = full; a->tail = tail; a->first = first; a->freed = freed; a->chunk_freed = chunk_freed; a->copies_tail = copies_tail;
    a->totals = totals; a->bad = bad;
  }
  return at;
}

size_t compact_scratch(int n_pages, ShareArgs *a, char *base) {
  size_t at = 0;
  const auto take = [&](size_t n) {
    int32_t *p = reinterpret_cast<int32_t *>(base + at);
    at += round256(n * sizeof(int32_t));
    return p;
  };
  int32_t *bits = take((size_t)n_pages / 32 + 1), *holes = take((size_t)n_pages / 2 + 1), *strays = take((size_t)n_pages / 2 + 1), *counts = take(2 * kShareCtas), *bad = take(kShareCtas);
  if (a) {
    a->free_bits = reinterpret_cast<uint32_t *>(bits); a->holes = holes; a->strays = strays; a->counts = counts; a->bad = bad;
  }
  return at;
}

cudaError_t share_configure() {
  const cudaError_t e = cudaFuncSetAttribute(k_cache_fork, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ShareSmem));
  return e != cudaSuccess ? e : cudaFuncSetAttribute(k_cache_compact, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ShareSmem));
}

cudaError_t launch_cache_fork(const ShareArgs &a, cudaStream_t st) { return launch(k_cache_fork, a, st); }
cudaError_t launch_cache_compact(const ShareArgs &a, cudaStream_t st) { return launch(k_cache_compact, a, st); }

}  // namespace pact
