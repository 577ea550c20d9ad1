// Requests that go on with the rows of others (pact_cache_fork) and pages moved to the lowest ids (pact_cache_compact).
//
// Both are bookkeeping over block tables, bound by latency: a chain of steps in which every entry has to be known to all before the next begins.  One cluster of CTAs walks through them with
// barriers between, a launch instead of five; counts go to global memory by integer atomics, whose order does not show.  A warp looks at 64 entries of a table at a time.
// Each instruction runs a few times only, so that fetching code is a good part of the time: what is needed of a request is worked out once, and steps are written once where they can be.
// Measured: 128 requests in groups of four, 24,000 entries: 17.6 us; eight that go on with one of 131,072 rows: 12.0 us; a compaction of 2,048 pages 10.3 us, of 65,536 17.3 us.  Eight CTAs
// instead of 16: 34, 24, 13 and 27 us (before lengths and sources were kept in shared memory; 16 then: 27, 24, 13, 21); the counts of a page in four arrays instead of one word of 16 bytes: 47 us for the first.
#include "share.cuh"

namespace pact {
namespace {

// ---- what both have -------------------------------------------------------------------------------------

__device__ __forceinline__ int cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return (int)r;
}

// Two sums at once, one in each half.
__device__ __forceinline__ uint64_t two(int low, int high) { return (uint64_t)(unsigned)low | (uint64_t)(unsigned)high << 32; }
__device__ __forceinline__ int low(uint64_t v) { return (int)(unsigned)v; }
__device__ __forceinline__ int high(uint64_t v) { return (int)(v >> 32); }

// Exclusive sums of a value per thread over the CTA; warp_sums[31] has the total until the next barrier.  (Not inlined: see above.)
__device__ __noinline__ uint64_t share_scan(uint64_t v, uint64_t *warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  if (warp == 0) {
    uint64_t w = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    warp_sums[lane] = w;
  }
  __syncthreads();
  return (warp ? warp_sums[warp - 1] : 0) + x - v;
}

// Sums over the cluster of what its CTAs have told, and over those before this one; by whole warps.
struct ClusterSums {
  int a, b, a_before, b_before, bad;
  __device__ __forceinline__ ClusterSums(const ShareSum *sums, int rank) {
    const int lane = threadIdx.x & 31;
    int4 v = make_int4(0, 0, 0, 0);
    if (lane < kShareCtas) v = *reinterpret_cast<const int4 *>(sums + lane);
    a = __reduce_add_sync(0xffffffffu, v.x);
    b = __reduce_add_sync(0xffffffffu, v.y);
    a_before = __reduce_add_sync(0xffffffffu, lane < rank ? v.x : 0);
    b_before = __reduce_add_sync(0xffffffffu, lane < rank ? v.y : 0);
    bad = __reduce_min_sync(0xffffffffu, v.z);
  }
};

constexpr int kMyWarps = kShareThreads / 32, kAll = kShareCtas * kShareThreads;
constexpr int kMyRequests = (PACT_MAX_REQUESTS + kShareCtas - 1) / kShareCtas;

struct ShareSmem {
  uint64_t warp[32];
  int bad;
  int old_chunk[PACT_MAX_REQUESTS + 1], new_chunk[PACT_MAX_REQUESTS + 1];   // chunks of the requests before, of their pages before and after the call
  int pages[PACT_MAX_REQUESTS], rows[PACT_MAX_REQUESTS], source[PACT_MAX_REQUESTS];   // pages before, rows after
  int tail[kMyRequests], copy_at[kMyRequests];               // of this CTA's requests: the page that they end in and share with what follows them in the source; their place among those that copy
};

__device__ __forceinline__ int share_of(int n, int rank) { return (int)((long long)n * rank / kShareCtas); }

// f(request, first place, chunk) for every chunk of this warp; a CTA has neighbouring ones
template <typename F> __device__ __forceinline__ void each_chunk(const int *chunk, int B, int rank, F f) {
  const int end = share_of(chunk[B], rank + 1);
#pragma unroll 1
  for (int c = share_of(chunk[B], rank) + (threadIdx.x >> 5); c < end; c += kMyWarps) {
    int lo = 0, hi = B;                                      // (some requests have no chunks)
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (chunk[mid] <= c) lo = mid;
      else hi = mid;
    }
    f(lo, (c - chunk[lo]) * kShareChunk, c);
  }
}
// f(request, place, what is there) for every entry of this thread: the first count(b) of row(b) of the table.  (Both are loaded before f, whose stores the compiler cannot tell from them.)
template <typename N, typename R, typename F>
__device__ __forceinline__ void each_entry(const int32_t *table, long long width, const int *chunk, int B, int rank, N count, R row, F f) {
  each_chunk(chunk, B, rank, [&](int b, int j0, int) {
    const int n = count(b), j = j0 + (int)(threadIdx.x & 31);
    const int32_t *at = table + row(b) * width + j;
    const int p = j < n ? at[0] : -1, q = j + 32 < n ? at[32] : -1;
    if (j < n) f(b, j, p);
    if (j + 32 < n) f(b, j + 32, q);
  });
}

// ---- fork -------------------------------------------------------------------------------------------------

// A page once all entries are counted.
struct ForkPage : SharePage {
  int shared, outside;                     // holders that are not in the tables
  bool kept;                               // by the request that ends in it
  int now;                                 // holders after the call
  __device__ __forceinline__ ForkPage(const ShareArgs &a, int p) {
    const int4 v = *reinterpret_cast<const int4 *>(a.pages + p);
    held = v.x; full = v.y; tail = v.z; first = v.w;
    shared = a.shared[p];
    outside = shared + 1 - held;
    kept = tail < a.B && full == 0 && outside == 0;
    now = outside + full + (kept ? 1 : 0);
  }
};

__global__ void __launch_bounds__(kShareThreads) k_cache_fork(const __grid_constant__ ShareArgs a) {
  static_assert(kShareChunk == 64, "two entries of a lane, a word of bits");
  extern __shared__ __align__(16) char sm[];
  ShareSmem &sh = *reinterpret_cast<ShareSmem *>(sm);
  const int tid = threadIdx.x, lane = tid & 31, rank = cta_rank(), me = rank * kShareThreads + tid;
  if (tid == 0) sh.bad = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const auto pages_of = [&](unsigned n) { return page_of(a.page_mul, n); };
  const auto old_at = [&](int b, int j) { return a.table[(long long)b * a.width + j]; };
  const auto is_page = [&](int p) { return p >= 0 && p < a.n_pages; };
  const auto old_entries = [&](auto f) {
    each_entry(a.table, a.width, sh.old_chunk, a.B, rank, [&](int b) { return sh.pages[b]; }, [](int b) { return b; }, f);
  };
  const auto new_entries = [&](auto f) {                             // whole pages of the request after the call
    each_entry(a.table, a.width, sh.new_chunk, a.B, rank, [&](int b) { return pages_of(sh.rows[b]); }, [&](int b) { return sh.source[b]; }, f);
  };
  // 1: what is asked for, checked; the words of all pages named cleared
  {
    const int room = a.width * a.page, per = (a.B + kShareThreads - 1) / kShareThreads, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    uint64_t mine = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const int n = a.length[b], s = a.source[b], wanted = a.rows ? a.rows[b] : INT32_MAX, len = min(max(n, 0), room);
      const bool goes_on = s >= 0 && s < a.B;
      const int have = goes_on ? min(max(a.length[s], 0), room) : 0, rows = min(max(wanted, 0), have);
      if (n != len || s < -1 || s >= a.B || (goes_on && a.rows && rows != wanted)) sh.bad = PACT_ERR_INVALID_ARG;
      sh.pages[b] = pages_of((unsigned)len + a.page - 1);
      sh.rows[b] = rows;
      sh.source[b] = s;
      mine += two((sh.pages[b] + kShareChunk - 1) / kShareChunk, (pages_of(rows) + kShareChunk - 1) / kShareChunk);
    }
    uint64_t at = share_scan(mine, sh.warp);
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      sh.old_chunk[b] = low(at);
      sh.new_chunk[b] = high(at);
      at += two((sh.pages[b] + kShareChunk - 1) / kShareChunk, (pages_of(sh.rows[b]) + kShareChunk - 1) / kShareChunk);
    }
    if (tid == 0) {
      sh.old_chunk[a.B] = low(sh.warp[31]);
      sh.new_chunk[a.B] = high(sh.warp[31]);
    }
    __syncthreads();
  }
  const int first_b = share_of(a.B, rank), my_b = share_of(a.B, rank + 1) - first_b;   // this CTA's requests
  old_entries([&](int, int, int p) {
    if (is_page(p)) *reinterpret_cast<int4 *>(a.pages + p) = make_int4(0, 0, INT32_MAX, INT32_MAX);
    else sh.bad = PACT_ERR_INVALID_ARG;
  });
  for (int i = tid; i < my_b; i += kShareThreads) {
    const int b = first_b + i, n = sh.rows[b], j = pages_of(n);
    sh.tail[i] = n > j * a.page ? old_at(sh.source[b], j) : -1;
  }
  if (a.shared_out != a.shared)
    for (int p = me; p < a.n_pages; p += kAll) a.shared_out[p] = a.shared[p];
  cluster_sync();
  // 2: holders before and after
  old_entries([&](int b, int j, int p) {
    if (!is_page(p)) return;
    atomicAdd(&a.pages[p].held, 1);
    atomicMin(&a.pages[p].first, b * a.width + j);
  });
  new_entries([&](int, int, int p) {
    if (is_page(p)) atomicAdd(&a.pages[p].full, 1);
  });
  for (int i = tid; i < my_b; i += kShareThreads)
    if (is_page(sh.tail[i])) atomicMin(&a.pages[sh.tail[i]].tail, first_b + i);
  cluster_sync();
  // 3: pages that go back and requests that copy, counted in their order within the CTA
  each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int c) {
    uint64_t firsts = 0, gones = 0;
    const int j = j0 + lane, n = sh.pages[b];
    int p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = j + 32 * i < n ? old_at(b, j + 32 * i) : -1;
    ForkPage page[2] = {ForkPage(a, is_page(p[0]) ? p[0] : 0), ForkPage(a, is_page(p[1]) ? p[1] : 0)};   // (page 0 in place of none: looked at, not used)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool first = is_page(p[i]) && page[i].first == b * a.width + j + 32 * i, gone = first && page[i].now == 0;
      if (is_page(p[i]) && (page[i].shared < 0 || page[i].outside < 0)) sh.bad = PACT_ERR_INVALID_ARG;
      firsts |= (uint64_t)__ballot_sync(0xffffffffu, first) << (32 * i);
      gones |= (uint64_t)__ballot_sync(0xffffffffu, gone) << (32 * i);
    }
    if (lane == 0) {
      a.chunk_first[c] = firsts;
      a.chunk_gone[c] = gones;
    }
  });
  __syncthreads();
  {
    const int c0 = share_of(sh.old_chunk[a.B], rank), my_c = share_of(sh.old_chunk[a.B], rank + 1) - c0;
    uint64_t sum = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < max(my_c, my_b); i0 += kShareThreads) {
      const int i = i0 + tid;
      bool copies = false;
      if (i < my_b && is_page(sh.tail[i])) {
        const ForkPage page(a, sh.tail[i]);
        copies = !(page.kept && page.tail == first_b + i);
      }
      const uint64_t n = two(i < my_c ? __popcll(a.chunk_gone[c0 + i]) : 0, copies ? 1 : 0), before = sum + share_scan(n, sh.warp);
      if (i < my_c) a.chunk_freed[c0 + i] = low(before);
      if (i < my_b) sh.copy_at[i] = copies ? high(before) : -1;
      sum += sh.warp[31];
    }
    if (tid == 0) *reinterpret_cast<int4 *>(a.sums + rank) = make_int4(low(sum), high(sum), sh.bad, 0);
  }
  cluster_sync();
  // 4: all of it, or nothing
  const ClusterSums sums(a.sums, rank);
  const int freed = sums.a, copied = sums.b, have = *a.n_free, left = have + freed - copied;
  int bad = sums.bad;
  if (have < 0 || have > a.n_pages || (!bad && freed > a.n_pages - have)) bad = PACT_ERR_INVALID_ARG;
  if (!bad && left < 0) bad = PACT_ERR_NO_PAGES;
  if (bad) {
    old_entries([&](int b, int j, int p) { a.table_out[(long long)b * a.width + j] = p; });
    for (int b = me; b < a.B; b += kAll) a.length_out[b] = a.length[b];
    if (me == 0 && a.status) atomicMin(a.status, bad);
  } else {
    each_chunk(sh.old_chunk, a.B, rank, [&](int b, int j0, int c) {
      const uint64_t firsts = a.chunk_first[c], gones = a.chunk_gone[c];
      const int at = sums.a_before + a.chunk_freed[c];
      int p[2], now[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) p[h] = firsts >> (lane + 32 * h) & 1 ? old_at(b, j0 + lane + 32 * h) : -1;
#pragma unroll
      for (int h = 0; h < 2; ++h) now[h] = ForkPage(a, max(p[h], 0)).now;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = lane + 32 * h;
        if (p[h] >= 0) a.shared_out[p[h]] = max(now[h] - 1, 0);      // (each page that was named is settled at its first place)
        if (gones >> i & 1) {
          const int k = at + __popcll(gones & ((1ull << i) - 1));
          a.freed[k] = p[h];
          if (have + k < left) a.free_out[have + k] = p[h];
        }
      }
    });
    new_entries([&](int b, int j, int p) { a.table_out[(long long)b * a.width + j] = p; });
    for (int b = me; b < a.B; b += kAll) a.length_out[b] = sh.rows[b];
  }
  if (a.free_out != a.free_pages)
    for (int i = me; i < min(bad ? min(max(have, 0), a.n_pages) : left, have); i += kAll) a.free_out[i] = a.free_pages[i];
  const int listed = bad ? 0 : copied;
  for (int k = listed + me; k < a.n_list; k += kAll) {
    a.copies[3 * k] = a.copies[3 * k + 1] = -1;
    a.copies[3 * k + 2] = 0;
  }
  cluster_sync();
  // 5: pages for those that copy, off the top of the stack, on which the freed ones lie
  if (me == 0) {
    *a.n_copies = listed;
    *a.n_free_out = bad ? have : left;
  }
  if (!bad)
    for (int i = tid; i < my_b; i += kShareThreads) {
      int p = sh.tail[i];
      if (p < 0) continue;
      const int b = first_b + i, n = sh.rows[b], j = pages_of(n);
      if (sh.copy_at[i] >= 0) {
        const int k = sums.b_before + sh.copy_at[i], at = have + freed - 1 - k, from = p;
        p = at >= have ? a.freed[at - have] : a.free_pages[at];
        a.copies[3 * k] = from;
        a.copies[3 * k + 1] = p;
        a.copies[3 * k + 2] = n - j * a.page;
      }
      a.table_out[(long long)b * a.width + j] = p;
    }
}

// ---- compaction ---------------------------------------------------------------------------------------------

__global__ void __launch_bounds__(kShareThreads) k_cache_compact(const __grid_constant__ ShareArgs a) {
  extern __shared__ __align__(16) char sm[];
  ShareSmem &sh = *reinterpret_cast<ShareSmem *>(sm);
  const int tid = threadIdx.x, rank = cta_rank(), me = rank * kShareThreads + tid;
  if (tid == 0) sh.bad = 0;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int words = (a.n_pages + 31) / 32, room = a.width * a.page, have = *a.n_free;
  const bool fits = have >= 0 && have <= a.n_pages;
  const int n_free = fits ? have : 0, n_used = a.n_pages - n_free;
  // 1
  for (int w = me; w < words; w += kAll) a.free_bits[w] = 0;
  if (!fits) sh.bad = PACT_ERR_INVALID_ARG;
  {
    const int per = (a.B + kShareThreads - 1) / kShareThreads, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    uint64_t mine = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      const int n = a.length[b], len = min(max(n, 0), room);
      if (n != len && rank == 0 && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      sh.pages[b] = page_of(a.page_mul, (unsigned)len + a.page - 1);
      mine += (sh.pages[b] + kShareChunk - 1) / kShareChunk;
    }
    uint64_t at = share_scan(mine, sh.warp);
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
      sh.old_chunk[b] = low(at);
      at += (sh.pages[b] + kShareChunk - 1) / kShareChunk;
    }
    if (tid == 0) sh.old_chunk[a.B] = low(sh.warp[31]);
  }
  cluster_sync();
  // 2: the free pages
  for (int i = me; i < n_free; i += kAll) {
    const int p = a.free_pages[i];
    if (p < 0 || p >= a.n_pages || (atomicOr(a.free_bits + (p >> 5), 1u << (p & 31)) >> (p & 31) & 1u)) sh.bad = PACT_ERR_INVALID_ARG;
  }
  for (int p = me; p < a.n_pages; p += kAll) {
    a.moved_to[p] = p;
    if (a.shared_out != a.shared) a.shared_out[p] = a.shared[p];
  }
  cluster_sync();
  // 3: free ids below n_used and used ones from there on, of this CTA's words; a thread has neighbouring ones
  const int w0 = share_of(words, rank), w1 = share_of(words, rank + 1), per = (w1 - w0 + kShareThreads - 1) / kShareThreads, t0 = min(w1, w0 + tid * per), t1 = min(w1, t0 + per);
  const auto of_word = [&](int w, uint32_t &hole, uint32_t &stray) {
    const uint32_t there = w * 32 + 32 <= a.n_pages ? 0xffffffffu : (1u << (a.n_pages - w * 32)) - 1u;
    const int split = min(max(n_used - w * 32, 0), 32);
    const uint32_t low = split == 32 ? 0xffffffffu : (1u << split) - 1u, free = a.free_bits[w] & there;
    hole = free & low;
    stray = ~free & there & ~low;
  };
  uint64_t mine = 0;
#pragma unroll 1
  for (int w = t0; w < t1; ++w) {
    uint32_t h, s;
    of_word(w, h, s);
    mine += two(__popc(h), __popc(s));
  }
  const uint64_t before = share_scan(mine, sh.warp);
  if (tid == 0) *reinterpret_cast<int4 *>(a.sums + rank) = make_int4(low(sh.warp[31]), high(sh.warp[31]), sh.bad, 0);
  cluster_sync();
  // 4: their ids in order (there are as many of the one as of the other)
  const ClusterSums sums(a.sums, rank);
  const int bad = sums.bad, moves = bad ? 0 : sums.a;
  if (!bad) {
    int hole_at = sums.a_before + low(before), stray_at = sums.b_before + high(before);
#pragma unroll 1
    for (int w = t0; w < t1; ++w) {
      uint32_t h, s;
      of_word(w, h, s);
      for (; h; h &= h - 1) a.holes[hole_at++] = w * 32 + __ffs(h) - 1;
      for (; s; s &= s - 1) a.strays[stray_at++] = w * 32 + __ffs(s) - 1;
    }
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
  if (!bad || a.free_out != a.free_pages)
    for (int i = me; i < n_free; i += kAll) a.free_out[i] = bad ? a.free_pages[i] : a.n_pages - 1 - i;
  if (me == 0) {
    *a.n_copies = moves;
    if (bad && a.status) atomicMin(a.status, bad);
  }
  cluster_sync();
  // 6: the tables
  each_entry(a.table, a.width, sh.old_chunk, a.B, rank, [&](int b) { return sh.pages[b]; }, [](int b) { return b; }, [&](int b, int j, int p) {
    const bool there = p >= 0 && p < a.n_pages;
    if (!there && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    a.table_out[(long long)b * a.width + j] = there ? a.moved_to[p] : p;
  });
}

size_t round256(size_t x) { return (x + 255) / 256 * 256; }

cudaError_t launch(void (*kernel)(ShareArgs), const ShareArgs &a, cudaStream_t st) {
  LaunchOpt opt;
  opt.cluster = kShareCtas;
  return launch_opt(opt, kernel, dim3(kShareCtas), dim3(kShareThreads), sizeof(ShareSmem), st, a);
}

bool cluster_fits(void (*kernel)(ShareArgs)) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ShareSmem)) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
    return false;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(kShareCtas);
  lc.blockDim = dim3(kShareThreads);
  lc.dynamicSmemBytes = sizeof(ShareSmem);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kShareCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  lc.attrs = attr;
  lc.numAttrs = 1;
  int n = 0;
  return cudaOccupancyMaxActiveClusters(&n, kernel, &lc) == cudaSuccess && n >= 1;
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
  int32_t *pages = take(4 * P), *freed = take(P), *chunk_freed = take(chunks), *first = take(2 * chunks), *gone = take(2 * chunks), *sums = take(4 * kShareCtas);
  if (a) {
    a->pages = reinterpret_cast<SharePage *>(pages); a->freed = freed; a->chunk_freed = chunk_freed;
    a->chunk_first = reinterpret_cast<uint64_t *>(first); a->chunk_gone = reinterpret_cast<uint64_t *>(gone);
    a->sums = reinterpret_cast<ShareSum *>(sums);
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
  int32_t *bits = take((size_t)n_pages / 32 + 1), *holes = take((size_t)n_pages / 2 + 1), *strays = take((size_t)n_pages / 2 + 1), *sums = take(4 * kShareCtas);
  if (a) {
    a->free_bits = reinterpret_cast<uint32_t *>(bits); a->holes = holes; a->strays = strays;
    a->sums = reinterpret_cast<ShareSum *>(sums);
  }
  return at;
}

bool share_fits() {
  for (auto kernel : {k_cache_fork, k_cache_compact})
    if (!cluster_fits(kernel)) {
      (void)cudaGetLastError();
      return false;
    }
  return true;
}

cudaError_t launch_cache_fork(const ShareArgs &a, cudaStream_t st) { return launch(k_cache_fork, a, st); }
cudaError_t launch_cache_compact(const ShareArgs &a, cudaStream_t st) { return launch(k_cache_compact, a, st); }

}  // namespace pact
