// Block tables and slots of the rows that come next (pact_cache_plan).
//
// With had_b = ceil(length_b / page) and need_b = ceil((length_b + n_new_b) / page) - had_b, the k-th page that the call takes (by ascending
// request, then place) is entry n_free + F - 1 - k of the stack free_pages[0 .. n_free) followed by the F pages of the ended requests.
// Everything follows from three prefix sums over the requests (pages needed, pages given back, rows), which every CTA forms for itself:
// a trip to memory and a scan, where one CTA's scan for all of them would be a launch before this one.  What a launch reads it does
// not write (entries below had_b, the stack below n_free, lengths unless they are updated in place), so CTAs need not wait for one another;
// lengths in place are written by the one CTA of a small call after its barrier, and by a launch of their own behind a large one.
#include "paged.cuh"

namespace pact {
namespace {

constexpr int kPlanRequests = 256;         // requests up to which CTAs have 256 threads, beyond 1024
constexpr int kPlanRowsAlone = 1024;       // new rows up to which one CTA does everything
constexpr int kPlanRowsInPlace = 8192;     // the same where lengths are updated in place

struct Sums {
  long long need, freed, rows;
};

__device__ __forceinline__ Sums add(const Sums &x, const Sums &y) { return {x.need + y.need, x.freed + y.freed, x.rows + y.rows}; }

// last index b with pre[b] <= k, for pre ascending from 0 and k < pre[n]
__device__ __forceinline__ int find_share(const int *pre, int n, int k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_cache_plan(PlanArgs a) {
  extern __shared__ int s_plan[];
  __shared__ Sums s_warp[THREADS / 32];
  int *s_need = s_plan, *s_freed = s_need + a.B + 1, *s_rows = s_freed + a.B + 1, *s_len = s_rows + a.B + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.B + THREADS - 1) / THREADS;                   // requests of a thread
  pdl_wait();
  pdl_trigger();
  const long long n_free = *a.n_free;
  const long long room = (long long)a.width * a.page;
  const auto sums_of = [&](int len, int add_rows) {
    const bool ended = add_rows < 0;
    const unsigned rows = ended ? 0u : (unsigned)add_rows, had = ((unsigned)len + (unsigned)a.page - 1u) / (unsigned)a.page;
    // (len + rows < 2^32: both are below 2^31; what does not fit the table is refused before these are used)
    const unsigned all = (unsigned)(((unsigned long long)(unsigned)len + rows + (unsigned)a.page - 1u) / (unsigned)a.page);
    return Sums{ended ? 0ll : (long long)all - had, ended ? (long long)had : 0ll, (long long)rows};
  };
  Sums mine = {0, 0, 0};
  bool bad = n_free < 0 || n_free > a.n_pages;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b >= a.B) break;
    const int len = a.length[b], add_rows = a.n_new[b * a.n_new_stride];
    bad = bad || len < 0 || len + (long long)max(add_rows, 0) > room || (a.row_stride && add_rows > a.row_stride);
    const Sums x = sums_of(max(len, 0), add_rows);
    s_need[b] = (int)mine.need;                                    // so far: before this request, of this thread's
    s_freed[b] = (int)mine.freed;
    s_rows[b] = (int)mine.rows;
    s_len[b] = len;
    mine = add(mine, x);
  }
  Sums upto = mine;                                                // inclusive over the warp
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums other = {__shfl_up_sync(0xffffffffu, upto.need, o), __shfl_up_sync(0xffffffffu, upto.freed, o), __shfl_up_sync(0xffffffffu, upto.rows, o)};
    if (lane >= o) upto = add(upto, other);
  }
  if (lane == 31) s_warp[warp] = upto;
  const bool any_bad = __syncthreads_or(bad);
  Sums total = {0, 0, 0}, before = {0, 0, 0};
#pragma unroll 8
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w == warp) before = total;
    total = add(total, s_warp[w]);
  }
  const bool invalid = any_bad || total.rows > a.n_rows || n_free + total.freed > a.n_pages;
  const bool ok = !invalid && total.need <= n_free + total.freed;  // then every sum fits 32 bits
  const Sums at = {before.need + upto.need - mine.need, before.freed + upto.freed - mine.freed, before.rows + upto.rows - mine.rows};
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    if (b >= a.B) break;
    s_need[b] += (int)at.need;
    s_freed[b] += (int)at.freed;
    s_rows[b] += (int)at.rows;
  }
  if (tid == 0) {
    s_need[a.B] = (int)total.need;
    s_freed[a.B] = (int)total.freed;
    s_rows[a.B] = (int)total.rows;
  }
  __syncthreads();

  const int nf = (int)n_free, top = nf + (int)total.freed;
  const auto had_of = [&](int b) { return (int)(((unsigned)s_len[b] + (unsigned)a.page - 1u) / (unsigned)a.page); };
  const auto stack = [&](int i) {                                  // entry i of the free pages, those given back on top
    if (i < nf) return a.free_pages[i];
    const int b = find_share(s_freed, a.B, i - nf);
    return a.table[(long long)b * a.width + (i - nf - s_freed[b])];
  };
  const long long first = (long long)blockIdx.x * THREADS + tid, step = (long long)gridDim.x * THREADS;
  if (a.rows && ok) {
    for (long long k = first; k < total.need; k += step) {
      const int b = find_share(s_need, a.B, (int)k);
      a.table[(long long)b * a.width + had_of(b) + ((int)k - s_need[b])] = stack(top - 1 - (int)k);
    }
    for (long long i = nf + first; i < top - total.need; i += step) a.free_pages[i] = stack((int)i);
  }
  if (a.rows && a.slot) {
    for (long long r = first; r < a.n_rows; r += step) {
      long long v = -1;
      if (ok) {
        int b = 0, i = 0, n = 0;
        if (a.row_stride) {
          b = (int)(r / a.row_stride);
          i = (int)(r - (long long)b * a.row_stride);
          n = s_rows[b + 1] - s_rows[b];
        } else if (r < total.rows) {
          b = find_share(s_rows, a.B, (int)r);
          i = (int)r - s_rows[b];
          n = i + 1;
        }
        if (i < n) {
          const unsigned p = (unsigned)s_len[b] + (unsigned)i, place = p / (unsigned)a.page;
          const int had = had_of(b);
          const int id = (int)place < had ? a.table[(long long)b * a.width + place] : stack(top - 1 - (s_need[b] + (int)place - had));
          v = (long long)id * a.page + (p - place * (unsigned)a.page);
        }
      }
      a.slot[r] = v;
    }
  }
  if (a.commit && blockIdx.x == 0) {
    for (int b = tid; b < a.B; b += THREADS) {
      const int add_rows = ok ? a.n_new[b * a.n_new_stride] : 0;
      a.length_out[b] = add_rows < 0 ? 0 : s_len[b] + add_rows;
      if (a.row_start) a.row_start[b] = ok ? s_rows[b] : 0;
    }
    if (tid == 0) {
      *a.n_free_out = ok ? top - (int)total.need : (int)n_free;
      if (a.row_start) a.row_start[a.B] = ok ? s_rows[a.B] : 0;
      if (!ok && a.status) atomicMin(a.status, invalid ? (int)PACT_ERR_INVALID_ARG : (int)PACT_ERR_NO_PAGES);
    }
  }
}

}  // namespace

cudaError_t launch_cache_plan(PlanArgs a, int sm_count, cudaStream_t st, int *launches) {
  const size_t smem = ((size_t)a.B * 4 + 3) * sizeof(int);
  const bool in_place = a.length_out == a.length || a.n_free_out == a.n_free, wide = a.B > kPlanRequests || (in_place && a.n_rows > kPlanRowsAlone);
  void (*kernel)(PlanArgs) = wide ? k_cache_plan<1024> : k_cache_plan<256>;
  const int threads = wide ? 1024 : 256;
  a.rows = a.commit = true;
  *launches = 1;
  if (a.n_rows <= (in_place ? kPlanRowsInPlace : kPlanRowsAlone)) return launch_k(kernel, dim3(1), dim3(threads), smem, st, true, a);
  const long long ctas = (a.n_rows + 4 * threads - 1) / (4 * threads), most = wide ? sm_count : 4 * sm_count;
  a.commit = !in_place;
  cudaError_t e = launch_k(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(threads), smem, st, true, a);
  if (e != cudaSuccess || !in_place) return e;
  a.rows = false;
  a.commit = true;
  *launches = 2;
  return launch_k(kernel, dim3(1), dim3(threads), smem, st, true, a);
}

cudaError_t plan_configure() {
  return cudaFuncSetAttribute(k_cache_plan<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(((size_t)PACT_MAX_REQUESTS * 4 + 3) * sizeof(int)));
}

}  // namespace pact
