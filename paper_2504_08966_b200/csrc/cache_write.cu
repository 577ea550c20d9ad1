// Rows into their slots of the paged cache, and the bounds of the pages' keys (pact_cache_write).
//
// A copy: every row is read once and written once, so HBM bounds it for prompts and latency for one new row per request.  A CTA
// takes a block of consecutive rows of one key head.  The bounds of a page are the minimum and maximum over the rows that this call
// puts into it (and the old bounds, where the page was begun earlier); its rows are a run of neighbours in the call, and the CTA in whose
// block the run begins reduces all of it.  The rows of the run that lie in the next block are read again: they come from the L2, and the
// bounds need neither atomics nor a second kernel.  Minimum and maximum are exact in any order.
#include "paged.cuh"

namespace pact {
namespace {

constexpr int kWriteThreads = 256;
constexpr int kWriteRows = 64;             // most rows of a block

// element-wise minimum and maximum of 16-byte vectors; a NaN gives way to a number
template <typename T> struct Bound;
template <> struct Bound<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t lo1(uint32_t x, uint32_t y) {
    const __nv_bfloat162 r = __hmin2(*reinterpret_cast<__nv_bfloat162 *>(&x), *reinterpret_cast<__nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
  static __device__ __forceinline__ uint32_t hi1(uint32_t x, uint32_t y) {
    const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&x), *reinterpret_cast<__nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&r);
  }
};
template <> struct Bound<float> {
  static __device__ __forceinline__ uint32_t lo1(uint32_t x, uint32_t y) { return __float_as_uint(fminf(__uint_as_float(x), __uint_as_float(y))); }
  static __device__ __forceinline__ uint32_t hi1(uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }
};
template <typename T> __device__ __forceinline__ void widen_bounds(uint4 &lo, uint4 &hi, const uint4 &l, const uint4 &h) {
  lo = make_uint4(Bound<T>::lo1(lo.x, l.x), Bound<T>::lo1(lo.y, l.y), Bound<T>::lo1(lo.z, l.z), Bound<T>::lo1(lo.w, l.w));
  hi = make_uint4(Bound<T>::hi1(hi.x, h.x), Bound<T>::hi1(hi.y, h.y), Bound<T>::hi1(hi.z, h.z), Bound<T>::hi1(hi.w, h.w));
}

template <typename T>
__global__ void __launch_bounds__(kWriteThreads) k_cache_write(WriteArgs a, int R) {
  // slots of rows c0 - 1 .. c0 + R + page - 1, and a bit for every row from c0 on that does not continue the run of the row before it
  extern __shared__ long long s_slot[];
  __shared__ uint32_t s_begins[(kWriteRows + 1024) / 32 + 1];
  __shared__ int s_run[kWriteRows], s_len[kWriteRows], s_n_runs, s_longest;
  __shared__ int2 s_at[kWriteRows];                             // page and place of the rows of the block, page -1: none
  __shared__ uint4 s_lo[kWriteThreads], s_hi[kWriteThreads];
  constexpr int V = Vec<T>::N;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long c0 = (long long)blockIdx.x * R, cap = (long long)a.n_pages * a.page;
  const int head = blockIdx.y, nv = a.d_h / V, reach = a.bounds ? R + a.page : R;
  pdl_wait();
  pdl_trigger();
  for (int i = tid; i <= reach; i += kWriteThreads) {
    const long long r = c0 - 1 + i;
    long long s = r >= 0 && r < a.n_rows ? a.slot[r] : -1;
    if (s >= cap) {
      s = -1;
      if (a.status && head == 0 && i > 0 && i <= R) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    }
    s_slot[i] = s;
    if (i > 0 && i <= R) {
      const long long page = s / a.page;
      s_at[i - 1] = s < 0 ? make_int2(-1, 0) : make_int2((int)page, (int)(s - page * a.page));
    }
  }
  if (tid == 0) s_n_runs = s_longest = 0;
  __syncthreads();

  const T *Kn = static_cast<const T *>(a.Kn) + head * a.ld_head, *Vn = static_cast<const T *>(a.Vn) + head * a.ld_head;
  T *K = static_cast<T *>(a.K) + head * a.k_head, *Vc = static_cast<T *>(a.V) + head * a.v_head;
  constexpr int U = 4;                                          // vectors of K and of V that a thread has in flight
  for (int i0 = tid; i0 < R * nv; i0 += U * kWriteThreads) {
    uint4 k[U], v[U];
    int2 at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kWriteThreads, r = i / nv, c = (i - r * nv) * V;
      at[u] = i < R * nv ? s_at[r] : make_int2(-1, 0);
      if (at[u].x >= 0) {
        k[u] = __ldg(reinterpret_cast<const uint4 *>(Kn + (c0 + r) * a.ld_row + c));
        v[u] = __ldg(reinterpret_cast<const uint4 *>(Vn + (c0 + r) * a.ld_row + c));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kWriteThreads, c = (i - i / nv * nv) * V;
      if (at[u].x >= 0) {
        *reinterpret_cast<uint4 *>(K + at[u].x * a.k_page + at[u].y * a.k_row + c) = k[u];
        *reinterpret_cast<uint4 *>(Vc + at[u].x * a.v_page + at[u].y * a.v_row + c) = v[u];
      }
    }
  }
  if (a.logw && head == 0 && tid < R && s_at[tid].x >= 0)
    a.logw[(long long)s_at[tid].x * a.page + s_at[tid].y] = a.logw_new ? a.logw_new[c0 + tid] : 0.f;
  if (!a.bounds) return;

  // runs: rows whose slots follow one another within a page
  for (int i0 = warp * 32; i0 < reach; i0 += kWriteThreads) {
    const int i = i0 + lane;
    bool begins = true;
    if (i < reach) {
      const long long s = s_slot[i + 1], prev = s_slot[i];
      begins = !(s >= 0 && prev >= 0 && s == prev + 1 && s % a.page != 0);
    }
    const uint32_t bits = __ballot_sync(0xffffffffu, begins);
    if (lane == 0) s_begins[i0 / 32] = bits;
  }
  __syncthreads();
  if (tid < R && s_at[tid].x >= 0 && (s_begins[tid / 32] >> (tid & 31) & 1)) {
    int w = tid / 32;                                          // the next beginning; a run ends with its page, so there is one within reach
    uint32_t bits = s_begins[w] & (0xfffffffeu << (tid & 31));
    while (!bits && (w + 1) * 32 < reach) bits = s_begins[++w];
    const int end = bits ? min(reach, w * 32 + __ffs(bits) - 1) : reach;
    const int k = atomicAdd(&s_n_runs, 1);                     // (the order of the runs changes nothing)
    s_run[k] = tid;
    s_len[k] = end - tid;
    atomicMax(&s_longest, end - tid);
  }
  __syncthreads();
  const int n_runs = s_n_runs;
  T *bounds = static_cast<T *>(a.bounds);
  const auto store = [&](int first, int c, uint4 lo, uint4 hi) {
    T *to = bounds + ((long long)s_at[first].x * a.n_kvh + head) * 2 * a.d_h + c;
    if (s_at[first].y)                                         // the page was begun earlier
      widen_bounds<T>(lo, hi, *reinterpret_cast<const uint4 *>(to), *reinterpret_cast<const uint4 *>(to + a.d_h));
    *reinterpret_cast<uint4 *>(to) = lo;
    *reinterpret_cast<uint4 *>(to + a.d_h) = hi;
  };
  if (s_longest <= 4) {                                        // a thread per run and vector: the one or few new rows of many requests
    for (int i = tid; i < n_runs * nv; i += kWriteThreads) {
      const int run = i / nv, c = (i - run * nv) * V, first = s_run[run];
      const T *p = Kn + (c0 + first) * a.ld_row + c;
      uint4 lo = __ldg(reinterpret_cast<const uint4 *>(p)), hi = lo;
      for (int r = 1; r < s_len[run]; ++r) {
        const uint4 k = __ldg(reinterpret_cast<const uint4 *>(p + r * a.ld_row));
        widen_bounds<T>(lo, hi, k, k);
      }
      store(first, c, lo, hi);
    }
  } else {                                                     // the CTA on one run after the other
    const int groups = kWriteThreads / nv, g = tid / nv, c = (tid - g * nv) * V;
    for (int run = 0; run < n_runs; ++run) {
      const int first = s_run[run], len = s_len[run];
      if (g < groups && g < len) {
        const T *p = Kn + (c0 + first) * a.ld_row + c;
        uint4 lo = __ldg(reinterpret_cast<const uint4 *>(p + g * a.ld_row)), hi = lo;
#pragma unroll 4
        for (int r = g + groups; r < len; r += groups) {
          const uint4 k = __ldg(reinterpret_cast<const uint4 *>(p + r * a.ld_row));
          widen_bounds<T>(lo, hi, k, k);
        }
        s_lo[tid] = lo;
        s_hi[tid] = hi;
      }
      __syncthreads();
      if (tid < nv) {
        uint4 lo = s_lo[tid], hi = s_hi[tid];
        for (int o = 1; o < min(groups, len); ++o) widen_bounds<T>(lo, hi, s_lo[o * nv + tid], s_hi[o * nv + tid]);
        store(first, c, lo, hi);
      }
      __syncthreads();
    }
  }
  if (head == 0)
    for (int run = warp; run < n_runs; run += kWriteThreads / 32) {
      const int first = s_run[run];
      float top = a.logw_new ? -INFINITY : 0.f;
      if (a.logw_new)
        for (int r = lane; r < s_len[run]; r += 32) top = fmaxf(top, a.logw_new[c0 + first + r]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (lane == 0) a.w_max[s_at[first].x] = s_at[first].y ? fmaxf(top, a.w_max[s_at[first].x]) : top;
    }
}

}  // namespace

cudaError_t launch_cache_write(const WriteArgs &a, bool bf16, int sm_count, cudaStream_t st) {
  int R = kWriteRows;                                          // smaller blocks until every SM has two CTAs
  while (R > 8 && (a.n_rows + R - 1) / R * a.n_kvh < 2 * sm_count) R /= 2;
  const dim3 grid((unsigned)((a.n_rows + R - 1) / R), (unsigned)a.n_kvh);
  const size_t smem = (size_t)(R + (a.bounds ? a.page : 0) + 1) * sizeof(long long);
  return bf16 ? launch_k(k_cache_write<__nv_bfloat16>, grid, dim3(kWriteThreads), smem, st, true, a, R)
              : launch_k(k_cache_write<float>, grid, dim3(kWriteThreads), smem, st, true, a, R);
}

}  // namespace pact
