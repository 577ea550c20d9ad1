// Rows into their slots of the paged cache, and the bounds of the pages' keys (pact_cache_write).
//
// A copy: every row is read once and written once, so HBM bounds it for prompts and latency for one new row per request.  The bounds of a page are the
// minimum and maximum over the rows that this call puts into it (and the old bounds, where the page was begun earlier); its rows are a run of
// neighbours in the call.  A CTA takes the runs of one key head that begin in its block of rows, all of their rows and no others, so that a page's bounds are one
// CTA's, without atomics or a second kernel, from rows that it has just copied and finds in its L1.  Its warps share out the runs, or a run.
// Minimum and maximum are exact in any order.
// 16 prompts of 2948 rows at most, 4 key heads of 128, pages of 64, bf16 (119 MB): 27.5 us, without bounds 23 to 24.  Others: bounds from pieces of runs kept in
// registers 44 to 51 us, a warp per run 32, bounds in registers on the way through the copy 29.
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

constexpr int kWriteWarps = kWriteThreads / 32;
constexpr int kMaxReach = kWriteRows + 1024;   // rows that a CTA may have: those of its block, and of a page that goes on behind it

template <typename T>
__global__ void __launch_bounds__(kWriteThreads) k_cache_write(WriteArgs a, int R) {
  // of rows c0 .. c0 + R + page - 1: page and place (page -1: none), and a bit for those that do not continue the run of the row before them
  extern __shared__ int2 s_at[];
  __shared__ uint32_t s_begins[kMaxReach / 32 + 1];
  __shared__ int s_run[kWriteRows], s_len[kWriteRows], s_n_runs;
  __shared__ uint4 s_lo[kWriteWarps][32], s_hi[kWriteWarps][32];
  constexpr int V = Vec<T>::N;
  constexpr uint32_t kNone = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu;   // NaN, which gives way to any number
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long c0 = (long long)blockIdx.x * R, cap = (long long)a.n_pages * a.page;
  const int head = blockIdx.y, nv = a.d_h / V, reach = R + a.page;
  pdl_wait();
  pdl_trigger();
  if (tid == 0) s_n_runs = 0;
  for (int i0 = warp * 32; i0 < reach; i0 += kWriteThreads) {
    const int i = i0 + lane;
    const long long r = c0 + i;
    long long s = i < reach && r < a.n_rows ? a.slot[r] : -1, prev = __shfl_up_sync(0xffffffffu, s, 1);
    if (lane == 0) prev = r > 0 && r - 1 < a.n_rows ? a.slot[r - 1] : -1;
    if (s >= cap) {
      if (a.status && head == 0 && i < R) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      s = -1;
    }
    const long long page = cap >> 32 ? s / a.page : (unsigned)s / (unsigned)a.page;
    const int2 at = s < 0 ? make_int2(-1, 0) : make_int2((int)page, (int)(s - page * a.page));
    if (i < reach) s_at[i] = at;
    // (the row before a continued one has a slot of this cache: it is one less than this row's)
    const uint32_t bits = __ballot_sync(0xffffffffu, !(at.x >= 0 && at.y != 0 && s == prev + 1));
    if (lane == 0) s_begins[i0 / 32] = bits;
  }
  __syncthreads();
  const auto next_begin = [&](int i) {                          // the first at or behind i, at most `reach`
    for (int w = i >> 5; w * 32 < reach; ++w) {
      const uint32_t bits = s_begins[w] & (w == i >> 5 ? 0xffffffffu << (i & 31) : 0xffffffffu);
      if (bits) return min(reach, w * 32 + __ffs(bits) - 1);
    }
    return reach;
  };
  const int lo_row = next_begin(0), hi_row = next_begin(R);     // this CTA's rows (a run ends with its page, so the last one ends within reach)
  if (lo_row >= R) return;
  if (tid < R && s_at[tid].x >= 0 && (s_begins[tid / 32] >> (tid & 31) & 1)) {
    const int k = atomicAdd(&s_n_runs, 1);                      // (the order of the runs changes nothing)
    s_run[k] = tid;
    s_len[k] = next_begin(tid + 1) - tid;
  }

  const T *Kn = static_cast<const T *>(a.Kn) + head * a.ld_head, *Vn = static_cast<const T *>(a.Vn) + head * a.ld_head;
  T *K = static_cast<T *>(a.K) + head * a.k_head, *Vc = static_cast<T *>(a.V) + head * a.v_head;
  constexpr int U = 4;                                          // vectors of K and of V that a thread has in flight
  const int n_vec = (hi_row - lo_row) * nv;
  for (int i0 = tid; i0 < n_vec; i0 += U * kWriteThreads) {
    uint4 k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kWriteThreads, r = i / nv, c = (i - r * nv) * V;
      if (i < n_vec && s_at[lo_row + r].x >= 0) {
        k[u] = __ldg(reinterpret_cast<const uint4 *>(Kn + (c0 + lo_row + r) * a.ld_row + c));
        v[u] = __ldg(reinterpret_cast<const uint4 *>(Vn + (c0 + lo_row + r) * a.ld_row + c));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * kWriteThreads, r = i / nv, c = (i - r * nv) * V;
      if (i < n_vec && s_at[lo_row + r].x >= 0) {
        const int2 at = s_at[lo_row + r];
        *reinterpret_cast<uint4 *>(K + at.x * a.k_page + at.y * a.k_row + c) = k[u];
        *reinterpret_cast<uint4 *>(Vc + at.x * a.v_page + at.y * a.v_row + c) = v[u];
      }
    }
  }
  if (a.logw && head == 0)
    for (int r = lo_row + tid; r < hi_row; r += kWriteThreads)
      if (s_at[r].x >= 0) a.logw[(long long)s_at[r].x * a.page + s_at[r].y] = a.logw_new ? a.logw_new[c0 + r] : 0.f;
  if (!a.bounds) return;
  __syncthreads();

  // a team of warps per run: 1 for five runs and more, 2, 4, and all eight for a single one; 32 / nv rows at a time
  const int n_runs = s_n_runs, team = n_runs >= 5 ? 1 : n_runs >= 3 ? 2 : n_runs == 2 ? 4 : 8, member = warp & (team - 1);
  const int at_once = 32 / nv, sub = lane / nv, c = (lane - sub * nv) * V;
  const auto store = [&](int first, uint4 lo, uint4 hi) {       // by the first nv lanes
    T *to = static_cast<T *>(a.bounds) + ((long long)s_at[first].x * a.n_kvh + head) * 2 * a.d_h + c;
    if (s_at[first].y)                                          // the page was begun earlier
      widen_bounds<T>(lo, hi, *reinterpret_cast<const uint4 *>(to), *reinterpret_cast<const uint4 *>(to + a.d_h));
    *reinterpret_cast<uint4 *>(to) = lo;
    *reinterpret_cast<uint4 *>(to + a.d_h) = hi;
  };
  for (int run = warp / team; run < n_runs; run += kWriteWarps / team) {   // (once, unless a team is one warp)
    const int first = s_run[run], len = s_len[run], step = at_once * team;
    const T *p = Kn + (c0 + first) * a.ld_row + c;
    uint4 lo = make_uint4(kNone, kNone, kNone, kNone), hi = lo;
    if (sub < at_once) {
      constexpr int W = 4;                                      // vectors in flight
      for (int x0 = member * at_once + sub; x0 < len; x0 += W * step) {
        uint4 k[W];
#pragma unroll
        for (int u = 0; u < W; ++u)
          if (x0 + u * step < len) k[u] = __ldg(reinterpret_cast<const uint4 *>(p + (x0 + u * step) * a.ld_row));
#pragma unroll
        for (int u = 0; u < W; ++u)
          if (x0 + u * step < len) widen_bounds<T>(lo, hi, k[u], k[u]);
      }
    }
    __syncwarp();
    for (int x = 1; x < at_once; ++x) {
      const int from = (lane + x * nv) & 31;
      const uint4 l = make_uint4(__shfl_sync(0xffffffffu, lo.x, from), __shfl_sync(0xffffffffu, lo.y, from), __shfl_sync(0xffffffffu, lo.z, from), __shfl_sync(0xffffffffu, lo.w, from));
      const uint4 h = make_uint4(__shfl_sync(0xffffffffu, hi.x, from), __shfl_sync(0xffffffffu, hi.y, from), __shfl_sync(0xffffffffu, hi.z, from), __shfl_sync(0xffffffffu, hi.w, from));
      if (sub == 0) widen_bounds<T>(lo, hi, l, h);
    }
    if (team == 1) {
      if (sub == 0) store(first, lo, hi);
    } else {
      s_lo[warp][lane] = lo;
      s_hi[warp][lane] = hi;
    }
    if (head == 0 && member == 0) {
      float top = a.logw_new ? -INFINITY : 0.f;
      if (a.logw_new)
        for (int x = lane; x < len; x += 32) top = fmaxf(top, a.logw_new[c0 + first + x]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      if (lane == 0) a.w_max[s_at[first].x] = s_at[first].y ? fmaxf(top, a.w_max[s_at[first].x]) : top;
    }
  }
  if (team == 1) return;
  __syncthreads();
  if (member == 0 && warp / team < n_runs && sub == 0) {
    uint4 lo = s_lo[warp][lane], hi = s_hi[warp][lane];
    for (int w = 1; w < team; ++w) widen_bounds<T>(lo, hi, s_lo[warp + w][lane], s_hi[warp + w][lane]);
    store(s_run[warp / team], lo, hi);
  }
}

}  // namespace

cudaError_t launch_cache_write(const WriteArgs &a, bool bf16, int sm_count, cudaStream_t st) {
  int R = kWriteRows;                                          // smaller blocks until every SM has two CTAs
  while (R > 8 && (a.n_rows + R - 1) / R * a.n_kvh < 2 * sm_count) R /= 2;
  const dim3 grid((unsigned)((a.n_rows + R - 1) / R), (unsigned)a.n_kvh);
  const size_t smem = (size_t)(R + a.page) * sizeof(int2);
  return bf16 ? launch_k(k_cache_write<__nv_bfloat16>, grid, dim3(kWriteThreads), smem, st, true, a, R)
              : launch_k(k_cache_write<float>, grid, dim3(kWriteThreads), smem, st, true, a, R);
}

}  // namespace pact
