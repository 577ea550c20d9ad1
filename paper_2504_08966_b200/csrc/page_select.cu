// Pages that one new token should attend to (pact_page_select).
//
// k_page_scores: for a page with key bounds lo, hi and a query q, the largest q.k over all k with lo <= k <= hi is
// sum_c (max(q_c, 0) hi_c + min(q_c, 0) lo_c), so scale times it, plus the page's largest bias, bounds every logit of the page.  The order of
// the scores decides what is selected, and with thousands of pages two scores that differ by 1e-6 of themselves are common.  So they
// are formed in double: products of bf16 or fp32 numbers are exact there and the sums good to 1e-15.
// A lane keeps DL coordinates of eight pages and takes four query heads at a time; the 32 sums over the lanes are then folded together (31
// exchanges in all, where 32 sums by themselves would take 160).
// k_page_pick: a CTA per request and key head finds the n-th largest key (histograms of ten bits from the first bit in which the keys
// differ, then ranks among the keys of one bin) and writes the selected places in order from a bit mask.
#include "paged.cuh"

namespace pact {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 64;            // pages of a CTA, eight of a warp
constexpr int kHeadsAtOnce = 4;

// unsigned integers that order like the doubles; NaN with minus infinity
__device__ __forceinline__ unsigned long long order_key(double s) {
  if (s != s) s = -INFINITY;
  const unsigned long long b = (unsigned long long)__double_as_longlong(s + 0.0);   // (-0 orders as +0)
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

__device__ __forceinline__ double shfl_xor_f64(double v, int o) {
  return __hiloint2double(__shfl_xor_sync(0xffffffffu, __double2hiint(v), o), __shfl_xor_sync(0xffffffffu, __double2loint(v), o));
}

// Sums of x[0..N) over the lanes: value i ends up in x[0] of the lanes whose bits from `bit` down spell i.
template <int N> __device__ __forceinline__ void fold(double (&x)[N], int lane, int bit) {
  if constexpr (N > 1) {
    double y[N / 2];
    const bool up = lane & bit;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const double keep = up ? x[N / 2 + i] : x[i], give = up ? x[i] : x[N / 2 + i];
      y[i] = keep + shfl_xor_f64(give, bit);
    }
    fold<N / 2>(y, lane, bit >> 1);
    x[0] = y[0];
  }
}

template <typename T, int DL> struct Lane;   // DL consecutive elements of a row
template <int DL> struct Lane<__nv_bfloat16, DL> {
  static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&x)[DL]) {
    uint32_t w[DL / 2];
    if constexpr (DL == 2) w[0] = __ldg(reinterpret_cast<const uint32_t *>(p));
    else if constexpr (DL == 4) {
      const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
      w[0] = v.x; w[1] = v.y;
    } else {
      const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
#pragma unroll
    for (int i = 0; i < DL / 2; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
};
template <int DL> struct Lane<float, DL> {
  static __device__ __forceinline__ void load(const float *p, float (&x)[DL]) {
#pragma unroll
    for (int i = 0; i < DL; i += 2) {
      const float2 v = __ldg(reinterpret_cast<const float2 *>(p + i));
      x[i] = v.x; x[i + 1] = v.y;
    }
  }
};

__device__ __forceinline__ int pages_of(const SelectArgs &a, int b, bool report) {
  const int len = a.length[b];
  const long long room = (long long)a.width * a.page;
  if (len < 0 || len > room) {
    if (report && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    return len < 0 ? 0 : a.width;
  }
  return (int)(((unsigned)len + (unsigned)a.page - 1u) / (unsigned)a.page);
}

template <typename T, int DL>
__global__ void __launch_bounds__(kScoreThreads) k_page_scores(SelectArgs a) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = blockIdx.y, b = blockIdx.z, p0 = blockIdx.x * kScorePages + warp * 8;
  const int c = lane * DL;
  const bool mine = c < a.d_h;                             // (d_h is a multiple of DL)
  pdl_wait();
  pdl_trigger();
  const int np = pages_of(a, b, false);
  if (p0 >= np) return;
  int id = -1;                                             // page of lane & 7
  if (lane < 8 && p0 + lane < np) {
    id = a.table[(long long)b * a.width + p0 + lane];
    if (id < 0 || id >= a.n_pages) {
      id = -1;
      if (a.status && head == 0) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    }
  }
  const T *bounds = static_cast<const T *>(a.bounds), *Q = static_cast<const T *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  float lo[8][DL], hi[8][DL];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int at = __shfl_sync(0xffffffffu, id, p);
    if (mine && at >= 0) {
      const T *row = bounds + ((long long)at * a.n_kvh + head) * 2 * a.d_h + c;
      Lane<T, DL>::load(row, lo[p]);
      Lane<T, DL>::load(row + a.d_h, hi[p]);
    } else {
#pragma unroll
      for (int e = 0; e < DL; ++e) lo[p][e] = hi[p][e] = 0.f;
    }
  }
  double best = -INFINITY;                                 // of page lane >> 2, over the heads of this lane
  for (int h0 = 0; h0 < a.group; h0 += kHeadsAtOnce) {
    double sum[8 * kHeadsAtOnce];
#pragma unroll
    for (int h = 0; h < kHeadsAtOnce; ++h) {
      float q[DL];
#pragma unroll
      for (int e = 0; e < DL; ++e) q[e] = 0.f;
      if (mine && h0 + h < a.group) Lane<T, DL>::load(Q + (h0 + h) * a.ldQh + c, q);
      double qp[DL], qn[DL];
#pragma unroll
      for (int e = 0; e < DL; ++e) {
        qp[e] = q[e] > 0.f ? q[e] : q[e] == q[e] ? 0.f : q[e];
        qn[e] = q[e] < 0.f ? q[e] : 0.f;
      }
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < DL; ++e) s = fma(qp[e], (double)hi[p][e], fma(qn[e], (double)lo[p][e], s));
        sum[p * kHeadsAtOnce + h] = s;
      }
    }
    fold<8 * kHeadsAtOnce>(sum, lane, 16);
    const double s = sum[0] * (double)a.scale;
    if (h0 + (lane & (kHeadsAtOnce - 1)) < a.group) best = fmax(best, s);   // (drops a NaN)
  }
#pragma unroll
  for (int o = 1; o < kHeadsAtOnce; o <<= 1) best = fmax(best, shfl_xor_f64(best, o));
  const int at = __shfl_sync(0xffffffffu, id, lane >> 2);
  const int p = p0 + (lane >> 2);
  if ((lane & 3) == 0 && p < np) {
    const double s = at < 0 ? -INFINITY : best + (double)a.w_max[at];
    a.keys[((long long)b * a.n_kvh + head) * a.width + p] = order_key(s);
  }
}

constexpr int kPickThreads = 512;
constexpr int kPickBits = 10;
constexpr int kPickKeys = 8192;            // keys of a request and head that are kept in shared memory
constexpr int kPickRank = kPickThreads;    // keys of one bin that are ranked by comparing all of them

struct PickShared {
  uint32_t mask[kMaxSelectPages / 32];
  int hist[1 << kPickBits];
  unsigned long long cand[kPickRank];
  int cand_at[kPickRank];
  unsigned long long w_max[kPickThreads / 32], w_min[kPickThreads / 32];
  int w_sum[kPickThreads / 32];
  int bin, above, in_bin, n_cand;
};

// exclusive prefix sum over the CTA's threads; *total: over all of them
__device__ __forceinline__ int scan_block(int v, int *w_sum, int *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) w_sum[warp] = x;
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kPickThreads / 32; ++w) {
    if (w == warp) before = all;
    all += w_sum[w];
  }
  *total = all;
  return before + x - v;
}

__global__ void __launch_bounds__(kPickThreads) k_page_pick(SelectArgs a) {
  extern __shared__ unsigned long long s_keys[];
  __shared__ PickShared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = blockIdx.x, b = blockIdx.y;
  int32_t *out = a.selected + ((long long)b * a.n_kvh + head) * a.n_select;
  pdl_wait();
  pdl_trigger();
  const int np = pages_of(a, b, tid == 0 && head == 0);
  if (np <= a.n_select) {                                  // all of them
    for (int i = tid; i < a.n_select; i += kPickThreads) out[i] = i < np ? i : -1;
    return;
  }
  const int first = a.n_first, end = np - a.n_last;        // the scores decide between these (n_first + n_last <= n_select < np)
  int need = a.n_select - a.n_first - a.n_last;
  const unsigned long long *keys = a.keys + ((long long)b * a.n_kvh + head) * a.width;
  const bool kept = np <= kPickKeys;
  unsigned long long kmax = 0, kmin = ~0ull;
  for (int i = first + tid; i < end; i += kPickThreads) {
    const unsigned long long k = keys[i];
    if (kept) s_keys[i] = k;
    kmax = max(kmax, k);
    kmin = min(kmin, k);
  }
  if (kept) keys = s_keys;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    kmax = max(kmax, __shfl_xor_sync(0xffffffffu, kmax, o));
    kmin = min(kmin, __shfl_xor_sync(0xffffffffu, kmin, o));
  }
  if (lane == 0) {
    s.w_max[warp] = kmax;
    s.w_min[warp] = kmin;
  }
  if (tid == 0) s.n_cand = 0;
  __syncthreads();
  for (int w = 0; w < kPickThreads / 32; ++w) {
    kmax = max(kmax, s.w_max[w]);
    kmin = min(kmin, s.w_min[w]);
  }
  // Keys whose bits from `shift` up are larger than `prefix` are selected, those whose bits are smaller are not; `need` of the `agree` keys
  // that agree with it are still to be found.
  int shift = kmax <= kmin ? 0 : 64 - __clzll((long long)(kmax ^ kmin));
  const auto high = [](unsigned long long k, int sh) { return sh == 64 ? 0ull : k >> sh; };
  unsigned long long prefix = high(kmax, shift);
  int agree = end - first;
  while (need > 0 && need < agree && agree > kPickRank && shift > 0) {
    const int lower = max(0, shift - kPickBits), bins = 1 << (shift - lower);
    for (int i = tid; i < bins; i += kPickThreads) s.hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < end; i += kPickThreads)
      if (high(keys[i], shift) == prefix) atomicAdd(&s.hist[(int)(keys[i] >> lower) & (bins - 1)], 1);
    __syncthreads();
    // two bins per thread, the largest first
    const int i0 = bins - 1 - 2 * tid, n0 = i0 >= 0 ? s.hist[i0] : 0, n1 = i0 >= 1 ? s.hist[i0 - 1] : 0;
    int all;
    const int before = scan_block(n0 + n1, s.w_sum, &all);
    if (before < need && before + n0 >= need) { s.bin = i0; s.above = before; s.in_bin = n0; }
    else if (before + n0 < need && before + n0 + n1 >= need) { s.bin = i0 - 1; s.above = before + n0; s.in_bin = n1; }
    __syncthreads();
    prefix = (shift == 64 ? 0ull : prefix << (shift - lower)) | (unsigned long long)s.bin;
    need -= s.above;
    agree = s.in_bin;
    shift = lower;
    __syncthreads();
  }
  // the mask: the first and last pages, all larger keys, and of those that agree all, none, the highest ranks, or (equal keys) the lowest places
  const int words = (np + 31) / 32;
  const bool some = need > 0 && need < agree, rank = some && agree <= kPickRank;
  int taken = 0;                                           // equal keys in the words before this round's
  for (int w0 = 0; w0 < words; w0 += kPickThreads / 32) {
    const int w = w0 + warp, i = w * 32 + lane;
    const bool in = i >= first && i < end;
    const unsigned long long k = in ? keys[i] : 0ull, h = high(k, shift);
    const bool more = in ? h > prefix : i < np, same = in && h == prefix;
    uint32_t m = __ballot_sync(0xffffffffu, more || (same && need > 0 && need >= agree));
    const uint32_t eq = __ballot_sync(0xffffffffu, same);
    if (rank && same) {
      const int at = atomicAdd(&s.n_cand, 1);              // (ranks do not depend on the order here)
      s.cand[at] = k;
      s.cand_at[at] = i;
    }
    if (some && !rank) {                                   // more equal keys than are ranked
      if (lane == 0) s.w_sum[warp] = __popc(eq);
      __syncthreads();
      int before = taken, all = 0;
      for (int v = 0; v < kPickThreads / 32; ++v) {
        if (v < warp) before += s.w_sum[v];
        all += s.w_sum[v];
      }
      taken += all;
      __syncthreads();
      m |= __ballot_sync(0xffffffffu, same && before + __popc(eq & ((1u << lane) - 1u)) < need);
    }
    if (lane == 0 && w < words) s.mask[w] = m;
  }
  __syncthreads();
  if (rank && tid < agree) {
    const unsigned long long k = s.cand[tid];
    const int at = s.cand_at[tid];
    int r = 0;
    for (int j = 0; j < agree; ++j) r += s.cand[j] > k || (s.cand[j] == k && s.cand_at[j] < at);
    if (r < need) atomicOr(&s.mask[at >> 5], 1u << (at & 31));
  }
  __syncthreads();
  int base = 0;
  for (int w0 = 0; w0 < words; w0 += kPickThreads) {
    const int w = w0 + tid;
    uint32_t m = w < words ? s.mask[w] : 0u;
    int all;
    int at = base + scan_block(__popc(m), s.w_sum, &all);
    base += all;
    for (; m; m &= m - 1) out[at++] = w * 32 + __ffs(m) - 1;
  }
}

}  // namespace

cudaError_t select_pages_configure() {
  return cudaFuncSetAttribute(k_page_pick, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kPickKeys * sizeof(unsigned long long)));
}

cudaError_t launch_page_select(const SelectArgs &a, bool bf16, cudaStream_t st, int *launches) {
  *launches = 1;
  if (a.width > a.n_select) {                              // otherwise all pages are selected whatever the lengths
    const dim3 grid((unsigned)((a.width + kScorePages - 1) / kScorePages), (unsigned)a.n_kvh, (unsigned)a.B);
    void (*kernel)(SelectArgs) = bf16 ? (a.d_h <= 64 ? k_page_scores<__nv_bfloat16, 2> : a.d_h <= 128 ? k_page_scores<__nv_bfloat16, 4> : k_page_scores<__nv_bfloat16, 8>)
                                      : (a.d_h <= 64 ? k_page_scores<float, 2> : k_page_scores<float, 4>);
    const cudaError_t e = launch_k(kernel, grid, dim3(kScoreThreads), 0, st, true, a);
    if (e != cudaSuccess) return e;
    *launches = 2;
  }
  const int keys = a.width <= a.n_select ? 0 : a.width < kPickKeys ? a.width : kPickKeys;
  return launch_k(k_page_pick, dim3((unsigned)a.n_kvh, (unsigned)a.B), dim3(kPickThreads), (size_t)keys * sizeof(unsigned long long), st, true, a);
}

}  // namespace pact
