// Pages that one new token should attend to (pact_page_select).
//
// For a page with key bounds lo, hi and a query q, the largest q.k over all k with lo <= k <= hi is sum_c (max(q_c, 0) hi_c + min(q_c, 0) lo_c), so
// scale times it, plus the page's largest bias, bounds every logit of the page.  The order of the scores decides what is selected, and with
// thousands of pages two scores that differ by 1e-6 of themselves are common: the order is that of scores formed in double (products of bf16 or
// fp32 numbers are exact there, sums good to 1e-15).  Doubles for all of them cost 20 times what the bytes do (82 us where HBM would need 7), so
// k_page_scores forms the scores in fp32, with a bound of their error, and k_page_pick forms in double only those that the bound leaves in doubt,
// a few per request.
// k_page_scores, bf16: pages (16) by query heads (8) on mma.sync; rows are loaded 16 bytes per lane straight into operands (a dot product does not
// mind the order of its columns, so keys and queries take the same convenient one).  fp32: fused multiply-adds, folded over the lanes.
// k_page_pick: a CTA per request and key head finds the bin of the n-th largest score (histograms of ten bits from the first bit in which the
// scores differ), decides what lies near it in double, and writes the selected places in order from a bit mask.
#include "paged.cuh"

namespace pact {
namespace {

constexpr int kScoreThreads = 128;

// unsigned integers that order like the floats; NaN with minus infinity
__device__ __forceinline__ unsigned long long order_key(double s) {
  if (s != s) s = -INFINITY;
  const unsigned long long b = (unsigned long long)__double_as_longlong(s + 0.0);   // (-0 orders as +0)
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t order_key(float s) {
  const uint32_t b = __float_as_uint(s + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_order_key(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

__device__ __forceinline__ int pages_of(const SelectArgs &a, int b, bool report) {
  const int len = a.length[b];
  const long long room = (long long)a.width * a.page;
  if (len < 0 || len > room) {
    if (report && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    return len < 0 ? 0 : a.width;
  }
  return (int)(((unsigned)len + (unsigned)a.page - 1u) / (unsigned)a.page);
}

// Score in fp32 and a bound of its error: `size` bounds the sum of the absolute products of a head, times |scale|.  512 products at most, each addition off
// by 2^-23 of what it adds up to at most (tensor cores cut off): 2^-14 of `size`; the addition of w by 2^-24 of the result.
// What fp32 cannot hold, infinities and NaN get an unlimited error: they are decided in double.
constexpr float kScoreErr = 1.f / 16384.f;
__device__ __forceinline__ uint2 approx(float best, float size, float w) {
  if (w == -INFINITY) return make_uint2(order_key(-INFINITY), 0u);
  const float s = best + w;
  float err = size * kScoreErr + fabsf(w) * (1.f / 4194304.f);
  if (!(err < 1e30f) || !(fabsf(s) < 1e30f)) {
    err = INFINITY;
    return make_uint2(order_key(0.f), __float_as_uint(err));
  }
  return make_uint2(order_key(s), __float_as_uint(err));
}

__device__ __forceinline__ uint32_t bf2_max(uint32_t x, uint32_t y) {
  const __nv_bfloat162 r = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&x), *reinterpret_cast<__nv_bfloat162 *>(&y));
  return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ uint32_t bf2_min(uint32_t x, uint32_t y) {
  const __nv_bfloat162 r = __hmin2(*reinterpret_cast<__nv_bfloat162 *>(&x), *reinterpret_cast<__nv_bfloat162 *>(&y));
  return *reinterpret_cast<const uint32_t *>(&r);
}
__device__ __forceinline__ void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// bf16.  A warp has 16 pages of one key head; lane 4 r + c reads columns 32 j + 8 c .. + 7 of pages r and r + 8.  ND: blocks of 32 columns.
constexpr int kScorePages = 16 * kScoreThreads / 32;   // pages of a CTA

template <int ND>
__global__ void __launch_bounds__(kScoreThreads) k_page_scores(SelectArgs a) {
  using T = __nv_bfloat16;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.y, b = blockIdx.z, p0 = blockIdx.x * kScorePages + warp * 16;
  const int r = lane / 4, c = lane % 4;
  pdl_wait();
  pdl_trigger();
  const int np = pages_of(a, b, false);
  if (p0 >= np) return;
  int id = -1;                                             // page of lane & 15
  if (lane < 16 && p0 + lane < np) {
    id = a.table[(long long)b * a.width + p0 + lane];
    if (id < 0 || id >= a.n_pages) {
      id = -1;
      if (a.status && head == 0) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    }
  }
  const int id0 = __shfl_sync(0xffffffffu, id, r), id1 = __shfl_sync(0xffffffffu, id, r + 8);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const T *bounds = static_cast<const T *>(a.bounds) + (long long)head * 2 * a.d_h, *Q = static_cast<const T *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  const T *row0 = bounds + (long long)id0 * a.n_kvh * 2 * a.d_h, *row1 = bounds + (long long)id1 * a.n_kvh * 2 * a.d_h;
  const auto ld = [&](const T *p, bool there, int col) { return there && col < a.d_h ? __ldg(reinterpret_cast<const uint4 *>(p + col)) : zero; };
  float best0 = -INFINITY, best1 = -INFINITY, size0 = 0.f, size1 = 0.f;   // over the heads of this lane; pages r and r + 8
  for (int h0 = 0; h0 < a.group; h0 += 8) {
    float s[4] = {0.f, 0.f, 0.f, 0.f}, q1 = 0.f;
    uint32_t top0 = 0, top1 = 0;                           // largest absolute bound of this lane's columns
    constexpr int U = ND < 4 ? ND : 4;                     // blocks of columns in flight
#pragma unroll
    for (int j0 = 0; j0 < ND; j0 += U) {
      uint4 x[U][4], q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int col = (j0 + u) * 32 + c * 8;
        x[u][0] = ld(row0, id0 >= 0, col);
        x[u][1] = ld(row1, id1 >= 0, col);
        x[u][2] = ld(row0 + a.d_h, id0 >= 0, col);
        x[u][3] = ld(row1 + a.d_h, id1 >= 0, col);
        q[u] = ld(Q + (h0 + r) * a.ldQh, h0 + r < a.group, col);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t qw[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
        uint32_t qp[4], qn[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qp[i] = bf2_max(qw[i], 0u);
          qn[i] = bf2_min(qw[i], 0u);
          q1 += fabsf(__uint_as_float(qw[i] << 16)) + fabsf(__uint_as_float(qw[i] & 0xFFFF0000u));
        }
        const uint4 lo0 = x[u][0], lo1 = x[u][1], hi0 = x[u][2], hi1 = x[u][3];
        mma_16x8(s, lo0.x, lo1.x, lo0.y, lo1.y, qn[0], qn[1]);
        mma_16x8(s, lo0.z, lo1.z, lo0.w, lo1.w, qn[2], qn[3]);
        mma_16x8(s, hi0.x, hi1.x, hi0.y, hi1.y, qp[0], qp[1]);
        mma_16x8(s, hi0.z, hi1.z, hi0.w, hi1.w, qp[2], qp[3]);
        // absolute values of bf16 numbers, NaN above infinity, order like the integers
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 v = x[u][i];
          uint32_t &top = i & 1 ? top1 : top0;
          top = __vmaxu2(top, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
        }
      }
    }
    // |q| of head r over the four lanes, the largest over the heads; the largest bound over the four lanes
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      q1 += __shfl_xor_sync(0xffffffffu, q1, o);
      top0 = __vmaxu2(top0, __shfl_xor_sync(0xffffffffu, top0, o));
      top1 = __vmaxu2(top1, __shfl_xor_sync(0xffffffffu, top1, o));
    }
    q1 = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(q1)));   // (not negative, and NaN is above all)
    const float t0 = __uint_as_float(max(top0 << 16, top0 & 0xFFFF0000u)), t1 = __uint_as_float(max(top1 << 16, top1 & 0xFFFF0000u));
    // fmaxf drops a NaN, so the larger one is taken as integers, which have it above all
    size0 = __uint_as_float(max(__float_as_uint(size0), __float_as_uint(q1 * t0) & 0x7fffffffu));
    size1 = __uint_as_float(max(__float_as_uint(size1), __float_as_uint(q1 * t1) & 0x7fffffffu));
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (h0 + 2 * c + i < a.group) {
        best0 = fmaxf(best0, s[i] * a.scale);
        best1 = fmaxf(best1, s[2 + i] * a.scale);
      }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    best0 = fmaxf(best0, __shfl_xor_sync(0xffffffffu, best0, o));
    best1 = fmaxf(best1, __shfl_xor_sync(0xffffffffu, best1, o));
  }
  if (c < 2) {                                             // lane 4 r writes page r, lane 4 r + 1 page r + 8
    const int p = p0 + r + 8 * c, at = c ? id1 : id0;
    if (p < np)
      a.approx[((long long)b * a.n_kvh + head) * a.width + p] =
          approx(c ? best1 : best0, fabsf(a.scale) * (c ? size1 : size0), at < 0 ? -INFINITY : a.w_max[at]);
  }
}

// fp32.  A warp has eight pages; a lane has DL columns of them and takes four query heads at a time.
constexpr int kHeadsAtOnce = 4;

// Sums of x[0..N) over the lanes: value i ends up in x[0] of the lanes whose bits from `bit` down spell i (31 exchanges for 32 sums, where 32
// sums by themselves would take 160).
template <int N> __device__ __forceinline__ void fold(float (&x)[N], int lane, int bit) {
  if constexpr (N > 1) {
    float y[N / 2];
    const bool up = lane & bit;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) y[i] = (up ? x[N / 2 + i] : x[i]) + __shfl_xor_sync(0xffffffffu, up ? x[i] : x[N / 2 + i], bit);
    fold<N / 2>(y, lane, bit >> 1);
    x[0] = y[0];
  }
}

template <int DL>
__global__ void __launch_bounds__(kScoreThreads) k_page_scores_f32(SelectArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int head = blockIdx.y, b = blockIdx.z, p0 = (blockIdx.x * (kScoreThreads / 32) + warp) * 8;
  const int c = lane * DL;
  const bool mine = c < a.d_h;                             // (d_h is a multiple of 4)
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
  const float *bounds = static_cast<const float *>(a.bounds), *Q = static_cast<const float *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  const auto load = [&](const float *p, bool there, float (&x)[DL]) {
#pragma unroll
    for (int i = 0; i < DL; i += 2) {
      const float2 v = there ? __ldg(reinterpret_cast<const float2 *>(p + i)) : make_float2(0.f, 0.f);
      x[i] = v.x; x[i + 1] = v.y;
    }
  };
  float lo[8][DL], hi[8][DL];
  uint32_t top[8];                                         // largest absolute bound of a page, as bits (NaN above all)
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int at = __shfl_sync(0xffffffffu, id, p);
    const float *row = bounds + ((long long)at * a.n_kvh + head) * 2 * a.d_h + c;
    load(row, mine && at >= 0, lo[p]);
    load(row + a.d_h, mine && at >= 0, hi[p]);
    top[p] = 0;
#pragma unroll
    for (int e = 0; e < DL; ++e) top[p] = max(top[p], max(__float_as_uint(lo[p][e]) & 0x7fffffffu, __float_as_uint(hi[p][e]) & 0x7fffffffu));
  }
  float best = -INFINITY;                                  // of page lane >> 2, over the heads of this lane
  uint32_t q1 = 0;                                         // largest |q| of a head
  for (int h0 = 0; h0 < a.group; h0 += kHeadsAtOnce) {
    float sum[8 * kHeadsAtOnce];
#pragma unroll
    for (int h = 0; h < kHeadsAtOnce; ++h) {
      float q[DL], n = 0.f;
      load(Q + (h0 + h) * a.ldQh + c, mine && h0 + h < a.group, q);
#pragma unroll
      for (int e = 0; e < DL; ++e) n += fabsf(q[e]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
      q1 = max(q1, __float_as_uint(n) & 0x7fffffffu);
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < DL; ++e) s = fmaf(fmaxf(q[e], 0.f), hi[p][e], fmaf(fminf(q[e], 0.f), lo[p][e], s));
        sum[p * kHeadsAtOnce + h] = s;
      }
    }
    fold<8 * kHeadsAtOnce>(sum, lane, 16);
    if (h0 + (lane & (kHeadsAtOnce - 1)) < a.group) best = fmaxf(best, sum[0] * a.scale);
  }
#pragma unroll
  for (int o = 1; o < kHeadsAtOnce; o <<= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
  uint32_t my_top = 0;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const uint32_t t = __reduce_max_sync(0xffffffffu, top[p]);
    if (p == lane >> 2) my_top = t;
  }
  const int at = __shfl_sync(0xffffffffu, id, lane >> 2), p = p0 + (lane >> 2);
  if ((lane & 3) == 0 && p < np)
    a.approx[((long long)b * a.n_kvh + head) * a.width + p] =
        approx(best, fabsf(a.scale) * __uint_as_float(q1) * __uint_as_float(my_top), at < 0 ? -INFINITY : a.w_max[at]);
}

// The score of page p in double, by a warp.
template <typename T> __device__ double exact_score(const SelectArgs &a, int b, int head, int p) {
  const int lane = threadIdx.x & 31, id = a.table[(long long)b * a.width + p];
  if (id < 0 || id >= a.n_pages) return -INFINITY;
  const T *row = static_cast<const T *>(a.bounds) + ((long long)id * a.n_kvh + head) * 2 * a.d_h, *Q = static_cast<const T *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  double best = -INFINITY;
  for (int h = 0; h < a.group; ++h) {
    double s = 0.0;
    for (int c = lane; c < a.d_h; c += 32) {
      const float q = (float)Q[h * a.ldQh + c];
      const double qp = q > 0.f ? q : q == q ? 0.f : q, qn = q < 0.f ? q : 0.f;
      s = fma(qp, (double)(float)row[a.d_h + c], fma(qn, (double)(float)row[c], s));
    }
    best = fmax(best, warp_sum(s) * (double)a.scale);      // (drops a NaN)
  }
  return best + (double)a.w_max[id];
}

constexpr int kPickThreads = 256;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kPickBits = 10;
constexpr int kPickKeys = 8192;            // scores of a request and head that are kept in shared memory
constexpr int kPickDoubt = 256;            // most scores in doubt that are ranked by comparing them with one another

struct PickShared {
  uint32_t mask[kMaxSelectPages / 32];
  int hist[1 << kPickBits];
  unsigned long long cand[kPickDoubt];
  int cand_at[kPickDoubt];
  unsigned long long w_max[kPickWarps], w_min[kPickWarps];
  uint32_t w_err[kPickWarps];
  int w_sum[kPickWarps];
  int bin, above, in_bin, n_cand, n_sure;
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
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) {
    if (w == warp) before = all;
    all += w_sum[w];
  }
  *total = all;
  return before + x - v;
}

// Where the need-th largest of keys [first, end) lies: keys whose bits from `shift` up are larger than `prefix` come before it, those whose bits are
// smaller behind it, and `need` of the `agree` keys that agree with `prefix` are to be found among them.  Stops once no more than `enough` agree, or all or
// none of those that agree are needed.
template <typename K> struct Cut {
  K prefix;
  int shift, need, agree;
  static __device__ __forceinline__ K high(K k, int sh) { return sh >= (int)sizeof(K) * 8 ? K(0) : k >> sh; }
};
template <typename K, typename F>
__device__ __forceinline__ Cut<K> find_cut(PickShared &s, F key, int first, int end, int need, K kmax, K kmin, int enough) {
  const int tid = threadIdx.x;
  Cut<K> cut;
  cut.shift = kmax <= kmin ? 0 : sizeof(K) == 8 ? 64 - __clzll((long long)(kmax ^ kmin)) : 32 - __clz((int)(kmax ^ kmin));
  cut.prefix = Cut<K>::high(kmax, cut.shift);
  cut.need = need;
  cut.agree = end - first;
  while (cut.need > 0 && cut.need < cut.agree && cut.agree > enough && cut.shift > 0) {
    const int lower = max(0, cut.shift - kPickBits), bins = 1 << (cut.shift - lower);
    for (int i = tid; i < bins; i += kPickThreads) s.hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < end; i += kPickThreads) {
      const K k = key(i);
      if (Cut<K>::high(k, cut.shift) == cut.prefix) atomicAdd(&s.hist[(int)(k >> lower) & (bins - 1)], 1);
    }
    __syncthreads();
    constexpr int PER = (1 << kPickBits) / kPickThreads;   // bins of a thread, the largest first
    int n[PER], sum = 0, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = bins - 1 - (tid * PER + i);
      n[i] = at >= 0 ? s.hist[at] : 0;
      sum += n[i];
    }
    int before = scan_block(sum, s.w_sum, &all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (before < cut.need && before + n[i] >= cut.need) {
        s.bin = bins - 1 - (tid * PER + i);
        s.above = before;
        s.in_bin = n[i];
      }
      before += n[i];
    }
    __syncthreads();
    cut.prefix = (cut.shift == (int)sizeof(K) * 8 ? K(0) : K(cut.prefix << (cut.shift - lower))) | (K)s.bin;
    cut.need -= s.above;
    cut.agree = s.in_bin;
    cut.shift = lower;
    __syncthreads();
  }
  return cut;
}

template <typename T>
__global__ void __launch_bounds__(kPickThreads) k_page_pick(SelectArgs a) {
  extern __shared__ uint32_t s_keys[];
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
  const int need = a.n_select - a.n_first - a.n_last;
  const long long row = ((long long)b * a.n_kvh + head) * a.width;
  const uint2 *apx = a.approx + row;
  const bool kept = np <= kPickKeys;
  uint32_t kmax = 0, kmin = ~0u, err = 0;
  for (int i = first + tid; i < end; i += kPickThreads) {
    const uint2 k = apx[i];
    if (kept) s_keys[i] = k.x;
    kmax = max(kmax, k.x);
    kmin = min(kmin, k.x);
    err = max(err, k.y);                                   // (not negative: orders like the bits)
  }
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  err = __reduce_max_sync(0xffffffffu, err);
  if (lane == 0) {
    s.w_max[warp] = kmax;
    s.w_min[warp] = kmin;
    s.w_err[warp] = err;
  }
  if (tid == 0) s.n_cand = s.n_sure = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPickWarps; ++w) {
    kmax = max(kmax, (uint32_t)s.w_max[w]);
    kmin = min(kmin, (uint32_t)s.w_min[w]);
    err = max(err, s.w_err[w]);
  }
  const auto key = [&](int i) { return kept ? s_keys[i] : apx[i].x; };
  const int words = (np + 31) / 32;
  // Of two scores whose fp32 values differ by more than twice the largest error the larger one is the larger one in double as well.  [low, high]: fp32
  // values that may lie on either side of the need-th largest; `sure` ones are larger.
  uint32_t low = 0, high = ~0u;
  if (err < 0x7f800000u) {
    const Cut<uint32_t> cut = find_cut<uint32_t>(s, key, first, end, need, kmax, kmin, 1);
    // the need-th largest agrees with the prefix
    const uint32_t least = cut.shift >= 32 ? 0u : cut.prefix << cut.shift, most = cut.shift >= 32 ? ~0u : least | ((1u << cut.shift) - 1u);
    const float e2 = 2.f * __uint_as_float(err);
    low = order_key(__fsub_rd(from_order_key(max(least, kmin)), e2));
    high = order_key(__fadd_ru(from_order_key(min(most, kmax)), e2));
  }
  for (int w = warp; w < words; w += kPickWarps) {
    const int i = w * 32 + lane;
    const bool in = i >= first && i < end;
    const uint32_t k = in ? key(i) : 0u;
    const bool sure = in && need > 0 && k > high, doubt = in && need > 0 && k >= low && k <= high;
    const uint32_t m = __ballot_sync(0xffffffffu, sure || (!in && i < np)), ms = __ballot_sync(0xffffffffu, sure);
    if (lane == 0) {
      s.mask[w] = m;
      if (ms) atomicAdd(&s.n_sure, __popc(ms));
    }
    if (doubt) {
      const int at = atomicAdd(&s.n_cand, 1);              // (their order changes nothing)
      if (at < kPickDoubt) s.cand_at[at] = i;
    }
  }
  __syncthreads();
  const int doubts = s.n_cand, more = need - s.n_sure;     // `more` of the ones in doubt are selected: 0 <= more <= doubts
  if (more > 0 && more == doubts && doubts <= kPickDoubt) {
    for (int j = tid; j < doubts; j += kPickThreads) atomicOr(&s.mask[s.cand_at[j] >> 5], 1u << (s.cand_at[j] & 31));
  } else if (more > 0 && doubts <= kPickDoubt) {
    for (int j = warp; j < doubts; j += kPickWarps) {
      const double x = exact_score<T>(a, b, head, s.cand_at[j]);
      if (lane == 0) s.cand[j] = order_key(x);
    }
    __syncthreads();
    for (int j = tid; j < doubts; j += kPickThreads) {
      const unsigned long long k = s.cand[j];
      const int at = s.cand_at[j];
      int before = 0;
      for (int i = 0; i < doubts; ++i) before += s.cand[i] > k || (s.cand[i] == k && s.cand_at[i] < at);
      if (before < more) atomicOr(&s.mask[at >> 5], 1u << (at & 31));
    }
  } else if (more > 0) {                                   // many scores (nearly) equal, or beyond fp32: all that are in doubt in double
    unsigned long long *exact = a.keys + row;              // 0 for what is not in doubt: below every score
    unsigned long long xmax = 0, xmin = ~0ull;
    for (int i = first + warp; i < end; i += kPickWarps) {
      const uint32_t k = key(i);
      unsigned long long x = 0;
      if (k >= low && k <= high) {
        x = order_key(exact_score<T>(a, b, head, i));
        xmin = min(xmin, x);
      }
      xmax = max(xmax, x);
      if (lane == 0) exact[i] = x;
    }
    if (lane == 0) {
      s.w_max[warp] = xmax;
      s.w_min[warp] = doubts < end - first ? 0ull : xmin;
    }
    __syncthreads();
    for (int w = 0; w < kPickWarps; ++w) {
      xmax = max(xmax, s.w_max[w]);
      xmin = min(xmin, s.w_min[w]);
    }
    const auto ekey = [&](int i) { return exact[i]; };
    const Cut<unsigned long long> cut = find_cut<unsigned long long>(s, ekey, first, end, more, xmax, xmin, 0);
    int taken = 0;                                         // equal scores in the words before this round's
    for (int w0 = 0; w0 < words; w0 += kPickWarps) {
      const int w = w0 + warp, i = w * 32 + lane;
      const unsigned long long k = i >= first && i < end ? exact[i] : 0ull, h = Cut<unsigned long long>::high(k, cut.shift);
      const bool same = k != 0 && h == cut.prefix;
      const uint32_t eq = __ballot_sync(0xffffffffu, same), gt = __ballot_sync(0xffffffffu, k != 0 && h > cut.prefix);
      if (lane == 0) s.w_sum[warp] = __popc(eq);
      __syncthreads();
      int before = taken, all = 0;
      for (int v = 0; v < kPickWarps; ++v) {
        if (v < warp) before += s.w_sum[v];
        all += s.w_sum[v];
      }
      taken += all;
      __syncthreads();
      const uint32_t m = gt | __ballot_sync(0xffffffffu, same && before + __popc(eq & ((1u << lane) - 1u)) < cut.need);
      if (lane == 0 && w < words) s.mask[w] |= m;
    }
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
  const cudaError_t e = cudaFuncSetAttribute(k_page_pick<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kPickKeys * sizeof(uint32_t)));
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(k_page_pick<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kPickKeys * sizeof(uint32_t)));
}

cudaError_t launch_page_select(const SelectArgs &a, bool bf16, cudaStream_t st, int *launches) {
  *launches = 1;
  if (a.width > a.n_select) {                              // otherwise all pages are selected whatever the lengths
    const int pages = bf16 ? kScorePages : kScorePages / 2;
    const dim3 grid((unsigned)((a.width + pages - 1) / pages), (unsigned)a.n_kvh, (unsigned)a.B);
    void (*kernel)(SelectArgs) = bf16 ? (a.d_h <= 64 ? k_page_scores<2> : a.d_h <= 128 ? k_page_scores<4> : k_page_scores<8>)
                                      : (a.d_h <= 64 ? k_page_scores_f32<2> : k_page_scores_f32<4>);
    const cudaError_t e = launch_k(kernel, grid, dim3(kScoreThreads), 0, st, true, a);
    if (e != cudaSuccess) return e;
    *launches = 2;
  }
  const int keys = a.width <= a.n_select ? 0 : a.width < kPickKeys ? a.width : kPickKeys;
  return launch_k(bf16 ? k_page_pick<__nv_bfloat16> : k_page_pick<float>, dim3((unsigned)a.n_kvh, (unsigned)a.B), dim3(kPickThreads), (size_t)keys * sizeof(uint32_t), st, true, a);
}

}  // namespace pact
