// Pages that one new token should attend to (pact_page_select).
//
// For a page with key bounds lo, hi and a query q, the largest q.k over all k with lo <= k <= hi is the sum of q_c hi_c where q_c > 0 and q_c lo_c where q_c < 0, so
// scale times it, plus the page's largest bias, bounds every logit of the page.  (As max(q_c, 0) hi_c + min(q_c, 0) lo_c in the fp32 scores: the same but for
// infinite bounds, where 0 times infinity has no place in the sum; those scores are formed again in double.)  The order of the scores decides what is selected, and with
// thousands of pages two scores that differ by 1e-6 of themselves are common: the order is that of scores formed in double (products of bf16 or
// fp32 numbers are exact there, sums good to 1e-15).  Doubles for all of them cost 12 times what the bytes do (82 us where HBM would need 7), so
// the scores are formed in fp32 with a bound of their error, and in double only those that the bound leaves in doubt, a few per request.
//
// One kernel, a cluster of CTAs per request and key head (one CTA where there are enough of them): all CTAs score pages, the first one has the scores in
// its shared memory and selects.  (As two kernels: 22.2 us against 18.3 for 32 requests of 16384 rows, 16.5 against 14.6 for two of 131072; now 16.6 and
// 9.2, of which the scores take 7 and 3.7 and the selection, a chain of dependent steps in one CTA, 5.)
// Scores, bf16: pages (16) by query heads (8) on mma.sync; rows are loaded 16 bytes per lane straight into operands (a dot product does not
// mind the order of its columns, so keys and queries take the same convenient one).  fp32: fused multiply-adds, folded over the lanes.
// Selection: the bin of the n-th largest score (histograms of ten bits from the first bit in which the scores differ), what lies near it in
// double, and the selected places in order from a bit mask.
#include "paged.cuh"
#include "tma.cuh"

namespace pact {
namespace {

constexpr int kSelectThreads = 256;
constexpr int kSelectWarps = kSelectThreads / 32;
constexpr int kSelectPages = 16 * kSelectWarps;   // pages that a CTA scores at once
constexpr int kMaxSelectCluster = 16;

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

// A page's score in fp32 as an integer, and a bound of its error.  `size` is the sum of the absolute products, the largest over the heads, times |scale|;
// rel: what the additions are off by, as a part of it; the addition of w is off by 2^-24 of the result.
// What fp32 cannot hold is marked: the first CTA forms these scores in double.  (An unlimited error for all scores of the request instead, which decides every one of them in
// double: one infinite key among 4096 pages 1.7 ms against 18 us, among 65536 pages 28 ms
// against 0.26.)
// Below the normal numbers errors are no part of the value: sums of products are off by a few hundred times 2^-126 at most (where tensor cores drop them), which is
// less than any rel of kTiny, and everything else by steps of 2^-149 (kLast: seven of them).
constexpr float kTiny = 1e-28f, kLast = 1e-44f;
constexpr uint32_t kMarked = ~0u;              // in place of a score
constexpr uint32_t kAnyMarked = 0x80000000u;   // beside the largest error
constexpr uint32_t kUnlimited = 0x7f800000u;   // an error
__device__ __forceinline__ uint32_t approx(float best, float size, float rel, float w, uint32_t &err) {
  if (w == -INFINITY) return order_key(-INFINITY);
  const float s = best + w, e = size * rel + (size + fabsf(w)) * (1.f / 4194304.f) + kLast;
  if (!(e < 1e30f) || !(fabsf(s) < 1e30f)) {
    err |= kAnyMarked;
    return kMarked;
  }
  err = max(err & ~kAnyMarked, __float_as_uint(e)) | (err & kAnyMarked);
  return order_key(s);
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

// bf16: scores of pages p0 .. p0 + 15 by a warp, into put(page, score as an integer); id: page of this lane, of the first 16 (fp32: 8).  Lane 4 r + c reads columns 32 j + 8 c .. + 7 of pages r and r + 8.
// ND: blocks of 32 columns.  Error of a sum: an instruction adds 17 numbers, which tensor cores align to the largest and cut off, each off by 2^-23 of the absolute sum at most; four
// of them make the sum of a block, and the sums of the blocks are added with rounding.  (All in one chain: the same time, but every instruction off by a part of
// the whole, four times as many scores in doubt; every instruction's result added by itself: 2 to 4 us more.)
template <int ND, typename F> __device__ __forceinline__ void score_pages(const SelectArgs &a, int b, int head, int p0, int id, int np, uint32_t &err, F put) {
  using T = __nv_bfloat16;
  constexpr float kRel = (4 * 17 + ND) / 8388608.f;
  const int lane = threadIdx.x & 31, r = lane / 4, c = lane % 4;
  const int id0 = __shfl_sync(0xffffffffu, id, r), id1 = __shfl_sync(0xffffffffu, id, r + 8);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const T *bounds = static_cast<const T *>(a.bounds) + (long long)head * 2 * a.d_h, *Q = static_cast<const T *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  const T *row0 = bounds + (long long)id0 * a.n_kvh * 2 * a.d_h, *row1 = bounds + (long long)id1 * a.n_kvh * 2 * a.d_h;
  const float w = c < 2 && (c ? id1 : id0) >= 0 ? __ldg(a.w_max + (c ? id1 : id0)) : -INFINITY;
  const auto ld = [&](const T *p, bool there, int col) { return there && col < a.d_h ? __ldg(reinterpret_cast<const uint4 *>(p + col)) : zero; };
  float best0 = -INFINITY, best1 = -INFINITY;              // over the heads of this lane; pages r and r + 8
  uint32_t size0 = 0, size1 = 0;                           // (as integers: not negative, and NaN is above all)
  for (int h0 = 0; h0 < a.group; h0 += 8) {
    float s[4] = {0.f, 0.f, 0.f, 0.f}, t[4] = {0.f, 0.f, 0.f, 0.f};
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
        const uint32_t lo0[4] = {x[u][0].x, x[u][0].y, x[u][0].z, x[u][0].w}, lo1[4] = {x[u][1].x, x[u][1].y, x[u][1].z, x[u][1].w};
        const uint32_t hi0[4] = {x[u][2].x, x[u][2].y, x[u][2].z, x[u][2].w}, hi1[4] = {x[u][3].x, x[u][3].y, x[u][3].z, x[u][3].w};
        uint32_t m0[4], m1[4];                             // absolute values of bf16 numbers order like the integers, NaN above infinity
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m0[i] = __vmaxu2(lo0[i] & 0x7FFF7FFFu, hi0[i] & 0x7FFF7FFFu);
          m1[i] = __vmaxu2(lo1[i] & 0x7FFF7FFFu, hi1[i] & 0x7FFF7FFFu);
        }
        float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          mma_16x8(y, lo0[i], lo1[i], lo0[i + 1], lo1[i + 1], bf2_min(qw[i], 0u), bf2_min(qw[i + 1], 0u));
          mma_16x8(y, hi0[i], hi1[i], hi0[i + 1], hi1[i + 1], bf2_max(qw[i], 0u), bf2_max(qw[i + 1], 0u));
          mma_16x8(t, m0[i], m1[i], m0[i + 1], m1[i + 1], qw[i] & 0x7FFF7FFFu, qw[i + 1] & 0x7FFF7FFFu);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += y[e];
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (h0 + 2 * c + i < a.group) {
        best0 = fmaxf(best0, s[i] * a.scale);
        best1 = fmaxf(best1, s[2 + i] * a.scale);
        size0 = max(size0, __float_as_uint(t[i]) & 0x7fffffffu);
        size1 = max(size1, __float_as_uint(t[2 + i]) & 0x7fffffffu);
      }
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    best0 = fmaxf(best0, __shfl_xor_sync(0xffffffffu, best0, o));
    best1 = fmaxf(best1, __shfl_xor_sync(0xffffffffu, best1, o));
    size0 = max(size0, __shfl_xor_sync(0xffffffffu, size0, o));
    size1 = max(size1, __shfl_xor_sync(0xffffffffu, size1, o));
  }
  const int p = p0 + r + 8 * c;                            // lane 4 r has page r, lane 4 r + 1 page r + 8
  if (c < 2 && p < np) put(p, approx(c ? best1 : best0, fabsf(a.scale) * (__uint_as_float(c ? size1 : size0) + kTiny), kRel, w, err));
}

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

// fp32: scores of pages p0 .. p0 + 7 by a warp.  A lane has DL columns and takes four query heads at a time.  Error: 2 DL additions in a lane and five over
// the lanes, of 2^-24 each.
template <int DL, typename F> __device__ __forceinline__ void score_pages_f32(const SelectArgs &a, int b, int head, int p0, int id, int np, uint32_t &err, F put) {
  constexpr float kRel = (2 * DL + 5) / 16777216.f;
  const int lane = threadIdx.x & 31, c = lane * DL;
  const bool mine = c < a.d_h;                             // (d_h is a multiple of 4)
  const float *bounds = static_cast<const float *>(a.bounds), *Q = static_cast<const float *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  const auto load = [&](const float *p, bool there, float (&x)[DL]) {
#pragma unroll
    for (int i = 0; i < DL; i += 2) {
      const float2 v = there ? __ldg(reinterpret_cast<const float2 *>(p + i)) : make_float2(0.f, 0.f);
      x[i] = v.x; x[i + 1] = v.y;
    }
  };
  float lo[8][DL], hi[8][DL];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const int at = __shfl_sync(0xffffffffu, id, p);
    const float *row = bounds + ((long long)at * a.n_kvh + head) * 2 * a.d_h + c;
    load(row, mine && at >= 0, lo[p]);
    load(row + a.d_h, mine && at >= 0, hi[p]);
  }
  const int at = __shfl_sync(0xffffffffu, id, lane >> 2);
  const float w = at >= 0 ? __ldg(a.w_max + at) : -INFINITY;
  float best = -INFINITY;                                  // of page lane >> 2, over the heads of this lane
  uint32_t size = 0;                                       // (as an integer: not negative, and NaN is above all)
  for (int h0 = 0; h0 < a.group; h0 += kHeadsAtOnce) {
    float sum[8 * kHeadsAtOnce], abs[8 * kHeadsAtOnce];
#pragma unroll
    for (int h = 0; h < kHeadsAtOnce; ++h) {
      float q[DL];
      load(Q + (h0 + h) * a.ldQh + c, mine && h0 + h < a.group, q);
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        float s = 0.f, t = 0.f;
#pragma unroll
        for (int e = 0; e < DL; ++e) {
          s = fmaf(fmaxf(q[e], 0.f), hi[p][e], fmaf(fminf(q[e], 0.f), lo[p][e], s));
          t = fmaf(fabsf(q[e]), fabsf(lo[p][e]) + fabsf(hi[p][e]), t);
        }
        sum[p * kHeadsAtOnce + h] = s;
        abs[p * kHeadsAtOnce + h] = t;
      }
    }
    fold<8 * kHeadsAtOnce>(sum, lane, 16);
    fold<8 * kHeadsAtOnce>(abs, lane, 16);
    if (h0 + (lane & (kHeadsAtOnce - 1)) < a.group) {
      best = fmaxf(best, sum[0] * a.scale);
      size = max(size, __float_as_uint(abs[0]) & 0x7fffffffu);
    }
  }
#pragma unroll
  for (int o = 1; o < kHeadsAtOnce; o <<= 1) {
    best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o));
    size = max(size, __shfl_xor_sync(0xffffffffu, size, o));
  }
  const int p = p0 + (lane >> 2);
  if ((lane & 3) == 0 && p < np) put(p, approx(best, fabsf(a.scale) * (__uint_as_float(size) + kTiny), kRel, w, err));
}

// The score of page p in double, by a warp.
template <typename T> __device__ __noinline__ double exact_score(const SelectArgs &a, int b, int head, int p) {
  const int lane = threadIdx.x & 31, id = a.table[(long long)b * a.width + p];
  if (id < 0 || id >= a.n_pages) return -INFINITY;
  const T *row = static_cast<const T *>(a.bounds) + ((long long)id * a.n_kvh + head) * 2 * a.d_h, *Q = static_cast<const T *>(a.Q) + b * a.ldQ + (long long)head * a.group * a.ldQh;
  const double w = a.w_max[id];
  double best = -INFINITY;
  for (int h0 = 0; h0 < a.group; h0 += 4) {
    double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1                              // (its code is cold: unrolled it takes 0.4 us more)
    for (int c = lane; c < a.d_h; c += 32) {
      const float lo = (float)row[c], hi = (float)row[a.d_h + c];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const float q = h0 + h < a.group ? (float)Q[(h0 + h) * a.ldQh + c] : 0.f;
        s[h] = fma((double)q, (double)(q > 0.f ? hi : q < 0.f ? lo : q), s[h]);   // (0 and NaN by themselves)
      }
    }
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const double x = warp_sum(s[h]) * (double)a.scale;
      if (h0 + h < a.group) best = fmax(best, x);          // (drops a NaN)
    }
  }
  return best + w;
}

constexpr int kPickBits = 10;
constexpr int kPickNear = 256;             // most scores near the n-th largest that are decided by comparing them with one another
constexpr int kPickBin = 64;               // a bin of no more scores than this is not divided further

struct PickShared {
  uint32_t mask[kMaxSelectPages / 32];
  int hist[1 << kPickBits];
  uint32_t near_key[kPickNear];            // scores near the n-th largest, in fp32
  int near_at[kPickNear];
  int doubt[kPickNear];                    // of these, the ones that fp32 leaves in doubt
  unsigned long long cand[kPickNear];      // their scores in double
  unsigned long long w_max[kSelectWarps], w_min[kSelectWarps];
  uint32_t range[3][kMaxSelectCluster * kSelectWarps];   // largest and smallest score and largest error of every warp of the cluster
  int w_sum[kSelectWarps];
  int bin, above, in_bin, n_near, n_sure, n_doubt;
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
  for (int w = 0; w < kSelectWarps; ++w) {
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
    for (int i = tid; i < bins; i += kSelectThreads) s.hist[i] = 0;
    __syncthreads();
    for (int i = first + tid; i < end; i += kSelectThreads) {
      const K k = key(i);
      if (Cut<K>::high(k, cut.shift) == cut.prefix) atomicAdd(&s.hist[(int)(k >> lower) & (bins - 1)], 1);
    }
    __syncthreads();
    constexpr int PER = (1 << kPickBits) / kSelectThreads;   // bins of a thread, the largest first
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

__device__ __forceinline__ void st_cluster_u32(const uint32_t *p, int rank, uint32_t v) {
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}

// W: columns of a row, in blocks of 64 (bf16 and fp32)
template <typename T, int W>
__global__ void __launch_bounds__(kSelectThreads, W * sizeof(T) <= 4 ? 2 : 1) k_page_select(const __grid_constant__ SelectArgs a) {
  extern __shared__ uint32_t s_keys[];
  __shared__ PickShared s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int head = blockIdx.y, b = blockIdx.z, rank = blockIdx.x, ctas = gridDim.x;   // (a cluster is a row of the grid)
  int32_t *out = a.selected + ((long long)b * a.n_kvh + head) * a.n_select;
  cluster_arrive();                                        // the first CTA's shared memory is written once that CTA runs
  pdl_wait();
  pdl_trigger();
  const int np = pages_of(a, b, rank == 0 && tid == 0 && head == 0);
  const bool all = np <= a.n_select;
  const int first = a.n_first, end = np - a.n_last;        // the scores decide between these (n_first + n_last <= n_select < np)
  const long long row = ((long long)b * a.n_kvh + head) * a.width;
  const bool kept = np <= kPickKeys;                       // in shared memory, otherwise in the workspace
  cluster_wait();
  if (!all) {
    uint32_t kmax = 0, kmin = ~0u, err = 0;                // (of all pages; the range may be wider than that of the ones the scores decide between)
    const auto put = [&](int p, uint32_t k) {
      kmax = max(kmax, k);
      kmin = min(kmin, k);
      if (kept) st_cluster_u32(s_keys + p, 0, k);
      else a.approx[row + p] = k;
    };
    constexpr int PER = sizeof(T) == 2 ? 16 : 8;           // pages of a warp
    const int step = ctas * kSelectWarps * PER;
    const auto page_at = [&](int p) { return lane < PER && p + lane < np ? a.table[(long long)b * a.width + p + lane] : -1; };
    int p0 = (rank * kSelectWarps + warp) * PER, next = page_at(p0);
    for (; p0 < np; p0 += step) {
      int id = next;
      next = page_at(p0 + step);                           // (a trip ahead of the pages themselves)
      if (lane < PER && p0 + lane < np && (id < 0 || id >= a.n_pages)) {
        id = -1;
        if (a.status && head == 0) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      }
      if constexpr (sizeof(T) == 2) score_pages<2 * W>(a, b, head, p0, id, np, err, put);
      else score_pages_f32<2 * W>(a, b, head, p0, id, np, err, put);
    }
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    kmin = __reduce_min_sync(0xffffffffu, kmin);
    err = __reduce_max_sync(0xffffffffu, err & ~kAnyMarked) | __reduce_or_sync(0xffffffffu, err & kAnyMarked);
    if (lane < 3) st_cluster_u32(s.range[lane] + rank * kSelectWarps + warp, 0, lane == 0 ? kmax : lane == 1 ? kmin : err);
  }
  cluster_sync();
  if (rank) return;
  if (all) {
    for (int i = tid; i < a.n_select; i += kSelectThreads) out[i] = i < np ? i : -1;
    return;
  }
  const int need = a.n_select - a.n_first - a.n_last;
  const uint32_t *apx = a.approx + row;
  uint32_t kmax = 0, kmin = ~0u, err = 0;                  // (every warp for itself)
  for (int i = lane; i < ctas * kSelectWarps; i += 32) {
    kmax = max(kmax, s.range[0][i]);
    kmin = min(kmin, s.range[1][i]);
    err = max(err, s.range[2][i]);
  }
  kmax = __reduce_max_sync(0xffffffffu, kmax);
  kmin = __reduce_min_sync(0xffffffffu, kmin);
  err = __reduce_max_sync(0xffffffffu, err);
  const auto key = [&](int i) { return kept ? s_keys[i] : apx[i]; };
  if (err & kAnyMarked) {
    err = 0;
    for (int i = 0; i < ctas * kSelectWarps; ++i) err = max(err, s.range[2][i] & ~kAnyMarked);
    kmax = 0;                                              // (a mark is above all scores)
    if (tid == 0) s.n_near = 0;
    __syncthreads();
    for (int i = tid; i < np; i += kSelectThreads) {
      const uint32_t k = key(i);
      if (k != kMarked) {
        kmax = max(kmax, k);
      } else {
        const int at = atomicAdd(&s.n_near, 1);
        if (at < kPickNear) s.near_at[at] = i;
      }
    }
    __syncthreads();
    const int n = s.n_near;
    if (n > kPickNear) err = kUnlimited;
    for (int j = warp; j < min(n, kPickNear); j += kSelectWarps) {
      const int p = s.near_at[j];
      const double x = exact_score<T>(a, b, head, p);
      uint32_t k;
      if (fabs(x) < 1e30) {
        k = order_key((float)x);
        err = max(err, __float_as_uint((float)fabs(x) * (1.f / 8388608.f) + kLast));
      } else {                                             // infinities (NaN as minus infinity) as they are; what is beyond fp32: all scores are decided in double
        k = order_key(x == INFINITY ? INFINITY : x > -INFINITY ? 0.f : -INFINITY);
        if (fabs(x) < INFINITY) err = kUnlimited;
      }
      kmax = max(kmax, k);
      kmin = min(kmin, k);
      if (lane == 0) {
        if (kept) s_keys[p] = k;
        else a.approx[row + p] = k;
      }
    }
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    __syncthreads();                                       // (all have read the ranges of the cluster)
    if (lane < 3) s.range[lane][warp] = lane == 0 ? kmax : lane == 1 ? kmin : err;
    __syncthreads();
    for (int w = 0; w < kSelectWarps; ++w) {
      kmax = max(kmax, s.range[0][w]);
      kmin = min(kmin, s.range[1][w]);
      err = max(err, s.range[2][w]);
    }
  }
  if (tid == 0) s.n_near = s.n_sure = s.n_doubt = 0;
  __syncthreads();
  const int words = (np + 31) / 32;
  // Of two scores whose fp32 values differ by more than twice the largest error the larger one is the larger one in double as well.  [low, high]: fp32
  // values that may lie on either side of the need-th largest; those above it are selected.
  const float e2 = 2.f * __uint_as_float(err);
  const auto below = [&](uint32_t k) { return order_key(__fsub_rd(from_order_key(k), e2)); };
  const auto above = [&](uint32_t k) { return order_key(__fadd_ru(from_order_key(k), e2)); };
  uint32_t low = 0, high = ~0u;
  if (err < kUnlimited) {
    const Cut<uint32_t> cut = find_cut<uint32_t>(s, key, first, end, need, kmax, kmin, kPickBin);
    // the need-th largest agrees with the prefix
    const uint32_t least = cut.shift >= 32 ? 0u : cut.prefix << cut.shift, most = cut.shift >= 32 ? ~0u : least | ((1u << cut.shift) - 1u);
    low = below(max(least, kmin));
    high = above(min(most, kmax));
  }
  for (int w = warp; w < words; w += kSelectWarps) {
    const int i = w * 32 + lane;
    const bool in = i >= first && i < end;
    const uint32_t k = in ? key(i) : 0u;
    const bool sure = in && need > 0 && k > high, near = in && need > 0 && k >= low && k <= high;
    const uint32_t m = __ballot_sync(0xffffffffu, sure || (!in && i < np)), ms = __ballot_sync(0xffffffffu, sure);
    if (lane == 0) {
      s.mask[w] = m;
      if (ms) atomicAdd(&s.n_sure, __popc(ms));
    }
    if (near) {
      const int at = atomicAdd(&s.n_near, 1);              // (their order changes nothing)
      if (at < kPickNear) {
        s.near_at[at] = i;
        s.near_key[at] = k;
      }
    }
  }
  __syncthreads();
  const int near = s.n_near, more = need - s.n_sure;       // `more` of the near ones are selected: 0 <= more <= near
  if (more > 0 && near <= kPickNear) {
    // each against the others: `over` of them are larger whatever the errors, `maybe` may be (itself among them)
    int in = 0;
    for (int j = tid; j < near; j += kSelectThreads) {
      const uint32_t k = s.near_key[j], up = err < kUnlimited ? above(k) : ~0u, down = err < kUnlimited ? below(k) : 0u;
      int over = 0, maybe = 0;
      for (int i = 0; i < near; ++i) {
        over += s.near_key[i] > up;
        maybe += s.near_key[i] >= down;
      }
      if (maybe <= more) {
        ++in;
        atomicOr(&s.mask[s.near_at[j] >> 5], 1u << (s.near_at[j] & 31));
      } else if (over < more) {
        s.doubt[atomicAdd(&s.n_doubt, 1)] = s.near_at[j];
      }
    }
    if (tid < 32) s.w_sum[0] = 0;
    __syncthreads();
    if (in) atomicAdd(&s.w_sum[0], in);
    __syncthreads();
    const int doubts = s.n_doubt, rest = more - s.w_sum[0];   // `rest` of the ones in doubt are selected
    for (int j = warp; j < doubts; j += kSelectWarps) {
      const double x = exact_score<T>(a, b, head, s.doubt[j]);
      if (lane == 0) s.cand[j] = order_key(x);
    }
    if (doubts) __syncthreads();
    for (int j = tid; j < doubts; j += kSelectThreads) {
      const unsigned long long k = s.cand[j];
      const int at = s.doubt[j];
      int before = 0;
      for (int i = 0; i < doubts; ++i) before += s.cand[i] > k || (s.cand[i] == k && s.doubt[i] < at);
      if (before < rest) atomicOr(&s.mask[at >> 5], 1u << (at & 31));
    }
  } else if (more > 0) {                                   // many scores (nearly) equal, or beyond fp32: all near ones in double
    unsigned long long *exact = a.keys + row;              // 0 for what is not near: below every score
    unsigned long long xmax = 0, xmin = ~0ull;
    for (int i = first + warp; i < end; i += kSelectWarps) {
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
      s.w_min[warp] = near < end - first ? 0ull : xmin;
    }
    __syncthreads();
    for (int w = 0; w < kSelectWarps; ++w) {
      xmax = max(xmax, s.w_max[w]);
      xmin = min(xmin, s.w_min[w]);
    }
    const auto ekey = [&](int i) { return exact[i]; };
    const Cut<unsigned long long> cut = find_cut<unsigned long long>(s, ekey, first, end, more, xmax, xmin, 0);
    int taken = 0;                                         // equal scores in the words before this round's
    for (int w0 = 0; w0 < words; w0 += kSelectWarps) {
      const int w = w0 + warp, i = w * 32 + lane;
      const unsigned long long k = i >= first && i < end ? exact[i] : 0ull, h = Cut<unsigned long long>::high(k, cut.shift);
      const bool same = k != 0 && h == cut.prefix;
      const uint32_t eq = __ballot_sync(0xffffffffu, same), gt = __ballot_sync(0xffffffffu, k != 0 && h > cut.prefix);
      if (lane == 0) s.w_sum[warp] = __popc(eq);
      __syncthreads();
      int before = taken, all = 0;
      for (int v = 0; v < kSelectWarps; ++v) {
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
  for (int w0 = 0; w0 < words; w0 += kSelectThreads) {
    const int w = w0 + tid;
    uint32_t m = w < words ? s.mask[w] : 0u;
    int all;
    int at = base + scan_block(__popc(m), s.w_sum, &all);
    base += all;
    for (; m; m &= m - 1) out[at++] = w * 32 + __ffs(m) - 1;
  }
}

}  // namespace

using SelectKernel = void (*)(SelectArgs);
static SelectKernel select_kernel(int d_h, bool bf16) {
  if (!bf16) return d_h <= 64 ? k_page_select<float, 1> : k_page_select<float, 2>;
  return d_h <= 64 ? k_page_select<__nv_bfloat16, 1> : d_h <= 128 ? k_page_select<__nv_bfloat16, 2> : k_page_select<__nv_bfloat16, 4>;
}

cudaError_t select_pages_configure(int d_h, bool bf16) {
  const cudaError_t e = cudaFuncSetAttribute(select_kernel(d_h, bf16), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(kPickKeys * sizeof(uint32_t)));
  return e != cudaSuccess ? e : cudaFuncSetAttribute(select_kernel(d_h, bf16), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}

cudaError_t launch_page_select(const SelectArgs &a, bool bf16, int most_ctas, int sm_count, cudaStream_t st) {
  // As many CTAs as give every SM one, no more than there are pages for.  (Two per SM, 32 requests of 8 key heads in clusters of 2: 16.6 -> 21 us, with CTAs of half
  // the threads 17.0.)
  int size = 1;
  const int pages = bf16 ? kSelectPages : kSelectPages / 2;
  while (size * 2 <= most_ctas && size * 2 <= kMaxSelectCluster && (long long)a.B * a.n_kvh * size < sm_count && size * pages < a.width) size *= 2;
  if (a.width <= a.n_select) size = 1;                     // all pages are selected whatever the lengths
  const int keys = a.width <= a.n_select ? 0 : a.width < kPickKeys ? a.width : kPickKeys;
  LaunchOpt opt;
  opt.cluster = size > 1 ? size : 0;
  return launch_opt(opt, select_kernel(a.d_h, bf16), dim3((unsigned)size, (unsigned)a.n_kvh, (unsigned)a.B), dim3(kSelectThreads), (size_t)keys * sizeof(uint32_t), st, a);
}

}  // namespace pact
