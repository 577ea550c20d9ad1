// Attention of one new token per request over a paged cache (pact_paged_attention): Eq. 11 of the paper for the tokens that follow.
//
//   s_p = scale q.k_p + logw_p,   out = sum_p exp(s_p - m) v_p / sum_p exp(s_p - m),   m = max_p s_p
//
// Keys and values are read once and each is used by the few query heads of its key head, so HBM bounds it: 4 d_h bytes per row and key
// head in bf16 against 4 d_h g operations for g query heads.  (Once for up to 16 query heads of a key head, in fp32 8; wider groups are several tiles of heads, which read them once each.)
//
// Split.  The rows of all requests and key heads, in tiles of 64, form one line of T tiles that G CTAs share out evenly: CTA i takes tiles
// [i T / G, (i + 1) T / G).  No length, batch or number of heads leaves SMs idle, at most G - 1 cuts are made in all, and k_attend_join puts
// the parts of what was cut together.  The shares follow from prefix sums over the lengths, which every CTA forms itself: lengths are known on
// the device only.  (Smaller units behind shares of four fifths, which CTAs took over as they were done: the CTAs ended within 3 us instead of
// 9, but no earlier, since HBM was busy all the time, and the more parts cost the join 3 to 25 us.)
// Short tables and few requests: a cluster of CTAs per request and key head instead, which put their parts together through shared memory.
//
// Pipeline.  One warp copies: each lane works out page ids and row counts of one tile, 32 tiles at a time, and tiles arrive as boxes of
// 128-byte columns through the tensor-copy unit (swizzled, so that ldmatrix meets no bank conflicts) in a ring that runs on across requests.
// Four warps compute; each has 16 rows of every tile and its own running maximum, sum and output, so they meet only at the end of a request.
// A warp whose wait runs out gives up for its CTA: it gives no stage back any more, so that the copying warp fills none whose copies have not been waited for
// and stops within a ring; all go on through the barriers, and the copies under way land before the CTA ends.
//
// bf16: logits as K (16 rows x 16) by q^T (16 x 8 heads) on mma.sync, so that eight heads are one operand; the output as V^T (16 columns x 16 rows)
// by P^T (16 rows x 8 heads), also without padding.  tcgen05 would want 64 or 128 rows per instruction and its results through tensor memory,
// where HBM delivers a tile every 1400 clocks of an SM and the warps need less.  Probabilities go in as three bf16 terms, which hold all of fp32's 24 bits.  (Two are
// off by 2^-17: two rows, worst relative error of a result 5.8e-6 against less than 2^-20; of 28672 bf16 results over 2500 rows 28 were not the nearest number, with three 7.  The third costs 0.5 %
// of a call that HBM bounds.)
// The products of 16 rows are summed by themselves, the small terms first, and added with rounding: an instruction cuts its sum off towards 0, so that a running sum in its
// accumulator loses some 2^-25 at each (values of one sign, 1048576 rows: the mean of the results 2.9e-5 too small, now below 2^-20; 128 requests of 8192 rows 408 -> 412 us).
// fp32: fused multiply-adds; for the logits a lane has one row and half of the columns, for the output four columns of all rows.
#include "paged.cuh"
#include "paged_tiles.h"
#include "umma.cuh"

namespace pact {
namespace {

constexpr int kConsumers = 4;              // computing warps
constexpr int kAttendThreads = (kConsumers + 1) * 32;
constexpr int kMaxAttendStages = 8;
constexpr int kBoxBytes = 128;             // columns of a box
constexpr int kBlockBytes = kTile * kBoxBytes;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCluster = 16;
template <int HEADS> constexpr int kScratch = (kRowsOfWarp + 1) * HEADS;   // fp32: floats of a warp for probabilities and factors

// What the copying warp has worked out about a tile.
struct __align__(16) TilePlan {
  int id[4];                               // page of every 16 rows
  uint32_t rows, place;                    // rows that count of every 16, their place in the page in 16 rows: a byte each
  uint32_t bytes;                          // to be copied
  int first;                               // the first of its part of a request
  int b, h;
};

// Offsets in dynamic shared memory (the ring comes first: swizzled boxes lie at multiples of 1024 bytes).
struct AttendSmem {
  int stage;                               // bytes of K and V of a stage
  int bias, q, q_row, q_own, slots, ml, tiles, bars, meta, pre, total;
};
__host__ __device__ inline AttendSmem attend_smem(int stages, int blocks, int heads, int elt, int B) {
  AttendSmem m;
  m.stage = 2 * blocks * kBlockBytes;
  m.bias = stages * m.stage;
  m.q = m.bias + stages * kTile * 4;
  m.q_row = blocks * kBoxBytes + 16;       // (16 bytes more: rows of different heads begin in different banks)
  m.q_own = m.q + stages * heads * m.q_row;
  m.slots = m.q_own + (elt == 4 ? heads * m.q_row : 0);
  m.ml = m.slots + 2 * heads * (blocks * kBoxBytes / elt + 4) * 4;
  m.tiles = m.ml + kConsumers * heads * 8;
  m.bars = m.tiles + 32 * (int)sizeof(TilePlan);
  m.meta = m.bars + 2 * stages * 8;
  m.pre = m.meta + stages * 4 + 8;
  m.total = m.pre + (B + 1 + kAttendThreads / 32) * 4;
  return m;
}

__device__ __forceinline__ void tma_load_5d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y, int z, int w, int v) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(v) : "memory");
}
__device__ __forceinline__ void copy16(void *dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void arrive_after_copies(uint64_t *bar) {   // once this thread's 16-byte copies so far have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ float4 lds4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float fma4(const float4 &x, const float4 &y, float s) { return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s)))); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t in_cta(const void *p, uint32_t rank) {   // the same place in the shared memory of another CTA of the cluster
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float2 ld_cluster2(uint32_t at) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}

__device__ __forceinline__ void consumers_meet() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers * 32) : "memory"); }

// Logits stay in natural units: a bias of the lowest float times log2 e would be minus infinity, and rows that all have it share the attention.
// exp(s - m), 0 for s = -inf whatever m is
__device__ __forceinline__ float exp_below(float s, float m) { return ex2_approx((s - (m == -INFINITY ? 0.f : m)) * kLog2e); }
// how much a sum with maximum m counts beside one with maximum `to` (m - to is NaN where both are infinite)
__device__ __forceinline__ float weight(float m, float to) { return m == -INFINITY ? 0.f : m == to ? 1.f : ex2_approx((m - to) * kLog2e); }

// One warp's part of a request and key head: running maximum of the logits, sum and output of its rows.
template <typename T, int NB, int NT> struct Part;

template <int NB, int NT> struct Part<__nv_bfloat16, NB, NT> {
  static constexpr int kHeads = 8 * NT, kCols = NB * 64;
  uint32_t q[NB * 4][NT][2];               // q^T: columns 16 k + 2 (lane % 4) + {0, 1} (+ 8), head lane / 4
  float m[NT][2], l[NT][2];                // heads 2 (lane % 4) + {0, 1}; the sums are of this lane's rows
  float o[NB * 4][NT][4];                  // columns 16 c + lane / 4 (+ 8 in the upper two), the same heads

  __device__ __forceinline__ void begin(const char *sq, int q_row, char *, int lane, int) {
#pragma unroll
    for (int k = 0; k < NB * 4; ++k)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          q[k][n][i] = *reinterpret_cast<const uint32_t *>(sq + (n * 8 + lane / 4) * q_row + (k * 16 + i * 8 + (lane % 4) * 2) * 2);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int c = 0; c < NB * 4; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[c][n][i] = 0.f;
    }
  }

  // 16 rows, of which the first `rows` count: K from sk on, V from sv on, 128 bytes of each and `block` bytes to the next 128 of their columns
  __device__ __forceinline__ void step(uint32_t sk, uint32_t sv, uint32_t block, const float *bias, bool has_bias, int rows, float scale, int lane, float *) {
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] = 0.f;
    {
      const int r = lane & 15, x = r & 7;
      const uint32_t at = sk + r * kBoxBytes;
#pragma unroll
      for (int k = 0; k < NB * 4; ++k) {
        uint32_t a[4];
        ldsm4(a, at + (k / 4) * block + ((((k % 4) * 2 + (lane >> 4)) ^ x) << 4));
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(s[n], a, q[k][n][0], q[k][n][1]);
      }
    }
    const int r0 = lane / 4, r1 = r0 + 8;
    float b0 = 0.f, b1 = 0.f;
    if (has_bias) {
      b0 = bias[r0];
      b1 = bias[r1];
    }
    const bool in0 = r0 < rows && b0 != -INFINITY, in1 = r1 < rows && b1 != -INFINITY;
    float top[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[n][i] = in0 ? fmaf(s[n][i], scale, b0) : -INFINITY;
        s[n][2 + i] = in1 ? fmaf(s[n][2 + i], scale, b1) : -INFINITY;
        top[n][i] = fmaxf(s[n][i], s[n][2 + i]);
      }
#pragma unroll
    for (int w = 4; w < 32; w <<= 1)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) top[n][i] = fmaxf(top[n][i], __shfl_xor_sync(0xffffffffu, top[n][i], w));
    bool grows = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) grows = grows || top[n][i] > m[n][i];
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float to = fmaxf(m[n][i], top[n][i]), f = weight(m[n][i], to);
          m[n][i] = to;
          l[n][i] *= f;
#pragma unroll
          for (int c = 0; c < NB * 4; ++c) {
            o[c][n][i] *= f;
            o[c][n][2 + i] *= f;
          }
        }
    }
    uint32_t hi[NT][2], lo[NT][2], rest[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = exp_below(s[n][i], m[n][i & 1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) l[n][i] += p[i] + p[2 + i];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t h = pack_bf16(p[2 * i], p[2 * i + 1]);
        hi[n][i] = transpose8(h);
        const float x = p[2 * i] - __uint_as_float(h << 16), y = p[2 * i + 1] - __uint_as_float(h & 0xFFFF0000u);   // (exact)
        const uint32_t g = pack_bf16(x, y);
        lo[n][i] = transpose8(g);
        rest[n][i] = transpose8(pack_bf16(x - __uint_as_float(g << 16), y - __uint_as_float(g & 0xFFFF0000u)));
      }
    }
    // values of rows that do not count are cleared: zero times an infinity or a NaN would not be zero
    uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
    const uint32_t rows0 = __ballot_sync(0xffffffffu, in0), rows1 = __ballot_sync(0xffffffffu, in1);
    const bool clear = (rows0 & rows1) != 0xffffffffu;
    if (clear) {                               // lane 4 r speaks for row r; this lane's registers hold rows 2 (lane % 4) + {0, 1} (+ 8)
      const int r = (lane % 4) * 8;
      keep0 = ((rows0 >> r) & 1 ? 0xFFFFu : 0u) | ((rows0 >> (r + 4)) & 1 ? 0xFFFF0000u : 0u);
      keep1 = ((rows1 >> r) & 1 ? 0xFFFFu : 0u) | ((rows1 >> (r + 4)) & 1 ? 0xFFFF0000u : 0u);
    }
    {
      const int r = (lane & 7) + (lane >> 4) * 8, x = r & 7;
      const uint32_t at = sv + r * kBoxBytes;
#pragma unroll
      for (int c = 0; c < NB * 4; ++c) {
        uint32_t a[4];
        ldsm4_t(a, at + (c / 4) * block + ((((c % 4) * 2 + ((lane >> 3) & 1)) ^ x) << 4));
        if (clear) {
          a[0] &= keep0;
          a[1] &= keep0;
          a[2] &= keep1;
          a[3] &= keep1;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float y[4] = {0.f, 0.f, 0.f, 0.f};
          mma_bf16(y, a, rest[n][0], rest[n][1]);
          mma_bf16(y, a, lo[n][0], lo[n][1]);
          mma_bf16(y, a, hi[n][0], hi[n][1]);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[c][n][i] += y[i];
        }
      }
    }
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int w = 4; w < 32; w <<= 1)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], w);
  }
  // f(head, m, l), once for every head
  template <typename F> __device__ __forceinline__ void each_head(int lane, F f) {
    if (lane < 4)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) f(n * 8 + lane * 2 + i, m[n][i], l[n][i]);
  }
  // x = f(head, m), then g(x, o, head, column) for every element of o of this lane
  template <typename F, typename G> __device__ __forceinline__ void each(int lane, F f, G g) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int head = n * 8 + (lane % 4) * 2 + i;
        const auto x = f(head, m[n][i]);
#pragma unroll
        for (int c = 0; c < NB * 4; ++c) {
          g(x, o[c][n][i], head, c * 16 + lane / 4);
          g(x, o[c][n][2 + i], head, c * 16 + lane / 4 + 8);
        }
      }
  }
};

// NT: 1 for eight heads, 0 for two (models with as many key heads as query heads would pay for eight: 212 rows 9.1 -> 8.1 us)
template <int NB, int NT> struct Part<float, NB, NT> {
  static constexpr int kHeads = NT ? 8 : 2, kHalf = kHeads / 2, kCols = NB * 32;
  static constexpr int kChunks = NB * 8;                       // 16-byte columns of a row
  static constexpr int kGroups = kChunks <= 8 ? 4 : kChunks <= 16 ? 2 : 1;   // groups of lanes that share out the rows for the output
  static constexpr int kGroupLanes = 32 / kGroups;
  uint32_t q;                              // in shared memory
  int q_row;
  float m[kHalf], l[kHalf];                // heads kHalf (lane / 16) + {0 ..}; the sums are of this lane's row
  float o[kHeads][4];                           // columns 4 (lane % kGroupLanes) + {0 .. 3}, rows of the lane's group

  // q is read in every step, and the copying warp may be ahead by now with the next request's in the same stage: the warps make a copy.
  // (The barrier also parts the probabilities to come, which lie in the slots, from reads of the slots at the end of the request before.)
  __device__ __forceinline__ void begin(const char *sq, int row, char *own, int, int tid) {
    for (int i = tid * 16; i < kHeads * row; i += kConsumers * 32 * 16) *reinterpret_cast<uint4 *>(own + i) = *reinterpret_cast<const uint4 *>(sq + i);
    consumers_meet();
    q = smem_u32(own);
    q_row = row;
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[h][i] = 0.f;
  }

  // scratch: 16 rows of probabilities and a row of factors, this warp's
  __device__ __forceinline__ void step(uint32_t sk, uint32_t sv, uint32_t block, const float *bias, bool has_bias, int rows, float scale, int lane, float *scratch) {
    const int r = lane & 15, half = lane >> 4, x = r & 7;
    float s[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) s[h] = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 2 * i + half;
        const float4 k = lds4(sk + nb * block + r * kBoxBytes + ((c ^ x) << 4));
#pragma unroll
        for (int h = 0; h < kHeads; ++h) s[h] = fma4(k, lds4(q + h * q_row + nb * kBoxBytes + c * 16), s[h]);
      }
    const float b = has_bias ? bias[r] : 0.f;
    const bool in = r < rows && b != -INFINITY;
    float t[kHalf], top[kHalf];
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {         // both halves of the columns; a lane goes on with half of the heads
      const float give = half ? s[i] : s[kHalf + i], got = __shfl_xor_sync(0xffffffffu, give, 16);
      t[i] = in ? fmaf((half ? s[kHalf + i] : s[i]) + got, scale, b) : -INFINITY;
      top[i] = t[i];
    }
#pragma unroll
    for (int w = 1; w < 16; w <<= 1)
#pragma unroll
      for (int i = 0; i < kHalf; ++i) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], w));
    bool grows = false;
#pragma unroll
    for (int i = 0; i < kHalf; ++i) grows = grows || top[i] > m[i];
    const bool rescale = __any_sync(0xffffffffu, grows);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) {
      if (rescale) {
        const float to = fmaxf(m[i], top[i]), f = weight(m[i], to);
        m[i] = to;
        l[i] *= f;
        if (r == 0) scratch[kRowsOfWarp * kHeads + half * kHalf + i] = f;
      }
      t[i] = exp_below(t[i], m[i]);
      l[i] += t[i];
    }
    if constexpr (kHalf == 4) *reinterpret_cast<float4 *>(scratch + r * 8 + half * 4) = make_float4(t[0], t[1], t[2], t[3]);
    else scratch[r * 2 + half] = t[0];
    const uint32_t live = __ballot_sync(0xffffffffu, in) & 0xffffu;
    __syncwarp();
    if (rescale) {
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float f = scratch[kRowsOfWarp * kHeads + h];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[h][i] *= f;
      }
    }
    const int c = lane % kGroupLanes;
    if (c < kChunks) {
#pragma unroll 4
      for (int k = lane / kGroupLanes; k < kRowsOfWarp; k += kGroups) {
        if (!(live >> k & 1)) continue;       // zero times an infinity or a NaN would not be zero
        const float4 v = lds4(sv + (c / 8) * block + k * kBoxBytes + (((c % 8) ^ (k & 7)) << 4));
        float p[kHeads];
        if constexpr (kHeads == 8) {
          const float4 p0 = *reinterpret_cast<const float4 *>(scratch + k * 8), p1 = *reinterpret_cast<const float4 *>(scratch + k * 8 + 4);
          p[0] = p0.x; p[1] = p0.y; p[2] = p0.z; p[3] = p0.w;
          p[4] = p1.x; p[5] = p1.y; p[6] = p1.z; p[7] = p1.w;
        } else {
          const float2 p0 = *reinterpret_cast<const float2 *>(scratch + k * 2);
          p[0] = p0.x; p[1] = p0.y;
        }
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          o[h][0] = fmaf(p[h], v.x, o[h][0]);
          o[h][1] = fmaf(p[h], v.y, o[h][1]);
          o[h][2] = fmaf(p[h], v.z, o[h][2]);
          o[h][3] = fmaf(p[h], v.w, o[h][3]);
        }
      }
    }
    __syncwarp();
  }

  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int w = 1; w < 16; w <<= 1)
#pragma unroll
      for (int i = 0; i < kHalf; ++i) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
#pragma unroll
    for (int w = kGroupLanes; w < 32; w <<= 1)
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[h][i] += __shfl_xor_sync(0xffffffffu, o[h][i], w);
  }
  template <typename F> __device__ __forceinline__ void each_head(int lane, F f) {
    if ((lane & 15) == 0)
#pragma unroll
      for (int i = 0; i < kHalf; ++i) f((lane >> 4) * kHalf + i, m[i], l[i]);
  }
  template <typename F, typename G> __device__ __forceinline__ void each(int lane, F f, G g) {
    float mh[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) mh[h] = __shfl_sync(0xffffffffu, m[h % kHalf], h / kHalf * 16);
    if (lane < kGroupLanes && lane < kChunks)
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const auto x = f(h, mh[h]);
#pragma unroll
        for (int i = 0; i < 4; ++i) g(x, o[h][i], h, lane * 4 + i);
      }
  }
};

__device__ __forceinline__ void store4(const AttendArgs &a, int b, int head, int c, const float4 &v) {
  const long long at = b * a.ldO + head * a.ldOh + c;
  if (a.out_bf16) *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
  else *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = v;
}

constexpr int attend_ctas(int blocks, int tiles_of_heads) { return blocks <= 2 && tiles_of_heads <= 1 ? 2 : 1; }   // of an SM

// CLUSTER: CTA (rank, key head and head tile, request) has a share of that request's tiles alone.
template <typename T, int NB, int NT, bool CLUSTER>
__global__ void __launch_bounds__(kAttendThreads, attend_ctas(NB, NT))
    k_attend(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttendArgs a) {
  using P = Part<T, NB, NT>;
  extern __shared__ __align__(1024) char sm[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttendSmem at = attend_smem(a.stages, NB, P::kHeads, sizeof(T), CLUSTER ? 1 : a.B);
  uint64_t *full = reinterpret_cast<uint64_t *>(sm + at.bars), *empty = full + a.stages;
  uint32_t *meta = reinterpret_cast<uint32_t *>(sm + at.meta);
  int *abort = reinterpret_cast<int *>(meta + a.stages), *filled = abort + 1;   // tiles that the copying warp has asked for
  int *pre = reinterpret_cast<int *>(sm + at.pre), *w_sum = pre + (CLUSTER ? 1 : a.B) + 1;
  TilePlan *plan = reinterpret_cast<TilePlan *>(sm + at.tiles);
  if (tid < a.stages) {
    mbar_init(full + tid, a.logw ? 1 + kTile / 4 : 1);          // (the biases: 16 bytes of a lane each)
    mbar_init(empty + tid, kConsumers);
  }
  if (tid == 0) *abort = 0;
  // columns past d_h and heads past the last are zero in q (of K and V the copies fill them in)
  for (int i = tid * 16; i < at.q_own - at.q; i += kAttendThreads * 16) *reinterpret_cast<uint4 *>(sm + at.q + i) = make_uint4(0, 0, 0, 0);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  // What this lane copies of a tile: of box `x` of rows K, then V, all of their 128-byte blocks at once if they are whole, otherwise one after
  // the other (columns past d_h are filled in then).  A box lies in a stage as its blocks, each with all rows of the box.
  const int boxes = kTile / a.box_rows, per_box = a.box_rows / kRowsOfWarp, at_once = a.whole_blocks ? NB : 1, copies = 2 * NB / at_once;
  constexpr int kRoles = (4 * 2 * NB + 31) / 32;
  int my_box[kRoles], my_copy[kRoles];
#pragma unroll
  for (int r = 0; r < kRoles; ++r) {
    my_box[r] = (lane + 32 * r) / copies;
    my_copy[r] = lane + 32 * r - my_box[r] * copies;
  }

  pdl_wait();
  pdl_trigger();
  const long long room = (long long)a.width * a.page;
  const auto rows_of = [&](int len) { return len < 0 ? 0 : len > room ? (int)room : len; };
  const auto tiles_of = [&](int len) { return tiles_of_request(rows_of(len), a.page, a.selected != nullptr, a.n_select); };
  const int Hn = a.n_kvh * a.head_tiles;
  if constexpr (CLUSTER) {
    const int b = blockIdx.z, len = a.length[b];
    if (tid == 0) {
      pre[0] = 0;
      pre[1] = tiles_of(len);
      if (blockIdx.x == 0 && blockIdx.y == 0 && a.status && (len < 0 || len > room)) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
    }
    __syncthreads();
  } else {
    // tiles before each request, of one key head
    const int per = (a.B + kAttendThreads - 1) / kAttendThreads, b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
      const int len = a.length[b], n = tiles_of(len);
      if (blockIdx.x == 0 && a.status && (len < 0 || len > room)) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      pre[b] = mine;
      mine += n;
    }
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) w_sum[warp] = x;
    __syncthreads();
    int sum = x - mine;
    for (int w = 0; w < warp; ++w) sum += w_sum[w];
    for (int b = b0; b < b1; ++b) pre[b] += sum;
    sum += mine;
    if (b0 < a.B && b1 == a.B) pre[a.B] = sum;
    __syncthreads();
  }
  // this CTA's tiles
  const long long T_all = CLUSTER ? pre[1] : (long long)pre[a.B] * Hn;
  const long long G = CLUSTER ? cluster_size() : min((long long)gridDim.x, T_all), me = CLUSTER ? cluster_rank() : blockIdx.x;
  const long long t0 = me < G ? share_begin(me, G, T_all) : T_all, t1 = me < G ? share_begin(me + 1, G, T_all) : T_all;
  // where tile t lies: request, key head and head tile, place
  const auto find = [&](long long t, int &b, int &h, int &j) {
    if constexpr (CLUSTER) {
      b = blockIdx.z;
      h = blockIdx.y;
      j = (int)t;
    } else if (T_all >> 31) {
      int lo = 0, hi = a.B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((long long)pre[mid] * Hn <= t) lo = mid;
        else hi = mid;
      }
      b = lo;
      h = divide_small(t - (long long)pre[lo] * Hn, pre[lo + 1] - pre[lo], &j);
    } else {                                                   // (the same in 32 bits)
      int lo = 0, hi = a.B;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pre[mid] * Hn <= (int)t) lo = mid;
        else hi = mid;
      }
      b = lo;
      h = divide_small((int)t - pre[lo] * Hn, pre[lo + 1] - pre[lo], &j);
    }
  };
  if constexpr (CLUSTER) {
    if (t0 == t1 && tid < P::kHeads) reinterpret_cast<float2 *>(sm + at.ml)[2 * P::kHeads + tid] = make_float2(-INFINITY, 0.f);   // this CTA has no part
  } else {
    // requests without any row
    for (int b = blockIdx.x; b < a.B; b += gridDim.x)
      if (pre[b + 1] == pre[b]) {
        for (int i = tid * 4; i < a.n_kvh * a.group * a.d_h; i += kAttendThreads * 4) store4(a, b, i / a.d_h, i % a.d_h, make_float4(0.f, 0.f, 0.f, 0.f));
        if (a.lse)
          for (int i = tid; i < a.n_kvh * a.group; i += kAttendThreads) a.lse[(long long)b * a.n_kvh * a.group + i] = -INFINITY;
      }
    if (t0 == t1 && tid == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  }

  if (warp == kConsumers) {
    // ---- the copying warp ----
    int st = 0;
    uint32_t ph = 0;
    int tiles = 0;
    bool given_up = false;
    for (long long base = t0; base < t1 && !given_up; base += 32) {
      const int n = (int)min(32ll, t1 - base);
      if (lane < n) {
        int b, h, j;
        find(base + lane, b, h, j);
        const int kv = h / a.head_tiles, ht = h - kv * a.head_tiles;
        const TileRows at_rows = locate_rows(j, rows_of(a.length[b]), a.page, per_box, a.table + (long long)b * a.width, a.n_pages,
                                             a.selected ? a.selected + ((long long)b * a.n_kvh + kv) * a.n_select : nullptr, a.n_select);
        if (at_rows.bad && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
        TilePlan p;
        p.rows = at_rows.rows;
        p.place = 0;
        p.first = j == 0 || base + lane == t0;
        p.bytes = p.first ? min(P::kHeads, a.group - ht * P::kHeads) * a.d_h * (int)sizeof(T) : 0;
        p.b = b;
        p.h = h;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          p.id[g] = at_rows.id[g];
          p.place |= (uint32_t)(at_rows.off[g] / kRowsOfWarp) << (8 * g);
          // a box is copied if any of its rows counts: its first 16 do then
          if (g % per_box == 0 && (at_rows.rows >> (8 * g) & 0xffu)) p.bytes += a.box_rows * 2 * NB * kBoxBytes;
        }
        plan[lane] = p;
      }
      __syncwarp();
      for (int i = 0; i < n; ++i) {
        const uint32_t rows = plan[i].rows, place = plan[i].place;
        if (!mbar_wait_warp_polls(abort, empty + st, ph ^ 1, a.polls)) {
          given_up = true;
          if (lane == 0) {
            atomicExch(abort, 1);
            if (a.status) atomicMin(a.status, (int)PACT_ERR_TIMEOUT);
          }
          break;
        }
        ++tiles;
        if (lane == 0) {
          meta[st] = rows;
          mbar_arrive_expect_tx(full + st, plan[i].bytes);
        }
        __syncwarp();
        const int h = plan[i].h, kv = h / a.head_tiles;
#pragma unroll
        for (int r = 0; r < kRoles; ++r) {
          const int x = my_box[r], k = my_copy[r], g = 8 * x * per_box;
          if (x < boxes && (rows >> g & 0xffu)) {
            const int page = plan[i].id[x * per_box], row = (int)(place >> g & 0xffu) * kRowsOfWarp;
            const int nb = k * at_once % NB, of_v = k * at_once / NB, block = a.box_rows * kBoxBytes;
            char *to = sm + st * at.stage + of_v * NB * kBlockBytes + (x * NB + nb) * block;
            tma_load_5d(to, of_v ? &map_v : &map_k, full + st, nb * (kBoxBytes / (int)sizeof(T)), row, 0, kv, page);
          }
        }
        if (a.logw && lane < kTile / 4) {
          const int g = lane / 4, box = g / per_box * per_box;   // (16 rows of four lanes)
          if (rows >> (8 * g) & 0xffu)
            copy16(sm + at.bias + (st * kTile + lane * 4) * 4, a.logw + (long long)plan[i].id[box] * a.page + (place >> (8 * box) & 0xffu) * kRowsOfWarp + (lane * 4 - box * kRowsOfWarp));
          arrive_after_copies(full + st);
        }
        if (plan[i].first) {
          const int ht = h - kv * a.head_tiles;
          if (lane < min(P::kHeads, a.group - ht * P::kHeads)) {
            const T *q = static_cast<const T *>(a.Q) + plan[i].b * a.ldQ + (long long)(kv * a.group + ht * P::kHeads + lane) * a.ldQh;
            bulk_load(sm + at.q + (st * P::kHeads + lane) * at.q_row, q, a.d_h * (int)sizeof(T), full + st);
          }
        }
        if (++st == a.stages) {
          st = 0;
          ph ^= 1;
        }
      }
      __syncwarp();
    }
    if (lane == 0) *filled = tiles;
  } else {
    // ---- the computing warps ----
    P part;
    int st = 0;
    uint32_t ph = 0;
    float *slots = reinterpret_cast<float *>(sm + at.slots);
    float2 *ml = reinterpret_cast<float2 *>(sm + at.ml);
    constexpr int kRow = P::kCols + 4, kSlot = P::kHeads * kRow;
    static_assert(sizeof(T) == 2 || 2 * kSlot >= kConsumers * kScratch<P::kHeads>, "the probabilities lie in the slots, which are free between ends");
    // this warp's rows of a stage
    const uint32_t block = a.box_rows * kBoxBytes, of_warp = warp / per_box * NB * block + warp % per_box * kRowsOfWarp * kBoxBytes;
    bool ok = true;
    int b = 0, h = 0, j = 0;
    if (t0 < t1) {
      find(t0, b, h, j);
      if (!CLUSTER && tid == 0) {                            // what the CTAs before this one have of the request at t0
        int4 d = make_int4(0, 0, 0, 0);
        if (j > 0) {
          const long long ts = t0 - j, te = ts + (pre[b + 1] - pre[b]);
          const long long i0 = share_of(ts, G, T_all), i1 = share_of(te - 1, G, T_all);
          if (i0 == me - 1) d = make_int4(ts == share_begin(i0, G, T_all) ? 1 : 2, (int)i1, b, h);
        }
        a.desc[blockIdx.x] = d;
      }
    }
    for (long long t = t0; t < t1;) {
      const int n = CLUSTER ? pre[1] : pre[b + 1] - pre[b], j1 = (int)min((long long)n, j + (t1 - t));
      for (int i = j; i < j1; ++i) {
        if (ok && !mbar_wait_warp_polls(abort, full + st, ph, a.polls)) {
          ok = false;
          if (lane == 0) {
            atomicExch(abort, 1);
            if (a.status) atomicMin(a.status, (int)PACT_ERR_TIMEOUT);
          }
        }
        if (i == j) part.begin(sm + at.q + st * P::kHeads * at.q_row, at.q_row, sm + at.q_own, lane, tid);
        const int rows = (int)(meta[st] >> (8 * warp) & 0xffu);
        if (rows > 0 && ok) {
          const uint32_t sk = smem_u32(sm + st * at.stage) + of_warp;
          part.step(sk, sk + NB * kBlockBytes, block, reinterpret_cast<const float *>(sm + at.bias) + st * kTile + warp * kRowsOfWarp, a.logw != nullptr, rows, a.scale, lane,
                    slots + warp * kScratch<P::kHeads>);
        }
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(empty + st);          // (a warp that has given up keeps its stage)
        if (++st == a.stages) {
          st = 0;
          ph ^= 1;
        }
      }
      // ---- the four warps' parts, two and two ----
      part.finish();
      consumers_meet();                                      // (the slots of the request before have been read)
      if (warp >= 2) {
        float *slot = slots + (warp - 2) * kSlot;
        part.each(lane, [](int, float) { return 0; }, [&](int, float o, int head, int c) { slot[head * kRow + c] = o; });
      }
      part.each_head(lane, [&](int head, float m, float l) { ml[warp * P::kHeads + head] = make_float2(m, l); });
      consumers_meet();
      if (warp < 2) {
        float *slot = slots + warp * kSlot;
        part.each(
            lane,
            [&](int head, float m) {
              const float mo = ml[(warp + 2) * P::kHeads + head].x, to = fmaxf(m, mo);
              return make_float2(weight(m, to), weight(mo, to));
            },
            [&](float2 f, float o, int head, int c) {
              float &s = slot[head * kRow + c];
              s = o * f.x + s * f.y;
            });
        part.each_head(lane, [&](int head, float m, float l) {
          const float2 other = ml[(warp + 2) * P::kHeads + head];
          const float to = fmaxf(m, other.x);
          ml[warp * P::kHeads + head] = make_float2(to, l * weight(m, to) + other.y * weight(other.x, to));
        });
      }
      consumers_meet();
      const int kv = h / a.head_tiles, ht = h - kv * a.head_tiles, heads = min(P::kHeads, a.group - ht * P::kHeads);
      const bool whole = !CLUSTER && j == 0 && j1 == n;
      const long long slot_out = 2 * me + (t == t0 ? 0 : 1);
      for (int i = tid; i < heads * (P::kCols / 4); i += kConsumers * 32) {
        const int hd = i / (P::kCols / 4), c = (i - hd * (P::kCols / 4)) * 4;
        const float2 x = ml[hd], y = ml[P::kHeads + hd];
        const float to = fmaxf(x.x, y.x), fx = weight(x.x, to), fy = weight(y.x, to), l = x.y * fx + y.y * fy;
        const float4 u = *reinterpret_cast<const float4 *>(slots + hd * kRow + c), v = *reinterpret_cast<const float4 *>(slots + kSlot + hd * kRow + c);
        const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        const float4 o = make_float4((u.x * fx + v.x * fy) * inv, (u.y * fx + v.y * fy) * inv, (u.z * fx + v.z * fy) * inv, (u.w * fx + v.w * fy) * inv);
        if constexpr (CLUSTER) {                             // for the other CTAs to read
          *reinterpret_cast<float4 *>(slots + hd * kRow + c) = o;
          if (c == 0) ml[2 * P::kHeads + hd] = make_float2(to, l);
        } else if (whole) {
          const int head = kv * a.group + ht * P::kHeads + hd;
          if (c < a.d_h) store4(a, b, head, c, o);
          if (c == 0 && a.lse) a.lse[(long long)b * a.n_kvh * a.group + head] = l == 0.f ? -INFINITY : to + logf(l);
        } else {
          *reinterpret_cast<float4 *>(a.part_o + (slot_out * P::kHeads + hd) * P::kCols + c) = o;
          if (c == 0) a.part_ml[slot_out * P::kHeads + hd] = make_float2(to, l);
        }
      }
      t += j1 - j;
      j = 0;
      if (!CLUSTER && ++h == Hn) {
        h = 0;
        do ++b;
        while (b < a.B && pre[b + 1] == pre[b]);
      }
    }
  }
  if constexpr (CLUSTER) {
    // The parts of the CTAs of a request and key head: a group of lanes per eight columns, a lane per CTA, so that all is asked for in one trip.
    cluster_sync();
    const int b = blockIdx.z, h = blockIdx.y, kv = h / a.head_tiles, ht = h - kv * a.head_tiles, heads = min(P::kHeads, a.group - ht * P::kHeads);
    const int rank = cluster_rank(), size = cluster_size(), r = tid & (size - 1), items = heads * (P::kCols / 8);
    constexpr int kRow = P::kCols + 4;
    const float *slots = reinterpret_cast<const float *>(sm + at.slots);
    const float2 *ml = reinterpret_cast<const float2 *>(sm + at.ml) + 2 * P::kHeads;
    for (int i0 = 0; i0 < items; i0 += kAttendThreads) {       // (as many groups in all CTAs together)
      const int i = i0 + (rank * kAttendThreads + tid) / size, hd = i / (P::kCols / 8), c = (i - hd * (P::kCols / 8)) * 8;
      float2 x = make_float2(-INFINITY, 0.f);
      float4 u = make_float4(0.f, 0.f, 0.f, 0.f), v = u;
      if (i < items) {
        const uint32_t from = in_cta(slots + hd * kRow + c, r);
        x = ld_cluster2(in_cta(ml + hd, r));
        u = ld_cluster4(from);
        v = ld_cluster4(from + 16);
        if (x.x == -INFINITY && x.y == 0.f) u = v = make_float4(0.f, 0.f, 0.f, 0.f);   // no part, or none of its rows counts
      }
      float top = x.x;
      for (int o = 1; o < size; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const float f = weight(x.x, top);
      float y[9] = {u.x * f, u.y * f, u.z * f, u.w * f, v.x * f, v.y * f, v.z * f, v.w * f, x.y * f};
      for (int o = 1; o < size; o <<= 1)
#pragma unroll
        for (int e = 0; e < 9; ++e) y[e] += __shfl_xor_sync(0xffffffffu, y[e], o);
      if (i < items && r < 2) {                                // a lane for each four of them
        const float l = y[8], inv = l == 0.f ? 0.f : 1.f / l;
        const int head = kv * a.group + ht * P::kHeads + hd;
        const float4 z = r ? make_float4(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv) : make_float4(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        if (c + 4 * r < a.d_h) store4(a, b, head, c + 4 * r, z);
        if (c + 4 * r == 0 && a.lse) a.lse[(long long)b * a.n_kvh * a.group + head] = l == 0.f ? -INFINITY : top + logf(l);
      }
    }
    cluster_sync();                                            // (the others have read)
  } else {
    __syncthreads();
  }
  if (*abort && tid < min(a.stages, *filled)) {              // each stage's last copies, which still write to this CTA's shared memory
    const int rounds = (*filled - 1 - tid) / a.stages;
    mbar_wait_slow(full + tid, rounds & 1);
  }
}

// Parts of the requests and key heads that were cut.  Few parts (a batch): CTA i < `shares` has what was cut at the beginning of share i and not before it, a
// warp per head.  Many (a long request): a CTA per head, whose warps share out the parts; there are at most shares / kFewParts of these, and
// the CTAs from `shares` on look for the one that is theirs.  A warp asks for its first sums together with the maxima.
constexpr int kJoinWarps = 8;
constexpr int kMaxParts = 512;             // most CTAs of k_attend
constexpr int kFewParts = 8;

template <int CH>                          // 16-byte columns of a lane
__global__ void __launch_bounds__(kJoinWarps * 32) k_attend_join(const __grid_constant__ AttendArgs a, int tile_heads, int cols, int shares, int head_ctas) {
  __shared__ float s_w[kJoinWarps][kMaxParts / kJoinWarps + 1];
  __shared__ float4 s_o[kJoinWarps][CH * 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quads = cols / 4;
  pdl_wait();
  pdl_trigger();
  const bool few = blockIdx.x < shares;
  int unit = blockIdx.x, first_head = warp;
  if (!few) {
    __shared__ int s_count[kJoinWarps], s_unit;
    const int e = blockIdx.x - shares;
    first_head = e % head_ctas;
    int before = e / head_ctas;                                // of the requests of many parts
    if (threadIdx.x == 0) s_unit = -1;
    for (int u0 = 0; u0 < shares; u0 += kJoinWarps * 32) {
      const int u = u0 + threadIdx.x;
      const int4 x = u < shares ? a.desc[u] : make_int4(0, 0, 0, 0);
      const bool many = x.x && x.y - (u - 1) + 1 > kFewParts;
      const uint32_t bits = __ballot_sync(0xffffffffu, many);
      if (lane == 0) s_count[warp] = __popc(bits);
      __syncthreads();
      int at = before, all = 0;
      for (int w = 0; w < kJoinWarps; ++w) {
        if (w < warp) at -= s_count[w];
        all += s_count[w];
      }
      if (many && at == __popc(bits & ((1u << lane) - 1u))) s_unit = u;
      before -= all;
      __syncthreads();
    }
    unit = s_unit;
    if (unit < 0) return;
  }
  const int4 d = a.desc[unit];
  const int i0 = unit - 1, n = d.y - i0 + 1, b = d.z, kv = d.w / a.head_tiles, ht = d.w - kv * a.head_tiles;
  if (!d.x || (few && n > kFewParts)) return;
  const int heads = min(tile_heads, a.group - ht * tile_heads);
  const int p0 = few ? 0 : warp * n / kJoinWarps, p1 = few ? n : (warp + 1) * n / kJoinWarps;
  for (int hd = first_head; hd < heads; hd += few ? kJoinWarps : head_ctas) {
    const auto slot = [&](int p) { return (2 * (long long)(i0 + p) + (p == 0 ? d.x - 1 : 0)) * tile_heads + hd; };
    const auto sum_of = [&](int p, int k) { return *reinterpret_cast<const float4 *>(a.part_o + slot(p) * cols + (lane + 32 * k) * 4); };
    const auto add = [&](const float4 &v, float f, float4 &to) {
      to.x = fmaf(v.x, f, to.x);
      to.y = fmaf(v.y, f, to.y);
      to.z = fmaf(v.z, f, to.z);
      to.w = fmaf(v.w, f, to.w);
    };
    constexpr int U = 8;
    float4 x[U][CH], o[CH];
    float2 ml = make_float2(-INFINITY, 0.f);
    if (lane < n) ml = a.part_ml[slot(lane)];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int k = 0; k < CH; ++k)
        if (p0 + u < p1 && lane + 32 * k < quads) x[u][k] = sum_of(p0 + u, k);
    float top = ml.x, l = 0.f;
    for (int p = 32 + lane; p < n; p += 32) top = fmaxf(top, a.part_ml[slot(p)].x);
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    for (int p = lane; p < n; p += 32) {
      const float2 y = p < 32 ? ml : a.part_ml[slot(p)];
      const float f = weight(y.x, top);
      l += y.y * f;
      if (p >= p0 && p < p1) s_w[warp][p - p0] = f;
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) l += __shfl_xor_sync(0xffffffffu, l, w);
    __syncwarp();
#pragma unroll
    for (int k = 0; k < CH; ++k) o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = p0; p < p1; p += U) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p + u < p1)
#pragma unroll
          for (int k = 0; k < CH; ++k)
            if (lane + 32 * k < quads) add(x[u][k], s_w[warp][p + u - p0], o[k]);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < CH; ++k)
          if (p + U + u < p1 && lane + 32 * k < quads) x[u][k] = sum_of(p + U + u, k);
    }
    if (!few) {
#pragma unroll
      for (int k = 0; k < CH; ++k) s_o[warp][lane + 32 * k] = o[k];
      __syncthreads();
      if (warp == 0)
        for (int w = 1; w < kJoinWarps; ++w)
#pragma unroll
          for (int k = 0; k < CH; ++k) add(s_o[w][lane + 32 * k], 1.f, o[k]);
      __syncthreads();
    }
    if (few || warp == 0) {
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int head = kv * a.group + ht * tile_heads + hd;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        const int c = (lane + 32 * k) * 4;
        if (c < a.d_h) store4(a, b, head, c, make_float4(o[k].x * inv, o[k].y * inv, o[k].z * inv, o[k].w * inv));
      }
      if (lane == 0 && a.lse) a.lse[(long long)b * a.n_kvh * a.group + head] = l == 0.f ? -INFINITY : top + logf(l);
    }
    __syncwarp();
  }
}

// ---- host side -----------------------------------------------------------------------------------

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Pages as [page][head][128-byte block][row][column], boxes of box_rows rows and all blocks; rows that are no whole number of blocks as one block, boxes
// of 128 bytes of it.
bool encode_pages(const PagedCfg &cfg, CUtensorMap *map, void *base, bool bf16, const AttendArgs &a, long long ld_page, long long ld_head, long long ld_row) {
  const int elt = bf16 ? 2 : 4, blocks = a.whole_blocks ? cfg.blocks : 1;
  const cuuint64_t dims[5] = {(cuuint64_t)(a.whole_blocks ? kBoxBytes / elt : a.d_h), (cuuint64_t)a.page, (cuuint64_t)blocks, (cuuint64_t)a.n_kvh, (cuuint64_t)a.n_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)ld_row * elt, (cuuint64_t)kBoxBytes, (cuuint64_t)ld_head * elt, (cuuint64_t)ld_page * elt};
  const cuuint32_t box[5] = {(cuuint32_t)(kBoxBytes / elt), (cuuint32_t)a.box_rows, (cuuint32_t)blocks, 1, 1}, estr[5] = {1, 1, 1, 1, 1};
  return reinterpret_cast<EncodeTiledFn>(cfg.encode_tiled)(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 5, base, dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

using AttendKernel = void (*)(CUtensorMap, CUtensorMap, AttendArgs);
template <bool CLUSTER> AttendKernel attend_kernel(const PagedCfg &cfg, bool bf16) {
  const bool few = cfg.tile_heads == 2, wide = cfg.tile_heads == 16;
  if (bf16) switch (cfg.blocks) {
    case 1: return wide ? k_attend<__nv_bfloat16, 1, 2, CLUSTER> : k_attend<__nv_bfloat16, 1, 1, CLUSTER>;
    case 2: return wide ? k_attend<__nv_bfloat16, 2, 2, CLUSTER> : k_attend<__nv_bfloat16, 2, 1, CLUSTER>;
    case 3: return wide ? k_attend<__nv_bfloat16, 3, 2, CLUSTER> : k_attend<__nv_bfloat16, 3, 1, CLUSTER>;
    case 4: return wide ? k_attend<__nv_bfloat16, 4, 2, CLUSTER> : k_attend<__nv_bfloat16, 4, 1, CLUSTER>;
  }
  else switch (cfg.blocks) {
    case 1: return few ? k_attend<float, 1, 0, CLUSTER> : k_attend<float, 1, 1, CLUSTER>;
    case 2: return few ? k_attend<float, 2, 0, CLUSTER> : k_attend<float, 2, 1, CLUSTER>;
    case 3: return few ? k_attend<float, 3, 0, CLUSTER> : k_attend<float, 3, 1, CLUSTER>;
    case 4: return few ? k_attend<float, 4, 0, CLUSTER> : k_attend<float, 4, 1, CLUSTER>;
  }
  return nullptr;
}

constexpr size_t kSmSmem = 228 * 1024, kCtaReserve = 1024;   // shared memory of an SM, and what the system takes of it for each CTA

// CTAs of a cluster per request and key head, 0: no clusters.  `n` tiles of one at most, `heads` of them.
// Clusters leave SMs idle where there are few heads and give every request the time of the longest, the line of tiles costs a second kernel.  One request
// of 28 heads on 4: 1000 rows 7.1 us in clusters against 10.3, 5000 10.1 / 13.2, 9000 12.8 / 13.4, 16000 17.7 / 15.0; eight of them (clusters of 8, two CTAs
// per SM): 1000 9.5 / 13.2, 5000 16.8 / 19.6, 9000 31.7 / 35.5, 16000 48.4 / 52.7 where all are as long, but of eight between 0 and 9000 the longest counts, 23.1 / 22.3, of 0 to 16000 39.0 / 36.5: no clusters
// beyond 8192 rows.  fp32, 2 heads on 2: 200 rows 6.2 / 7.6, 4000 9.2 / 10.6, 9000 13.8 / 13.5.
int cluster_for(const PagedCfg &cfg, long long n, long long heads, int sm_count) {
  for (int size = cfg.cluster; size >= 2; size /= 2) {
    const int i = size == 2 ? 0 : size == 4 ? 1 : size == 8 ? 2 : 3;
    const int most = heads * size > sm_count ? 16 : 8;         // tiles of a CTA
    if (heads <= cfg.clusters[i] && n <= (long long)size * most) return size;
  }
  return 0;
}

}  // namespace

cudaError_t paged_configure(PagedCfg *cfg, const DeviceCfg &dev, int n_qh, int n_kvh, int d_h, bool bf16) {
  void *fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
  if (e != cudaSuccess) return e;
  if (qres != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
  cfg->encode_tiled = fn;
  e = plan_configure();
  const int blocks = (d_h * (bf16 ? 2 : 4) + kBoxBytes - 1) / kBoxBytes, group = n_qh / n_kvh;
  if (e != cudaSuccess || blocks > 4) return e;
  e = select_pages_configure(d_h, bf16);
  if (e != cudaSuccess) return e;
  cfg->blocks = blocks;
  cfg->tile_heads = bf16 ? (group > 8 ? 16 : 8) : group > 2 ? 8 : 2;
  cfg->head_tiles = (group + cfg->tile_heads - 1) / cfg->tile_heads;
  e = cudaFuncSetAttribute(attend_kernel<false>(*cfg, bf16), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dev.smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_kernel<true>(*cfg, bf16), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)dev.smem_optin);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(attend_kernel<true>(*cfg, bf16), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  // clusters of how many CTAs can be launched at all
  cfg->cluster = 1;
  for (int size = 2; size <= kMaxCluster; size *= 2) {
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(size);
    lc.blockDim = dim3(kAttendThreads);
    lc.dynamicSmemBytes = kSmSmem / attend_ctas(cfg->blocks, cfg->tile_heads / 8) - kCtaReserve;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = size;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    int n = 0;
    e = cudaOccupancyMaxActiveClusters(&n, attend_kernel<true>(*cfg, bf16), &lc);
    if (e != cudaSuccess || n < 1) {
      (void)cudaGetLastError();
      break;
    }
    cfg->cluster = size;
    cfg->clusters[size == 2 ? 0 : size == 4 ? 1 : size == 8 ? 2 : 3] = n;
  }
  return cudaSuccess;
}

size_t attend_scratch(const PagedCfg &cfg, const DeviceCfg &dev, bool bf16, AttendArgs *a, char *base) {
  if (!cfg.blocks) return 0;
  const size_t ctas = (size_t)dev.sm_count * attend_ctas(cfg.blocks, cfg.tile_heads / 8), slots = ctas * 2 * cfg.tile_heads;
  const size_t o = slots * (cfg.blocks * kBoxBytes / (bf16 ? 2 : 4)) * sizeof(float), ml = slots * sizeof(float2);   // multiples of 128 bytes
  if (a) {
    a->part_o = reinterpret_cast<float *>(base);
    a->part_ml = reinterpret_cast<float2 *>(base + o);
    a->desc = reinterpret_cast<int4 *>(base + o + ml);
  }
  return (o + ml + ctas * sizeof(int4) + 255) / 256 * 256;
}

cudaError_t launch_attend(AttendArgs a, const pact_paged_cache &cache, const PagedCfg &cfg, const DeviceCfg &dev, bool bf16, cudaStream_t st, int *launches) {
  a.head_tiles = cfg.head_tiles;
  a.box_rows = a.page % 64 == 0 ? 64 : a.page % 32 == 0 ? 32 : 16;
  a.whole_blocks = a.d_h * (bf16 ? 2 : 4) % kBoxBytes == 0;
  CUtensorMap mk, mv;
  if (!encode_pages(cfg, &mk, cache.K, bf16, a, cache.k_page, cache.k_head, cache.k_row) ||
      !encode_pages(cfg, &mv, cache.V, bf16, a, cache.v_page, cache.v_head, cache.v_row))
    return cudaErrorInvalidValue;
  const int per_sm = attend_ctas(cfg.blocks, cfg.tile_heads / 8), elt = bf16 ? 2 : 4, Hn = a.n_kvh * cfg.head_tiles;
  const int ctas = dev.sm_count * per_sm;
  // the most tiles that a request and key head can have
  const long long n = ((long long)(a.selected && a.n_select < a.width ? a.n_select : a.width) * a.page + kTile - 1) / kTile;
  const int size = cluster_for(cfg, n, (long long)a.B * Hn, dev.sm_count);
  const int B = size ? 1 : a.B;
  const size_t most = kSmSmem / per_sm - kCtaReserve;
  a.stages = kMaxAttendStages;
  while (a.stages > 2 && (size_t)attend_smem(a.stages, cfg.blocks, cfg.tile_heads, elt, B).total > most) --a.stages;
  const int smem = attend_smem(a.stages, cfg.blocks, cfg.tile_heads, elt, B).total;
  *launches = 1;
  if (size) {
    LaunchOpt opt;
    opt.cluster = size;
    return launch_opt(opt, attend_kernel<true>(cfg, bf16), dim3((unsigned)size, (unsigned)Hn, (unsigned)a.B), dim3(kAttendThreads), (size_t)smem, st, mk, mv, a);
  }
  cudaError_t e = launch_k(attend_kernel<false>(cfg, bf16), dim3((unsigned)ctas), dim3(kAttendThreads), (size_t)smem, st, true, mk, mv, a);
  if (e != cudaSuccess || n == 1) return e;                    // (a request and key head of one tile is never cut)
  *launches = 2;
  const int cols = cfg.blocks * kBoxBytes / elt, heads = a.group < 8 ? a.group : 8;
  return launch_k(cols <= 128 ? k_attend_join<1> : k_attend_join<2>, dim3((unsigned)(ctas + ctas / kFewParts * heads)), dim3(kJoinWarps * 32), 0, st, true, a, cfg.tile_heads,
                  cols, ctas, heads);
}

}  // namespace pact
