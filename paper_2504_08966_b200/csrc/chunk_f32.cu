// Attention of several new tokens per request over a paged cache of fp32 rows (pact_chunk_attention): the formulas of chunk_attention.cu in fp32 multiply-adds.
//
// 4 d_h operations per row of an item and cached row, 128 multiply-adds a clock and SM.  An item is 64 rows (token, head) against tiles of 64 cached rows; a thread of
// 16 x 16 has four rows with four logits each and 4 x 8 columns of the results, so that eight 16-byte loads feed 64 multiply-adds and three feed 32.  Bound by these loads: shared memory
// hands a warp a float per lane and clock, 32 clocks for what four schedulers multiply in 16.  Tiles arrive by 16-byte asynchronous copies, the next one while this one is used.  Warps
// without rows keep step only.  A logit that a token must not see is handed on as the probability -1, beside which values are left out.
//
// Measured: 234 tokens of 32 heads of 128 over 4,731 rows 596 us, 30 TFLOP/s; 16 requests of five tokens over 3,000 rows 194 us (273 us when all warps took part).  Eight rows per thread
// were 547 us in the first case, but 322 us in the second and 46 instead of 43 us for two heads, and were left out.
#include <type_traits>

#include "chunk_row.cuh"

namespace pact {
namespace {

constexpr int kThreads = 256, kRows = 64, kTileF = 64, kMaxD = 128;
constexpr int kPStride = kRows + 4;                                  // floats: rows of probabilities begin in different banks

struct ShapeF32 {
  float q[kRows][kMaxD], k[2][kTileF][kMaxD], v[2][kTileF][kMaxD];   // q, k: 16-byte columns exchanged by the row's last three bits
  float p[kTileF][kPStride];
  float bias[2][kTileF];
  ChunkLineKept line;
};
static_assert(sizeof(ChunkLineSetup) <= sizeof(float) * kTileF * kMaxD, "");

__device__ __forceinline__ void copy16_f32(void *dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ float dot4(const float4 &x, const float4 &y, float s) { return fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, s)))); }

struct PagesF32 {
  const float *K, *V;
  long long k_page, k_head, k_row, v_page, v_head, v_row;
};

// TWO: more than 64 columns
template <bool TWO>
__global__ void __launch_bounds__(kThreads, 1) k_chunk_f32(const __grid_constant__ ChunkArgs a, const __grid_constant__ PagesF32 pages) {
  extern __shared__ __align__(128) char smem_raw[];
  ShapeF32 &sh = *reinterpret_cast<ShapeF32 *>(smem_raw);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  pdl_wait();
  pdl_trigger();
  ChunkCuts cuts;
  ChunkLine line = chunk_line<kThreads, kRows, kTileF>(a, sh.line, *reinterpret_cast<ChunkLineSetup *>(sh.k[0]), cuts);
  if (tid < 32) cuts.write<kRows, kTileF>(a, line);
  ChunkSegment s = {};
  const int chunks = a.d_h / 4;
  // rows [row0, row0 + 64) of a request, those it has; each thread a quarter of a row
  const auto load = [&](int j, int buf) {
    const int row = tid >> 2, pos = j * kTileF + row;
    int id = -1, off = 0;
    if (pos < s.len) {
      const int place = pos / a.page;
      off = pos - place * a.page;
      id = a.table[(long long)s.b * a.width + place];
      if (id < 0 || id >= a.n_pages) {
        id = -1;
        if (a.status && (tid & 3) == 0) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      }
    }
    if (id >= 0) {
      const float *k = pages.K + id * pages.k_page + s.kv * pages.k_head + off * pages.k_row, *v = pages.V + id * pages.v_page + s.kv * pages.v_head + off * pages.v_row;
      for (int c = tid & 3; c < chunks; c += 4) {
        copy16_f32(&sh.k[buf][row][(c ^ (row & 7)) * 4], k + c * 4);
        copy16_f32(&sh.v[buf][row][c * 4], v + c * 4);
      }
    }
    if ((tid & 3) == 0) sh.bias[buf][row] = id < 0 ? -INFINITY : a.logw ? a.logw[(long long)id * a.page + off] : 0.f;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  while (line.next<kRows, kTileF>(a, s)) {
    const int n = s.j1 - s.j0;
    __syncthreads();                                                 // (the segment before is done with the shared memory)
    load(s.j0, 0);
    for (int i = tid; i < kRows * chunks; i += kThreads) {
      const int r = i / chunks, c = i - r * chunks, at = s.first + r, token = at / a.group, head = s.kv * a.group + at - token * a.group;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < s.rows) v = __ldg(reinterpret_cast<const float4 *>(static_cast<const float *>(a.Q) + (s.row0 + token) * a.ldQ + head * a.ldQh + c * 4));
      *reinterpret_cast<float4 *>(&sh.q[r][(c ^ (r & 7)) * 4]) = v;
    }
    const bool idle = tid / 32 * 8 >= s.rows;                        // no row of this warp is there; rows that are not, beside some that are, take part as if they were the last
    int limit[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) limit[i] = s.limit((s.first + min(ty * 4 + i, s.rows - 1)) / a.group, a.causal);
    float m[4], l[4], o[4][TWO ? 8 : 4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < (TWO ? 8 : 4); ++c) o[i][c] = 0.f;
    }
    for (int j = 0; j < n; ++j) {
      const int buf = j & 1, row0 = (s.j0 + j) * kTileF;
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncthreads();
      if (j + 1 < n) load(s.j0 + j + 1, buf ^ 1);
      if (idle) {                                                    // (it only keeps step)
        __syncthreads_and(true);
        __syncthreads();
        continue;
      }
      float x[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = 0.f;
#pragma unroll 4
      for (int c = 0; c < chunks; ++c) {
        float4 q[4], k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4 *>(&sh.q[ty * 4 + i][(c ^ ((ty * 4 + i) & 7)) * 4]);
#pragma unroll
        for (int e = 0; e < 4; ++e) k[e] = *reinterpret_cast<const float4 *>(&sh.k[buf][tx + 16 * e][(c ^ (tx & 7)) * 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i][e] = dot4(q[i], k[e], x[i][e]);
      }
      float bias[4];
      bool all = true;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bias[e] = sh.bias[buf][tx + 16 * e];
#pragma unroll
        for (int i = 0; i < 4; ++i) all = all && bias[e] != -INFINITY && row0 + tx + 16 * e < limit[i];
      }
      const bool whole = __syncthreads_and(all);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bool seen[4];
        float top = -INFINITY;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          seen[e] = bias[e] != -INFINITY && row0 + tx + 16 * e < limit[i];
          x[i][e] = seen[e] ? fmaf(x[i][e], a.scale, bias[e]) : -INFINITY;
          top = fmaxf(top, x[i][e]);
        }
#pragma unroll
        for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        const float to = fmaxf(m[i], top), f = part_weight(m[i], to), ref = to == -INFINITY ? 0.f : to;
        m[i] = to;
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < (TWO ? 8 : 4); ++c) o[i][c] *= f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = ex2_approx((x[i][e] - ref) * kChunkLog2e);
          l[i] += p;
          x[i][e] = seen[e] ? p : -1.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<float4 *>(&sh.p[tx + 16 * e][ty * 4]) = make_float4(x[0][e], x[1][e], x[2][e], x[3][e]);
      __syncthreads();
      const auto add = [&](auto masked) {
#pragma unroll 4
        for (int r = 0; r < kTileF; ++r) {
          const float4 p4 = *reinterpret_cast<const float4 *>(&sh.p[r][ty * 4]);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
          const float4 v0 = *reinterpret_cast<const float4 *>(&sh.v[buf][r][tx * 4]);
          float v[8] = {v0.x, v0.y, v0.z, v0.w, 0.f, 0.f, 0.f, 0.f};
          if constexpr (TWO) {
            const float4 v1 = *reinterpret_cast<const float4 *>(&sh.v[buf][r][64 + tx * 4]);
            v[4] = v1.x; v[5] = v1.y; v[6] = v1.z; v[7] = v1.w;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!decltype(masked)::value || !(p[i] < 0.f))
#pragma unroll
              for (int c = 0; c < (TWO ? 8 : 4); ++c) o[i][c] = fmaf(p[i], v[c], o[i][c]);
        }
      };
      if (whole) add(std::false_type());
      else add(std::true_type());
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
      const int r = ty * 4 + i, at = s.first + r, token = at / a.group, head = s.kv * a.group + at - token * a.group;
      if (r < s.rows) {
        const float inv = s.slot >= 0 ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
        for (int h = 0; h < (TWO ? 2 : 1); ++h) {
          const int c = h * 64 + tx * 4;
          const float4 v = make_float4(o[i][4 * h] * inv, o[i][4 * h + 1] * inv, o[i][4 * h + 2] * inv, o[i][4 * h + 3] * inv);
          if (c >= a.d_h) {
          } else if (s.slot >= 0) {
            reinterpret_cast<float4 *>(a.part_o)[((long long)s.slot * (kMaxD / 4) + c / 4) * kRows + r] = v;
          } else {
            store4(a, (s.row0 + token) * a.ldO + head * a.ldOh + c, v);
          }
        }
        if (tx == 0) {
          if (s.slot >= 0) a.part_ml[(long long)s.slot * kRows + r] = make_float2(m[i], l[i]);
          else if (a.lse) a.lse[(s.row0 + token) * (a.n_kvh * a.group) + head] = l[i] == 0.f ? -INFINITY : m[i] + logf(l[i]);
        }
      }
    }
  }
}

}  // namespace

ChunkFormF32 chunk_form_f32() { return {kRows, kTileF, kMaxD}; }

cudaError_t chunk_configure_f32(const ChunkCfg &cfg, int d_h) {
  return cudaFuncSetAttribute(d_h > 64 ? k_chunk_f32<true> : k_chunk_f32<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ShapeF32));
}

cudaError_t launch_chunk_f32(const ChunkArgs &a, const pact_paged_cache &c, const ChunkCfg &cfg, cudaStream_t st) {
  const PagesF32 pages = {static_cast<const float *>(c.K), static_cast<const float *>(c.V), c.k_page, c.k_head, c.k_row, c.v_page, c.v_head, c.v_row};
  return launch_k(a.d_h > 64 ? k_chunk_f32<true> : k_chunk_f32<false>, dim3((unsigned)cfg.ctas), dim3(kThreads), sizeof(ShapeF32), st, true, a, pages);
}

}  // namespace pact
