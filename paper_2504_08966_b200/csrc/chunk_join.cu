// The parts of the items of pact_chunk_attention that several CTAs shared, put together: a reference, a sum and unscaled results of each row.
#include "chunk_row.cuh"

namespace pact {
namespace {

// Items that were cut.  A warp takes 32 rows and 16 columns of one: a row per lane, so that parts are read 512 bytes at a time.
constexpr int kChunkJoinThreads = 384;
static_assert(kChunkJoinThreads >= 2 * kChunkMaxSms, "");

__global__ void __launch_bounds__(kChunkJoinThreads) k_chunk_join(const __grid_constant__ ChunkArgs a, int rows, int width, int G) {
  __shared__ int s_warp[32], s_units[2 * kChunkMaxSms + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, groups = (a.d_h + 15) / 16;
  pdl_wait();
  pdl_trigger();
  int units = 0, all;
  if (tid < 2 * G && a.cut[tid].cut) units = (a.cut[tid].rows + 31) / 32 * groups;
  const int before = chunk_scan<kChunkJoinThreads>(units, s_warp, &all);
  if (tid < 2 * G) s_units[tid] = before;
  __syncthreads();
  for (int u = blockIdx.x * (kChunkJoinThreads / 32) + warp; u < all; u += gridDim.x * (kChunkJoinThreads / 32)) {
    int q = 0, hi = 2 * G;
    while (hi - q > 1) {
      const int mid = (q + hi) >> 1;
      if (s_units[mid] <= u) q = mid;
      else hi = mid;
    }
    const ChunkCut cut = a.cut[q];
    const int at = u - s_units[q], c4 = at % groups * 4, row = at / groups * 32 + lane;
    const bool there = row < cut.rows;
    const int parts = cut.last - cut.first + 2;                      // the first: of the CTA that began the item, if one did
    const auto slot = [&](int p) { return p == 0 ? (cut.head ? q : -1) : a.tail[cut.first + p - 1] > 0 ? G + q + cut.first + p - 1 : -1; };
    float top = -INFINITY, l = 0.f, o[16];
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const int x = slot(p);
      if (x >= 0 && there) top = fmaxf(top, a.part_ml[(long long)x * rows + row].x);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = 0.f;
#pragma unroll 2
    for (int p = 0; p < parts; ++p) {
      const int x = slot(p);
      if (x < 0 || !there) continue;
      const float2 ml = a.part_ml[(long long)x * rows + row];
      const float4 *from = reinterpret_cast<const float4 *>(a.part_o) + ((long long)x * (width / 4) + c4) * rows + row;
      float4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = from[i * rows];
      const float f = part_weight(ml.x, top);
      l = fmaf(ml.y, f, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[4 * i] = fmaf(v[i].x, f, o[4 * i]);
        o[4 * i + 1] = fmaf(v[i].y, f, o[4 * i + 1]);
        o[4 * i + 2] = fmaf(v[i].z, f, o[4 * i + 2]);
        o[4 * i + 3] = fmaf(v[i].w, f, o[4 * i + 3]);
      }
    }
    if (!there) continue;
    const int at_row = cut.first_row + row, token = at_row / a.group, head = cut.kv * a.group + at_row - token * a.group;
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] *= inv;
    const long long to = (cut.row0 + token) * a.ldO + head * a.ldOh + c4 * 4;
#pragma unroll
    for (int i = 0; i < 16; i += 8) {
      if (c4 * 4 + i + 8 <= a.d_h) store8(a, to + i, o + i);
      else if (c4 * 4 + i < a.d_h) store4(a, to + i, make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]));
    }
    if (c4 == 0 && a.lse) a.lse[(cut.row0 + token) * (a.n_kvh * a.group) + head] = l == 0.f ? -INFINITY : top + logf(l);
  }
}

}  // namespace

cudaError_t launch_chunk_join(const ChunkArgs &a, const ChunkCfg &cfg, cudaStream_t st) {
  return launch_k(k_chunk_join, dim3((unsigned)(2 * cfg.ctas)), dim3(kChunkJoinThreads), 0, st, true, a, cfg.rows, cfg.width, cfg.ctas);
}

}  // namespace pact
