// The parts of the items of pact_chunk_attention that several CTAs shared, put together: a reference, a sum and unscaled results of each row.
//
// A warp takes 32 rows and 8 columns of an item, a row per lane, so that parts are read 512 bytes at a time; eight parts are asked for at once, since a call with few items has
// many of each and waits for nothing else.
#include "chunk_row.cuh"

namespace pact {
namespace {

constexpr int kChunkJoinThreads = 384, kChunkJoinWarps = kChunkJoinThreads / 32;
static_assert(kChunkJoinThreads >= 2 * kChunkMaxSms, "");

__global__ void __launch_bounds__(kChunkJoinThreads) k_chunk_join(const __grid_constant__ ChunkArgs a, int rows, int width, int G) {
  __shared__ int s_warp[32], s_units[2 * kChunkMaxSms], s_tail[kChunkMaxSms], s_slot[kChunkJoinWarps][kChunkMaxSms + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, groups = (a.d_h + 7) / 8;
  pdl_wait();
  pdl_trigger();
  int units = 0, all;
  if (tid < 2 * G && a.cut[tid].cut) units = (a.cut[tid].rows + 31) / 32 * groups;
  if (tid < G) s_tail[tid] = a.tail[tid];
  const int before = chunk_scan<kChunkJoinThreads>(units, s_warp, &all);
  if (tid < 2 * G) s_units[tid] = before;
  __syncthreads();
  // neighbouring warps are of different CTAs: few units are spread over the device
  for (int u = warp * gridDim.x + blockIdx.x; u < all; u += gridDim.x * kChunkJoinWarps) {
    int q = 0, hi = 2 * G;
    while (hi - q > 1) {
      const int mid = (q + hi) >> 1;
      if (s_units[mid] <= u) q = mid;
      else hi = mid;
    }
    const ChunkCut cut = a.cut[q];
    const int at = u - s_units[q], c0 = at % groups * 8, row = at / groups * 32 + lane;
    // slots of the parts: of the CTA that began the item, if one did, and of those that share the rest
    int *slots = s_slot[warp], n = 0;
    if (cut.head) {
      if (lane == 0) slots[0] = q;
      n = 1;
    }
    for (int c = cut.first; c <= cut.last; c += 32) {
      const bool has = c + lane <= cut.last && s_tail[c + lane] > 0;
      const uint32_t who = __ballot_sync(0xffffffffu, has);
      if (has) slots[n + __popc(who & ((1u << lane) - 1u))] = G + q + c + lane;
      n += __popc(who);
    }
    __syncwarp();
    float top = -INFINITY, l = 0.f, o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.f;
    const bool there = row < cut.rows;
    constexpr int U = 8;
    if (there)
      for (int p = 0; p < n; p += U) {
        float2 ml[U];
        float4 v[U][2];
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (p + k < n) {
            const long long x = slots[p + k];
            ml[k] = a.part_ml[x * rows + row];
            const float4 *from = reinterpret_cast<const float4 *>(a.part_o) + (x * (width / 4) + c0 / 4) * rows + row;
            v[k][0] = from[0];
            v[k][1] = from[rows];                                    // (a part is at least eight columns wide)
          }
        float to = top;
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (p + k < n) to = fmaxf(to, ml[k].x);
        const float f0 = part_weight(top, to);
        top = to;
        l *= f0;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= f0;
#pragma unroll
        for (int k = 0; k < U; ++k)
          if (p + k < n) {
            const float f = part_weight(ml[k].x, top), *y = &v[k][0].x;
            l = fmaf(ml[k].y, f, l);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(i < 4 ? y[i] : (&v[k][1].x)[i - 4], f, o[i]);
          }
      }
    __syncwarp();                                                    // (the slots have been read)
    if (there) {
      const int at_row = cut.first_row + row, token = at_row / a.group, head = cut.kv * a.group + at_row - token * a.group;
      const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= inv;
      const long long to = (cut.row0 + token) * a.ldO + head * a.ldOh + c0;
      if (c0 + 8 <= a.d_h) store8(a, to, o);
      else store4(a, to, make_float4(o[0], o[1], o[2], o[3]));
      if (c0 == 0 && a.lse) a.lse[(cut.row0 + token) * (a.n_kvh * a.group) + head] = l == 0.f ? -INFINITY : top + logf(l);
    }
  }
}

}  // namespace

cudaError_t launch_chunk_join(const ChunkArgs &a, const ChunkCfg &cfg, cudaStream_t st) {
  return launch_k(k_chunk_join, dim3((unsigned)(2 * cfg.ctas)), dim3(kChunkJoinThreads), 0, st, true, a, cfg.rows, cfg.width, cfg.ctas);
}

}  // namespace pact
