// What the kernels of the attention of several new tokens have in common beside their shares: weights of parts, results to memory.
#pragma once
#include "chunk_line.cuh"
#include "umma.cuh"

namespace pact {

constexpr float kChunkLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
// how much a sum with reference m counts beside one with reference `to` (m - to is NaN where both are infinite)
__device__ __forceinline__ float part_weight(float m, float to) { return m == -INFINITY ? 0.f : m == to ? 1.f : ex2_approx((m - to) * kChunkLog2e); }

__device__ __forceinline__ void store8(const ChunkArgs &a, long long at, const float *x) {   // eight columns of a result
  if (a.out_bf16) {
    const uint4 v = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    __nv_bfloat16 *p = static_cast<__nv_bfloat16 *>(a.out) + at;
    if (a.store_bytes >= 16) {
      *reinterpret_cast<uint4 *>(p) = v;
    } else {
      *reinterpret_cast<uint2 *>(p) = make_uint2(v.x, v.y);
      *reinterpret_cast<uint2 *>(p + 4) = make_uint2(v.z, v.w);
    }
  } else {
    float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// sixteen: 32 bytes at a time where they lie so (a lane has a row, and a store of a warp takes as long as it has rows, whatever its width)
__device__ __forceinline__ void store16(const ChunkArgs &a, long long at, const float *x) {
  if (a.store_bytes < 32) {
    store8(a, at, x);
    store8(a, at + 8, x + 8);
    return;
  }
  if (a.out_bf16) {
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<__nv_bfloat16 *>(a.out) + at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float *y = x + 8 * h;
      asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(static_cast<float *>(a.out) + at + 8 * h), "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]),
                   "f"(y[5]), "f"(y[6]), "f"(y[7]) : "memory");
    }
  }
}
__device__ __forceinline__ void store4(const ChunkArgs &a, long long at, const float4 &x) {
  if (a.out_bf16) *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(a.out) + at) = make_uint2(bf16_pair(x.x, x.y), bf16_pair(x.z, x.w));
  else *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = x;
}

}  // namespace pact
