// Rows of pages onto other pages (pact_page_copy), for one layer: keys, values, biases and bounds.
//
// Bound by memory: a warp takes the rows of one head of K or of V of a copy, which lie together or at one stride, 16 bytes a lane and eight of them under way at once.  The number of copies is known
// on the device only, so a fixed grid goes through them.
#include "share.cuh"

namespace pact {
namespace {

constexpr int kCopyThreads = 256, kCopyWarps = kCopyThreads / 32, kUnder = 8;

// `rows` rows of `vecs` 16-byte vectors, `from_row` and `to_row` bytes apart
__device__ __forceinline__ void copy_rows(const char *from, char *to, long long stride, int rows, int vecs, int lane) {
  const bool together = stride == (long long)vecs * 16;
  const int n = rows * vecs;
  for (int i0 = lane; i0 < n; i0 += 32 * kUnder) {
    uint4 v[kUnder];
    long long at[kUnder];
#pragma unroll
    for (int u = 0; u < kUnder; ++u) {
      const int i = i0 + 32 * u;
      at[u] = (long long)i * 16;
      if (!together) {
        const int r = i / vecs;
        at[u] = r * stride + (i - r * vecs) * 16;
      }
      if (i < n) v[u] = *reinterpret_cast<const uint4 *>(from + at[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnder; ++u)
      if (i0 + 32 * u < n) *reinterpret_cast<uint4 *>(to + at[u]) = v[u];
  }
}

__global__ void __launch_bounds__(kCopyThreads) k_page_copy(const __grid_constant__ PageCopyArgs a) {
  const int lane = threadIdx.x & 31, warps = gridDim.x * kCopyWarps;
  pdl_wait();
  pdl_trigger();
  const int n = min(max(a.n_copies ? *a.n_copies : a.n_list, 0), a.n_list), parts = 2 * a.n_kvh + 1;
  const int vecs = a.d_h * a.elt / 16;
  for (long long u = blockIdx.x * kCopyWarps + (threadIdx.x >> 5); u < (long long)n * parts; u += warps) {
    const int k = (int)(u / parts), part = (int)(u - (long long)k * parts);
    const int from = a.copies[3 * k], to = a.copies[3 * k + 1], rows = a.copies[3 * k + 2];
    if (from < 0 || rows <= 0) continue;
    if (from >= a.n_pages || to < 0 || to >= a.n_pages || rows > a.page || from == to) {
      if (lane == 0 && part == 0 && a.status) atomicMin(a.status, (int)PACT_ERR_INVALID_ARG);
      continue;
    }
    if (part < 2 * a.n_kvh) {
      const bool of_v = part >= a.n_kvh;
      const long long page = of_v ? a.v_page : a.k_page, row = (of_v ? a.v_row : a.k_row) * a.elt, head = (part - (of_v ? a.n_kvh : 0)) * (of_v ? a.v_head : a.k_head);
      char *base = static_cast<char *>(of_v ? a.V : a.K);
      copy_rows(base + (from * page + head) * a.elt, base + (to * page + head) * a.elt, row, rows, vecs, lane);
    } else {
      if (a.logw)                          // (a page is a multiple of 16 rows)
        for (int r = lane; r < rows; r += 32) a.logw[(long long)to * a.page + r] = a.logw[(long long)from * a.page + r];
      if (a.bounds) {
        const long long bytes = 2ll * a.n_kvh * a.d_h * a.elt;
        char *base = static_cast<char *>(a.bounds);
        copy_rows(base + from * bytes, base + to * bytes, bytes, 1, (int)(bytes / 16), lane);
        if (lane == 0) a.w_max[to] = a.w_max[from];
      }
    }
  }
}

}  // namespace

cudaError_t launch_page_copy(const PageCopyArgs &a, int sm_count, cudaStream_t st) {
  const long long units = (long long)a.n_list * (2 * a.n_kvh + 1), ctas = (units + kCopyWarps - 1) / kCopyWarps, most = (long long)sm_count * (2048 / kCopyThreads);
  return launch_k(k_page_copy, dim3((unsigned)(ctas < most ? ctas : most)), dim3(kCopyThreads), 0, st, true, a);
}

}  // namespace pact
