"""Pages that several requests hold, on the host: devices that cannot launch the kernels' cluster."""
import os
import shutil

import pytest

from tests.test_paged_cpu import CSRC, _run


def test_a_device_without_clusters_of_16(tmp_path):
    """The occupancy query and the attributes answer as such a device would: the two calls are refused, no error is left behind for others to find, and a context is as good for everything else."""
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    _run(tmp_path, r"""
#include <stdio.h>
#include <string.h>
#include "context.h"
static cudaError_t attribute = cudaSuccess, occupancy = cudaSuccess, last = cudaSuccess;
static int clusters = 1, asked = 0;
template <typename K> static cudaError_t fake_attribute(K, cudaFuncAttribute, int) { return last = attribute; }
template <typename K> static cudaError_t fake_occupancy(int *n, K, const cudaLaunchConfig_t *lc) {
  if (lc->gridDim.x != 16 || lc->blockDim.x != 1024 || lc->numAttrs != 1 || lc->attrs[0].val.clusterDim.x != 16 || lc->dynamicSmemBytes < 65536) return cudaErrorUnknown;
  ++asked;
  *n = clusters;
  return last = occupancy;
}
static cudaError_t fake_last() { const cudaError_t e = last; last = cudaSuccess; return e; }
static cudaError_t fake_device(int *d) { *d = 0; return cudaSuccess; }
#define cudaFuncSetAttribute fake_attribute
#define cudaOccupancyMaxActiveClusters fake_occupancy
#define cudaGetLastError fake_last
#define cudaGetDevice fake_device
#include "cache_share.cu"
#include "share_api.cu"
namespace pact {
cudaError_t launch_page_copy(const PageCopyArgs &, int, cudaStream_t) { return cudaSuccess; }
}
alignas(256) char buf[1 << 16];
int main() {
  if (!share_fits() || asked != 2) return 1;
  clusters = 0;
  if (share_fits() || last != cudaSuccess) return 2;
  clusters = 1;
  occupancy = cudaErrorInvalidClusterSize;
  if (share_fits() || last != cudaSuccess) return 3;
  occupancy = cudaSuccess;
  attribute = cudaErrorInvalidValue;
  if (share_fits() || last != cudaSuccess) return 4;
  pact_ctx ctx = {};
  ctx.d = 512; ctx.n_qh = 4; ctx.n_kvh = 2; ctx.d_h = 128; ctx.d_k = 256; ctx.in = ctx.out = PACT_BF16; ctx.elt = 2; ctx.paged.blocks = 2; ctx.dev.sm_count = 148;
  ctx.no_share = true;
  int32_t *const W = (int32_t *)buf, *const W2 = (int32_t *)(buf + 4096);
  pact_fork f;
  memset(&f, 0, sizeof f);
  f.page_rows = 32; f.n_pages = 8; f.n_requests = 2; f.max_pages = 4; f.block_table = f.length = f.source = f.shared = f.free_pages = f.n_free = W;
  f.block_table_out = f.length_out = W2; f.shared_out = f.free_out = f.n_free_out = f.copies = f.n_copies = W; f.ws = buf; f.ws_bytes = sizeof buf;
  if (pact_cache_fork(&ctx, &f, nullptr) != PACT_ERR_UNSUPPORTED) return 5;
  f.page_rows = 20;
  if (pact_cache_fork(&ctx, &f, nullptr) != PACT_ERR_INVALID_ARG) return 6;
  pact_compact m;
  memset(&m, 0, sizeof m);
  m.page_rows = 32; m.n_pages = 9; m.n_requests = 2; m.max_pages = 4; m.block_table = m.length = m.shared = m.free_pages = m.n_free = W;
  m.block_table_out = m.shared_out = m.free_out = m.moved_to = m.copies = m.n_copies = W; m.n_list = 4; m.ws = buf; m.ws_bytes = sizeof buf;
  if (pact_cache_compact(&ctx, &m, nullptr) != PACT_ERR_UNSUPPORTED || ctx.launches) return 7;
  return 0;
}""", [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "--expt-relaxed-constexpr", "-I", CSRC])
