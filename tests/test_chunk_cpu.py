"""Attention of several new tokens and pages that several requests hold, on the host: struct layout, refusals of the C calls and of the binding, the arithmetic that shares out the
attention's work (csrc/chunk_tiles.h), and the plain implementations by hand."""
import os
import shutil

import numpy as np
import pytest
import torch

from oracle import chunk_oracle as co
from oracle import paged_oracle as po
from tests.test_paged_cpu import CSRC, ROOT, _run, _stub_context


def test_struct_layouts(tmp_path):
    from paper_2504_08966_b200 import binding
    out = _run(tmp_path, r"""
#include <stdio.h>
#include <string.h>
#include "pact.h"
template <typename T> void dump(const T &x) {
  for (size_t i = 0; i < sizeof(x); ++i) printf("%02x", ((const unsigned char *)&x)[i]);
  printf("\n");
}
#define P(n) ((char *)0 + n)
#define I(n) ((int32_t *)P(n))
int main() {
  pact_chunk c; memset(&c, 0, sizeof c);
  c.Q = P(1); c.ldQ = 2; c.ldQh = 3; c.block_table = I(4); c.length = I(5); c.n_new = I(6); c.n_new_stride = 7; c.row_start = I(8); c.n_rows = 9; c.row_stride = 10; c.n_requests = 11;
  c.max_pages = 12; c.causal = 13; c.scale = 14; c.out = P(16); c.ldO = 17; c.ldOh = 18; c.lse = (float *)P(19); c.status = I(20); c.ws = P(21); c.ws_bytes = 22;
  dump(c);
  pact_fork f; memset(&f, 0, sizeof f);
  f.page_rows = 1; f.n_pages = 2; f.n_requests = 3; f.max_pages = 4; f.block_table = I(5); f.length = I(6); f.source = I(7); f.rows = I(8); f.shared = I(9); f.free_pages = I(10); f.n_free = I(11);
  f.block_table_out = I(12); f.length_out = I(13); f.shared_out = I(14); f.free_out = I(15); f.n_free_out = I(16); f.copies = I(17); f.n_copies = I(18); f.status = I(19); f.ws = P(20);
  f.ws_bytes = 21;
  dump(f);
  pact_compact k; memset(&k, 0, sizeof k);
  k.page_rows = 1; k.n_pages = 2; k.n_requests = 3; k.max_pages = 4; k.block_table = I(5); k.length = I(6); k.shared = I(7); k.free_pages = I(8); k.n_free = I(9); k.block_table_out = I(10);
  k.shared_out = I(11); k.free_out = I(12); k.moved_to = I(13); k.copies = I(14); k.n_list = 15; k.n_copies = I(17); k.status = I(18); k.ws = P(19); k.ws_bytes = 20;
  dump(k);
  pact_copies p; memset(&p, 0, sizeof p);
  p.copies = I(1); p.n_copies = I(2); p.status = I(3); p.n_list = 4;
  dump(p);
}""", ["g++", "-std=c++17", "-I", os.path.join(ROOT, "include")]).split()
    assert binding._CHUNK.pack(*range(1, 15), 0, *range(16, 23)).hex() == out[0]
    assert binding._FORK.pack(*range(1, 22)).hex() == out[1]
    assert binding._COMPACT.pack(*range(1, 16), 0, *range(17, 21)).hex() == out[2]
    assert binding._COPIES.pack(*range(1, 5), 0).hex() == out[3]


def test_items_and_tiles_are_counted_as_they_are(tmp_path):
    """Sums over the items of a head in closed form against one by one, the tiles of an item against the last row that its tokens see, and the largest numbers."""
    _run(tmp_path, r"""
#include <stdio.h>
#include <stdlib.h>
#include "chunk_tiles.h"
using namespace pact;
#define BAD(...) do { printf(__VA_ARGS__); return 1; } while (0)
int main() {
  srand(1);
  for (int trial = 0; trial < 300000; ++trial) {
    const int rows = trial % 3 == 0 ? 64 : trial % 3 == 1 ? 128 : 256, tile = trial % 2 ? 64 : 128, group = 1 + rand() % (trial % 5 ? 8 : 300);
    ChunkLengths q;
    q.want = rand() % (trial % 7 ? 300 : 3000);
    q.n = trial % 4 ? q.want : rand() % (q.want + 1);                  // (tokens without a row of Q)
    q.len = trial % 6 ? q.want + rand() % 2000 : rand() % (q.want + 1);   // (more tokens than rows)
    const int items = chunk_items(q, group, rows);
    if ((long long)items * rows < (long long)q.n * group || (long long)(items - 1) * rows >= (long long)q.n * group) BAD("items %d of %d x %d\n", items, q.n, group);
    for (int causal = 0; causal < 2; ++causal) {
      unsigned long long sum = 0;
      for (int i = 0; i < items; ++i) {
        const int k = chunk_tiles(q, i, group, rows, tile, causal);
        sum += k;
        long long last = 0;                                             // rows that the last token of the item sees
        for (long long r = (long long)i * rows; r < (long long)(i + 1) * rows && r < (long long)q.n * group; ++r) {
          const long long token = r / group, sees = causal ? q.len - q.want + token + 1 : q.len;
          if (sees > last) last = sees;
        }
        if (last > q.len) BAD("a token sees too much\n");
        if (k < 1 || (long long)k * tile < last) BAD("item %d: %d tiles for %lld rows\n", i, k, last);
        // none that nothing is in, but where all tokens come before the first row
        if (q.len >= q.want && k > 1 && (long long)(k - 1) * tile >= last) BAD("item %d: %d tiles, %lld rows would do with fewer\n", i, k, last);
      }
      if (chunk_tiles_of_head(q, group, rows, tile, causal) != sum) BAD("%llu instead of %llu\n", chunk_tiles_of_head(q, group, rows, tile, causal), sum);
    }
  }
  for (int trial = 0; trial < 20000; ++trial) {
    const unsigned long long n = rand() % 400, m = 1 + rand() % (trial % 2 ? 50 : 1 << 20), a = rand() % (trial % 3 ? 300 : 1 << 24), b = rand() % (1 << 24);
    unsigned long long sum = 0;
    for (unsigned long long i = 0; i < n; ++i) sum += (a * i + b) / m;
    if (floor_sum(n, m, a, b) != sum) BAD("floor_sum(%llu, %llu, %llu, %llu)\n", n, m, a, b);
  }
  // the largest: 2^31 - 1 rows of an item line, cached rows up to 2^31 - 1
  {
    const ChunkLengths q = {INT32_MAX, INT32_MAX, INT32_MAX};
    if (chunk_items(q, 1, 256) != 1 << 23 || chunk_tiles(q, (1 << 23) - 1, 1, 256, 128, true) != 1 << 24 || chunk_tiles(q, 0, 1, 256, 128, true) != 2 || chunk_tiles(q, 5, 1, 256, 128, false) != 1 << 24)
      BAD("largest\n");
    unsigned long long sum = 0;
    for (int i = 0; i < 1 << 23; ++i) sum += chunk_tiles(q, i, 1, 256, 128, true);
    if (chunk_tiles_of_head(q, 1, 256, 128, true) != sum) BAD("largest sum\n");
    const ChunkLengths wide = {1 << 20, 1 << 20, INT32_MAX};
    sum = 0;
    for (int i = 0; i < chunk_items(wide, 2047, 256); ++i) sum += chunk_tiles(wide, i, 2047, 256, 128, true);
    if (chunk_tiles_of_head(wide, 2047, 256, 128, true) != sum) BAD("many heads\n");
  }
  return 0;
}""", ["g++", "-O2", "-std=c++17", "-I", CSRC])


def test_refusals_of_the_c_calls(tmp_path):
    """The host side alone: a context made by hand, and launchers that only count."""
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    main = r"""
#include <math.h>
#include <stdio.h>
#include <string.h>
#include <functional>
#include "context.h"
static int launched, device_now = 0;
static cudaError_t fake_get_device(int *d) { *d = device_now; return cudaSuccess; }
static cudaError_t fake_last_error() { return cudaSuccess; }
#define cudaGetDevice fake_get_device
#define cudaGetLastError fake_last_error
#include "chunk_api.cu"
#include "share_api.cu"
static ChunkArgs seen;
namespace pact {
cudaError_t launch_chunk(ChunkArgs a, const pact_paged_cache &, const ChunkCfg &, cudaStream_t, int *n) { seen = a; ++launched; *n = 2; return cudaSuccess; }
size_t chunk_scratch(const ChunkCfg &cfg, int, ChunkArgs *, char *) { return cfg.blocks ? 4096 : 0; }
size_t fork_scratch(int, int, int, ShareArgs *, char *) { return 4096; }
size_t compact_scratch(int, ShareArgs *, char *) { return 2048; }
cudaError_t launch_cache_fork(const ShareArgs &, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_cache_compact(const ShareArgs &, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_page_copy(const PageCopyArgs &, int, cudaStream_t) { ++launched; return cudaSuccess; }
}
int failures = 0;
void want(const char *what, pact_status got, pact_status wanted, int launches) {
  if (got != wanted || launched != launches) { printf("%s: status %d instead of %d, %d launches\n", what, (int)got, (int)wanted, launched); ++failures; }
  launched = 0;
}
#define GOOD(change) { Args x = ok; change; want(#change, x.call(), PACT_OK, 1); }
#define REFUSED(change) { Args x = ok; change; want(#change, x.call(), PACT_ERR_INVALID_ARG, 0); }
#define UNSUPPORTED(change) { Args x = ok; change; want(#change, x.call(), PACT_ERR_UNSUPPORTED, 0); }
#define WORKSPACE(change) { Args x = ok; change; want(#change, x.call(), PACT_ERR_WORKSPACE, 0); }
alignas(256) char buf[1 << 16];
int32_t *const W = (int32_t *)buf, *const W2 = (int32_t *)(buf + 4096);
struct Args {
  pact_ctx *ctx; pact_paged_cache c; bool cache_null = false; pact_chunk k; pact_fork f; pact_compact m; pact_copies p;
  std::function<pact_status(Args &)> call_;
  pact_status call() { return call_(*this); }
};
int main() {
  pact_ctx ctx = {};
  ctx.d = 512; ctx.n_qh = 4; ctx.n_kvh = 2; ctx.d_h = 128; ctx.d_k = 256; ctx.in = ctx.out = PACT_BF16; ctx.elt = 2; ctx.device = 0;
  ctx.paged.blocks = 2; ctx.dev.sm_count = 148; ctx.chunk.blocks = 2; ctx.chunk.rows = 256; ctx.chunk.tile = 128;
  Args ok;
  ok.ctx = &ctx;
  ok.c = {buf, buf, 2 * 32 * 128, 32 * 128, 128, 2 * 32 * 128, 32 * 128, 128, (float *)buf, buf, (float *)buf, 8, 32};
  memset(&ok.k, 0, sizeof ok.k); memset(&ok.f, 0, sizeof ok.f); memset(&ok.m, 0, sizeof ok.m); memset(&ok.p, 0, sizeof ok.p);
  ok.k.Q = buf; ok.k.ldQ = 512; ok.k.ldQh = 128; ok.k.block_table = ok.k.length = ok.k.n_new = ok.k.row_start = W; ok.k.n_new_stride = 1; ok.k.n_rows = 8; ok.k.n_requests = 2; ok.k.max_pages = 4;
  ok.k.causal = 1; ok.k.scale = 0.1f; ok.k.out = buf; ok.k.ldO = 512; ok.k.ldOh = 128; ok.k.ws = buf; ok.k.ws_bytes = sizeof buf;
  ok.f.page_rows = 32; ok.f.n_pages = 8; ok.f.n_requests = 2; ok.f.max_pages = 4; ok.f.block_table = ok.f.length = ok.f.source = ok.f.shared = ok.f.free_pages = ok.f.n_free = W;
  ok.f.block_table_out = ok.f.length_out = W2; ok.f.shared_out = ok.f.free_out = ok.f.n_free_out = ok.f.copies = ok.f.n_copies = W; ok.f.ws = buf; ok.f.ws_bytes = sizeof buf;
  ok.m.page_rows = 32; ok.m.n_pages = 9; ok.m.n_requests = 2; ok.m.max_pages = 4; ok.m.block_table = ok.m.length = ok.m.shared = ok.m.free_pages = ok.m.n_free = W;
  ok.m.block_table_out = ok.m.shared_out = ok.m.free_out = ok.m.moved_to = ok.m.copies = ok.m.n_copies = W; ok.m.n_list = 4; ok.m.ws = buf; ok.m.ws_bytes = sizeof buf;
  ok.p.copies = W; ok.p.n_list = 3;
  if (pact_chunk_attention(&ctx, nullptr, nullptr, nullptr) != -1 || pact_chunk_attention(nullptr, nullptr, nullptr, nullptr) != -1 || pact_cache_fork(&ctx, nullptr, nullptr) != -1 ||
      pact_cache_compact(&ctx, nullptr, nullptr) != -1 || pact_page_copy(&ctx, nullptr, nullptr, nullptr) != -1)
    return 1;
  if (pact_chunk_workspace_bytes(nullptr, 1) || pact_chunk_workspace_bytes(&ctx, 0) || pact_chunk_workspace_bytes(&ctx, PACT_MAX_REQUESTS + 1) || pact_chunk_workspace_bytes(&ctx, 5) != 4096) return 1;
  if (pact_share_workspace_bytes(nullptr, 1, 1, 1) || pact_share_workspace_bytes(&ctx, 0, 1, 1) || pact_share_workspace_bytes(&ctx, 1, 0, 1) || pact_share_workspace_bytes(&ctx, 1, 1, 0) ||
      pact_share_workspace_bytes(&ctx, PACT_MAX_REQUESTS + 1, 1, 1) || pact_share_workspace_bytes(&ctx, 1, 1, 1) != 4096)
    return 1;
  // n / page by a multiplication, up to the ends of its range
  for (int page = 16; page <= 1024; page += 16)
    for (unsigned k = 0; k <= ((1u << 31) + 1024) / page; k += k < 3000 ? 1 : 977)
      for (unsigned n : {k * page, k * page + page / 2, k * page + page - 1, (1u << 31) - 1 - k, (1u << 31) + 1023 - k % 1024})
        if (n < (1u << 31) + 1024 && page_of(page_mul_of(page), n) != (int)(n / page)) { printf("%u / %d\n", n, page); return 1; }
  const auto with_cache = [&] {
    REFUSED(x.ctx = nullptr) REFUSED(x.cache_null = true) REFUSED(x.c.K = nullptr) REFUSED(x.c.V = nullptr) REFUSED(x.c.K = buf + 8) REFUSED(x.c.k_row = 120) REFUSED(x.c.k_row = 129)
    REFUSED(x.c.v_head = 0) REFUSED(x.c.v_page = -4096) UNSUPPORTED(x.c.k_page = 1ll << 40) REFUSED(x.c.logw = (float *)(buf + 4)) REFUSED(x.c.bounds = nullptr) REFUSED(x.c.n_pages = 0)
    REFUSED(x.c.page_rows = 24) REFUSED(x.c.page_rows = 1040)
    device_now = 1;
    REFUSED((void)x)
    device_now = 0;
  };
  // ---- attention
  ok.call_ = [](Args &x) { return pact_chunk_attention(x.ctx, x.cache_null ? nullptr : &x.c, &x.k, nullptr); };
  GOOD((void)x) GOOD(x.c.bounds = nullptr; x.c.w_max = nullptr; x.c.logw = nullptr) GOOD(x.k.row_start = nullptr; x.k.row_stride = 4) GOOD(x.k.causal = 0) GOOD(x.k.scale = -1.f) GOOD(x.k.scale = 0.f)
  GOOD(x.k.n_rows = 0; x.k.Q = nullptr; x.k.out = nullptr) GOOD(x.k.ldO = 1 << 20; x.k.ldOh = 132) GOOD(x.k.out = buf + 8)
  if (seen.store_bytes != 8 || seen.group != 2 || seen.polls != ctx.copy_polls) return 1;
  with_cache();
  REFUSED(x.k.Q = nullptr) REFUSED(x.k.Q = buf + 2) REFUSED(x.k.ldQ = 0) REFUSED(x.k.ldQh = 127) REFUSED(x.k.ldQh = 132) REFUSED(x.k.block_table = nullptr) REFUSED(x.k.length = nullptr)
  REFUSED(x.k.n_new = nullptr) REFUSED(x.k.n_new_stride = 0) REFUSED(x.k.row_start = nullptr) REFUSED(x.k.row_stride = 4) REFUSED(x.k.row_start = nullptr; x.k.row_stride = 3)
  REFUSED(x.k.row_stride = -4) REFUSED(x.k.n_rows = -1) REFUSED(x.k.causal = 2) REFUSED(x.k.causal = -1) REFUSED(x.k.scale = NAN) REFUSED(x.k.scale = -INFINITY) REFUSED(x.k.out = nullptr)
  REFUSED(x.k.out = buf + 4) REFUSED(x.k.ldO = 100) REFUSED(x.k.ldOh = 130) REFUSED(x.k.n_requests = 0) REFUSED(x.k.max_pages = 0) UNSUPPORTED(x.k.n_requests = PACT_MAX_REQUESTS + 1)
  UNSUPPORTED(x.k.max_pages = 1 << 27) UNSUPPORTED(x.k.n_rows = 1ll << 30) UNSUPPORTED(x.k.n_rows = 1ll << 62) UNSUPPORTED(x.k.n_rows = 1ll << 28; x.k.max_pages = 1 << 20)
  WORKSPACE(x.k.ws = nullptr) WORKSPACE(x.k.ws = buf + 16) WORKSPACE(x.k.ws_bytes = 100)
  ctx.chunk.blocks = 0;
  UNSUPPORTED((void)x)
  if (pact_chunk_workspace_bytes(&ctx, 5)) return 1;
  ctx.chunk.blocks = 2;
  // ---- fork
  ok.call_ = [](Args &x) { return pact_cache_fork(x.ctx, &x.f, nullptr); };
  GOOD((void)x) GOOD(x.f.rows = W) GOOD(x.f.status = W)
  REFUSED(x.ctx = nullptr) REFUSED(x.f.page_rows = 20) REFUSED(x.f.page_rows = 0) REFUSED(x.f.n_pages = 0) REFUSED(x.f.n_requests = 0) REFUSED(x.f.max_pages = 0)
  UNSUPPORTED(x.f.n_requests = PACT_MAX_REQUESTS + 1) UNSUPPORTED(x.f.max_pages = 1 << 27) UNSUPPORTED(x.f.n_requests = 4096; x.f.max_pages = 1 << 20)
  REFUSED(x.f.block_table = nullptr) REFUSED(x.f.length = nullptr) REFUSED(x.f.source = nullptr) REFUSED(x.f.shared = nullptr) REFUSED(x.f.free_pages = nullptr) REFUSED(x.f.n_free = nullptr)
  REFUSED(x.f.block_table_out = nullptr) REFUSED(x.f.length_out = nullptr) REFUSED(x.f.shared_out = nullptr) REFUSED(x.f.free_out = nullptr) REFUSED(x.f.n_free_out = nullptr)
  REFUSED(x.f.copies = nullptr) REFUSED(x.f.n_copies = nullptr) REFUSED(x.f.block_table_out = W) REFUSED(x.f.length_out = W)
  WORKSPACE(x.f.ws = nullptr) WORKSPACE(x.f.ws = buf + 4) WORKSPACE(x.f.ws_bytes = 4095)
  device_now = 1;
  REFUSED((void)x)
  device_now = 0;
  // ---- compaction
  ok.call_ = [](Args &x) { return pact_cache_compact(x.ctx, &x.m, nullptr); };
  GOOD((void)x) GOOD(x.m.n_pages = 1; x.m.n_list = 0)
  REFUSED(x.ctx = nullptr) REFUSED(x.m.page_rows = 20) REFUSED(x.m.n_pages = 0) REFUSED(x.m.n_requests = 0) REFUSED(x.m.max_pages = 0) UNSUPPORTED(x.m.n_requests = 4096; x.m.max_pages = 1 << 20)
  REFUSED(x.m.block_table = nullptr) REFUSED(x.m.length = nullptr) REFUSED(x.m.shared = nullptr) REFUSED(x.m.free_pages = nullptr) REFUSED(x.m.n_free = nullptr)
  REFUSED(x.m.block_table_out = nullptr) REFUSED(x.m.shared_out = nullptr) REFUSED(x.m.free_out = nullptr) REFUSED(x.m.moved_to = nullptr) REFUSED(x.m.copies = nullptr)
  REFUSED(x.m.n_copies = nullptr) REFUSED(x.m.n_list = 3) REFUSED(x.m.n_list = -1) WORKSPACE(x.m.ws = nullptr) WORKSPACE(x.m.ws = buf + 4) WORKSPACE(x.m.ws_bytes = 2047)
  device_now = 1;
  REFUSED((void)x)
  device_now = 0;
  // ---- copies
  ok.call_ = [](Args &x) { return pact_page_copy(x.ctx, x.cache_null ? nullptr : &x.c, &x.p, nullptr); };
  GOOD((void)x) GOOD(x.p.n_copies = W; x.p.status = W)
  { Args x = ok; x.p.n_list = 0; x.p.copies = nullptr; want("no entries", x.call(), PACT_OK, 0); }
  with_cache();
  REFUSED(x.p.n_list = -1) REFUSED(x.p.copies = nullptr)
  ctx.paged.blocks = 0;
  UNSUPPORTED((void)x)
  return failures;
}"""
    _run(tmp_path, main, [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "--expt-relaxed-constexpr", "-I", CSRC])


def _stub(n_kvh=2):
    ctx = _stub_context(n_kvh=n_kvh)
    ctx._chunk_workspace = lambda: (0, 0, None)
    ctx._share_workspace = lambda B, W, P: (0, 0, None)
    return ctx


def _refused(call, *args, word="wanted", **kw):
    from paper_2504_08966_b200 import binding as pb
    with pytest.raises(pb.PactError, match=word):
        call(*args, **kw)


NULL = "status -1"                                            # past the checks of the binding: the library sees the null handle


def test_refusals_of_the_binding(monkeypatch):
    from paper_2504_08966_b200 import binding as pb
    monkeypatch.setattr(pb, "_stream", lambda: 0)
    ctx, bf, i32 = _stub(), torch.bfloat16, torch.int32
    K = torch.zeros(6, 2, 16, 64, dtype=bf)
    cache = pb.PagedCache(K, K.clone())
    good = dict(Q=torch.zeros(7, 4, 64, dtype=bf), block_table=torch.zeros(3, 5, dtype=i32), length=torch.zeros(3, dtype=i32), n_new=torch.zeros(3, 2, dtype=i32)[:, 1], out=torch.zeros(7, 4, 64),
                row_start=torch.zeros(4, dtype=i32), lse=torch.zeros(7, 4), status=torch.zeros(1, dtype=i32))

    def call(cache=cache, ctx=ctx, **change):
        kw = {**good, **change}
        ctx.pact_chunk_attention(cache, *(kw.pop(k) for k in ("Q", "block_table", "length", "n_new", "out")), **kw)

    _refused(call, word=NULL)
    _refused(call, row_start=good["row_start"][:3], lse=None, status=None, word=NULL)
    _refused(call, Q=torch.zeros(7, 5, 72, dtype=bf)[:, :4, :64], out=torch.zeros(7, 5, 72)[:, :4, :64], word=NULL)
    _refused(call, Q=good["Q"].float())
    _refused(call, Q=good["Q"][:, :3])
    _refused(call, Q=torch.zeros(7, 64, 4, dtype=bf).transpose(1, 2), word="contiguous")
    _refused(call, out=good["out"][:6])
    _refused(call, out=good["out"].to(bf))
    _refused(call, out=torch.zeros(7, 4, 128)[..., ::2], word="contiguous")
    _refused(call, block_table=good["block_table"].long())
    _refused(call, block_table=good["block_table"].T)
    _refused(call, block_table=good["block_table"][0])
    _refused(call, length=good["length"][:2])
    _refused(call, n_new=good["n_new"].long())
    _refused(call, n_new=good["n_new"][:2])
    _refused(call, row_start=good["row_start"][:2])
    _refused(call, row_start=good["row_start"].long())
    _refused(call, lse=good["lse"][:, :3])
    _refused(call, lse=good["lse"].double())
    _refused(call, status=torch.zeros(2, dtype=i32))
    other = _stub(n_kvh=1)
    _refused(call, ctx=other, word="not one of")

    P, B = 6, 3
    one, pages, per = torch.zeros(1, dtype=i32), torch.zeros(P, dtype=i32), torch.zeros(B, dtype=i32)
    table = good["block_table"]
    fork = dict(block_table=table, length=per, source=per, shared=pages, free_pages=pages, n_free=one, block_table_out=table.clone(), length_out=per.clone(), shared_out=pages, free_out=pages,
                n_free_out=one, copies=torch.zeros(B, 3, dtype=i32), n_copies=one, rows=per, status=one)
    _refused(lambda: ctx.pact_cache_fork(16, **fork), word=NULL)
    _refused(lambda: ctx.pact_cache_fork(16, **{**fork, "rows": None, "status": None}), word=NULL)
    for name, x in fork.items():
        _refused(lambda: ctx.pact_cache_fork(16, **{**fork, name: x.long()}))
        _refused(lambda: ctx.pact_cache_fork(16, **{**fork, name: torch.zeros(x.numel() + 1, dtype=i32)}))
        _refused(lambda: ctx.pact_cache_fork(16, **{**fork, name: torch.zeros(*x.shape, 2, dtype=i32)[..., 0]})) if x.numel() > 1 else None
    compact = dict(block_table=table, length=per, shared=pages, free_pages=pages, n_free=one, block_table_out=table, shared_out=pages, free_out=pages, moved_to=pages,
                   copies=torch.zeros(3, 3, dtype=i32), n_copies=one, status=one)
    _refused(lambda: ctx.pact_cache_compact(16, **compact), word=NULL)
    for name, x in compact.items():
        _refused(lambda: ctx.pact_cache_compact(16, **{**compact, name: x.long()}))
        _refused(lambda: ctx.pact_cache_compact(16, **{**compact, name: torch.zeros(x.numel() + 1, dtype=i32)}))
    entries = torch.zeros(4, 3, dtype=i32)
    _refused(ctx.pact_page_copy, cache, entries, word=NULL)
    _refused(ctx.pact_page_copy, cache, entries, one, one, word=NULL)
    _refused(ctx.pact_page_copy, cache, entries.long())
    _refused(ctx.pact_page_copy, cache, entries[:, :2])
    _refused(ctx.pact_page_copy, cache, entries[0])
    _refused(ctx.pact_page_copy, cache, entries, torch.zeros(2, dtype=i32))
    _refused(other.pact_page_copy, cache, entries, word="not one of")


def test_workspaces_that_are_outgrown_are_kept(monkeypatch):
    """A captured graph goes on with the one it was recorded with; the attention's is one for all calls."""
    ctx = _stub_context()
    monkeypatch.setattr(type(ctx), "_cuda", lambda self: torch.device("cpu"))
    ctx._share_ws, ctx._share_need, ctx._chunk_ws = [], {(1, 1, 1): 1000, (4, 1, 1): 1500, (9, 1, 1): 9000}, None
    got = [ctx._share_workspace(b, 1, 1) for b in (1, 4, 1, 9, 4)]
    assert [n for _, n, _ in got] == [1000, 2000, 2000, 9000, 9000]
    assert len({a for a, _, _ in got}) == 3 and len(ctx._share_ws) == 3
    assert ctx._chunk_workspace() is ctx._chunk_workspace()


# ---- the plain implementations ------------------------------------------------------------------------------------------

def test_oracle_attention_by_hand():
    K, V = np.zeros((2, 1, 16, 4)), np.arange(128.0).reshape(2, 1, 16, 4)
    q, table = np.zeros((5, 2, 4)), np.array([[1, 0]])
    touched, out, lse, _, _ = co.attend(q, K, V, None, table, [18], [3], [1], 16, 1.0, True, 5)
    rows = np.concatenate([V[1, 0], V[0, 0]])
    assert list(touched) == [False, True, True, True, False] and not out[0].any() and lse[0, 0] == -np.inf
    for i in range(3):                                        # tokens 15, 16 and 17 see 16, 17 and 18 rows, all alike
        assert np.allclose(out[1 + i], rows[:16 + i].mean(0)) and np.allclose(lse[1 + i], np.log(16 + i))
    _, out, _, _, _ = co.attend(q, K, V, None, table, [18], [3], [1], 16, 1.0, False, 5)
    assert np.allclose(out[1:4], rows[:18].mean(0))
    w = np.full((2, 16), -np.inf)
    w[0, 1] = 5.0                                             # one row counts, which is the last token's own
    _, out, lse, _, _ = co.attend(q, K, V, w, table, [18], [3], [1], 16, 1.0, True, 5)
    assert not out[1:3].any() and np.array_equal(out[3, 1], V[0, 0, 1]) and lse[3, 1] == 5.0 and (lse[1:3] == -np.inf).all()
    touched, out, lse, _, _ = co.attend(q, K, V, None, table, [2], [4], [0], 16, 1.0, True, 5)      # more new tokens than rows: the first two see nothing
    assert not out[:2].any() and np.array_equal(out[2, 0], V[1, 0, 0]) and (lse[:2] == -np.inf).all()
    assert list(touched) == [True] * 4 + [False]
    touched = co.attend(q, K, V, None, np.array([[1, 9], [0, 1]]), [18, 18], [9, 2], [0, 4], 16, 1.0, True, 5, 3)[0]       # three rows of Q each, and one that is there
    assert list(touched) == [True, True, True, False, True]


def test_oracle_fork_by_hand():
    table, F = np.array([[5, 6, 7], [3, -1, -1], [-1, -1, -1]]), [0, 1, 2, 4]
    # request 0 goes on in 0 and 2, request 1 ends; both end in page 7: the first keeps it, the other takes the page that request 1 gave back
    r = co.fork(16, table, [40, 10, 0], [0, -1, 0], None, [0] * 8, F, 4)
    assert r == (po.OK, [[5, 6, 7], [], [5, 6, 3]], [40, 0, 40], [0, 0, 0, 0, 0, 1, 1, 0], [0, 1, 2, 4], [[7, 3, 8]])
    # cut at a page's end: nothing to copy, and what is behind goes back in the order of its places
    r = co.fork(16, table, [40, 10, 0], [0, 1, 0], [16, 10, 32], [0] * 8, F, 4)
    assert r == (po.OK, [[5], [3], [5, 6]], [16, 10, 32], [0, 0, 0, 0, 0, 1, 0, 0], [0, 1, 2, 4, 7], [])
    # a page that somebody else holds is not kept for writing, and does not go back
    r = co.fork(16, table, [40, 10, 0], [0, -1, -1], [24, 0, 0], [0, 0, 0, 0, 0, 0, 1, 0], F, 4)
    assert r == (po.OK, [[5, 3], [], []], [24, 0, 0], [0] * 8, [0, 1, 2, 4, 7], [[6, 3, 8]])
    assert co.fork(16, table, [40, 10, 0], [0, 1, 0], None, [0] * 8, F, 0)[0] == po.NO_PAGES
    assert co.fork(16, table, [40, 10, 0], [0, 1, 3], None, [0] * 8, F, 4)[0] == po.INVALID


def test_oracle_compaction_by_hand():
    table, shared = np.array([[5, 1, -1], [5, 6, -1]]), [0, 0, 0, 0, 0, 1, 0, 0]
    # used: 1, 5, 6; free: 0, 2, 3, 4, 7.  5 goes to 0 and 6 to 2
    r = co.compact(16, table, [32, 20], shared, [4, 7, 0, 3, 2], 5)
    assert r == (po.OK, [[0, 1], [0, 2]], [1, 0, 0, 0, 0, 0, 0, 0], [7, 6, 5, 4, 3], [0, 1, 2, 3, 4, 0, 2, 7], [[5, 0, 16], [6, 2, 16]])
    assert co.compact(16, table, [32, 20], shared, [4, 4], 2)[0] == po.INVALID
