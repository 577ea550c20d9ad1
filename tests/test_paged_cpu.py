"""The paged cache on the host: struct layout, refusals of the C calls and of the binding, and the arithmetic that shares out the attention's
work and finds its rows (csrc/paged_tiles.h), gone through with bad page ids among them."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_08966_b200", "csrc")


def _run(tmp_path, text, cmd):
    src, exe = tmp_path / ("t.cu" if "nvcc" in cmd[0] else "t.cpp"), str(tmp_path / "t")
    src.write_text(text)
    subprocess.check_call(cmd + [str(src), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_struct_layouts(tmp_path):
    """The binding packs the three argument structs with the struct module and the cache with ctypes."""
    from paper_2504_08966_b200 import binding
    out = _run(tmp_path, r"""
#include <stdio.h>
#include <stddef.h>
#include <string.h>
#include "pact.h"
template <typename T> void dump(const T &x) {
  for (size_t i = 0; i < sizeof(x); ++i) printf("%02x", ((const unsigned char *)&x)[i]);
  printf("\n");
}
#define P(n) ((char *)0 + n)
int main() {
  pact_paged_cache c; memset(&c, 0, sizeof c);
  c.K = P(1); c.V = P(2); c.k_page = 3; c.k_head = 4; c.k_row = 5; c.v_page = 6; c.v_head = 7; c.v_row = 8; c.logw = (float *)P(9); c.bounds = P(10); c.w_max = (float *)P(11);
  c.n_pages = 12; c.page_rows = 13;
  dump(c);
  pact_plan p; memset(&p, 0, sizeof p);
  p.page_rows = 1; p.n_pages = 2; p.n_requests = 3; p.max_pages = 4; p.block_table = (int32_t *)P(5); p.length = (int32_t *)P(6); p.n_new = (int32_t *)P(7); p.n_new_stride = 8;
  p.free_pages = (int32_t *)P(9); p.n_free = (int32_t *)P(10); p.length_out = (int32_t *)P(11); p.n_free_out = (int32_t *)P(12); p.row_start = (int32_t *)P(13); p.slot = (int64_t *)P(14);
  p.n_rows = 15; p.row_stride = 16; p.status = (int32_t *)P(18);
  dump(p);
  pact_new_rows r; memset(&r, 0, sizeof r);
  r.K = P(1); r.V = P(2); r.ld_row = 3; r.ld_head = 4; r.logw = (float *)P(5); r.slot = (int64_t *)P(6); r.n_rows = 7; r.status = (int32_t *)P(8);
  dump(r);
  pact_query q; memset(&q, 0, sizeof q);
  q.Q = P(1); q.ldQ = 2; q.ldQh = 3; q.block_table = (int32_t *)P(4); q.length = (int32_t *)P(5); q.n_requests = 6; q.max_pages = 7; q.selected = (int32_t *)P(8); q.n_select = 9;
  q.n_first = 10; q.n_last = 11; q.scale = 12; q.out = P(13); q.ldO = 14; q.ldOh = 15; q.lse = (float *)P(16); q.status = (int32_t *)P(17); q.ws = P(18); q.ws_bytes = 19;
  dump(q);
}""", ["g++", "-I", os.path.join(ROOT, "include")]).split()
    assert bytes(binding.PagedCacheDesc(*range(1, 14))).hex() == out[0]
    assert binding._PLAN.pack(*range(1, 17), 0, 18).hex() == out[1]
    assert binding._NEW_ROWS.pack(*range(1, 9)).hex() == out[2]
    assert binding._QUERY.pack(*range(1, 20)).hex() == out[3]


def test_status_text():
    from paper_2504_08966_b200 import binding, build
    build.build()
    assert b"free pages" in binding.lib().pact_status_string(-6)


def test_every_tile_has_one_owner_and_every_row_is_found_once(tmp_path):
    _run(tmp_path, r"""
#include <stdio.h>
#include <stdlib.h>
#include <vector>
#include "paged_tiles.h"
using namespace pact;
#define BAD(...) do { printf(__VA_ARGS__); return 1; } while (0)
int main() {
  // shares: together all tiles, sizes that differ by one at most, and the owner of a tile is the share it lies in
  const long long Gs[] = {1, 2, 3, 7, 148, 296};
  for (long long G : Gs)
    for (long long T = G; T < 5000; T += T < 1200 ? 1 : 97) {
      if (share_begin(0, G, T) != 0 || share_begin(G, G, T) != T) BAD("ends %lld %lld\n", G, T);
      for (long long i = 0; i < G; ++i) {
        const long long a = share_begin(i, G, T), b = share_begin(i + 1, G, T);
        if (b - a < T / G || b - a > T / G + 1 || b <= a) BAD("share %lld of %lld in %lld\n", i, T, G);
        for (long long t = a; t < b; ++t)
          if (share_of(t, G, T) != i) BAD("owner of %lld, %lld in %lld\n", t, T, G);
      }
    }
  for (long long T : {1ll << 31, (1ll << 33) + 12345, 1ll << 40})                    // far beyond 32 bits
    for (long long i = 0; i < 296; ++i)
      for (long long t : {share_begin(i, 296, T), share_begin(i + 1, 296, T) - 1})
        if (share_of(t, 296, T) != i) BAD("owner, long\n");
  for (int trial = 0; trial < 2000000; ++trial) {
    const int n = trial % 2 ? 1 + rand() % 1000 : 1 + rand() % (1 << 26), h = rand() % 256;
    const long long u = (long long)h * n + (trial % 5 == 0 ? 0 : trial % 5 == 1 ? n - 1 : rand() % n);
    int rest;
    if (divide_small(u, n, &rest) != h || rest != u - (long long)h * n) BAD("%lld / %d\n", u, n);
    if (u <= 0x7fffffff && (divide_small((int)u, n, &rest) != h || rest != u - (long long)h * n)) BAD("%lld / %d, 32 bits\n", u, n);
  }
  // the ends of the range: a request of almost 2^31 rows
  {
    const int32_t last[1] = {5};
    std::vector<int32_t> table((1 << 21) - 1, 3);
    const int len = ((1 << 21) - 1) * 1024, j = tiles_of_request(len, 1024, false, 0) - 1;
    const TileRows t = locate_rows(j, len, 1024, 4, table.data(), 4, nullptr, 0);
    if (t.bad || t.id[0] != 3 || t.off[0] != 960 || t.rows != 0x10101010u) BAD("last tile\n");
    const TileRows s = locate_rows(0, len, 1024, 4, table.data(), 4, last, 1);
    if (s.bad || s.id[0] != 3 || s.rows != 0x10101010u) BAD("listed\n");
  }
  // rows: whatever page size, length, list of pages and bad ids, every row that counts is found exactly once, none else, ids stay inside the cache
  srand(1);
  for (int trial = 0; trial < 60000; ++trial) {
    const int page = 16 * (1 + rand() % (trial % 3 ? 8 : 64)), box = page % 64 == 0 ? 4 : page % 32 == 0 ? 2 : 1;
    const int width = 1 + rand() % 9, n_pages = 1 + rand() % 30;
    const int len = rand() % 4 == 0 ? width * page : rand() % (width * page + 1);
    const bool sel = rand() % 2;
    const int n_select = sel ? 1 + rand() % 12 : 0;
    std::vector<int32_t> table(width), list(n_select);
    for (auto &x : table) x = rand() % 9 ? rand() % n_pages : rand() % 2 ? -1 - rand() % 3 : n_pages + rand() % 5;
    for (auto &x : list) x = rand() % 9 ? rand() % width : rand() % 2 ? -1 : width + rand() % 5;
    const int pages = (len + page - 1) / page;
    const int listed = sel && n_select < pages ? n_select : pages;
    const int tiles = tiles_of_request(len, page, sel, n_select);
    if ((len == 0) != (tiles == 0) && !sel) BAD("no tiles\n");
    long long at = 0;                                         // the row of the list of pages that comes next
    bool bad = false, bad_seen = false;
    for (int j = 0; j < tiles; ++j) {
      const TileRows t = locate_rows(j, len, page, box, table.data(), n_pages, sel ? list.data() : nullptr, n_select);
      bad_seen = bad_seen || t.bad;
      for (int r = 0; r < kTile; ++r, ++at) {
        const int g = r / 16, g0 = g / box * box, n = t.rows >> (8 * g) & 255;
        const bool counts = r % 16 < n;
        long long place = at / page;
        place = place < listed ? (sel ? list[place] : place) : -1;
        bool want = place >= 0 && place < pages && place * page + at % page < len;
        if (want && !(table[place] >= 0 && table[place] < n_pages)) { want = false; bad = true; }
        if (n > 16 || counts != want) BAD("row %lld: %d, %d\n", at, counts, want);
        if (counts && (t.id[g0] != table[place] || t.off[g0] + r - 16 * g0 != at % page || t.off[g0] + 16 * box > page)) BAD("place of row %lld\n", at);
        // a box is copied if its first 16 rows have one that counts; then no other 16 of it may count without it
        if (n && !(t.rows >> (8 * g0) & 255)) BAD("box of row %lld\n", at);
      }
    }
    if (bad != bad_seen) BAD("bad ids\n");
    for (; at < (long long)listed * page; ++at)              // past the last tile only places behind the request's rows are left
      if (sel || at < len) BAD("rows past the last tile\n");
  }
}""", ["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC])


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
#include "paged_api.cu"
namespace pact {
cudaError_t launch_cache_plan(PlanArgs, int, cudaStream_t, int *n) { ++launched; *n = 1; return cudaSuccess; }
cudaError_t launch_cache_write(const WriteArgs &, bool, int, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_page_select(const SelectArgs &, bool, int, int, cudaStream_t) { ++launched; return cudaSuccess; }
cudaError_t launch_attend(AttendArgs, const pact_paged_cache &, const PagedCfg &, const DeviceCfg &, bool, cudaStream_t, int *n) { ++launched; *n = 2; return cudaSuccess; }
size_t attend_scratch(const PagedCfg &, const DeviceCfg &, bool, AttendArgs *, char *) { return 4096; }
}
int failures = 0;
void want(const char *what, pact_status got, pact_status wanted, int launches) {
  if (got != wanted || launched != launches) { printf("%s: status %d instead of %d, %d launches\n", what, (int)got, (int)wanted, launched); ++failures; }
  launched = 0;
}
#define REFUSED(change, status) { Args x = ok; change; want(#change, x.call(), status, 0); }
alignas(256) char buf[1 << 16];
struct Args {
  pact_ctx *ctx; pact_paged_cache c; const pact_paged_cache *cp = nullptr; bool cache_null = false;
  void *q = buf, *out = buf, *ws = buf; int32_t *table = (int32_t *)buf, *length = (int32_t *)buf, *sel = (int32_t *)buf, *n_new = (int32_t *)buf, *free_pages = (int32_t *)buf,
       *n_free = (int32_t *)buf, *length_out = (int32_t *)buf, *n_free_out = (int32_t *)buf;
  int64_t *slot = (int64_t *)buf; int64_t ldq = 512, ldqh = 128, ldo = 512, ldoh = 128, n_rows = 8, new_stride = 1; size_t ws_bytes = 1 << 16;
  int B = 2, width = 4, n_select = 3, n_first = 1, n_last = 1, row_stride = 0, page = 32, n_pages = 8; float scale = 0.1f;
  std::function<pact_status(Args &)> f;
  pact_status call() { return f(*this); }
};
int main() {
  pact_ctx ctx = {};
  ctx.d = 512; ctx.n_qh = 4; ctx.n_kvh = 2; ctx.d_h = 128; ctx.d_k = 256; ctx.in = ctx.out = PACT_BF16; ctx.elt = 2; ctx.device = 0;
  ctx.paged.blocks = 2; ctx.paged.tile_heads = 8; ctx.paged.head_tiles = 1; ctx.dev.sm_count = 148;
  Args ok;
  ok.ctx = &ctx;
  ok.c = {buf, buf, 2 * 32 * 128, 32 * 128, 128, 2 * 32 * 128, 32 * 128, 128, (float *)buf, buf, (float *)buf, 8, 32};
  const auto cache = [](Args &x) { return x.cache_null ? nullptr : &x.c; };
  const auto query = [](Args &x) {
    return pact_query{x.q, x.ldq, x.ldqh, x.table, x.length, x.B, x.width, x.sel, x.n_select, x.n_first, x.n_last, x.scale, x.out, x.ldo, x.ldoh, nullptr, nullptr, x.ws, x.ws_bytes};
  };
  if (pact_paged_attention(&ctx, nullptr, nullptr, nullptr) != -1 || pact_page_select(&ctx, nullptr, nullptr, nullptr) != -1 || pact_cache_write(&ctx, nullptr, nullptr, nullptr) != -1 ||
      pact_cache_plan(&ctx, nullptr, nullptr) != -1)
    return 1;
  // ---- attention
  ok.f = [&](Args &x) { const pact_query q = query(x); return pact_paged_attention(x.ctx, cache(x), &q, nullptr); };
  want("attention", ok.call(), PACT_OK, 1);
  { Args x = ok; x.sel = nullptr; x.n_select = 0; want("no list", x.call(), PACT_OK, 1); }
  { Args x = ok; x.c.bounds = nullptr; x.c.w_max = nullptr; x.c.logw = nullptr; want("no biases", x.call(), PACT_OK, 1); }
  const auto common = [&](bool attends) {
    REFUSED(x.ctx = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.cache_null = true, PACT_ERR_INVALID_ARG)
    REFUSED(x.c.K = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.c.V = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.c.K = buf + 8, PACT_ERR_INVALID_ARG)
    REFUSED(x.c.k_row = 120, PACT_ERR_INVALID_ARG) REFUSED(x.c.k_row = 129, PACT_ERR_INVALID_ARG) REFUSED(x.c.v_head = 0, PACT_ERR_INVALID_ARG) REFUSED(x.c.v_page = -4096, PACT_ERR_INVALID_ARG)
    REFUSED(x.c.k_page = 1ll << 40, PACT_ERR_UNSUPPORTED) REFUSED(x.c.logw = (float *)(buf + 4), PACT_ERR_INVALID_ARG)
    REFUSED(x.c.bounds = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.c.w_max = nullptr, PACT_ERR_INVALID_ARG)
    REFUSED(x.c.n_pages = 0, PACT_ERR_INVALID_ARG) REFUSED(x.c.page_rows = 0, PACT_ERR_INVALID_ARG) REFUSED(x.c.page_rows = 24, PACT_ERR_INVALID_ARG) REFUSED(x.c.page_rows = 1040, PACT_ERR_INVALID_ARG)
    device_now = 1;
    REFUSED((void)x, PACT_ERR_INVALID_ARG)
    device_now = 0;
    if (!attends) return;
    REFUSED(x.table = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.length = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.q = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.q = buf + 2, PACT_ERR_INVALID_ARG)
    REFUSED(x.ldq = 0, PACT_ERR_INVALID_ARG) REFUSED(x.ldqh = 127, PACT_ERR_INVALID_ARG) REFUSED(x.ldqh = 132, PACT_ERR_INVALID_ARG)
    REFUSED(x.B = 0, PACT_ERR_INVALID_ARG) REFUSED(x.B = PACT_MAX_REQUESTS + 1, PACT_ERR_UNSUPPORTED) REFUSED(x.width = 0, PACT_ERR_INVALID_ARG) REFUSED(x.width = 1 << 27, PACT_ERR_UNSUPPORTED)
    REFUSED(x.scale = NAN, PACT_ERR_INVALID_ARG) REFUSED(x.scale = INFINITY, PACT_ERR_INVALID_ARG) REFUSED(x.n_select = 0, PACT_ERR_INVALID_ARG)
    REFUSED(x.ws = nullptr, PACT_ERR_WORKSPACE) REFUSED(x.ws = buf + 16, PACT_ERR_WORKSPACE) REFUSED(x.ws_bytes = 100, PACT_ERR_WORKSPACE)
    ctx.paged.blocks = 0;
    REFUSED((void)x, PACT_ERR_UNSUPPORTED)
    ctx.paged.blocks = 2;
  };
  common(true);
  REFUSED(x.out = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.out = buf + 4, PACT_ERR_INVALID_ARG) REFUSED(x.ldo = 100, PACT_ERR_INVALID_ARG) REFUSED(x.ldoh = 130, PACT_ERR_INVALID_ARG)
  // ---- selection
  ok.f = [&](Args &x) { const pact_query q = query(x); return pact_page_select(x.ctx, cache(x), &q, nullptr); };
  want("selection", ok.call(), PACT_OK, 1);
  common(true);
  REFUSED(x.sel = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.n_first = -1, PACT_ERR_INVALID_ARG) REFUSED(x.n_last = 3, PACT_ERR_INVALID_ARG) REFUSED(x.n_first = 1 << 30; x.n_last = 1 << 30, PACT_ERR_INVALID_ARG)
  REFUSED(x.width = 65537, PACT_ERR_UNSUPPORTED) REFUSED(x.c.bounds = nullptr; x.c.w_max = nullptr, PACT_ERR_INVALID_ARG)
  // ---- writing
  ok.f = [&](Args &x) { const pact_new_rows r = {x.q, x.out, x.ldq, x.ldqh, nullptr, x.slot, x.n_rows, nullptr}; return pact_cache_write(x.ctx, cache(x), &r, nullptr); };
  want("writing", ok.call(), PACT_OK, 1);
  { Args x = ok; x.n_rows = 0; x.q = nullptr; want("no rows", x.call(), PACT_OK, 0); }
  common(false);
  REFUSED(x.q = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.out = buf + 4, PACT_ERR_INVALID_ARG) REFUSED(x.slot = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.n_rows = -1, PACT_ERR_INVALID_ARG)
  REFUSED(x.ldq = 64, PACT_ERR_INVALID_ARG) REFUSED(x.n_rows = 1ll << 31, PACT_ERR_UNSUPPORTED)
  // ---- planning
  ok.f = [&](Args &x) { const pact_plan p = {x.page, x.n_pages, x.B, x.width, x.table, x.length, x.n_new, x.new_stride, x.free_pages, x.n_free, x.length_out, x.n_free_out, nullptr,
                                              x.slot, x.n_rows, x.row_stride, 0, nullptr}; return pact_cache_plan(x.ctx, &p, nullptr); };
  want("planning", ok.call(), PACT_OK, 1);
  { Args x = ok; x.slot = nullptr; want("no slots", x.call(), PACT_OK, 1); }
  { Args x = ok; x.row_stride = 4; want("padded", x.call(), PACT_OK, 1); }
  REFUSED(x.ctx = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.page = 20, PACT_ERR_INVALID_ARG) REFUSED(x.page = 0, PACT_ERR_INVALID_ARG) REFUSED(x.n_pages = 0, PACT_ERR_INVALID_ARG)
  REFUSED(x.B = 0, PACT_ERR_INVALID_ARG) REFUSED(x.B = 4097, PACT_ERR_UNSUPPORTED) REFUSED(x.width = 0, PACT_ERR_INVALID_ARG) REFUSED(x.width = 1 << 27, PACT_ERR_UNSUPPORTED)
  REFUSED(x.table = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.length = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.n_new = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.new_stride = 0, PACT_ERR_INVALID_ARG)
  REFUSED(x.free_pages = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.n_free = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.length_out = nullptr, PACT_ERR_INVALID_ARG) REFUSED(x.n_free_out = nullptr, PACT_ERR_INVALID_ARG)
  REFUSED(x.n_rows = -1, PACT_ERR_INVALID_ARG) REFUSED(x.row_stride = -4, PACT_ERR_INVALID_ARG) REFUSED(x.row_stride = 5, PACT_ERR_INVALID_ARG) REFUSED(x.n_rows = 1ll << 31, PACT_ERR_UNSUPPORTED)
  device_now = 1;
  REFUSED((void)x, PACT_ERR_INVALID_ARG)
  return failures;
}"""
    _run(tmp_path, main, [nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "--expt-relaxed-constexpr", "-I", CSRC])


def _stub_context(n_qh=4, n_kvh=2, d_h=64):
    """A context without a device: tensors on the CPU pass the device check, the library refuses the null handle."""
    from paper_2504_08966_b200 import binding, build
    build.build()
    ctx = object.__new__(binding.Context)
    ctx._L, ctx.handle = binding.lib(), C.c_void_p()
    ctx.n_qh, ctx.n_kvh, ctx.d_h, ctx.in_dtype, ctx.out_dtype, ctx.device = n_qh, n_kvh, d_h, torch.bfloat16, torch.float32, -1
    ctx._paged_ws, ctx._paged_need = [], {}
    ctx._paged_workspace = lambda B, W: (0, 0, None)
    ctx._make_args()
    return ctx


def test_refusals_of_the_binding(monkeypatch):
    from paper_2504_08966_b200 import binding as pb
    monkeypatch.setattr(pb, "_stream", lambda: 0)
    ctx = _stub_context()
    bf, i32 = torch.bfloat16, torch.int32
    K = torch.zeros(6, 2, 16, 64, dtype=bf)
    logw, bounds, w_max = torch.zeros(6, 16), torch.zeros(6, 2, 2, 64, dtype=bf), torch.zeros(6)
    cache = pb.PagedCache(K, K.clone(), logw, bounds, w_max)
    assert (cache.desc.k_page, cache.desc.k_head, cache.desc.k_row) == (2 * 16 * 64, 16 * 64, 64)
    turned = pb.PagedCache(*(torch.zeros(6, 16, 2, 64, dtype=bf).transpose(1, 2) for _ in range(2)))
    assert (turned.desc.k_page, turned.desc.k_head, turned.desc.k_row) == (2 * 16 * 64, 64, 2 * 64)
    one = pb.PagedCache(*(torch.zeros(1, 1, 16, 64, dtype=bf) for _ in range(2)))
    assert min(one.desc.k_page, one.desc.k_head) >= 64
    for bad in (lambda: pb.PagedCache(K, K[:5]), lambda: pb.PagedCache(K, K.float()), lambda: pb.PagedCache(K, K, logw[:5]), lambda: pb.PagedCache(K, K, logw.double()),
                lambda: pb.PagedCache(K, K, logw, bounds.float(), w_max), lambda: pb.PagedCache(K, K, logw, bounds, w_max[:2]), lambda: pb.PagedCache(K[0], K[0]),
                lambda: pb.PagedCache(K.transpose(2, 3), K.transpose(2, 3))):
        with pytest.raises(pb.PactError):
            bad()
    Q, out, table, length = torch.zeros(3, 4, 64, dtype=bf), torch.zeros(3, 4, 64), torch.zeros(3, 5, dtype=i32), torch.zeros(3, dtype=i32)
    sel = torch.zeros(3, 2, 4, dtype=i32)

    def refused(call, *args, word="wanted", **kw):
        with pytest.raises(pb.PactError, match=word):
            call(*args, **kw)

    null = "status -1"                                        # past the checks of the binding: the library sees the null handle
    refused(ctx.pact_paged_attention, cache, Q, table, length, out, word=null)
    refused(ctx.pact_paged_attention, cache, Q, table, length, out, selected=sel, word=null)
    refused(ctx.pact_page_select, cache, Q, table, length, sel, word=null)
    for change in (dict(Q=Q.float()), dict(Q=Q[:, :3]), dict(Q=Q[..., :32]), dict(table=table.long()), dict(table=table[0]), dict(table=table.t().contiguous().t()), dict(length=length[:2]),
                   dict(length=length.long()), dict(out=out.to(bf)), dict(out=out[:, :2]), dict(lse=torch.zeros(3, 5)), dict(selected=sel[:, :1]), dict(selected=sel.long()),
                   dict(status=torch.zeros(2, dtype=i32))):
        kw = dict(Q=Q, table=table, length=length, out=out, lse=None, selected=None, status=None)
        kw.update(change)
        refused(ctx.pact_paged_attention, cache, kw["Q"], kw["table"], kw["length"], kw["out"], lse=kw["lse"], selected=kw["selected"], status=kw["status"])
    refused(ctx.pact_paged_attention, cache, Q[:2], table, length, out)
    refused(ctx.pact_paged_attention, cache, Q, table, length, out[:2])
    refused(ctx.pact_paged_attention, turned, Q.transpose(1, 2).contiguous().transpose(1, 2), table, length, out, word="last axis")
    refused(_stub_context(n_kvh=1).pact_paged_attention, cache, Q, table, length, out, word="not one of")
    refused(ctx.pact_page_select, cache, Q, table, length, sel[:2])
    rows, slot = torch.zeros(7, 2, 64, dtype=bf), torch.zeros(7, dtype=torch.int64)
    refused(ctx.pact_cache_write, cache, rows, rows, None, slot, word=null)
    refused(ctx.pact_cache_write, cache, rows, rows, None, slot.int())
    refused(ctx.pact_cache_write, cache, rows, rows, torch.zeros(6), slot)
    refused(ctx.pact_cache_write, cache, rows, torch.zeros(7, 2, 128, dtype=bf)[..., :64], None, slot, word="same strides")
    refused(ctx.pact_cache_write, cache, rows[:, :1], rows[:, :1], None, slot)
    one_i = torch.zeros(1, dtype=i32)

    def plan(**change):
        kw = dict(table=table, length=length, n_new=length, free=torch.zeros(6, dtype=i32), n_free=one_i, length_out=length, n_free_out=one_i, row_start=None, slot=slot)
        kw.update(change)
        n_rows = kw.pop("n_rows", None)
        ctx.pact_cache_plan(16, *kw.values(), n_rows=n_rows)

    refused(plan, word=null)
    refused(plan, slot=None, n_rows=9, word=null)
    refused(plan, n_new=torch.zeros(3, 16, dtype=i32)[:, 0], word=null)
    refused(plan, slot=None)
    refused(plan, n_rows=9, word="length of slot")
    refused(plan, n_new=length[:2])
    refused(plan, n_new=length.long())
    refused(plan, length_out=length[:2])
    refused(plan, row_start=length)
    refused(plan, slot=slot.int())
    refused(plan, n_free=length)


def test_workspaces_that_are_outgrown_are_kept(monkeypatch):
    """A captured graph may hold the address of the smaller one."""
    ctx = _stub_context()
    del ctx._paged_workspace
    sizes = {(1, 1): 1000, (4, 4): 1500, (9, 9): 9000}
    monkeypatch.setattr(type(ctx), "_cuda", lambda self: torch.device("cpu"))
    ctx._paged_need.update(sizes)
    got = [ctx._paged_workspace(*k) for k in ((1, 1), (4, 4), (1, 1), (9, 9), (4, 4))]
    assert [n for _, n, _ in got] == [1000, 2000, 2000, 9000, 9000]
    assert len({a for a, _, _ in got}) == 3 and len(ctx._paged_ws) == 3


def test_a_large_workspace_grows_to_what_is_needed(monkeypatch):
    """Where two of them would not fit beside the outgrown one."""
    ctx = _stub_context()
    del ctx._paged_workspace
    monkeypatch.setattr(type(ctx), "_cuda", lambda self: torch.device("meta"))
    mb = 1 << 20
    ctx._paged_need.update({(1, 1): 20 * mb, (2, 2): 21 * mb, (3, 3): 50 * mb, (4, 4): 800 * mb, (5, 5): 801 * mb})
    got = [ctx._paged_workspace(i, i)[1] // mb for i in range(1, 6)]
    assert got == [20, 40, 64, 800, 801] and len(ctx._paged_ws) == 5


# ---- pins of the plain implementations ------------------------------------------------------------------------------

def test_oracle_plan_by_hand():
    table = np.array([[4, 9], [2, -1], [5, -1]], np.int32)
    # pages of 16: the first request grows from 17 rows into its open page, the second has ended, the third opens a page after filling one
    st, t, lens, stack, start, slot = po.plan(16, table, [17, 3, 16], [2, -1, 1], np.array([7, 1, 0], np.int32), 2, 4)
    assert st == 0 and lens == [19, 0, 17] and stack == [7, 1] and start == [0, 2, 2, 3]
    assert t.tolist() == [[4, 9], [2, -1], [5, 2]]            # page 2, given back last, is on top
    assert slot == [9 * 16 + 1, 9 * 16 + 2, 2 * 16, -1]
    assert po.plan(16, table, [17, 3, 16], [2, 0, 1], np.array([7, 1, 0], np.int32), 0, 4)[0] == po.NO_PAGES
    assert po.plan(16, table, [17, 3, 16], [2, 0, 1], np.array([7, 1, 0], np.int32), 2, 2)[0] == po.INVALID


def test_oracle_attention_by_hand():
    """Two rows, the second standing for three tokens: weights 1 : 3 for equal logits, as if it were there three times."""
    K = np.zeros((2, 1, 16, 4))
    V = np.arange(2 * 16 * 4, dtype=float).reshape(2, 1, 16, 4)
    logw = np.zeros((2, 16))
    logw[1, 1] = np.log(3.0)
    out, lse, _, _ = po.attend(np.ones((1, 1, 4)), K, V, logw, np.array([[1]], np.int32), [2], 16, 0.5)
    assert np.allclose(out[0, 0], (V[1, 0, 0] + 3 * V[1, 0, 1]) / 4) and np.isclose(lse[0, 0], np.log(4.0))
    logw[1] = -np.inf
    out, lse, _, _ = po.attend(np.ones((1, 1, 4)), K, V, logw, np.array([[1]], np.int32), [2], 16, 0.5)
    assert not out.any() and lse[0, 0] == -np.inf


def test_oracle_scores_bound_every_logit():
    rng = np.random.default_rng(0)
    K, q, logw = rng.normal(size=(40, 2, 16, 8)), rng.normal(size=(1, 6, 8)), rng.normal(size=(40, 16))
    bounds = np.stack([K.min(2), K.max(2)], 2)
    for h in range(2):
        s = po.page_scores(q[0, h * 3:h * 3 + 3], bounds[:, h], logw.max(1), range(40), 0.3)
        logits = np.einsum("gc,prc->pgr", q[0, h * 3:h * 3 + 3], K[:, h]) * 0.3 + logw[:, None]
        assert (s >= logits.max((1, 2)) - 1e-12).all()


def test_oracle_scores_bound_every_logit_beside_infinities():
    """A key with infinite coordinates: the page's other rows still have the logits that they have."""
    rng = np.random.default_rng(1)
    K, q = rng.normal(size=(60, 1, 16, 8)), rng.normal(size=(1, 5, 8))
    q[0, :, 3] = 0
    for page in range(60):
        for _ in range(page % 4):
            K[page, 0, rng.integers(16), rng.integers(8)] = rng.choice([np.inf, -np.inf])
    K[7, 0, :, 2] = -np.inf                                   # in every row: what of this page is a number is an infinity
    bounds = np.stack([K.min(2), K.max(2)], 2)
    s = po.page_scores(q[0], bounds[:, 0], np.zeros(60), range(60), 0.3)
    with np.errstate(invalid="ignore"):
        logits = np.einsum("gc,prc->pgr", q[0], K[:, 0]) * 0.3
    assert np.isnan(logits).any()
    assert (s >= np.where(np.isnan(logits), -np.inf, logits).max((1, 2)) - 1e-12).all()
