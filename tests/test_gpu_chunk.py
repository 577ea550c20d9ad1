"""Attention of several new tokens per request over the paged cache, on the GPU against its plain float64 implementation (oracle/chunk_oracle.py)."""
import itertools

import numpy as np
import pytest
import torch

from oracle import chunk_oracle as co
from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def pb():
    from paper_2504_08966_b200 import binding
    return binding


_ctx = {}


def context(pb, n_qh, n_kvh, d_h, dtype=BF, out=None):
    key = (n_qh, n_kvh, d_h, dtype, out or dtype)
    if key not in _ctx:
        _ctx[key] = pb.Context((n_qh * d_h + 7) // 8 * 8, n_qh, n_kvh, d_h, dtype, out or dtype)
    return _ctx[key]


def i32(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def cache_of(g, n_pages, H, page, D, dtype, heads_first=True, logw=True):
    shape = (n_pages, H, page, D) if heads_first else (n_pages, page, H, D)
    K, V = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if not heads_first:
        K, V = K.transpose(1, 2), V.transpose(1, 2)
    return K, V, torch.log(torch.floor(1 + 9 * torch.rand(n_pages, page, generator=g, device="cuda"))) if logw else None


def tables(rng, lens, width, page, n_pages):
    ids, table, at = rng.permutation(n_pages), np.full((len(lens), width), -1, np.int32), 0
    for b, n in enumerate(lens):
        k = po.pages_for(max(n, 0), page)
        table[b, :k] = ids[at:at + k]
        at += k
    return table


def tolerances(ref, mag, big, D, lens_max, dtype, out_dtype):
    """Of out and of lse.  Logits: a dot product of d_h terms in fp32 (every partial sum off by half a step, tensor cores by a whole one), scale, bias and exponent's argument rounded:
    (d_h + 8) 2^-23 of the largest sum of magnitudes; they move a weight and the sum of weights.  Weights: exponential 2^-21; bf16 results beside bf16 values: weights rounded to bf16,
    2^-8.  Sums: fp32 results beside bf16 rows: 24 instructions per 128 rows cut 2^-23 each, less than 2^-18, and a rounding (2^-24) per 128 rows; bf16 results: an instruction per 16 rows
    cuts 2^-23; fp32 rows: a rounding per row, 2^-24 each, in threads of their own.  The parts of an item: 160 at most, a rounding of the factor and one of the sum each, 2^-23."""
    delta = (D + 8) * 2.0 ** -23 * big
    if dtype == F32:
        sums = lens_max * 2.0 ** -24
    elif out_dtype == F32:
        sums = 2.0 ** -18 + lens_max / 128 * 2.0 ** -24
    else:
        sums = 2.0 ** -8 + lens_max / 16 * 2.0 ** -23
    rel = 2 * delta + 2.0 ** -20 + sums + 160 * 2.0 ** -23
    return mag * rel[..., None] + np.abs(ref) * torch.finfo(out_dtype).eps / 2 + 1e-30, delta + 2.0 ** -20 + lens_max * 2.0 ** -24 + 160 * 2.0 ** -23


def chunk_and_check(pb, dtype, out_dtype, n_qh, H, D, page, lens, new, heads_first=True, logw=True, causal=True, stride=0, seed=0, poison=None, mask=None, table=None, n_pages=None, scale=None,
                    want_status=0, q_strided=False, starts=None, n_rows=None, ctx=None, lse_too=True):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    B = len(lens)
    width = table.shape[1] if table is not None else max(max(po.pages_for(max(n, 0), page) for n in lens), 1) + 1
    n_pages = n_pages or sum(po.pages_for(max(n, 0), page) for n in lens) + 2
    K, V, w = cache_of(g, n_pages, H, page, D, dtype, heads_first, logw)
    if table is None:
        table = tables(rng, lens, width, page, n_pages)
    if mask is not None:
        mask(w, table)
    if starts is None:
        starts = [b * stride for b in range(B)] if stride else [sum(max(0, m) for m in new[:b]) for b in range(B)]
    if n_rows is None:
        n_rows = B * stride if stride else sum(max(0, m) for m in new) + 3
    Q = torch.randn(n_rows, n_qh + 1 if q_strided else n_qh, D + (8 if q_strided else 0), generator=g, device="cuda").to(dtype)[:, :n_qh, :D]
    Kc, Vc, wc = f64(K), f64(V), f64(w)
    if poison is not None:
        poison(K, V, w, table)
    scale = float(np.float32(D ** -0.5 if scale is None else scale))
    buf = torch.full((n_rows, n_qh, D + 8), -5.0, device="cuda").to(out_dtype)
    out, lse, status = buf[..., :D], torch.full((n_rows, n_qh), -5.0, device="cuda"), i32([0])
    ctx = ctx or context(pb, n_qh, H, D, dtype, out_dtype)
    kept = [x.clone() for x in (K, V)]
    call = lambda: ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, i32(table), i32(lens), i32(new), out, row_start=None if stride else i32(starts), row_stride=stride,   # noqa: E731
                                            lse=lse if lse_too else None, causal=causal, scale=scale, status=status)
    call()
    torch.cuda.synchronize()
    assert status.item() == want_status
    touched, ref, lse_ref, mag, big = co.attend(f64(Q), Kc, Vc, wc, table, lens, new, starts, page, scale, causal, n_rows, stride or None)
    assert (buf[..., D:] == -5).all() and (buf[torch.tensor(~touched, device="cuda")] == -5).all() and (lse[torch.tensor(~touched, device="cuda")] == -5).all()
    got, got_lse = f64(out)[touched], f64(lse)[touched]
    ref, lse_ref, mag, big = (x[touched] for x in (ref, lse_ref, mag, big))
    tol, tol_lse = tolerances(ref, mag, big, D, max(max(lens), 1), dtype, out_dtype)
    err = np.abs(got - ref)
    assert np.isfinite(got).all() and (err <= tol).all(), (err / tol).max()
    if lse_too:
        none = lse_ref == -np.inf
        assert np.array_equal(got_lse == -np.inf, none) and not got[none].any()
        assert (np.abs(got_lse[~none] - lse_ref[~none]) <= (tol_lse + 2.0 ** -22 * np.abs(np.where(none, 0, lse_ref)))[~none]).all()
    first = out.clone(), lse.clone()
    call()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])   # bitwise the same again
    assert poison is not None or all(torch.equal(x, y) for x, y in zip(kept, (K, V)))
    return got


LENS, NEW = [0, 1, 15, 64, 65, 127, 128, 129, 300, 700, 40], [0, 1, 15, 1, 65, 3, 128, 129, 150, 33, 0]


@pytest.mark.parametrize("n_qh,H,D,page", [(4, 4, 64, 16), (14, 2, 64, 32), (28, 4, 128, 64), (32, 8, 128, 16), (8, 1, 256, 64), (16, 1, 128, 128), (12, 1, 80, 48), (40, 1, 64, 16), (6, 2, 192, 32),
                                           (3, 1, 8, 16), (10, 1, 168, 1024), (2, 2, 24, 80), (1, 1, 136, 256)])
@pytest.mark.parametrize("out", [BF, F32])
def test_bf16(pb, n_qh, H, D, page, out):
    chunk_and_check(pb, BF, out, n_qh, H, D, page, LENS, NEW, heads_first=out == F32, logw=out == F32 or D == 64, seed=D + page, q_strided=out == BF, stride=160 if out == BF else 0)


@pytest.mark.parametrize("n_qh,H,D,page", [(2, 2, 64, 16), (14, 2, 64, 32), (8, 2, 128, 64), (9, 1, 100, 16), (4, 1, 96, 128), (32, 2, 32, 48), (3, 3, 4, 16), (60, 1, 128, 16), (100, 1, 32, 16)])
@pytest.mark.parametrize("out", [BF, F32])
def test_fp32(pb, n_qh, H, D, page, out):
    chunk_and_check(pb, F32, out, n_qh, H, D, page, LENS, NEW, heads_first=out == F32, logw=out == F32, seed=D + page, q_strided=out == BF, stride=160 if out == BF else 0)


@pytest.mark.parametrize("dtype,out,n_qh,H,D", [(BF, BF, 8, 2, 128), (BF, F32, 8, 2, 64), (F32, F32, 4, 2, 64), (BF, BF, 4, 1, 256)])
def test_all_rows_of_the_request(pb, dtype, out, n_qh, H, D):
    chunk_and_check(pb, dtype, out, n_qh, H, D, 32, [500, 0, 77, 1, 260], [300, 0, 2, 1, 64], causal=False, seed=D)


@pytest.mark.parametrize("dtype,out,n_qh,H,D,page,lens,new", [
    (BF, BF, 4, 1, 128, 64, [1], [1]), (BF, BF, 28, 4, 128, 64, [4000], [1]), (BF, F32, 28, 4, 128, 64, [5000], [3]), (BF, BF, 1, 1, 64, 16, [1500], [1500]), (BF, BF, 64, 64, 64, 16, [200], [200]),
    (BF, BF, 2, 1, 64, 16, [5, 0] * 150, [2, 0] * 150), (BF, BF, 2, 2, 64, 16, [(i * 37) % 90 for i in range(1200)], [min((i * 37) % 90, i % 7) for i in range(1200)]),
    (BF, F32, 16, 2, 128, 32, [900, 1, 901], [700, 1, 5]), (F32, F32, 8, 1, 128, 64, [2500, 77], [9, 70]), (F32, F32, 1, 1, 32, 16, list(range(0, 200, 9)), [n // 2 for n in range(0, 200, 9)]),
    (BF, BF, 125, 1, 64, 16, [40, 90], [40, 3]), (BF, BF, 50, 1, 160, 16, [40, 90], [20, 3]), (BF, F32, 256, 1, 16, 16, [40, 90], [20, 3])])
def test_few_and_many_requests(pb, dtype, out, n_qh, H, D, page, lens, new):
    chunk_and_check(pb, dtype, out, n_qh, H, D, page, lens, new, seed=len(lens))


@pytest.mark.parametrize("dtype,out,D", [(BF, BF, 64), (BF, F32, 128), (F32, F32, 64)])
def test_items_in_rounds_and_cut_ones(pb, dtype, out, D):
    """More items than two for every CTA, of very different lengths."""
    lens = [1200, 64, 1000, 5, 800, 300] * 8
    chunk_and_check(pb, dtype, out, 16, 16, D, 64, lens, [min(n, 20 if i % 3 else 300) for i, n in enumerate(lens)], seed=3)


def test_most_requests(pb):
    lens = [16 + i % 20 for i in range(4096)]
    chunk_and_check(pb, BF, BF, 2, 1, 64, 16, lens, [1 + i % 3 for i in range(4096)], seed=4)


def test_one_token_is_what_the_attention_of_one_token_gives(pb):
    g, page, n_qh, H, D = torch.Generator(device="cuda").manual_seed(1), 32, 28, 4, 128
    lens = [1000, 1, 33, 500]
    K, V, w = cache_of(g, 60, H, page, D, BF)
    table, Q = i32(tables(np.random.default_rng(0), lens, 40, page, 60)), torch.randn(4, n_qh, D, generator=g, device="cuda").to(BF)
    ctx, cache = context(pb, n_qh, H, D, BF, F32), pb.PagedCache(K, V, w)
    a, b, la, lb = torch.zeros(4, n_qh, D, device="cuda"), torch.zeros(4, n_qh, D, device="cuda"), torch.zeros(4, n_qh, device="cuda"), torch.zeros(4, n_qh, device="cuda")
    ctx.pact_paged_attention(cache, Q, table, i32(lens), a, la)
    ctx.pact_chunk_attention(cache, Q, table, i32(lens), i32([1] * 4), b, row_start=i32([0, 1, 2, 3]), lse=lb)
    # logits of each: off by (d_h + 8) 2^-23 of |q|.|k| / sqrt(d_h), 10 at most here; results: by twice that of sum p |v|, 2 at most where more than one row counts
    assert (a - b).abs().max() <= 4 * 136 * 2.0 ** -23 * 10 * 2 and (la - lb).abs().max() <= 2 * 136 * 2.0 ** -23 * 10 + 2.0 ** -19


# ---- masks, and what must not be seen ---------------------------------------------------------------------------------

def _mask_some(w, table):
    g = torch.Generator(device="cuda").manual_seed(1)
    w.masked_fill_(torch.rand(w.shape, generator=g, device="cuda") < 0.5, float("-inf"))
    w[torch.tensor(table[-1][table[-1] >= 0], device="cuda").long()] = float("-inf")
    w[int(table[0][0]), 1:] = float("-inf")


@pytest.mark.parametrize("dtype,out,D", [(BF, BF, 128), (BF, F32, 128), (BF, BF, 64), (BF, F32, 192), (F32, F32, 64), (F32, F32, 128)])
@pytest.mark.parametrize("masked", [False, True])
def test_rows_that_nobody_sees_may_hold_anything(pb, dtype, out, D, masked):
    lens, page = [100, 5, 64, 0, 700, 33, 90], 32

    def poison(K, V, w, table):
        seen = np.zeros((K.shape[0], page), bool)
        for b, n in enumerate(lens):
            for x in po.rows_of(table[b], n, page, K.shape[0]):
                seen[x] = float(w[x]) != -np.inf
        hide = torch.tensor(~seen, device="cuda")
        bad = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(dtype)[torch.randint(0, 3, K.shape, device="cuda")]
        K.copy_(torch.where(hide[:, None, :, None], bad, K))
        V.copy_(torch.where(hide[:, None, :, None], bad, V))
        w.copy_(torch.where(hide & (w != float("-inf")), float("nan"), w))

    chunk_and_check(pb, dtype, out, 8, 2, D, page, lens, [60, 5, 1, 0, 300, 33, 9], poison=poison, mask=_mask_some if masked else None, seed=D)


@pytest.mark.parametrize("dtype,out,n_qh,H,D", [(BF, BF, 4, 2, 128), (BF, F32, 4, 2, 128), (BF, BF, 1, 1, 64), (BF, BF, 2, 1, 256), (F32, F32, 4, 2, 64)])
@pytest.mark.parametrize("at", [190, 250, 299])
def test_what_is_not_finite_shows_to_the_tokens_that_see_it_only(pb, dtype, out, n_qh, H, D, at):
    """Infinite and NaN values in a row among the new tokens': earlier tokens have the results that they have without it, later ones a NaN or an infinity in its columns."""
    n, m, page = 300, 150, 16
    g = torch.Generator(device="cuda").manual_seed(D)
    K, V, w = cache_of(g, 19, H, page, D, dtype)
    table, Q = i32(np.arange(19)[None]), torch.randn(m, n_qh, D, generator=g, device="cuda").to(dtype)
    ctx, L, N, S = context(pb, n_qh, H, D, dtype, out), i32([n]), i32([m]), i32([0])
    clean, got = (torch.zeros(m, n_qh, D, dtype=out, device="cuda") for _ in range(2))
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, table, L, N, clean, row_start=S)
    V[at // page, 0, at % page, 1], V[at // page, 0, at % page, D - 1] = float("inf"), float("nan")
    lse = torch.zeros(m, n_qh, device="cuda")
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, table, L, N, got, row_start=S, lse=lse)
    first, heads = at - (n - m), n_qh // H
    assert torch.equal(got[:first], clean[:first]) and torch.equal(got[:, heads:], clean[:, heads:]) and torch.isfinite(lse).all()
    hit = got[first:, :heads]
    assert not torch.isfinite(hit[..., [1, D - 1]]).any()
    rest = [c for c in range(D) if c not in (1, D - 1)]
    assert torch.equal(hit[..., rest], clean[first:, :heads][..., rest])
    # a key or a bias that is not a number: the tokens that see it have nothing else
    V[at // page, 0, at % page] = 0
    K[at // page, 0, at % page, 2] = float("nan")
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, table, L, N, got, row_start=S, lse=lse)
    assert got[first:, :heads].isnan().all() and lse[first:, :heads].isnan().all() and torch.isfinite(got[:first]).all() and torch.isfinite(got[:, heads:]).all()
    K[at // page, 0, at % page, 2] = 0
    for bias in (float("nan"), float("inf")):
        w[at // page, at % page] = bias
        ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, table, L, N, got, row_start=S, lse=lse)
        assert got[first:].isnan().all() and not torch.isfinite(lse[first:]).any() and torch.equal(got[:first], clean[:first]) and torch.isfinite(lse[:first]).all()


@pytest.mark.parametrize("dtype,out,D", [(BF, BF, 64), (BF, F32, 64), (BF, BF, 128), (BF, F32, 200), (F32, F32, 64)])
def test_what_is_not_finite_in_many_short_requests(pb, dtype, out, D):
    """A tile each, every one with an infinity of its own among the new tokens' values: each shows in its request, its column and the tokens that see it, although values are looked at ahead."""
    B, H, n_qh, page = 1500, 2, 4, 32
    g, rng = torch.Generator(device="cuda").manual_seed(D), np.random.default_rng(D)
    K, V, w = cache_of(g, B, H, page, D, dtype)
    lens, new = rng.integers(8, page + 1, B), rng.integers(3, 8, B)
    starts, row, col, head = np.concatenate([[0], np.cumsum(new)[:-1]]), np.array([n - m + rng.integers(0, m) for n, m in zip(lens, new)]), rng.integers(0, D, B), rng.integers(0, H, B)
    Q = torch.randn(int(new.sum()), n_qh, D, generator=g, device="cuda").to(dtype)
    clean, got, status = torch.zeros(len(Q), n_qh, D, dtype=out, device="cuda"), torch.zeros(len(Q), n_qh, D, dtype=out, device="cuda"), i32([0])
    ctx, args = context(pb, n_qh, H, D, dtype, out), (i32(np.arange(B)[:, None]), i32(lens), i32(new))
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, *args, clean, row_start=i32(starts), status=status)
    at = torch.arange(B, device="cuda")
    V[at, torch.tensor(head, device="cuda"), torch.tensor(row, device="cuda"), torch.tensor(col, device="cuda")] = float("inf")
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, *args, got, row_start=i32(starts), status=status)
    hit = np.zeros((len(Q), n_qh, D), bool)
    for b in range(B):
        hit[starts[b] + row[b] - (lens[b] - new[b]):starts[b] + new[b], head[b] * 2:head[b] * 2 + 2, col[b]] = True
    hit = torch.tensor(hit, device="cuda")
    assert status.item() == 0 and torch.equal(~torch.isfinite(got), hit) and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
def test_masks_of_the_lowest_value_and_large_logits(pb, dtype, out):
    """The lowest float as a bias is a number: where all rows have it, they share the attention; beside others it is nothing."""
    lowest = torch.finfo(F32).min
    K, V = torch.zeros(2, 1, 16, 64, device="cuda"), torch.randn(2, 1, 16, 64, device="cuda")
    cache = pb.PagedCache(K.to(dtype), V.to(dtype), torch.full((2, 16), lowest, device="cuda"))
    o, lse = torch.zeros(3, 1, 64, dtype=out, device="cuda"), torch.zeros(3, 1, device="cuda")
    context(pb, 1, 1, 64, dtype, out).pact_chunk_attention(cache, torch.zeros(3, 1, 64, device="cuda", dtype=dtype), i32([[0, 1]]), i32([20]), i32([3]), o, row_start=i32([0]), lse=lse)
    rows = cache.V.double().reshape(32, 64)
    for i in range(3):                                 # equal weights are exact in bf16 as well
        want = rows[:18 + i].mean(0)
        assert ((o[i, 0].double() - want).abs() <= rows[:18 + i].abs().mean(0) * 2.0 ** -18 + want.abs() * torch.finfo(out).eps / 2).all() and lse[i].item() == lowest

    def some(w, table):
        w[int(table[0, 0])] = lowest
        w[int(table[1, 0]), 3:] = lowest

    chunk_and_check(pb, dtype, out, 2, 1, 64, 16, [40, 16], [30, 5], mask=some, seed=3, lse_too=out == F32)
    chunk_and_check(pb, dtype, out, 8, 1, 128, 64, [500, 64], [200, 64], scale=3.0, seed=5)     # logits of a few hundred
    chunk_and_check(pb, dtype, out, 8, 1, 64, 64, [500, 64], [200, 64], scale=-1.0, seed=5)
    chunk_and_check(pb, dtype, out, 8, 1, 64, 64, [500, 64], [200, 64], scale=0.0, seed=5)
    chunk_and_check(pb, dtype, out, 8, 1, 64, 64, [500, 64], [200, 64], scale=-0.5, logw=False, seed=6)


def test_bad_pages_lengths_and_rows(pb):
    rng, page, n_pages = np.random.default_rng(0), 16, 30
    table = rng.integers(0, n_pages, (3, 9)).astype(np.int32)
    bad = table.copy()
    bad[0, 2], bad[0, 5], bad[1, 0], bad[2, 8] = -1, n_pages, 1 << 30, -(1 << 31)
    for dtype, out, logw in ((BF, BF, True), (BF, F32, False), (F32, F32, True)):
        kw = dict(n_pages=n_pages, want_status=po.INVALID, logw=logw)
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [100, 10, 9 * page], [40, 3, 144], table=bad, **kw)
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, -3, 0], [20, 2, 0], table=table, **kw)
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, 9 * page + 1, 0], [5, 5, 0], table=table, **kw)
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, 30, 0], [25, 30, 3], table=table, **kw)                     # more new tokens than rows: the first see nothing
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, 30, 9], [5, 20, 3], table=table, starts=[0, 5, 25], n_rows=20, **kw)   # rows of Q that are not there
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, 30, 9], [5, 6, 3], table=table, starts=[2, -4, 1 << 30], n_rows=20, **kw)
        chunk_and_check(pb, dtype, out, 4, 2, 64, page, [20, 30, 9], [5, -1, 3], table=table, n_pages=n_pages, logw=logw, seed=2)   # a request that has ended


def test_a_page_that_two_requests_share_and_results_alone(pb):
    table = np.array([[0, 1, 2], [0, 1, 3], [0, 0, 0]], np.int32)
    chunk_and_check(pb, BF, BF, 8, 2, 128, 64, [150, 190, 192], [22, 62, 64], table=table, n_pages=4, lse_too=False)


def test_no_rows_at_all(pb):
    ctx = context(pb, 4, 2, 64)
    K = torch.zeros(2, 2, 16, 64, dtype=BF, device="cuda")
    empty = torch.zeros(0, 4, 64, dtype=BF, device="cuda")
    ctx.pact_chunk_attention(pb.PagedCache(K, K), empty, i32([[0]]), i32([5]), i32([0]), empty.clone(), row_start=i32([0]))
    chunk_and_check(pb, BF, BF, 4, 2, 64, 16, [5, 0, 40], [0, 0, 0])


@pytest.mark.parametrize("shift", [4, 8, 16])
def test_results_at_any_multiple_of_four_elements(pb, shift):
    g, D = torch.Generator(device="cuda").manual_seed(0), 64
    K, V, w = cache_of(g, 8, 2, 16, D, BF)
    Q = torch.randn(50, 4, D, generator=g, device="cuda").to(BF)
    want = torch.zeros(50, 4, D, dtype=BF, device="cuda")
    ctx, args = context(pb, 4, 2, D), (i32(np.arange(8)[None]), i32([120]), i32([50]))
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, *args, want, row_start=i32([0]))
    buf = torch.full((50 * 4 * (D + shift) + shift,), -5.0, dtype=BF, device="cuda")
    out = buf[shift:].view(50, 4, D + shift)[..., :D]
    ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, *args, out, row_start=i32([0]))
    assert torch.equal(out, want) and (buf[:shift] == -5).all() and (buf[shift:].view(50, 4, D + shift)[..., D:] == -5).all()


@pytest.mark.parametrize("n_qh,H,D", [(4, 4, 64), (8, 1, 128)])
def test_sums_of_fp32_results_are_not_biased(pb, n_qh, H, D):
    # Values of one sign, weights from the biases alone (queries 0).  24 instructions sum 128 rows, the small terms of every 16 first; an instruction cuts its running sum, which grows
    # from nothing, by half of 2^-23 in the mean: 24 / 2 * 2^-24 = 2^-20.4.  2^-19.5 leaves half as much again for the roundings of sums over groups, whose mean over thousands of
    # results is far smaller, and of the denominators.
    P, page, n, m = 64, 64, 1 << 16, 3
    g = torch.Generator(device="cuda").manual_seed(D)
    K = torch.zeros(P, H, page, D, dtype=BF, device="cuda")
    V, w = 1 + torch.rand(P, H, page, D, generator=g, device="cuda").to(BF), -torch.rand(P, page, generator=g, device="cuda")
    out = torch.empty(m, n_qh, D, device="cuda")
    table = torch.arange(n // page, dtype=I32, device="cuda")[None] % P
    context(pb, n_qh, H, D, BF, F32).pact_chunk_attention(pb.PagedCache(K, V, w), torch.zeros(m, n_qh, D, dtype=BF, device="cuda"), table, i32([n]), i32([m]), out, row_start=i32([0]), causal=False)
    p = torch.exp(w.double())
    want = (torch.einsum("pr,phrc->hc", p, V.double()) / p.sum()).repeat_interleave(n_qh // H, 0)
    assert abs(((out.double() - want) / want).mean().item()) <= 2.0 ** -19.5


def test_offsets_past_32_bits(pb):
    """A cache of more than 2^32 bytes and 2^31 elements: pages at its far end."""
    n_pages, H, page, D, m = 2050, 8, 1024, 128, 700
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("not enough memory")
    K, V = (torch.zeros(n_pages, H, page, D, dtype=BF, device="cuda") for _ in range(2))
    assert K.numel() > 1 << 31
    ids, g = [n_pages - 1, 0, n_pages - 3], torch.Generator(device="cuda").manual_seed(1)
    n = 2 * page + 500
    for i in ids:
        K[i], V[i] = torch.randn(H, page, D, generator=g, device="cuda"), torch.randn(H, page, D, generator=g, device="cuda")
    Q, out = torch.randn(m, H, D, generator=g, device="cuda").to(BF), torch.zeros(m, H, D, device="cuda")
    context(pb, H, H, D, BF, F32).pact_chunk_attention(pb.PagedCache(K, V), Q, i32([ids]), i32([n]), i32([m]), out, row_start=i32([0]))
    k, v = (X[ids].transpose(1, 2).reshape(-1, H, D)[:n].double() for X in (K, V))
    s = torch.einsum("mhc,nhc->hmn", Q.double(), k) * float(np.float32(D ** -0.5))
    s = s.masked_fill(torch.arange(n, device="cuda") > torch.arange(n - m, n, device="cuda")[:, None], -torch.inf)
    p = torch.softmax(s, 2)
    ref, mag = torch.einsum("hmn,nhc->mhc", p, v), torch.einsum("hmn,nhc->mhc", p, v.abs())
    # logits: (d_h + 8) 2^-23 of |q|.|k| / sqrt(d_h), at most 30 here; twice; sums less than 2^-17
    assert ((out.double() - ref).abs() <= mag * (2 * 136 * 2.0 ** -23 * 30 + 2.0 ** -17)).all()
    # rows of Q and of the result beyond 2^31 elements are told apart by 64-bit strides
    big = torch.zeros(1 << 14, 1, (1 << 17) + 64, dtype=BF, device="cuda")
    ctx = context(pb, 1, 1, 64)
    q = big[..., :64]
    q.copy_(torch.randn(1 << 14, 1, 64, generator=g, device="cuda"))
    K1, V1 = (torch.randn(4, 1, 16, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    a, b = torch.zeros(3, 1, 64, dtype=BF, device="cuda"), big[..., 64:128]
    last = (1 << 14) - 3
    ctx.pact_chunk_attention(pb.PagedCache(K1, V1), q[last:].contiguous(), i32([[0, 1, 2, 3]]), i32([60]), i32([3]), a, row_start=i32([0]))
    ctx.pact_chunk_attention(pb.PagedCache(K1, V1), q, i32([[0, 1, 2, 3]]), i32([60]), i32([3]), b, row_start=i32([last]))
    assert torch.equal(b[last:], a) and not b[:last].any()


# ---- graphs, streams, contexts ---------------------------------------------------------------------------------------

def test_captured_and_replayed_with_other_lengths_beside_eager_calls(pb):
    """Two captured graphs and eager calls of one context take turns on its workspace; the first call of the context is inside the capture."""
    rng, g = np.random.default_rng(0), torch.Generator(device="cuda").manual_seed(0)
    page, H, D, n_qh, n_pages, B, rows = 16, 2, 64, 8, 600, 5, 400
    K, V, w = cache_of(g, n_pages, H, page, D, BF)
    cache, ctx = pb.PagedCache(K, V, w), pb.Context(512, n_qh, H, D, BF, F32)
    table = rng.permutation(n_pages).astype(np.int32)[:B * 100].reshape(B, 100)
    T, L, N, S, Q = i32(table), i32([100] * B), i32([10] * B), i32([0] * B), torch.zeros(rows, n_qh, D, dtype=BF, device="cuda")
    out, out_all, out_e = (torch.zeros(rows, n_qh, D, device="cuda") for _ in range(3))
    one, two = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(one):
        ctx.pact_chunk_attention(cache, Q, T, L, N, out, row_start=S)
    with torch.cuda.graph(two):
        ctx.pact_chunk_attention(cache, Q, T, L, N, out_all, row_start=S, causal=False)
    scale = float(np.float32(D ** -0.5))
    for lens, new in (([100] * B, [10] * B), ([1600, 0, 3, 1, 999], [300, 0, 3, 1, 96]), ([0] * B, [0] * B), ([64] * B, [64, 1, 64, 0, 63]), ([1600] * B, [1] * B)):
        starts = [sum(new[:b]) for b in range(B)]
        for t, v in ((L, lens), (N, new), (S, starts)):
            t.copy_(i32(v))
        Q.copy_(torch.randn(rows, n_qh, D, generator=g, device="cuda"))
        for o in (out, out_all, out_e):
            o.zero_()
        one.replay()
        two.replay()
        ctx.pact_chunk_attention(cache, Q, T, L, N, out_e, row_start=S)
        one.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, out_e)
        for o, causal in ((out, True), (out_all, False)):
            touched, ref, _, mag, big = co.attend(f64(Q), f64(K), f64(V), f64(w), table, lens, new, starts, page, scale, causal, rows)
            tol, _ = tolerances(ref, mag, big, D, 1600, BF, F32)
            assert (np.abs(f64(o) - ref) <= tol).all() and not f64(o)[~touched].any()


def test_another_stream_and_two_calls_at_once_on_two_contexts(pb):
    g = torch.Generator(device="cuda").manual_seed(6)
    K, V, w = cache_of(g, 2000, 2, 64, 128, BF)
    T, L, N, S = torch.randperm(2000, device="cuda").int().view(2, 1000), i32([64000, 50001]), i32([100, 3]), i32([0, 100])
    runs = []
    for i in range(2):
        Q = torch.randn(103, 8, 128, device="cuda", generator=g).to(BF)
        ctx, s = pb.Context(1024, 8, 2, 128, BF, BF), torch.cuda.Stream()
        alone = torch.zeros(103, 8, 128, dtype=BF, device="cuda")
        ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, T, L, N, alone, row_start=S)
        runs.append((ctx, s, Q, alone, torch.zeros_like(alone)))
    torch.cuda.synchronize()
    for _, (ctx, s, Q, _, out) in itertools.product(range(10), runs):
        with torch.cuda.stream(s):
            ctx.pact_chunk_attention(pb.PagedCache(K, V, w), Q, T, L, N, out, row_start=S)
    torch.cuda.synchronize()
    for _, _, _, alone, out in runs:
        assert torch.equal(out, alone)


@pytest.mark.parametrize("out,n_qh,H,D,lens,new", [(BF, 8, 2, 64, [3000], [300]), (F32, 8, 2, 128, [6000, 5, 0, 2000], [3, 5, 0, 40]), (BF, 4, 1, 256, [900] * 3, [100] * 3), (BF, 4, 2, 128, [700, 300] * 12, [9, 200] * 12),
                                                   (F32, 16, 16, 64, [400] * 30, [300] * 30)])
def test_waits_that_run_out(pb, out, n_qh, H, D, lens, new):
    """Waits of a few polls: the call ends with its status, wherever a warp gave up, nothing outside the result is touched, and the next call is right."""
    rng, g, page = np.random.default_rng(0), torch.Generator(device="cuda").manual_seed(0), 16
    n_pages = sum(po.pages_for(n, page) for n in lens) + 1
    K, V, w = cache_of(g, n_pages, H, page, D, BF)
    table = i32(tables(rng, lens, max(po.pages_for(n, page) for n in lens), page, n_pages))
    ctx, cache, rows = pb.Context(n_qh * D, n_qh, H, D, BF, out), pb.PagedCache(K, V, w), sum(new)
    args = torch.randn(rows, n_qh, D, generator=g, device="cuda").to(BF), table, i32(lens), i32(new)
    S = i32([sum(new[:b]) for b in range(len(new))])
    want, buf, status = torch.zeros(rows, n_qh, D, dtype=out, device="cuda"), torch.full((rows + 2, n_qh, D), -5.0, dtype=out, device="cuda"), i32([0])
    copies = [x.clone() for x in (K, V, w)]
    ctx.pact_chunk_attention(cache, *args, want, row_start=S, status=status)
    assert status.item() == 0
    seen = set()
    for polls in (1, 2, 1, 3, 5, 9, 20, 50, 100, 1, 0):
        ctx.set_wait_limits(barrier_polls=polls)
        buf.fill_(-5)
        status.zero_()
        ctx.pact_chunk_attention(cache, *args, buf[1:-1], row_start=S, status=status)
        seen.add(status.item())
        assert status.item() in (0, -5) and (polls != 1 or status.item() == -5) and (polls or status.item() == 0)
        assert (buf[0] == -5).all() and (buf[-1] == -5).all()
        if status.item() == 0:
            assert torch.equal(buf[1:-1], want)
    assert seen == {0, -5} and all(torch.equal(x, y) for x, y in zip(copies, (K, V, w)))


def test_refusals_on_the_device(pb):
    ctx = context(pb, 4, 2, 64)
    K = torch.zeros(2, 2, 16, 64, dtype=BF, device="cuda")
    Q = torch.zeros(3, 4, 64, dtype=BF, device="cuda")
    args = i32([[0]]), i32([3]), i32([3])
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_chunk_attention(pb.PagedCache(K, K), Q, *args, Q.clone())                    # neither row_start nor row_stride
    with pytest.raises(pb.PactError, match="invalid"):
        ctx.pact_chunk_attention(pb.PagedCache(K, K), Q, *args, Q.clone(), row_stride=2)
    with pytest.raises(pb.PactError, match="wanted"):
        ctx.pact_chunk_attention(pb.PagedCache(K, K), Q.cpu(), *args, Q.clone(), row_start=i32([0]))
    with pytest.raises(pb.PactError, match="unsupported"):
        c = pb.Context(264, 1, 1, 264)
        K = torch.zeros(2, 1, 16, 264, dtype=BF, device="cuda")
        Q = torch.zeros(3, 1, 264, dtype=BF, device="cuda")
        c.pact_chunk_attention(pb.PagedCache(K, K), Q, *args, Q.clone(), row_start=i32([0]))
