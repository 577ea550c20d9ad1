"""How near the results of the attention of several new tokens are to the exact ones: terms of probabilities, sums over many tiles, large biases."""
import numpy as np
import pytest
import torch

from tests.test_gpu_chunk import BF, F32, I32, context, f64, i32, pb   # noqa: F401

pytestmark = pytest.mark.gpu


def half_step(x):
    """Of bf16, at x."""
    return 2.0 ** (np.floor(np.log2(np.abs(x))) - 8)


@pytest.mark.parametrize("B,n_qh,H,D,page,m", [(300, 1, 1, 64, 16, 1), (64, 8, 1, 128, 32, 2), (40, 8, 2, 128, 16, 100), (9, 2, 2, 64, 16, 200), (64, 4, 1, 192, 16, 3), (20, 8, 1, 256, 16, 40)])
def test_bf16_results_are_rounded_once(pb, B, n_qh, H, D, page, m):
    # Two rows with logits 0 and b (queries 0), values 0 and v: out = v x / (1 + x), x = exp(b), -1 <= b < 0.  In fp32 it is good to 2^-20: the argument of the exponential to 0.3, the exponential to
    # 1, the cuts of the products to 1.5, 1 + x, reciprocal and product to 0.75 units of 2^-22.  x as two bf16 terms: the first is off by half a step, 2^-9 where x is below 1, the second by half
    # of its own, 2^-18; x is above 1/4, at worst 1/2 with that step: 2^-17 of it.  Then one rounding, half a step.
    g = torch.Generator(device="cuda").manual_seed(D + m)
    K = torch.zeros(B, H, page, D, dtype=BF, device="cuda")
    V, w = K.clone(), torch.zeros(B, page, device="cuda")
    V[:, :, 1] = 1 + torch.rand(B, H, D, generator=g, device="cuda").to(BF)
    w[:, 1] = -torch.rand(B, generator=g, device="cuda")
    out = torch.empty(B * m, n_qh, D, dtype=BF, device="cuda")
    context(pb, n_qh, H, D, BF).pact_chunk_attention(pb.PagedCache(K, V, w), torch.zeros(B * m, n_qh, D, dtype=BF, device="cuda"), torch.arange(B, dtype=I32, device="cuda")[:, None], i32([2] * B),
                                                     i32([m] * B), out, row_stride=m, causal=False, status=None)
    x = np.exp(f64(w)[:, 1])[:, None, None, None]
    want = np.repeat(f64(V)[:, None, :, 1], n_qh // H, axis=2) * x / (1 + x)
    assert (np.abs(f64(out).reshape(B, m, n_qh, D) - want) <= half_step(want) + (2.0 ** -17 + 2.0 ** -20) * want).all()


@pytest.mark.parametrize("m,D", [(200, 64), (3, 64), (200, 128)])
def test_bf16_results_of_long_sums_are_not_cut_off(pb, m, D):
    # Values of one sign, weights from the biases alone (queries 0), and so many key heads that some have all 512 tiles in one CTA.  Two terms: 2^-17 of each weight.  The tensor cores sum 32 tiles,
    # 512 instructions, each of which cuts its running sum, which grows from nothing, by 2^-23 at most: 512 / 2 * 2^-23 = 2^-15.  16 such sums and 512 tiles' sums of weights, added with rounding:
    # (16 + 512) / 2 * 2^-24, and everything else 2^-20 as above.  Sums that are cut at every step would be off by 4,096 / 2 * 2^-24 = 2^-13 in the mean, more than all that.
    B, H, P, page, n = 5, 64, 32, 64, 1 << 16
    g = torch.Generator(device="cuda").manual_seed(D + m)
    K = torch.zeros(P, H, page, D, dtype=BF, device="cuda")
    V = (1 + torch.rand(1, H, 1, D, generator=g, device="cuda") + 0.5 * torch.rand(P, H, page, D, generator=g, device="cuda")).to(BF)
    w = -torch.rand(P, page, generator=g, device="cuda")
    out = torch.empty(B * m, H, D, dtype=BF, device="cuda")
    table = (torch.arange(n // page, dtype=I32, device="cuda") % P).repeat(B, 1)
    context(pb, H, H, D, BF).pact_chunk_attention(pb.PagedCache(K, V, w), torch.zeros(B * m, H, D, dtype=BF, device="cuda"), table, i32([n] * B), i32([m] * B), out, row_stride=m, causal=False)
    p = torch.exp(w.double())
    want = (torch.einsum("pr,phrc->hc", p, V.double()) / p.sum()).cpu().numpy()
    tol = 2.0 ** -17 + 2.0 ** -15 + 264 * 2.0 ** -24 + 2.0 ** -20
    assert (np.abs(f64(out) - want) <= half_step(want) + tol * want).all()


LOWEST = torch.finfo(F32).min


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("n_qh,H,D,lens,new", [(8, 2, 64, [3000], [300]), (2, 1, 128, [2000, 700], [3, 2]), (2, 2, 64, [300] * 200, [150] * 200), (1, 1, 64, [20] * 500, [2] * 500)])
def test_biases_as_large_as_floats_get(pb, dtype, out, n_qh, H, D, lens, new):
    """Where all rows have the same large bias, logits are lost in its last place: they share the attention, and the bias is the log-sum-exp.  In items that several CTAs share, in whole ones, in
    those of few rows and of one tile; beside rows without a bias such rows are nothing, or everything."""
    # equal weights are exact, in one term; values of both signs: fp32 sums of up to 3,000, 24 instructions that cut 2^-23 each at every 128 rows, or 8 of them at every 128 of 4,096, and a rounding
    # per row (fp32 rows) in sums that grow from nothing: less than 2^-12 of the mean of |v|
    g, page, B = torch.Generator(device="cuda").manual_seed(len(lens)), 16, len(lens)
    pages = [(n + page - 1) // page for n in lens]
    first = np.concatenate([[0], np.cumsum(pages)])
    K, V = (torch.randn(int(first[-1]), H, page, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = np.full((B, max(pages)), -1, np.int32)
    for b in range(B):
        table[b, :pages[b]] = np.arange(first[b], first[b + 1])
    starts, rows = np.concatenate([[0], np.cumsum(new)]), sum(new)
    Q, got, lse = torch.randn(rows, n_qh, D, generator=g, device="cuda").to(dtype), torch.zeros(rows, n_qh, D, dtype=out, device="cuda"), torch.zeros(rows, n_qh, device="cuda")
    w = torch.zeros(int(first[-1]), page, device="cuda")
    call = lambda: context(pb, n_qh, H, D, dtype, out).pact_chunk_attention(pb.PagedCache(K, V, w), Q, i32(table), i32(lens), i32(new), got, row_start=i32(starts), lse=lse)   # noqa: E731
    means = []
    for b in range(0, B, max(1, B // 4)):
        v = V[first[b]:first[b + 1]].double().transpose(1, 2).reshape(-1, H, D)[:lens[b]]
        n = torch.arange(lens[b] - new[b] + 1, lens[b] + 1, device="cuda")[:, None, None]
        means.append((b, (v.cumsum(0)[lens[b] - new[b]:] / n).repeat_interleave(n_qh // H, 1), (v.abs().cumsum(0)[lens[b] - new[b]:] / n).repeat_interleave(n_qh // H, 1)))
    for bias in (LOWEST, -3e38, -2.3e38, -2e38, -1.6e38, -1e30, 1e30, 1.6e38, 2.4e38, 3e38, -LOWEST):
        w.fill_(bias)
        call()
        assert (lse == w[0, 0]).all(), bias
        for b, mean, size in means:
            assert ((got[starts[b]:starts[b + 1]].double() - mean).abs() <= size * 2.0 ** -12 + mean.abs() * torch.finfo(out).eps / 2).all(), bias
    # every third row has the bias, the others none: what is left without it, and what it leaves
    plain = torch.arange(page, device="cuda") % 3 != 0
    w[:] = torch.where(plain, 0.0, -torch.inf)
    call()
    want, want_lse = got.clone(), lse.clone()
    for bias in (LOWEST, -2e38, -1.6e38):
        w[:] = torch.where(plain, 0.0, bias)
        call()
        seen = torch.isfinite(want_lse)
        assert torch.equal(got[seen], want[seen]) and torch.equal(lse[seen], want_lse[seen])
    for bias in (2e38, 3e38):
        w[:] = torch.where(plain, 0.0, bias)
        call()
        assert (lse == torch.tensor(bias, device="cuda")).all()
        w[:] = torch.where(plain, -torch.inf, bias)
        want = got.clone()
        call()
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype,out,n_qh,H,D", [(BF, BF, 4, 2, 128), (BF, F32, 4, 2, 128), (BF, BF, 1, 1, 64), (BF, F32, 2, 1, 256), (F32, F32, 4, 2, 64)])
@pytest.mark.parametrize("m", [1, 300])
def test_infinite_values_anywhere_are_that_infinity_or_nan(pb, dtype, out, n_qh, H, D, m):
    """In the first tile, which all tokens see in full, between, and in the last one: in the tokens that see the row an infinity of that sign or NaN, in its columns alone; and the same of the
    attention of one token."""
    n, page = 2000, 16
    g = torch.Generator(device="cuda").manual_seed(D)
    K, V = (torch.randn(n // page, H, page, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    Q, table = torch.randn(m, n_qh, D, generator=g, device="cuda").to(dtype), torch.arange(n // page, dtype=I32, device="cuda")[None]
    ctx, clean, got = context(pb, n_qh, H, D, dtype, out), torch.zeros(m, n_qh, D, dtype=out, device="cuda"), torch.zeros(m, n_qh, D, dtype=out, device="cuda")
    ctx.pact_chunk_attention(pb.PagedCache(K, V), Q, table, i32([n]), i32([m]), clean, row_start=i32([0]))
    for at in (0, 5, 700, n - m, n - 1):
        kept = V[at // page, 0, at % page].clone()
        V[at // page, 0, at % page, 1], V[at // page, 0, at % page, D - 1] = float("inf"), -float("inf")
        first, heads, rest = max(0, at - (n - m)), n_qh // H, [c for c in range(D) if c not in (1, D - 1)]
        ctx.pact_chunk_attention(pb.PagedCache(K, V), Q, table, i32([n]), i32([m]), got, row_start=i32([0]))
        assert torch.equal(got[:first], clean[:first]) and torch.equal(got[:, heads:], clean[:, heads:]) and torch.equal(got[first:, :heads][..., rest], clean[first:, :heads][..., rest]), at
        for c, sign in ((1, 1), (D - 1, -1)):
            hit = got[first:, :heads, c]
            assert (hit.isnan() | (hit == sign * float("inf"))).all(), at
        if m == 1:
            one = torch.zeros(1, n_qh, D, dtype=out, device="cuda")
            ctx.pact_paged_attention(pb.PagedCache(K, V), Q, table, i32([n]), one)
            assert all((x.isnan() | (x == s * float("inf"))).all() for x, s in ((one[0, :heads, 1], 1), (one[0, :heads, D - 1], -1))) and torch.isfinite(one[0, :heads][:, rest]).all()
        V[at // page, 0, at % page] = kept


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("m,n,slope,D", [(200, 4200, 64, 64), (200, 4400, 1024, 128), (200, 8300, 256, 64), (3, 8300, 64, 64), (3, 8450, 1024, 128), (100, 4200, 256, 256)])
def test_logits_that_grow_from_tile_to_tile(pb, out, m, n, slope, D):
    # Biases that rise with the rows (queries 0), so that sums of earlier tiles are rescaled before and after they are put aside, and so many key heads that some have all their tiles in one CTA.
    # 2^-17 and 2^-15 as above; a factor 2^-22 and a rounding or two 2^-24 for each of up to 60 times that the reference moves: 2^-15.8; the argument of an exponential, up to 2^5 where its weight
    # is 2^-24 or more, 2^-19; everything else 2^-20: less than 2^-13.9 (fp32 results: their rounding is within it).
    B, H, page = (10, 32, 32) if D == 256 else (5, 64, 32)
    P = (n + page - 1) // page
    g = torch.Generator(device="cuda").manual_seed(n + m)
    K = torch.zeros(P, H, page, D, dtype=BF, device="cuda")
    V = (1 + torch.rand(P, H, page, D, generator=g, device="cuda")).to(BF)
    w = torch.arange(P * page, device="cuda", dtype=F32).reshape(P, page) / slope
    got, lse = torch.empty(B * m, H, D, dtype=out, device="cuda"), torch.empty(B * m, H, device="cuda")
    context(pb, H, H, D, BF, out).pact_chunk_attention(pb.PagedCache(K, V, w), torch.zeros(B * m, H, D, dtype=BF, device="cuda"), torch.arange(P, dtype=I32, device="cuda").repeat(B, 1), i32([n] * B),
                                                       i32([m] * B), got, row_stride=m, lse=lse)
    s = w.reshape(-1)[:n].double()
    p = torch.exp(s - s[-1])
    sums, v = p.cumsum(0)[n - m:], V.transpose(0, 1).reshape(H, -1, D)[:, :n]
    last = torch.arange(n - m, n, device="cuda")
    want = torch.stack([((x.double() * p[:, None]).cumsum(0)[last] / sums[:, None]) for x in v], 1).cpu().numpy()
    err = np.abs(f64(got).reshape(B, m, H, D) - want)
    assert (err <= 2.0 ** -13.9 * want + (half_step(want) if out == BF else 0)).all()
    assert ((lse.double().view(B, m, H) - (s[-1] + torch.log(sums))[None, :, None]).abs() <= 2.0 ** -13.9 + 2.0 ** -23 * n / slope).all()
