"""Attention of several new tokens, on the GPU: calls at the ends of what is allowed, and beyond them."""
import pytest
import torch

from oracle import paged_oracle as po
from tests.test_gpu_chunk import BF, F32, I32, cache_of, context, i32, pb   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("B,n_rows", [(2, 5), (40, 300), (4096, 1 << 16)])
def test_requests_that_share_rows_of_q(pb, dtype, out, B, n_rows):
    """More rows named by all requests together than there are: nothing is served.  As many as there are, side by side: all of them."""
    g, D, page = torch.Generator(device="cuda").manual_seed(B), 64, 16
    K, V, w = cache_of(g, 8, 1, page, D, dtype)
    ctx, cache = context(pb, 2, 1, D, dtype, out), pb.PagedCache(K, V, w)
    Q, got, status = torch.randn(n_rows, 2, D, generator=g, device="cuda").to(dtype), torch.full((n_rows, 2, D), -5.0, dtype=out, device="cuda"), i32([0])
    lse, table, length = torch.full((n_rows, 2), -5.0, device="cuda"), torch.arange(8, dtype=I32, device="cuda").repeat(B, 1), i32([128] * B)
    ctx.pact_chunk_attention(cache, Q, table, length, i32([n_rows] * B), got, row_start=i32([0] * B), lse=lse, status=status)
    assert status.item() == po.INVALID and (got == -5).all() and (lse == -5).all()
    status.zero_()
    ctx.pact_chunk_attention(cache, Q, table, length, i32([(1 << 31) - 1] * B), got, row_start=i32(list(range(B))), lse=lse, status=status)
    assert status.item() == po.INVALID and (got == -5).all() and (lse == -5).all()
    status.zero_()
    m = n_rows // B
    ctx.pact_chunk_attention(cache, Q, table, length, i32([m] * B), got, row_start=i32([m * b for b in range(B)]), lse=lse, status=status)
    assert status.item() == 0 and torch.isfinite(got[:m * B]).all() and (got[:m * B] != -5).any(2).all() and (got[m * B:] == -5).all() and (lse[m * B:] == -5).all()


@pytest.mark.parametrize("dtype,out,page,n", [(BF, BF, 64, (1 << 31) - 64 - 10), (BF, F32, 64, (1 << 31) - 64 - 10), (BF, BF, 16, (1 << 31) - 16 - 3)])
def test_the_longest_requests(pb, dtype, out, page, n):
    """2^31 rows, but for the last few, of pages that lie in the table many times: what the last page holds behind them does not matter."""
    if torch.cuda.mem_get_info()[0] < 4 << 30:
        pytest.skip("not enough memory")
    D, width = 64, n // page + 1
    K, V = torch.zeros(2, 1, page, D, dtype=dtype, device="cuda"), torch.ones(2, 1, page, D, dtype=dtype, device="cuda")
    V[:, :, :, 1] = -2
    V[1, :, n % page:], K[1, :, n % page:] = float("nan"), float("inf")
    table = torch.zeros(1, width, dtype=I32, device="cuda")
    table[0, -1] = 1
    got, lse, status = torch.zeros(3, 1, D, dtype=out, device="cuda"), torch.zeros(3, 1, device="cuda"), i32([0])
    context(pb, 1, 1, D, dtype, out).pact_chunk_attention(pb.PagedCache(K, V), torch.ones(3, 1, D, dtype=dtype, device="cuda"), table, i32([n]), i32([3]), got, row_start=i32([0]), lse=lse,
                                                          status=status)
    # equal weights: exact sums are the values.  A CTA adds up 2^24 / 148 tiles (fp32 results: twice as many of half the size) in sums that grow from nothing, with rounding: 2^18 / 2 * 2^-24 at most
    # for the weights and as much for the results
    assert status.item() == 0 and ((got.double()[..., [0, 1]] - torch.tensor([1.0, -2.0], device="cuda")).abs() <= 2.0 ** -6).all()
    assert (got[..., 2:] == got[..., :1]).all() and ((lse.double() - torch.log(torch.tensor(float(n)))).abs() <= 2.0 ** -6).all()


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
def test_many_more_new_tokens_than_rows(pb, dtype, out):
    """Up to 2^31 - 1 new tokens of a request of 50 rows, of which 300 have a row: none of these sees anything, whatever lay in the places of their tiles before."""
    g, D, page = torch.Generator(device="cuda").manual_seed(0), 64, 16
    K, V, _ = cache_of(g, 300, 1, page, D, dtype)
    V[4:] = float("inf")
    K[4:] = float("nan")
    ctx, cache = context(pb, 1, 1, D, dtype, out), pb.PagedCache(K, V)
    table = torch.arange(4, 300, dtype=I32, device="cuda")[None].repeat(3, 1)
    table[1, :4] = torch.arange(4, dtype=I32, device="cuda")
    Q, got, lse, status = torch.randn(600, 1, D, generator=g, device="cuda").to(dtype), torch.full((600, 1, D), -5.0, dtype=out, device="cuda"), torch.full((600, 1), -5.0, device="cuda"), i32([0])
    for want in ((1 << 31) - 1, (1 << 31) - 200, 1 << 30, 1000):
        ctx.pact_chunk_attention(cache, Q, table[:1], i32([296 * page]), i32([300]), got, row_start=i32([0]))     # (infinities and NaN in all the tiles that shared memory holds)
        ctx.pact_chunk_attention(cache, Q, table[1:2], i32([50]), i32([want]), got, row_start=i32([300]), lse=lse, status=status)
        assert status.item() == po.INVALID and not got[300:].any() and (lse[300:] == -torch.inf).all(), want
        status.zero_()
