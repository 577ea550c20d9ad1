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
