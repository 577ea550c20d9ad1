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
