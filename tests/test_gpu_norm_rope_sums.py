"""Long sums in the gradient of the normed heads' weights."""
import pytest
import torch

from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu
F32 = torch.float32


def test_gradient_of_a_weight_over_thousands_of_terms():
    """Every thread adds up a thousand equal terms, which fp32 additions one after another would round the same way time and again: off by 1e-5
    of the sum for dy = 0.1. With runs of at most 64 of them in fp32 and all else in pairs: 63 x 2^-24 of the sum, the root's 2^-22,
    and 2^-23 for the product and the result."""
    D, H = 128, 100
    n = 16 * 304 * 1000 // H  # (16 tokens side by side in each of 304 CTAs)
    x = torch.ones(n, H, D, device="cuda")
    dy = 0.1 + 0.013 * torch.arange(D, dtype=F32, device="cuda")
    d = dy.expand(n, H, D).contiguous()
    w = torch.ones(D, device="cuda")
    _, _, gw, _ = ris.ris_norm_rope_backward(d, None, x, None, None, 1, None, w, eps=0.0, gq=d)
    want = dy.double() * (n * H)
    assert ((gw.double() - want).abs() <= (63 * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23) * want).all(), float(((gw.double() - want).abs() / want).max())


@pytest.mark.parametrize("n", [1, 3000])
def test_an_infinite_term(n):
    """An infinity among the terms of a channel: its sum is that, NaN with both signs or a NaN, and the other channels' are as without it."""
    D, H = 64, 2
    g = torch.Generator().manual_seed(n)
    x, d = (torch.randn(n, H, D, generator=g).cuda() for _ in range(2))
    x = x.abs() + 0.5
    w = torch.ones(D, device="cuda")

    def call(dy):
        return ris.ris_norm_rope_backward(dy, None, x, None, None, 1, None, w)[2]

    clean, bad = call(d), d.clone()
    inf, nan = float("inf"), float("nan")
    bad[n // 2, 0, 3], bad[n // 2, 1, 5], bad[0, 0, 7], bad[0, 0, 9], bad[n - 1, 1, 9] = inf, -inf, nan, inf, -inf
    got = call(bad)
    assert got[3] == inf and got[5] == -inf and got[7].isnan() and got[9].isnan()
    rest = [c for c in range(D) if c not in (3, 5, 7, 9)]
    assert torch.equal(got[rest], clean[rest])
