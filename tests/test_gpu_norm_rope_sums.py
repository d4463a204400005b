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
