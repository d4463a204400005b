"""Sines and cosines of normed and turned heads to what the arithmetic allows, at any position."""
import pytest
import torch

from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("D", [64, 128])
def test_angles(D, pairs):
    """Pairs (1, 0) come out as (cos, sin) of their angles. The angle is a fraction of a turn in 64 bits, good to 2^-52 of itself (the
    double frequency and its product with a constant: 200,000 x 2^-52 = 5e-11; as much for the 64-bit reference's), of which a
    correction by cos or sin times the last bits leaves out 2^-43 at most. Sine and cosine are good to two units in their last place (2^-22 of
    themselves), the correction and the products round three times more (3 x 2^-24): 2^-21 of the value + 2e-10, however small
    the value. An angle rounded to 24 bits is off by up to 9e-8."""
    g = torch.Generator().manual_seed(D)
    n = 2000
    pos = torch.randint(-200000, 200001, (n,), generator=g, dtype=torch.int32)
    pos[:5] = torch.tensor([0, 1, -1, 200000, -200000])
    rope = ris.rope_cfg(ris.ROPE_PLAIN, 1e4, 2048)
    f, _ = ris.ris_rope_freqs(rope, 200001, D)
    x = torch.zeros(n, 1, D)
    (x[..., 0::2] if pairs else x[..., :D // 2]).fill_(1.0)
    y, _ = ris.ris_norm_rope(x.cuda(), None, pos.cuda(), 200001, rope, pairs=pairs)
    y = y[:, 0].double().cpu()
    c, s = (y[:, 0::2], y[:, 1::2]) if pairs else (y[:, :D // 2], y[:, D // 2:])
    ang = pos.double()[:, None] * torch.tensor(f, dtype=torch.float64)
    for got, want in ((c, ang.cos()), (s, ang.sin())):
        assert ((want.abs() < 0.02).sum() > 100)  # (values so small that an angle's rounding would show)
        assert ((got - want).abs() <= 2.0 ** -21 * want.abs() + 2e-10).all()
