"""Scratch of the 4-bit attention with weights goes by the caller's bound of the lengths, not by the cache's capacity."""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, attend_plain, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("longest", [300, 301, 304, 1023])
def test_scratch_goes_by_the_bound_of_the_lengths(longest):
    B, Hq, Hkv, D, cap = 2, 16, 2, 64, 1 << 20
    lens = [300, 17]
    cache = ris.Cache4.empty(B, Hkv, D, cap)
    with ris.ris_pack_create(lens) as pack:
        k, v = (randn(sum(lens), Hkv, D, seed=s) for s in (1, 2))
        ris.ris_cache4_append(cache, pack, k, v, torch.arange(sum(lens), dtype=torch.int32, device="cuda"))
    q = randn(B, Hq, D, seed=3, dtype=BF16)
    w = torch.full_like(cache.weight, -1.0)
    torch.cuda.synchronize()
    before = ris.ris_memory_stats(reset_high_water=True)[0]
    ris.ris_cache4_attend(cache, q, weight_out=w, longest=longest)
    torch.cuda.synchronize()
    # (the scores of every head and slot take B Hq longest floats, the partial results of the CTAs some hundred KB)
    assert ris.ris_memory_stats()[1] - before <= 4 * B * Hq * (longest + 3) + (2 << 20)
    ris.ris_device_status()
    small = ris.Cache4.empty(B, Hkv, D, 304)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(small, name).copy_(getattr(cache, name)[:, :, :304])
    small.length.copy_(cache.length)
    _, _, rw = attend_plain(small, q, lens)
    for b, n in enumerate(lens):
        assert (w[b, :, :n].double().cpu() - rw[b, :, :n]).abs().max() <= 2e-5
        assert (w[b, :, n:] == -1.0).all()
