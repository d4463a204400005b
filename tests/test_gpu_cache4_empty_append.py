"""An append of no rows at given slots sets the lengths as one with rows does: within 0 .. capacity."""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [0, 1])
def test_lengths_stay_within_the_capacity(rows):
    """Sequences without rows: the same lengths whether another one has some or not."""
    B, H, D, cap = 300, 1, 64, 32
    cache = ris.Cache4.empty(B, H, D, cap)
    start = torch.arange(-20, B - 20, dtype=torch.int32, device="cuda")
    start[0], start[1], start[299] = -2 ** 31, 2 ** 31 - 1, 0
    k = randn(rows, H, D, dtype=BF16)
    with ris.ris_pack_create([0] * (B - 1) + [rows]) as pack:
        ris.ris_cache4_append(cache, pack, k, k, torch.zeros(rows, dtype=torch.int32, device="cuda"), start=start)
    ris.ris_device_status()
    want = start.clamp(0, cap).tolist()
    want[-1] = rows
    assert cache.length.tolist() == want
    rk, _ = ris.ris_cache4_read(cache)
    assert rk.shape == (B, H, cap, D)


def test_no_rows_after_the_slots_in_use():
    cache = ris.Cache4.empty(2, 1, 64, 16)
    cache.length.copy_(torch.tensor([5, 16]))
    k = randn(0, 1, 64, dtype=BF16)
    with ris.ris_pack_create([0, 0]) as pack:
        ris.ris_cache4_append(cache, pack, k, k, torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert cache.length.tolist() == [5, 16]
