"""An append of no rows after the slots in use sets the lengths as one with rows does: within 0 .. the sequence's slots."""
import pytest
import torch

from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [0, 1])
@pytest.mark.parametrize("given", [False, True])
def test_lengths_stay_within_the_slots(rows, given):
    """Sequences without rows: the same lengths whether another one has some or not, and whether `start` says them or not."""
    B, page, width = 300, 16, 2
    z = dict(dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(4, 1, page, 64, **z) for _ in range(2))
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    start = torch.arange(-20, B - 20, dtype=torch.int32, device="cuda")
    start[0], start[1], start[B - 1] = -2 ** 31, 2 ** 31 - 1, 0
    cache = ris.PagedCache(k, v, table, torch.full((B,), 7, dtype=torch.int32, device="cuda") if given else start.clone())
    x = torch.zeros(rows, 1, 64, **z)
    with ris.ris_pack_create([0] * (B - 1) + [rows]) as pack:
        ris.ris_paged_append(cache, pack, x, x, start=start if given else None)
    ris.ris_device_status()
    want = start.clamp(0, page * width).tolist()
    want[-1] = rows
    assert cache.length.tolist() == want
