"""ris_device_status: its cost beside a small copy's, and that it reports and clears what any of the kernels left."""
import time

import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, filled, randn

pytestmark = pytest.mark.gpu


def fastest(call, n=100):
    best = float("inf")
    for _ in range(7):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for _ in range(n):
            call()
        best = min(best, (time.perf_counter() - t) / n)
    return best


def test_status_costs_little_more_than_a_copy():
    x = torch.zeros(1, dtype=torch.int32, device="cuda")
    ris.ris_device_status()
    copy, status = fastest(lambda: x.item()), fastest(ris.ris_device_status)
    # a synchronisation, a launch and one copy; each further copy would add half a copy's time or more
    assert status <= 2.5 * copy + 2e-6, (status, copy)


def test_words_of_several_kernels_are_taken_at_once():
    cache, q = filled(1, 1, 64, 32, [32]), randn(1, 1, 64, dtype=BF16)
    k = randn(1, 1, 64, dtype=BF16)
    with ris.ris_pack_create([1]) as one:
        ris.ris_cache4_append(cache, one, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"))  # past the capacity
    try:
        ris.ris_debug_tile_stall(True, 4000)
        ris.ris_cache4_attend(cache, q)
        torch.cuda.synchronize()
    finally:
        ris.ris_debug_tile_stall(False, 0)
    with pytest.raises(ris.RisError) as e:
        ris.ris_device_status()
    assert e.value.status == ris.RIS_ERR_DEVICE_TIMEOUT  # the graver of the two
    ris.ris_device_status()
    with ris.ris_pack_create([1]) as one:
        ris.ris_cache4_append(cache, one, k, k, torch.zeros(1, dtype=torch.int32, device="cuda"))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with pytest.raises(ris.RisError) as e:
        ris.ris_device_status(stream=side)
    assert e.value.status == ris.RIS_ERR_INVALID
    ris.ris_device_status()
