"""Waits of the 4-bit attention that give up: reported, with nothing left on its way to shared memory, and the next calls right.

With its copies left out (ris_debug_tile_stall) the first wait gives up after a few thousand cycles; with short limits alone
a wait may end at any point, with copies under way.
"""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, F32, filled, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def defaults():
    ris.ris_device_status()
    yield
    ris.ris_debug_tile_stall(False, 0)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_copies_that_never_come(out, D):
    lens = [5000, 17, 0, 300]
    cache, q = filled(4, 2, D, 5008, lens), randn(4, 12, D, seed=1, dtype=BF16)
    w = torch.zeros_like(cache.weight)

    def call():
        return ris.ris_cache4_attend(cache, q, out_dtype=out, return_lse=True, weight_out=w) + (w.clone(),)

    ref = call()
    ris.ris_device_status()
    ris.ris_debug_tile_stall(True, 4000)
    call()
    torch.cuda.synchronize()
    ris.ris_debug_tile_stall(False, 0)
    with pytest.raises(ris.RisError) as e:
        ris.ris_device_status()
    assert e.value.status == ris.RIS_ERR_DEVICE_TIMEOUT
    for _ in range(2):
        again = call()
        ris.ris_device_status()  # (the word was cleared by the read)
        assert all(torch.equal(a, b) for a, b in zip(again, ref))


@pytest.mark.parametrize("out", [F32, BF16])
def test_waits_cut_short_with_copies_under_way(out):
    lens = [20000, 9000, 1, 16000, 700, 20000]
    cache, q = filled(6, 2, 128, 20000, lens), randn(6, 12, 128, seed=1, dtype=BF16)

    def call():
        return ris.ris_cache4_attend(cache, q, out_dtype=out, return_lse=True)

    ref = call()
    ris.ris_device_status()
    for limit in (1, 30, 100, 300, 600, 1000, 2000, 4000):
        ris.ris_debug_tile_stall(False, limit)
        call()
        torch.cuda.synchronize()
        ris.ris_debug_tile_stall(False, 0)
        try:
            ris.ris_device_status()
        except ris.RisError as e:
            assert e.status == ris.RIS_ERR_DEVICE_TIMEOUT
        again = call()
        ris.ris_device_status()
        assert all(torch.equal(a, b) for a, b in zip(again, ref)), limit
