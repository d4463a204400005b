"""Waits of the attention over pages that give up: reported, with nothing left on its way to shared memory, tensor memory released, and the
next calls right.

With its copies left out (ris_debug_tile_stall) the first wait on them gives up after a few thousand cycles; with short limits alone
a wait may end at any point, with copies and products under way.
"""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_paged import BF16, make, randn

pytestmark = pytest.mark.gpu

# rows of each sequence, keys before them, window, anchors: row tiles that several CTAs share, many short ones, few rows
CALLS = [([300, 1, 0, 40], [2000, 5000, 7, 0], 0, 0), ([900, 200], [50, 3000], 200, 70), ([1, 4, 1], [9000, 700, 0], 0, 0)]


@pytest.fixture(autouse=True)
def defaults():
    ris.ris_device_status()
    yield
    ris.ris_debug_tile_stall(False, 0)


def setup(q_lens, prior, window, anchors, D):
    Hq, Hkv = (12, 2) if D == 128 else (8, 2)
    cache, *_ = make([n + p for n, p in zip(q_lens, prior)], Hkv, D, 32, BF16, seed=1)
    q, pack = randn(sum(q_lens), Hq, D, seed=2, dtype=BF16), ris.ris_pack_create(q_lens)
    return lambda: ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", CALLS)
def test_copies_that_never_come(case, D):
    call = setup(*case, D)
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", CALLS)
def test_waits_cut_short_with_copies_and_products_under_way(case, D):
    call = setup(*case, D)
    ref = call()
    ris.ris_device_status()
    gave_up = 0
    for limit in (1, 30, 100, 300, 600, 1000, 2000, 4000):
        ris.ris_debug_tile_stall(False, limit)
        call()
        torch.cuda.synchronize()
        ris.ris_debug_tile_stall(False, 0)
        try:
            ris.ris_device_status()
        except ris.RisError as e:
            assert e.status == ris.RIS_ERR_DEVICE_TIMEOUT
            gave_up += 1
        again = call()
        ris.ris_device_status()
        assert all(torch.equal(a, b) for a, b in zip(again, ref)), limit
    assert gave_up > 0


@pytest.mark.parametrize("D", [64, 128])
def test_waits_cut_short_in_a_call_of_two_passes(D):
    """With a value that is not finite, in the middle of the rows."""
    q_lens, lengths = [300, 1], [2300, 900]
    Hq, Hkv = (12, 2) if D == 128 else (8, 2)
    cache, *_ = make(lengths, Hkv, D, 32, BF16, seed=1)
    cache.v[int(cache.table[0, 2150 // 32]), :, 2150 % 32, 5] = float("nan")
    q = randn(301, Hq, D, seed=2, dtype=BF16)
    with ris.ris_pack_create(q_lens) as pack:
        ref = ris.ris_paged_attend(cache, pack, q)[0]
        ris.ris_device_status()
        for limit in (30, 300, 1000, 2000, 4000):
            ris.ris_debug_tile_stall(False, limit)
            ris.ris_paged_attend(cache, pack, q)
            torch.cuda.synchronize()
            ris.ris_debug_tile_stall(False, 0)
            try:
                ris.ris_device_status()
            except ris.RisError as e:
                assert e.status == ris.RIS_ERR_DEVICE_TIMEOUT
            again = ris.ris_paged_attend(cache, pack, q)[0]
            ris.ris_device_status()
            assert torch.equal(again.view(torch.int16), ref.view(torch.int16)), limit
