"""Packs used on streams other than their own and freed while that work is still queued: the plan's memory must not be given to
the next pack before. Results are compared with those of the same calls made one by one."""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, F32, randn

pytestmark = pytest.mark.gpu
HQ, HKV, D = 4, 2, 64


def busy(x, n=60):
    """Some tens of milliseconds of work on the current stream."""
    y = x
    for _ in range(n):
        y = y @ x
    return y


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("how", ["free", "with", "dropped"])
def test_pack_freed_while_another_stream_has_yet_to_use_it(dtype, how):
    lens, other = [70, 200, 3], [3, 200, 70]
    n = sum(lens)
    q, k, v = (randn(n, h, D, seed=h + i, dtype=dtype) for i, h in enumerate((HQ, HKV, HKV)))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    with ris.ris_pack_create(lens) as pack:
        want = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=9)
        ref = ris.Cache4.empty(3, HKV, D, 208)
        ris.ris_cache4_append(ref, pack, k, v, pos)
    big = randn(4096, 4096, seed=5, scale=1 / 64)
    side = torch.cuda.Stream()
    for calls in ("attention", "append", "both"):
        cache = ris.Cache4.empty(3, HKV, D, 208)
        torch.cuda.synchronize()
        pack, got = ris.ris_pack_create(lens), None
        with torch.cuda.stream(side):
            busy(big)
            if calls != "append":
                got = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=9)
            if calls != "attention":
                ris.ris_cache4_append(cache, pack, k, v, pos)
        if how == "free":
            pack.free()
        elif how == "with":
            with pack:
                pass
        pack = None
        later = [ris.ris_pack_create(other) for _ in range(4)]  # (of the same size: the freed memory's next owners)
        torch.cuda.synchronize()
        ris.ris_device_status()
        if got is not None:
            for a, b in zip(got, want):
                assert torch.equal(a, b)
        if calls != "attention":
            for name in ("k", "v", "k_scale", "v_scale", "pos", "length"):
                assert torch.equal(getattr(cache, name), getattr(ref, name)), name
        for p in later:
            p.free()


def test_pack_of_many_streams_leaves_nothing_behind():
    torch.cuda.synchronize()
    lens = [5, 9]
    q, k, v = (randn(14, h, D, seed=h, dtype=BF16) for h in (HQ, HKV, HKV))
    side = [torch.cuda.Stream() for _ in range(5)]
    before = ris.ris_memory_stats()[0]
    outs = []
    for _ in range(3):
        with ris.ris_pack_create(lens) as pack:
            for s in side:
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    outs.append(ris.ris_attention_packed(pack, q, k, v)[0])
    torch.cuda.synchronize()
    assert ris.ris_memory_stats()[0] == before
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_pack_in_a_graph_captured_on_another_stream():
    lens = [70, 31]
    q, k, v = (randn(101, h, D, seed=h, dtype=BF16) for h in (HQ, HKV, HKV))
    with ris.ris_pack_create(lens) as pack:
        want, = ris.ris_attention_packed(pack, q, k, v)
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=side):
            got, = ris.ris_attention_packed(pack, q, k, v)
        for _ in range(2):
            got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)
