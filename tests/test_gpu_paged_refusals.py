"""What the calls on a cache in pages refuse with a pack at hand, before anything is launched, and allocations that fail."""
import ctypes

import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_failures import _sweep
from test_gpu_paged import BF16, F32, make, randn
from test_paged_refusals import paged
from test_serving_refusals import mem, refused  # noqa: F401

pytestmark = pytest.mark.gpu


def test_refused(mem):  # noqa: F811
    L, (_, p) = ris.lib(), mem
    pack, other, none = (ris.ris_pack_create(x) for x in ([3, 2], [3, 2, 1], [0, 0]))
    q = p + 16  # (addresses that are never read: every call below is refused, or has no rows)
    before = ris.ris_launch_count()
    d = ctypes.byref(paged(ris, p, length=p + 4))
    ok = dict(pack=pack, k=p, v=p, ks=256, vs=256, start=None)
    for c in (dict(pack=other), dict(k=None), dict(v=p + 8), dict(ks=128), dict(vs=260), dict(ks=2 ** 31 + 8), dict(start=p + 2), dict(start=p + 4)):
        a = dict(ok, **c)
        refused(ris, L.ris_paged_append(d, a["pack"].handle, a["k"], a["v"], a["ks"], a["vs"], a["start"], None))
    ok = dict(pack=pack, q=p, qs=512, heads=4, window=0, anchors=0, longest=0, out=p + 2 ** 20, lse=None)
    for c in (dict(pack=other), dict(q=None), dict(q=q + 4), dict(qs=256), dict(qs=516), dict(heads=3), dict(heads=0), dict(heads=65536), dict(window=-1),
              dict(window=4, anchors=-1), dict(anchors=1), dict(longest=-1), dict(longest=49), dict(out=None), dict(out=q + 8), dict(lse=p + 4)):
        a = dict(ok, **c)
        refused(ris, L.ris_paged_attend(d, a["pack"].handle, a["q"], a["qs"], a["heads"], a["window"], a["anchors"], a["longest"], a["out"],
                                        a["lse"], None))
    for at in (p, p + 16, p + 5 * 1024 - 16):  # (outputs over the queries, which are read again after outputs have been written)
        refused(ris, L.ris_paged_attend(d, pack.handle, p, 512, 4, 0, 0, 0, at, None, None))
        refused(ris, L.ris_paged_attend(d, pack.handle, at, 512, 4, 0, 0, 0, p, None, None))
    assert L.ris_paged_attend(d, none.handle, None, 0, 4, 0, 0, 0, None, None, None) == ris.RIS_OK  # (no rows: nothing to do)
    assert ris.ris_launch_count() == before


def test_binding_refuses():
    cache, *_ = make([20, 30], 2, 64, 16, BF16)
    q, k = randn(5, 4, 64, dtype=BF16), randn(5, 2, 64, dtype=BF16)
    before = ris.ris_launch_count()
    with ris.ris_pack_create([3, 2]) as pack:
        for bad in (randn(6, 4, 64, dtype=BF16), randn(5, 4, 128, dtype=BF16), randn(5, 8, 64, dtype=BF16)[:, ::2]):
            with pytest.raises(ValueError):
                ris.ris_paged_attend(cache, pack, bad)
        with pytest.raises(AssertionError):
            ris.ris_paged_attend(cache, pack, q.float())
        with pytest.raises(ris.RisError):
            ris.ris_paged_attend(cache, pack, q, out=q)
        with pytest.raises(AssertionError):
            ris.ris_paged_attend(cache, pack, q, out=torch.empty(5, 4, 64, device="cuda"))
        with pytest.raises(AssertionError):
            ris.ris_paged_attend(cache, pack, q, out=torch.empty(5, 8, 64, dtype=BF16, device="cuda")[:, :4])
        for bad in (randn(4, 2, 64, dtype=BF16), randn(5, 1, 64, dtype=BF16), randn(5, 2, 128, dtype=BF16)):
            with pytest.raises(ValueError):
                ris.ris_paged_append(cache, pack, bad, bad)
        with pytest.raises(ValueError):
            ris.ris_paged_append(cache, pack, k, k, start=torch.zeros(3, dtype=torch.int32, device="cuda"))
        with pytest.raises(ValueError):
            ris.ris_paged_append(cache, pack, k, k, start=torch.zeros(2, device="cuda"))
        with pytest.raises(AssertionError):
            ris.ris_paged_append(cache, pack, k.float(), k.float())
    assert ris.ris_launch_count() == before


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_allocations_that_fail(dtype):
    cache, *_ = make([300, 900], 2, 64, 16, dtype)
    q, out = randn(203, 4, 64, dtype=dtype), torch.empty(203, 4, 64, dtype=dtype, device="cuda")
    with ris.ris_pack_create([200, 3]) as pack:
        fails, _ = _sweep(lambda: ris.ris_paged_attend(cache, pack, q, out=out))
        assert fails == 1
        kept = out.clone()
        ris.ris_paged_attend(cache, pack, q, out=out)
        assert torch.equal(kept, out)
    d, w = randn(203, 4, 64, dtype=dtype), randn(64, dtype=dtype)
    gq = torch.empty_like(d)
    fails, _ = _sweep(lambda: ris.ris_norm_rope_backward(d, None, q, None, None, 1, None, w, gq=gq))
    assert fails == 1
    ris.ris_device_status()
