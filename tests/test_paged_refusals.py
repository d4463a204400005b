"""What the normed-head and paged-cache entry points refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest

from test_serving_refusals import mem, refused, ris  # noqa: F401  (fixtures)


def test_norm_rope(ris, mem):  # noqa: F811
    L, (_, p), before = ris.lib(), mem, ris.ris_launch_count()
    rope = ris.rope_cfg(1, 1e4, 2048)
    ok = dict(q=p, k=p, qo=p, ko=p, dt=1, n=3, heads=2, kv=1, D=128, qs=256, ks=128, qos=256, kos=128, pos=p, qw=p, kw=p, eps=1e-6, rot=0,
              pairs=0, ctx=100, rope=rope)
    bad = [dict(q=None), dict(q=p + 4), dict(qo=None), dict(k=None), dict(ko=p + 8), dict(dt=2), dict(n=-1), dict(n=2 ** 31), dict(heads=0),
           dict(kv=-1), dict(D=96), dict(qs=255), dict(qs=128), dict(ks=64), dict(qos=260), dict(kos=64), dict(pos=None), dict(pos=p + 2),
           dict(qw=p + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rot=8), dict(rot=144), dict(rot=40),
           dict(rot=-16), dict(pairs=2), dict(ctx=0), dict(rope=None, qw=None, kw=None), dict(rope=None, rot=64),
           dict(rope=ris.rope_cfg(0), qw=None, kw=None), dict(qos=512), dict(kv=0)]
    for c in bad:
        a = dict(ok, **c)
        r = None if a["rope"] is None else ctypes.byref(a["rope"])
        refused(ris, L.ris_norm_rope(a["q"], a["k"], a["qo"], a["ko"], a["dt"], a["n"], a["heads"], a["kv"], a["D"], a["qs"], a["ks"],
                                     a["qos"], a["kos"], a["pos"], a["qw"], a["kw"], a["eps"], a["rot"], a["pairs"], a["ctx"], r, None))
    ok.update(dq=p, dk=p, gq=p, gk=p, gqw=p, gkw=p, dqs=256, dks=128, gqs=256, gks=128)
    bad = [dict(dq=None), dict(dk=p + 8), dict(gq=None), dict(gk=p + 4), dict(q=None), dict(k=None), dict(gqw=None), dict(gkw=p + 2), dict(qw=None),
           dict(kw=None), dict(dqs=128), dict(dks=130), dict(gqs=257), dict(gks=0), dict(qs=512), dict(ks=256), dict(gqs=512), dict(dt=3),
           dict(n=-1), dict(rot=24), dict(pos=None), dict(kv=0)]
    for c in bad:
        a = dict(ok, **c)
        refused(ris, L.ris_norm_rope_backward(a["dq"], a["dk"], a["q"], a["k"], a["gq"], a["gk"], a["gqw"], a["gkw"], a["dt"], a["n"],
                                              a["heads"], a["kv"], a["D"], a["dqs"], a["dks"], a["qs"], a["ks"], a["gqs"], a["gks"], a["pos"],
                                              a["qw"], a["kw"], a["eps"], a["rot"], a["pairs"], a["ctx"], ctypes.byref(rope), None))
    assert ris.ris_launch_count() == before


def paged(ris, p, **kw):  # noqa: F811
    d = dict(batch=2, kv_heads=2, head_dim=128, page_size=16, dtype=1, n_pages=4, table_len=3, reserved=0, page_stride=4096, head_stride=2048,
             slot_stride=128, k=p, v=p, table=p, length=p)
    d.update(kw)
    return ris._PagedDesc(*[d[n] for n, _ in ris._PagedDesc._fields_])


def test_paged(ris, mem):  # noqa: F811
    L, (_, p), before = ris.lib(), mem, ris.ris_launch_count()
    pack = ctypes.c_void_p(0)
    # (every descriptor is refused before the pack is looked at, and a pack is refused where there is none)
    for c in (dict(batch=0), dict(batch=65536), dict(kv_heads=0), dict(kv_heads=4097), dict(head_dim=32), dict(page_size=8), dict(page_size=24),
              dict(page_size=2048), dict(dtype=2), dict(n_pages=0), dict(table_len=0), dict(table_len=2 ** 27), dict(reserved=1),
              dict(page_stride=64), dict(head_stride=0), dict(slot_stride=132), dict(slot_stride=-128), dict(page_stride=2 ** 37), dict(k=None),
              dict(v=p + 8), dict(table=None), dict(table=p + 2), dict(length=None), dict(length=p + 1), dict()):
        d = ctypes.byref(paged(ris, p, **c))
        refused(ris, L.ris_paged_append(d, pack, p, p, 256, 256, None, None))
        assert (b"pack" in L.ris_last_error()) == (not c)
        refused(ris, L.ris_paged_attend(d, pack, p, 512, 4, 0, 0, 0, p, None, None))
        assert (b"pack" in L.ris_last_error()) == (not c)
    refused(ris, L.ris_paged_append(None, pack, p, p, 256, 256, None, None))
    refused(ris, L.ris_paged_attend(None, pack, p, 512, 4, 0, 0, 0, p, None, None))
    assert ris.ris_launch_count() == before


def test_binding(ris):  # noqa: F811
    """What the binding itself refuses: tensors that are not on the GPU."""
    import torch

    k = torch.zeros(4, 2, 16, 64)
    t, n = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        ris.PagedCache(k, k, t, n)
    with pytest.raises(ValueError):
        ris.ris_norm_rope(torch.zeros(3, 2, 64), None, None, 10, None, torch.ones(64))
