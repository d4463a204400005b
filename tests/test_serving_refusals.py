"""What the serving entry points refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def ris():
    from paper_2607_21927_gb300 import build, ris as binding

    build.build()
    return binding


@pytest.fixture(scope="module")
def mem():
    buf = (ctypes.c_uint8 * 512)()
    p = ctypes.addressof(buf)
    return buf, p + (-p % 16)


def desc(ris, p, **kw):
    d = dict(batch=2, kv_heads=2, head_dim=128, reserved=0, capacity=32, k=p, v=p, k_scale=p, v_scale=p, pos=p, weight=p, length=p, sync=p)
    d.update(kw)
    return ris._Cache4Desc(*[d[n] for n, _ in ris._Cache4Desc._fields_])


def refused(ris, st, want=None):
    assert st == (ris.RIS_ERR_INVALID if want is None else want), (st, ris.ris_last_error())
    assert ris.ris_last_error() != ""


def test_pack_lengths(ris):
    L, h = ris.lib(), ctypes.c_void_p(1)
    one = (ctypes.c_int64 * 1)(5)
    for lens, klens, n in (([-1], None, 1), ([5], [-2], 1), ([5], None, 0), ([5], None, 65536), ([2 ** 31], None, 1),
                           ([2 ** 30, 2 ** 30], None, 2), ([2 ** 62, 2 ** 62, 2 ** 62], None, 3)):
        a = (ctypes.c_int64 * len(lens))(*lens)
        b = None if klens is None else (ctypes.c_int64 * len(klens))(*klens)
        refused(ris, L.ris_pack_create(a, b, n, ctypes.byref(h), None))
        assert h.value is None
    refused(ris, L.ris_pack_create(None, None, 1, ctypes.byref(h), None))
    refused(ris, L.ris_pack_create(one, None, 1, None, None))
    refused(ris, L.ris_pack_info(None, None, None, None, None, None))
    assert L.ris_pack_free(None) == ris.RIS_OK


def test_rope_axes(ris, mem):
    L, (_, p), before = ris.lib(), mem, ris.ris_launch_count()
    sec = (ctypes.c_int32 * 4)(16, 24, 24, 0)
    ok = dict(q=p, k=p, qo=p, ko=p, dt=1, n=3, heads=2, kv=1, D=128, qs=256, ks=128, pos=p, axes=3, sec=sec, il=0, ctx=100,
              rope=ris.rope_cfg(1, 1e4, 2048), inv=0)
    bad = [dict(q=None), dict(q=p + 4), dict(qo=None), dict(k=None), dict(ko=p + 8), dict(dt=2), dict(n=-1), dict(heads=0), dict(kv=-1),
           dict(D=96), dict(qs=255), dict(qs=260), dict(qs=128), dict(ks=64), dict(pos=None), dict(pos=p + 2), dict(axes=0),
           dict(axes=5), dict(sec=None), dict(axes=2), dict(il=2), dict(inv=-1), dict(ctx=0), dict(rope=None),
           dict(rope=ris.rope_cfg(0)), dict(sec=(ctypes.c_int32 * 4)(80, -8, -8, 0)), dict(qs=512)]
    for c in bad:
        a = dict(ok, **c)
        r = None if a["rope"] is None else ctypes.byref(a["rope"])
        refused(ris, L.ris_rope_axes(a["q"], a["k"], a["qo"], a["ko"], a["dt"], a["n"], a["heads"], a["kv"], a["D"], a["qs"], a["ks"],
                                     a["pos"], a["axes"], a["sec"], a["il"], a["ctx"], r, a["inv"], None))
    assert ris.ris_launch_count() == before


def test_cache4(ris, mem):
    L, (_, p), before = ris.lib(), mem, ris.ris_launch_count()
    good = desc(ris, p)
    bad = [dict(batch=0), dict(batch=65536), dict(kv_heads=0), dict(head_dim=32), dict(reserved=1), dict(capacity=0), dict(capacity=40),
           dict(capacity=2 ** 31), dict(k=None), dict(v=p + 8), dict(k_scale=None), dict(v_scale=p + 4), dict(pos=None),
           dict(weight=None), dict(length=None), dict(sync=None)]
    for c in bad:
        d = ctypes.byref(desc(ris, p, **c))
        refused(ris, L.ris_cache4_read(d, None, 1, p, p, None))
        refused(ris, L.ris_cache4_attend(d, p, 4, 1, 1, 0, p, None, None, None, None))
        refused(ris, L.ris_cache4_append(d, None, p, p, 256, 256, 1, p, None, None, None))
        refused(ris, L.ris_cache4_evict(d, ctypes.byref(good), 8, 0, p, None))
        refused(ris, L.ris_cache4_evict(ctypes.byref(good), d, 8, 0, p, None))
    g = ctypes.byref(good)
    refused(ris, L.ris_cache4_append(g, None, p, p, 256, 256, 1, p, None, None, None))
    for count, k in ((-1, p), (33, p), (1, None), (1, p + 4)):
        refused(ris, L.ris_cache4_read(g, None, count, k, p, None))
    ok = dict(q=p, heads=4, dt=1, odt=0, longest=0, out=p, lse=None, wi=None, wo=None)
    for c in [dict(q=None), dict(heads=3), dict(heads=0), dict(dt=5), dict(odt=-1), dict(longest=-1), dict(longest=33), dict(out=None),
              dict(lse=p + 4), dict(wi=p), dict(wo=p + 4)]:
        a = dict(ok, **c)
        refused(ris, L.ris_cache4_attend(g, a["q"], a["heads"], a["dt"], a["odt"], a["longest"], a["out"], a["lse"], a["wi"], a["wo"], None))
    one = ctypes.byref(desc(ris, p, kv_heads=1))
    refused(ris, L.ris_cache4_attend(one, p, 4097, 1, 1, 0, p, None, None, p, None), ris.RIS_ERR_UNSUPPORTED)
    other = desc(ris, p + 16)
    for s, d, budget, recent, kept in ((good, good, 0, 0, p), (good, good, 33, 0, p), (good, good, 8, 8, p), (good, good, 8, -1, p),
                                       (good, good, 8, 0, None), (good, desc(ris, p, capacity=16), 8, 0, p),
                                       (good, desc(ris, p + 16, v=p), 8, 0, p), (good, desc(ris, p + 16, batch=1), 8, 0, p),
                                       (good, desc(ris, p + 16, head_dim=64), 8, 0, p), (good, desc(ris, p + 16, capacity=16), 17, 0, p)):
        refused(ris, L.ris_cache4_evict(ctypes.byref(s), ctypes.byref(d), budget, recent, kept, None))
    assert ris.ris_launch_count() == before


def test_without_device_fails_loudly(ris, mem):
    import torch

    if torch.cuda.is_available():
        pytest.skip("host has a GPU")
    _, p = mem
    h, one = ctypes.c_void_p(), (ctypes.c_int64 * 1)(5)
    assert ris.lib().ris_pack_create(one, None, 1, ctypes.byref(h), None) == ris.RIS_ERR_CUDA and h.value is None
    assert ris.lib().ris_cache4_attend(ctypes.byref(desc(ris, p)), p, 4, 1, 1, 0, p, None, None, None, None) == ris.RIS_ERR_CUDA
