"""Packed prompts, positions on several axes and the 4-bit cache, against plain implementations in 64 bits.

Tolerances, from the arithmetic of each operator:
  rotation        fp32: the angle and its sine and cosine are good to about 2^-22, so a rotated pair is
                  off by at most 2e-6 of its norm; bf16 adds half an ulp, at most 2^-8 of the result (8 significant bits).
  fp32 attention  the parity bar of the fp32 path (relative L2 1e-5); log-sum-exp within 2e-5.
  bf16 attention  the parity bar of the bf16 path with bf16 outputs (1e-2 + 2^-8 |o|, relative L2 5e-3).
  4-bit cache     codes and copies are exact; attention on the values that the codes stand for: fp32
                  outputs 1e-5, bf16 outputs half an ulp (2^-8 |o|, of which half is taken from the next term) and 2^-9 of the
                  row's largest.
  key weights     fp32 sums of exponentials: 2e-5 of the largest.
"""
import math

import pytest
import torch

from helpers import check_bf16_path, check_f32_path, rel_l2, to_np
from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")


def randn(*shape, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


# ---------------------------------------------------------------- rotation
def rotate_plain(x, positions, sections, interleaved, f, mscale):
    """x [n, H, D] in 64 bits at positions [axes, n]."""
    half = x.shape[-1] // 2
    if interleaved:
        n = len(sections)
        axis = [c % n if c % n > 0 and c // n < sections[c % n] else 0 for c in range(half)]
    else:
        axis = [a for a, m in enumerate(sections) for _ in range(m)]
    ang = positions.double().cpu()[axis].T * torch.tensor(f, dtype=torch.float64)
    z = torch.polar(torch.ones_like(ang), ang)[:, None] * torch.complex(x[..., :half].double().cpu(), x[..., half:].double().cpu())
    return torch.cat([z.real, z.imag], -1) * mscale


@pytest.mark.parametrize("n,Hq,Hkv,D,sections,interleaved,dtype,kind", [
    (1, 12, 2, 128, [64], False, BF16, 1),
    (37, 4, 4, 64, [32], False, F32, 2),
    (1000, 12, 2, 128, [16, 24, 24], False, BF16, 1),
    (333, 7, 1, 64, [8, 12, 12], True, F32, 3),
    (65, 16, 1, 128, [24, 20, 20], True, BF16, 3),
    (19, 3, 3, 128, [0, 64, 0, 0], False, F32, 1),
])
def test_rope_axes(n, Hq, Hkv, D, sections, interleaved, dtype, kind):
    g = torch.Generator().manual_seed(n)
    pos = torch.randint(-50, 200000, (len(sections), n), generator=g, dtype=torch.int32).cuda()
    rope = ris.rope_cfg(kind, 1e6, 32768)
    f, ms = ris.ris_rope_freqs(rope, 200000, D)
    fused = randn(n, Hq + 2 * Hkv, D, seed=n, dtype=dtype)
    q, k = fused[:, :Hq], fused[:, Hq:Hq + Hkv]
    qo, ko = ris.ris_rope_axes(q, k, pos, sections, 200000, rope, interleaved=interleaved)
    for x, y in ((q, qo), (k, ko)):
        ref = rotate_plain(x, pos, sections, interleaved, f, ms)
        half = D // 2
        norm = torch.hypot(ref[..., :half], ref[..., half:]).repeat(1, 1, 2)
        tol = 2e-6 * norm + (2.0 ** -8 * (ref.abs() + 2e-6 * norm) if dtype == BF16 else 0) + 1e-30
        assert ((y.double().cpu() - ref).abs() <= tol).all()
    # in place, and without k
    q2 = q.contiguous()
    back, none = ris.ris_rope_axes(q2, None, pos, sections, 200000, rope, interleaved=interleaved, q_out=q2)
    assert none is None and back.data_ptr() == q2.data_ptr() and torch.equal(q2, qo)


def test_rope_axes_inverse_is_the_gradient():
    n, H, D, sections = 50, 2, 64, [8, 12, 12]
    pos = torch.randint(0, 9000, (3, n), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).cuda()
    rope = ris.rope_cfg(ris.ROPE_YARN, 1e4, 2048)
    f, ms = ris.ris_rope_freqs(rope, 9000, D)
    x, dy = randn(n, H, D, seed=3), randn(n, H, D, seed=4)
    dx, _ = ris.ris_rope_axes(dy, None, pos, sections, 9000, rope, inverse=True)
    xd = x.double().cpu().requires_grad_()
    rotate_plain(xd, pos, sections, False, f, ms).backward(dy.double().cpu())
    assert (dx.double().cpu() - xd.grad).abs().max() <= 2e-5
    # and against differences of the forward call itself: <dy, (f(x + h e) - f(x - h e)) / 2h> (linear: any h is exact)
    for seed in (5, 6):
        e = randn(n, H, D, seed=seed)
        up, _ = ris.ris_rope_axes(x + e, None, pos, sections, 9000, rope)
        dn, _ = ris.ris_rope_axes(x - e, None, pos, sections, 9000, rope)
        num = (dy.double() * (up.double() - dn.double()) / 2).sum()
        assert abs(float(num - (dx.double() * e.double()).sum())) <= 1e-5 * float(dy.norm() * e.norm())


# ---------------------------------------------------------------- packed prompts
def packed_plain(q, k, v, q_lens, k_lens, W):
    q, k, v = (x.double().cpu() for x in (q, k, v))
    Hq, D = q.shape[1:]
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, lse, w = torch.zeros_like(q), torch.full((Hq, q.shape[0]), -INF, dtype=torch.float64), torch.zeros(Hkv, k.shape[0], dtype=torch.float64)
    a = b = 0
    for n, m in zip(q_lens, k_lens):
        see = torch.arange(m) <= torch.arange(n)[:, None] + (m - n)
        for h in range(Hq):
            g = h // G
            s = (q[a:a + n, h] @ k[b:b + m, g].T / math.sqrt(D)).masked_fill(~see, -INF)
            s = torch.where(see, s, torch.full_like(s, -INF))
            l = torch.logsumexp(s, -1) if m else torch.full((n,), -INF, dtype=torch.float64)
            p = torch.where(see, torch.exp(s - l[:, None]), torch.zeros_like(s))
            vv = v[b:b + m, g]
            out[a:a + n, h] = torch.where(see[..., None], p[..., None] * vv, torch.zeros(())).sum(1) if not torch.isfinite(vv).all() else p @ vv
            lse[h, a:a + n] = l
            w[g, b:b + m] += p[max(0, n - W):].sum(0)
        a, b = a + n, b + m
    return out, lse, w


PACKS = [
    # q lengths, k lengths (None: the same)
    ([1], None),
    ([64], None),
    ([129], None),
    ([1, 0, 2, 127, 128, 300], None),
    ([5, 200], [133, 1000]),          # chunks behind earlier keys
    ([1, 1, 1], [257, 1, 64]),        # single tokens
    ([10, 7, 0], [4, 0, 9]),          # rows that see no key, keys without rows
    ([700], None),
    ([385, 130], [385 + 255, 130 + 1]),
]


@pytest.mark.parametrize("q_lens,k_lens", PACKS)
@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (5, 1, 64), (3, 3, 128), (8, 2, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_packed(q_lens, k_lens, Hq, Hkv, D, dtype):
    m = k_lens or q_lens
    nq, nk = sum(q_lens), sum(m)
    q = randn(nq, Hq, D, seed=nq, dtype=dtype, scale=1.5)
    k, v = randn(nk, Hkv, D, seed=nk + 1, dtype=dtype, scale=1.5), randn(nk, Hkv, D, seed=nk + 2, dtype=dtype)
    W = 37
    with ris.ris_pack_create(q_lens, k_lens) as pack:
        out, lse, w = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=W)
        ris.ris_device_status()
    ro, rl, rw = packed_plain(q, k, v, q_lens, m, W)
    if dtype == F32:
        check_f32_path(to_np(out), ro.numpy())
    else:
        check_bf16_path(to_np(out), ro.numpy(), out_bf16=True)
    empty = rl == -INF
    assert (lse.double().cpu()[empty] == -INF).all() and (out.cpu()[empty.T] == 0).all()
    assert ((lse.double().cpu() - rl)[~empty].abs() <= 2e-5 * (1 + rl[~empty].abs())).all()
    if nk:
        assert (w.double().cpu() - rw).abs().max() <= 2e-5 * max(1.0, float(rw.max()))


@pytest.mark.parametrize("dtype,D", [(F32, 128), (BF16, 128), (BF16, 64)])
def test_attention_packed_out_of_fused_rows(dtype, D):
    """q, k, v as views into a fused projection's rows; fp32 outputs of either type; two calls of one pack."""
    Hq, Hkv, lens = 12, 2, [200, 77, 301]
    x = randn(sum(lens), Hq + 2 * Hkv, D, seed=9, dtype=dtype)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    with ris.ris_pack_create(lens) as pack:
        a, = ris.ris_attention_packed(pack, q, k, v)
        b, = ris.ris_attention_packed(pack, q.contiguous(), k.contiguous(), v.contiguous())
        c, = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32)
    assert torch.equal(a, b)
    ro, _, _ = packed_plain(q, k, v, lens, lens, 1)
    (check_f32_path if dtype == F32 else check_bf16_path)(to_np(c), ro.numpy())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
def test_attention_packed_hidden_keys_take_no_part(dtype, bad):
    """An infinity or NaN in a key or value reaches only rows that see it (and no other sequence)."""
    lens, Hq, Hkv, D, at = [150, 140], 2, 1, 128, 70
    q, k, v = randn(290, Hq, D, seed=1, dtype=dtype), randn(290, Hkv, D, seed=2, dtype=dtype), randn(290, Hkv, D, seed=3, dtype=dtype)
    with ris.ris_pack_create(lens) as pack:
        good, = ris.ris_attention_packed(pack, q, k, v)
        for x in (k, v):
            y = x.clone()
            y[at, 0, 5] = bad
            y[149, 0, 6] = bad  # the last key of the first sequence: only the last row sees it
            got, = ris.ris_attention_packed(pack, q, y if x is k else k, y if x is v else v)
            ris.ris_device_status()
            rows = torch.ones(290, dtype=torch.bool, device="cuda")
            rows[at:150] = False
            tol = 0.0 if dtype == F32 or x is k else 2 ** -7
            assert torch.isfinite(got[rows]).all()
            assert ((got[rows].float() - good[rows].float()).abs() <= tol * good[rows].float().abs() + (tol > 0) * 1e-2).all()
            if x is v:
                assert not torch.isfinite(got[at:150, :, 5].float()).any()


def test_attention_packed_large_scores_and_values():
    """Scores of hundreds (one key takes the row) and values near fp16's limit and beyond."""
    lens, D = [300], 128
    q, k = randn(300, 2, D, seed=1, dtype=BF16, scale=8.0), randn(300, 1, D, seed=2, dtype=BF16, scale=8.0)
    for big in (1.0, 3e4, 1e6, 1e30, 1e-20):
        v = (randn(300, 1, D, seed=3) * big).to(BF16)
        with ris.ris_pack_create(lens) as pack:
            out, = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32)
        ro, _, _ = packed_plain(q, k, v, lens, lens, 1)
        assert rel_l2(to_np(out), ro.numpy()) <= 5e-3


def test_attention_packed_many_heads_per_group_and_long_row():
    lens = [1025, 3, 511]
    q, k, v = (randn(sum(lens), h, 128, seed=h, dtype=BF16) for h in (16, 1, 1))
    with ris.ris_pack_create(lens) as pack:
        out, w = ris.ris_attention_packed(pack, q, k, v, weight_rows=2000)  # all rows count
    ro, _, rw = packed_plain(q, k, v, lens, lens, 2000)
    check_bf16_path(to_np(out), ro.numpy(), out_bf16=True)
    assert (w.double().cpu() - rw).abs().max() <= 2e-5 * float(rw.max())
    # every row hands out one unit per head
    assert abs(float(w.double().sum()) - 16 * sum(lens)) <= 1e-3 * sum(lens)


# ---------------------------------------------------------------- the 4-bit cache
LEVELS = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise_plain(x):
    """Values that x [..., D] (fp32, on the CPU) is stored as, and the scales."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    s = (top * torch.tensor(1 / 6, dtype=F32)).to(BF16).float()
    s = torch.where(torch.isfinite(g).all(-1), s, torch.tensor(float("nan")))
    y = torch.where(s[..., None] > 0, g / s[..., None], torch.zeros(()))
    a = y.abs()
    d = (a[..., None] - LEVELS).abs()
    best = d.amin(-1, keepdim=True)
    cand = d == best                        # two at a tie: the even code
    idx = torch.where(cand, torch.arange(8), torch.tensor(99))
    lo, hi = idx.amin(-1), torch.where(cand, torch.arange(8), torch.tensor(-1)).amax(-1)
    code = torch.where(lo % 2 == 0, lo, hi).clamp(max=7)
    return (torch.copysign(LEVELS[code], y) * s[..., None]).flatten(-2), s


@pytest.mark.parametrize("D,Hkv,dtype", [(128, 2, BF16), (64, 3, F32), (128, 1, F32), (64, 4, BF16)])
def test_cache4_append_and_read(D, Hkv, dtype):
    lens, cap = [1, 0, 40, 17], 64
    n = sum(lens)
    x = randn(n, 3 * Hkv, D, seed=D, dtype=dtype, scale=3.0)
    x[0, 0, :32] = 0.0                                        # a group of zeros
    x[1, 0, :32] *= 1e-30 if dtype == F32 else 1e-20          # tiny and huge groups keep their scale
    x[2, Hkv, 32:64] *= 1e20
    x[3, 0, :8] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5], dtype=dtype)  # ties, with scale 1
    x[3, 0, 8:32] = torch.tensor(-0.75, dtype=dtype)
    k, v = x[:, :Hkv], x[:, 2 * Hkv:]
    pos = torch.arange(100, 100 + n, dtype=torch.int32, device="cuda")
    w = torch.rand(Hkv, n, generator=torch.Generator().manual_seed(1)).cuda()
    cache = ris.Cache4.empty(4, Hkv, D, cap)
    start = torch.tensor([5, 3, 0, 47], dtype=torch.int32, device="cuda")
    with ris.ris_pack_create(lens) as pack:
        ris.ris_cache4_append(cache, pack, k, v, pos, weight=w, start=start)
    ris.ris_device_status()
    assert cache.length.tolist() == [6, 3, 40, 64]
    rk, rv = ris.ris_cache4_read(cache, first=start, count=41)
    off = [0, 1, 1, 41, 58]
    for b, m in enumerate(lens):
        for got, src in ((rk, k), (rv, v)):
            ref, s = quantise_plain(src[off[b]:off[b + 1]].float().cpu())
            assert torch.equal(got[b, :, :m].cpu().transpose(0, 1), ref)
            assert (got[b, :, m:] == 0).all()
            err = (ref - src[off[b]:off[b + 1]].float().cpu()).abs().unflatten(-1, (-1, 32))
            assert (err <= s[..., None] * (1 + 6 * 2.0 ** -8)).all()
        sl = slice(int(start[b]), int(start[b]) + m)
        assert (cache.pos[b, :, sl] == pos[off[b]:off[b + 1]]).all()
        assert torch.equal(cache.weight[b, :, sl], w[:, off[b]:off[b + 1]])
    whole, _ = ris.ris_cache4_read(cache)
    assert whole.shape == (4, Hkv, cap, D) and torch.equal(whole[2, :, :40], rk[2, :, :40])


def test_cache4_append_token_by_token_and_overflow():
    """Appending after the slots in use gives the same cache as one call; what does not fit is left out and reported."""
    B, H, D, cap = 3, 2, 128, 16
    k, v = randn(B * 18, H, D, seed=1, dtype=BF16).view(B, 18, H, D), randn(B * 18, H, D, seed=2, dtype=BF16).view(B, 18, H, D)
    a, b = ris.Cache4.empty(B, H, D, cap), ris.Cache4.empty(B, H, D, cap)
    with ris.ris_pack_create([16] * B) as pack, ris.ris_pack_create([1] * B) as ones:
        pos = torch.arange(16, dtype=torch.int32, device="cuda").repeat(B)
        ris.ris_cache4_append(a, pack, k[:, :16].reshape(-1, H, D), v[:, :16].reshape(-1, H, D), pos)
        for t in range(16):
            ris.ris_cache4_append(b, ones, k[:, t].contiguous(), v[:, t].contiguous(), torch.full((B,), t, dtype=torch.int32, device="cuda"))
        for name in ("k", "v", "k_scale", "v_scale", "pos", "length"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        ris.ris_device_status()
        ris.ris_cache4_append(b, ones, k[:, 16].contiguous(), v[:, 16].contiguous(), torch.full((B,), 16, dtype=torch.int32, device="cuda"))
        with pytest.raises(ris.RisError) as e:
            ris.ris_device_status()
        assert e.value.status == ris.RIS_ERR_INVALID
        for name in ("k", "v", "k_scale", "v_scale", "pos", "length"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
        assert (b.sync == 0).all()


def test_cache4_append_not_finite():
    """A value that is not finite turns its own group into NaN and nothing else."""
    x = randn(3, 1, 64, seed=1)
    x[1, 0, 40], x[2, 0, 3] = INF, float("nan")
    cache = ris.Cache4.empty(1, 1, 64, 16)
    with ris.ris_pack_create([3]) as pack:
        ris.ris_cache4_append(cache, pack, x, x, torch.arange(3, dtype=torch.int32, device="cuda"))
    for y in ris.ris_cache4_read(cache, count=3):
        bad = torch.isnan(y[0, 0]).view(3, 2, 32)
        assert bad.all(-1).tolist() == [[False, False], [False, True], [True, False]]
        assert bad.any(-1).tolist() == bad.all(-1).tolist()


def filled(B, Hkv, D, cap, lens, seed=0, scale=1.0):
    cache = ris.Cache4.empty(B, Hkv, D, cap)
    cap = cache.capacity
    x, y = randn(B * cap, Hkv, D, seed=seed, scale=scale), randn(B * cap, Hkv, D, seed=seed + 1, scale=scale)
    with ris.ris_pack_create([cap] * B) as pack:
        ris.ris_cache4_append(cache, pack, x, y, torch.arange(B * cap, dtype=torch.int32, device="cuda"))
    cache.length.copy_(torch.tensor(lens, dtype=torch.int32))
    return cache


def attend_plain(cache, q, lens):
    k, v = (x.double().cpu() for x in (ris.ris_cache4_read(cache)))
    B, Hq, D = q.shape
    G = Hq // cache.kv_heads
    out, lse, w = torch.zeros(B, Hq, D, dtype=torch.float64), torch.full((B, Hq), -INF, dtype=torch.float64), torch.zeros(cache.weight.shape, dtype=torch.float64)
    for b, n in enumerate(lens):
        for h in range(Hq if n else 0):
            s = k[b, h // G, :n] @ q[b, h].double().cpu() / math.sqrt(D)
            lse[b, h] = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[b, h])
            out[b, h] = p @ v[b, h // G, :n]
            w[b, h // G, :n] += p
    return out, lse, w


@pytest.mark.parametrize("Hq,Hkv,D", [(12, 2, 128), (32, 4, 64), (8, 8, 128), (16, 1, 128), (20, 1, 64), (3, 1, 64)])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("cap,lens", [(16, [1, 16, 0]), (1040, [1039, 64, 65]), (300, [17, 304, 256]), (5008, [5003])])
def test_cache4_attend(Hq, Hkv, D, dtype, out, cap, lens):
    B = len(lens)
    cache = filled(B, Hkv, D, cap, lens, seed=cap)
    q = randn(B, Hq, D, seed=7, dtype=dtype, scale=2.0)
    w0 = torch.rand(cache.weight.shape, generator=torch.Generator().manual_seed(2)).cuda()
    w1 = torch.full_like(w0, -1.0)
    got, lse = ris.ris_cache4_attend(cache, q, out_dtype=out, return_lse=True, weight_in=w0, weight_out=w1)
    ris.ris_device_status()
    ro, rl, rw = attend_plain(cache, q, lens)
    if out == F32:
        assert rel_l2(to_np(got), ro.numpy()) <= 1e-5
    else:
        assert ((got.double().cpu() - ro).abs() <= 2.0 ** -9 * ro.abs() + 2.0 ** -9 * ro.abs().amax(-1, keepdim=True)).all()
    for b, n in enumerate(lens):
        if n == 0:
            assert (got[b] == 0).all() and (lse[b] == -INF).all()
            continue
        assert ((lse[b].double().cpu() - rl[b]).abs() <= 2e-5 * (1 + rl[b].abs())).all()
        ref = rw[b, :, :n] + w0[b, :, :n].double().cpu()
        assert (w1[b, :, :n].double().cpu() - ref).abs().max() <= 2e-5
    there = torch.arange(cache.capacity) < torch.tensor(lens)[:, None]
    assert (w1.cpu()[~there[:, None].expand(w1.shape)] == -1.0).all()  # slots that are not in use are left alone
    # without weights, with a bound on the lengths, in place: the same numbers
    again = ris.ris_cache4_attend(cache, q, out_dtype=out, longest=max(lens) or 1)
    assert rel_l2(to_np(again), to_np(got)) <= (1e-6 if out == F32 else 4e-3)
    w2 = w0.clone()
    ris.ris_cache4_attend(cache, q, out_dtype=out, weight_in=w2, weight_out=w2)
    assert torch.equal(w2.cpu()[there[:, None].expand(w1.shape)], w1.cpu()[there[:, None].expand(w1.shape)])


def test_cache4_attend_slots_not_in_use_may_hold_anything():
    lens = [5, 100]
    cache = filled(2, 2, 128, 128, lens)
    q = randn(2, 12, 128, seed=1, dtype=BF16)
    a = ris.ris_cache4_attend(cache, q, out_dtype=F32)
    for b, n in enumerate(lens):
        for s in (cache.k_scale, cache.v_scale):
            s[b, :, n:] = float("nan")
        cache.k[b, :, n:] = 255
    b = ris.ris_cache4_attend(cache, q, out_dtype=F32)
    assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e5, 1e30])
def test_cache4_attend_ranges_of_values_and_scores(scale):
    """Tiny and huge values; scores of hundreds; value scales that grow along the sequence."""
    n = 700
    cache = ris.Cache4.empty(1, 1, 128, 704)
    x, y = randn(n, 1, 128, seed=1, scale=6.0), randn(n, 1, 128, seed=2)
    y *= torch.logspace(-3, 0, n, device="cuda")[:, None, None] * scale
    with ris.ris_pack_create([n]) as pack:
        ris.ris_cache4_append(cache, pack, x, y, torch.arange(n, dtype=torch.int32, device="cuda"))
    q = randn(1, 4, 128, seed=3, scale=20.0)
    q[0, 3] = 0.0
    ro, rl, _ = attend_plain(cache, q, [n])
    got, lse = ris.ris_cache4_attend(cache, q, return_lse=True)
    assert rel_l2(to_np(got), ro.numpy()) <= 2e-5
    assert ((lse.double().cpu() - rl).abs() <= 2e-5 * (1 + rl.abs())).all()


def test_cache4_offsets_past_32_bits():
    """A cache whose code arrays are longer than 2^32 bytes: the last head's last slots."""
    B, H, D, cap = 1, 9, 128, 1 << 23
    cache = ris.Cache4.empty(B, H, D, cap)
    assert cache.k.numel() > 2 ** 32
    start = torch.tensor([cap - 500], dtype=torch.int32, device="cuda")
    x, y = randn(500, H, D, seed=1, dtype=BF16), randn(500, H, D, seed=2, dtype=BF16)
    cache.k_scale.zero_()
    with ris.ris_pack_create([500]) as pack:
        ris.ris_cache4_append(cache, pack, x, y, torch.arange(500, dtype=torch.int32, device="cuda"), start=start)
    rk, rv = ris.ris_cache4_read(cache, first=start, count=500)
    assert torch.equal(rk[0].cpu().transpose(0, 1), quantise_plain(x.float().cpu())[0])
    q = randn(1, 2 * H, D, seed=3, scale=4.0)
    out, lse = ris.ris_cache4_attend(cache, q, return_lse=True)
    for h in range(2 * H):  # the slots before hold zeros: score 0, value 0
        s = rk[0, h // 2].double() @ q[0, h].double() / math.sqrt(D)
        m = s.max().clamp(min=0)
        l = torch.exp(s - m).sum() + (cap - 500) * torch.exp(-m)
        o = torch.exp(s - m) @ rv[0, h // 2].double() / l
        assert rel_l2(to_np(out[0, h]), o.cpu().numpy()) <= 2e-5
        assert abs(float(lse[0, h]) - float(m + l.log())) <= 1e-3


# ---------------------------------------------------------------- eviction
def evict_plain(pos, weight, n, budget, recent):
    """Source slot of each place, by the definition, for one head: lists of Python numbers."""
    if n <= budget:
        return [j if j < n else -1 for j in range(budget)]
    newest = max(pos[:n])
    key = lambda j: (pos[j] <= newest - recent, math.isnan(weight[j]), 0.0 if math.isnan(weight[j]) else -weight[j], j)
    keep = set(sorted(range(n), key=key)[:budget])
    above = iter([j for j in range(budget, n) if j in keep])
    return [j if j in keep else next(above) for j in range(budget)]


@pytest.mark.parametrize("lens,budget,recent,D,kind", [
    ([40, 33, 32, 0, 5], 32, 4, 64, "random"),
    ([1000, 999, 400], 100, 99, 128, "random"),
    ([3000, 2049, 17], 2048, 0, 64, "ties"),
    ([500, 500], 1, 0, 128, "random"),
    ([700], 600, 100, 64, "nan"),
    ([900, 4000], 333, 200, 128, "positions"),
    ([10000, 9999, 8193], 4096, 512, 64, "random"),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_cache4_evict(lens, budget, recent, D, kind, in_place):
    B, H = len(lens), 2
    cap = max(max(lens), budget)
    src = filled(B, H, D, cap, lens, seed=cap)
    g = torch.Generator().manual_seed(budget)
    w = torch.rand(src.weight.shape, generator=g)
    pos = torch.arange(src.capacity, dtype=torch.int32).expand(src.pos.shape).clone()
    if kind == "ties":
        w = (w * 3).floor() - 1.0
        w[w == 0] = -0.0
    elif kind == "nan":
        w[:, :, ::7] = float("nan")
        w[:, :, 3::11] = -INF
        w[:, :, 5::13] = INF
    elif kind == "positions":  # any order, many alike
        pos = torch.randint(-100, 100, pos.shape, generator=g, dtype=torch.int32)
    src.weight.copy_(w)
    src.pos.copy_(pos)
    before = {n: getattr(src, n).clone() for n in ("k", "v", "k_scale", "v_scale", "pos", "weight")}
    dst = src if in_place else ris.Cache4.empty(B, H, D, budget + 5)
    kept = ris.ris_cache4_evict(src, dst, budget, recent).cpu()
    ris.ris_device_status()
    assert dst.length.tolist() == [min(n, budget) for n in lens]
    for b in range(B):
        for h in range(H):
            ref = evict_plain(pos[b, h].tolist(), w[b, h].tolist(), lens[b], budget, recent)
            assert kept[b, h].tolist() == ref
            at = torch.tensor([j for j in ref if j >= 0], dtype=torch.long, device="cuda")
            for name, x in before.items():
                assert torch.equal(getattr(dst, name)[b, h, :len(at)].view(torch.uint8), x[b, h][at].view(torch.uint8)), name
    if not in_place:
        for name, x in before.items():
            assert torch.equal(getattr(src, name).view(torch.uint8), x.view(torch.uint8)), name


def test_serving_round_trip():
    """Rotate, attend, append with the prompt's weights, cut back, generate: every call on a stream of its own,
    the decode steps as one replayed graph."""
    lens, Hq, Hkv, D, budget = [300, 120, 211], 12, 2, 128, 128
    n, rope = sum(lens), ris.rope_cfg(ris.ROPE_PLAIN, 1e6, 32768)
    side = torch.cuda.Stream()
    x = randn(n, Hq + 2 * Hkv, D, seed=1, dtype=BF16)
    step = randn(len(lens), Hq + 2 * Hkv, D, seed=2, dtype=BF16)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pack, ones = ris.ris_pack_create(lens), ris.ris_pack_create([1] * len(lens))
        pos = torch.cat([torch.arange(m, dtype=torch.int32) for m in lens]).cuda()
        q, k = ris.ris_rope_axes(x[:, :Hq], x[:, Hq:Hq + Hkv], pos[None], [D // 2], 300, rope)
        out, w = ris.ris_attention_packed(pack, q, k, x[:, Hq + Hkv:], weight_rows=32)
        cache = ris.Cache4.empty(len(lens), Hkv, D, 320)
        ris.ris_cache4_append(cache, pack, k, x[:, Hq + Hkv:], pos, weight=w)
        ris.ris_cache4_evict(cache, cache, budget, 16)
        now = torch.tensor(lens, dtype=torch.int32, device="cuda")
        got = torch.empty(len(lens), Hq, D, dtype=BF16, device="cuda")

        def token():
            q1, k1 = ris.ris_rope_axes(step[:, :Hq], step[:, Hq:Hq + Hkv], now[None], [D // 2], 400, rope)
            ris.ris_cache4_append(cache, ones, k1, step[:, Hq + Hkv:], now)
            ris.ris_cache4_attend(cache, q1, out=got, weight_in=cache.weight, weight_out=cache.weight, longest=192)
            now.add_(1)
            return q1

        token()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            q1 = token()
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    ris.ris_device_status()
    want = [min(m, budget) + 4 for m in lens]
    assert cache.length.tolist() == want and now.tolist() == [m + 4 for m in lens]
    ro, _, _ = attend_plain(cache, q1, want)
    assert ((got.double().cpu() - ro).abs() <= 2.0 ** -8 * ro.abs().amax(-1, keepdim=True)).all()
    for b, m in enumerate(lens):
        for h in range(Hkv):
            have = sorted(cache.pos[b, h, :want[b]].tolist())
            assert have[-20:] == list(range(m + 4 - 20, m + 4)) and len(set(have)) == len(have)


# ---------------------------------------------------------------- prompts behind many keys
LONG_KEYS = ([200, 130, 3, 0, 40], [5000, 6000, 1, 7, 20])  # short rows behind long prompts: the rows' tiles see some 30 key tiles each


@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (8, 2, 128), (2, 2, 128), (5, 1, 64), (4, 2, 64)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_attention_packed_behind_long_prompts(Hq, Hkv, D, out_dtype):
    n, m = LONG_KEYS
    q = randn(sum(n), Hq, D, seed=1, dtype=BF16, scale=2.0)
    kv = randn(sum(m), 2 * Hkv, D, seed=2, dtype=BF16)
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    with ris.ris_pack_create(n, m) as pack:
        out, lse, w = ris.ris_attention_packed(pack, q, k, v, out_dtype=out_dtype, return_lse=True, weight_rows=150)
        ris.ris_device_status()
    ro, rl, rw = packed_plain(q, k, v, n, m, 150)
    check_bf16_path(to_np(out), ro.numpy(), out_bf16=out_dtype == BF16)
    empty = rl == -INF
    assert empty.any() and (lse.double().cpu()[empty] == -INF).all() and (out.cpu()[empty.T] == 0).all()
    assert ((lse.double().cpu() - rl)[~empty].abs() <= 2e-5 * (1 + rl[~empty].abs())).all()
    assert (w.double().cpu() - rw).abs().max() <= 2e-5 * max(1.0, float(rw.max()))


@pytest.mark.parametrize("Hq,Hkv", [(3, 1), (4, 1)])
@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
def test_attention_packed_hidden_keys_behind_long_prompts(Hq, Hkv, bad):
    """An infinity or NaN among the last keys of the first sequence reaches only its rows that see it."""
    n, m = LONG_KEYS
    q = randn(sum(n), Hq, 128, seed=1, dtype=BF16)
    k, v = randn(sum(m), Hkv, 128, seed=2, dtype=BF16), randn(sum(m), Hkv, 128, seed=3, dtype=BF16)
    with ris.ris_pack_create(n, m) as pack:
        good, = ris.ris_attention_packed(pack, q, k, v)
        for x in (k, v):
            y = x.clone()
            y[4900, 0, 5] = bad  # seen by rows 100 .. 199
            y[4999, 0, 6] = bad
            got, = ris.ris_attention_packed(pack, q, y if x is k else k, y if x is v else v)
            ris.ris_device_status()
            rows = torch.ones(sum(n), dtype=torch.bool, device="cuda")
            rows[100:200] = False
            tol = 0.0 if x is k else 2 ** -7
            assert torch.isfinite(got[rows]).all()
            assert ((got[rows].float() - good[rows].float()).abs() <= tol * good[rows].float().abs() + (tol > 0) * 1e-2).all()
            if x is v:
                assert not torch.isfinite(got[100:200, :, 5].float()).any()


# ---------------------------------------------------------------- allocations that fail, streams, the example
@pytest.fixture
def allocations():
    yield ris.ris_debug_fail_allocation
    ris.ris_debug_fail_allocation(-1)


def test_serving_allocation_failures(allocations):
    """Every allocation of every call, failed in turn: the call reports it, nothing is kept, the next call is right."""
    lens, Hq, Hkv, D = [70, 200], 4, 2, 128
    q, k, v = (randn(270, h, D, seed=h, dtype=BF16) for h in (Hq, Hkv, Hkv))
    cache = filled(2, Hkv, D, 256, [256, 199])
    dst = ris.Cache4.empty(2, Hkv, D, 64)
    pack = ris.ris_pack_create(lens)
    qt = q[:2].contiguous()
    calls = [lambda: ris.ris_pack_create(lens),
             lambda: ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=8),
             lambda: ris.ris_cache4_attend(cache, qt, weight_out=dst_weight),
             lambda: ris.ris_cache4_evict(cache, dst, 64, 8)]
    dst_weight = torch.zeros_like(cache.weight)
    for call in calls:
        first = call()
        torch.cuda.synchronize()
        in_use = ris.ris_memory_stats()[0]
        failed = 0
        for n in range(8):
            ris.ris_debug_fail_allocation(n)
            try:
                call()
            except ris.RisError as e:
                assert e.status == ris.RIS_ERR_OOM
                failed += 1
                torch.cuda.synchronize()
                assert ris.ris_memory_stats()[0] == in_use
            else:
                break
            finally:
                ris.ris_debug_fail_allocation(-1)
        assert failed >= 1 and n < 7
        again = call()
        ris.ris_device_status()
        if isinstance(first, tuple):
            assert all(torch.equal(a, b) for a, b in zip(first, again))
        elif torch.is_tensor(first):
            assert torch.equal(first, again)


def test_example_serves_prompts():
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_prompts.py")
    spec = importlib.util.spec_from_file_location("serve_prompts", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    lens, tokens, budget, slack = [300, 33, 150], 21, 128, 8
    server, states = example.main(["--prompts", *map(str, lens), "--image", "4", "6", "--layers", "2", "--tokens", str(tokens),
                                   "--budget", str(budget), "--recent", "32", "--slack", str(slack)])
    assert states.shape == (tokens, 3, 12 * 128) and torch.isfinite(states.float()).all()
    # cuts before steps 8 and 16; the second sequence grows from 33 to 54 without reaching the budget
    assert server.layers[0].cache.length.tolist() == [128 + 5, 33 + 21, 128 + 5]
    assert server.token.tolist() == [n + tokens for n in lens]
    assert server.time.tolist() == [300 - 24 + 6 + tokens, 33 + tokens, 150 + tokens]
    for layer in server.layers:
        for b, n in enumerate(lens):
            have = layer.cache.pos[b, 0, :int(layer.cache.length[b])].tolist()
            assert len(set(have)) == len(have) and set(range(n + tokens - 32, n + tokens)) <= set(have)


def test_serving_calls_after_other_work_in_a_graph():
    """Each call right behind a memset, a copy, another stream's kernel and another library's, eagerly and as a replayed graph."""
    B, Hq, Hkv, D, cap = 3, 4, 2, 64, 64
    x = randn(B, Hq + 2 * Hkv, D, seed=1, dtype=BF16)
    src = x.clone()
    lens = torch.tensor([40, 7, 33], dtype=torch.int32, device="cuda")
    base = filled(B, Hkv, D, cap, lens.tolist())
    cache, small = filled(B, Hkv, D, cap, lens.tolist()), ris.Cache4.empty(B, Hkv, D, 32)
    rope = ris.rope_cfg(ris.ROPE_PLAIN, 1e4, 2048)
    ones, pos = ris.ris_pack_create([1] * B), torch.zeros(1, B, dtype=torch.int32, device="cuda")
    side, main = torch.cuda.Stream(), torch.cuda.Stream()
    big = randn(1024, 1024, seed=2)

    def steps():
        cache.length.zero_()                                   # memset
        cache.weight.zero_()
        cache.length.copy_(base.length)                        # copies
        x.copy_(src)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):                          # another stream's product, waited for
            y = big @ big
            pos.fill_(50)
        torch.cuda.current_stream().wait_stream(side)
        q, k = ris.ris_rope_axes(x[:, :Hq], x[:, Hq:Hq + Hkv], pos, [D // 2], 64, rope)
        ris.ris_cache4_append(cache, ones, k, x[:, Hq + Hkv:], pos[0])
        o = ris.ris_cache4_attend(cache, q, out_dtype=F32, weight_in=cache.weight, weight_out=cache.weight)
        z = o * 2.0                                            # another library's kernel
        pos.zero_()
        kept = ris.ris_cache4_evict(cache, small, 32, 4)
        small.weight.mul_(1.0)
        rk, rv = ris.ris_cache4_read(small)
        w, = ris.ris_attention_packed(ones, q, k, x[:, Hq + Hkv:])
        return [q, k, o, z, kept, rk, rv, w, cache.length.clone(), cache.weight.clone(), y]

    want = [t.clone() for t in steps()]
    torch.cuda.synchronize()
    ref, _, _ = attend_plain(cache, want[0], (lens + 1).tolist())
    assert rel_l2(to_np(want[2]), ref.numpy()) <= 1e-5 and torch.equal(want[3], want[2] * 2.0)
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            got = steps()
        for _ in range(3):
            for t in got:
                t.zero_()
            graph.replay()
    torch.cuda.synchronize()
    ris.ris_device_status()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 2, 64), (3, 1, 128)])
@pytest.mark.parametrize("step", [0.05, 0.4, 3.0, -0.4])
@pytest.mark.parametrize("late", [0, 64, 127])
def test_attention_packed_scores_that_grow_along_the_keys(Hq, Hkv, D, step, late):
    """Scores that rise (or fall) by `step` a key, so that a row's maximum moves by less than 2^8, by up to 2^15 and by far more in a
    tile, in its first half or its second; and one key of each tile far above the rest."""
    lens = [300, 513, 70]
    n = sum(lens)
    q, k, v = randn(n, Hq, D, seed=1, dtype=BF16), randn(n, Hkv, D, seed=2, dtype=BF16, scale=0.1), randn(n, Hkv, D, seed=3, dtype=BF16)
    q[..., 0], q[..., 1] = math.sqrt(D), math.sqrt(D)
    at = torch.cat([torch.arange(m) for m in lens]).cuda()
    k[..., 0] = (at * step).to(BF16)[:, None]
    k[..., 1] = ((at % 128 == late) * (at // 128 + 1) * 12.0).to(BF16)[:, None]
    with ris.ris_pack_create(lens) as pack:
        out, lse, w = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32, return_lse=True, weight_rows=40)
        ris.ris_device_status()
    ro, rl, rw = packed_plain(q, k, v, lens, lens, 40)
    check_bf16_path(to_np(out), ro.numpy())
    assert ((lse.double().cpu() - rl).abs() <= 2e-5 * (1 + rl.abs())).all()
    # a score of magnitude S is a sum of fp32 additions that cut off, 2^-23 S each, eight of them: 1e-6 S
    assert (w.double().cpu() - rw).abs().max() <= (2e-5 + 1e-6 * float(rl.abs().max())) * max(1.0, float(rw.max()))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_serving_token_strides_past_32_bits(dtype):
    """Tokens 2^20 elements apart: the last ones lie past 2^32 elements. The same bits as from contiguous copies."""
    n, Hq, Hkv, D = 4200, 3, 1, 64
    x = torch.empty(n, 1 << 20, dtype=dtype, device="cuda")
    heads = x[:, :(Hq + 2 * Hkv) * D].unflatten(1, (-1, D))
    heads.copy_(randn(n, Hq + 2 * Hkv, D, seed=1, dtype=dtype))
    q, k, v = heads[:, :Hq], heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:]
    lens = [4000, 0, 200]
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope = ris.rope_cfg(ris.ROPE_PLAIN, 1e4, 2048)
    got = []
    for a, b, c in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        cache = ris.Cache4.empty(3, Hkv, D, 4000)
        with ris.ris_pack_create(lens) as pack:
            ris.ris_cache4_append(cache, pack, b, c, pos)
            got.append([*ris.ris_rope_axes(a, b, pos[None], [D // 2], n, rope),
                        *ris.ris_attention_packed(pack, a, b, c, return_lse=True, weight_rows=16), cache.k, cache.v, cache.k_scale, cache.pos])
    ris.ris_device_status()
    for s, t in zip(*got):
        assert torch.equal(s, t)
    assert torch.isfinite(got[0][2].float()).all()


def test_attention_packed_outputs_past_31_bits():
    """11,000 prompts of 128 tokens: 2.2 billion output elements. The last prompts by themselves give the same bits."""
    S, m, Hq, Hkv, D, last = 11000, 128, 12, 2, 128, 3
    n = S * m
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(n, h, D, generator=g, device="cuda", dtype=BF16) for h in (Hq, Hkv, Hkv))
    assert q.numel() > 2 ** 31
    with ris.ris_pack_create([m] * S) as pack, ris.ris_pack_create([m] * last) as few:
        out, lse, w = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=8)
        t = n - last * m
        # (values are scaled by the call's largest magnitude, a power of two: the same bits where both scales are in fp16's normal range)
        o2, l2, w2 = ris.ris_attention_packed(few, q[t:], k[t:], v[t:], return_lse=True, weight_rows=8)
        ris.ris_device_status()
    assert rel_l2(to_np(out[t:]), to_np(o2)) <= 1e-4
    assert torch.equal(lse[:, t:], l2) and torch.equal(w[:, t:], w2)
    rows = torch.tensor([0, 127, 128, n // 2, n - 1], device="cuda")
    for i in rows.tolist():
        b = i // m * m
        s = torch.einsum("hd,jd->hj", q[i, :6].double(), k[b:i + 1, 0].double()) / math.sqrt(D)
        ref = torch.softmax(s, -1) @ v[b:i + 1, 0].double()
        check_bf16_path(to_np(out[i, :6]), ref.cpu().numpy(), out_bf16=True)
