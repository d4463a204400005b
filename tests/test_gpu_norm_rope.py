"""Queries and keys normed per head and turned in one pass, and the gradient, against plain implementations in 64 bits.

Tolerances, from the arithmetic. A turned pair is off by 2e-6 of its norm (angle, sine and cosine good to about 2^-22),
a normed channel by less than that of itself (the sum of squares: 128 terms of relative error 2^-23, halved by the root;
the root 2^-22; two products): 4e-6 of the pair's norm in all; bf16 results add half a step, 2^-8 of the result. Backwards
dx = r (u - h mean(u h)): u is off by 3e-6 of the head's largest, the mean by 6e-6 of the mean of |u h|, r and h by 1e-6:
1e-5 r (max |u| + |h| mean |u h|). A weight's gradient: each of its terms by 1e-5 of (pair's norm of g) |h|, the sums by less than
another 1e-5 of the sum of these (100 sequential additions at most in these sizes: 100 x 2^-24 = 6e-6)."""
import pytest
import torch

from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def randn(*shape, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def plain(x, w, pos, f, ms, rot, pairs, eps):
    """[n, H, D] in 64 bits on the CPU."""
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    if rot == 0:
        return x
    ang = pos.double().cpu()[:, None] * torch.tensor(f, dtype=torch.float64)
    c, s = (ms * ang.cos())[:, None], (ms * ang.sin())[:, None]
    z = x[..., :rot]
    a, b = (z[..., 0::2], z[..., 1::2]) if pairs else z.chunk(2, -1)
    u, v = a * c - b * s, b * c + a * s
    z = torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1)
    return torch.cat([z, x[..., rot:]], -1)


def pair_norm(x, rot, pairs):
    """|x| with the norm of its pair in the place of a turned channel."""
    y = x.abs().clone()
    z = x[..., :rot]
    if rot:
        n = torch.hypot(z[..., 0::2], z[..., 1::2]).repeat_interleave(2, -1) if pairs else torch.hypot(*z.chunk(2, -1)).repeat(1, 1, 2)
        y[..., :rot] = n
    return y


CASES = [
    # n, Hq, Hkv, D, rot, pairs, dtype, kind, weights of (q, k)
    (1, 12, 2, 128, 0, False, BF16, 1, (True, True)),
    (37, 4, 4, 64, 32, False, F32, 2, (True, True)),
    (333, 7, 1, 128, 96, True, BF16, 3, (True, False)),
    (65, 16, 1, 64, 16, True, F32, 1, (False, True)),
    (130, 3, 3, 128, 48, False, BF16, 1, (False, False)),
    (1000, 12, 2, 128, 128, True, F32, 3, (True, True)),
    (19, 5, 0, 64, 64, False, BF16, 1, (True, False)),
    (70, 2, 1, 128, 0, False, BF16, 0, (True, True)),   # the norm alone
    (70, 2, 1, 64, 0, False, F32, 0, (False, True)),
    (10007, 1, 1, 128, 128, False, F32, 1, (True, True)),  # a CTA takes several groups of tokens
    (9001, 1, 2, 64, 32, True, BF16, 1, (True, True)),
]


def setup(n, Hq, Hkv, D, rot, pairs, dtype, kind, weights):
    g = torch.Generator().manual_seed(n)
    pos = torch.randint(-50, 200000, (n,), generator=g, dtype=torch.int32).cuda()
    fused = randn(n, Hq + 2 * Hkv, D, seed=n, dtype=dtype, scale=3.0)
    q, k = fused[:, :Hq], fused[:, Hq:Hq + Hkv] if Hkv else None
    w = [1 + 0.3 * randn(D, seed=n + i) for i in range(2)]
    w = [x.to(dtype) if have else None for x, have in zip(w, weights)]
    rope = ris.rope_cfg(kind, 1e6, 32768) if kind else None
    real = (rot or D) if kind else 0
    f, ms = ris.ris_rope_freqs(rope, 200000, real) if kind else (None, 1.0)
    return q, k, pos, w, rope, real, f, ms


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    n, Hq, Hkv, D, rot, pairs, dtype, kind, _ = case
    q, k, pos, w, rope, real, f, ms = setup(*case)
    eps = 1e-5
    kw = dict(eps=eps, rot_dim=rot, pairs=pairs)
    qo, ko = ris.ris_norm_rope(q, k, pos if kind else None, 200000, rope, w[0], w[1], **kw)
    for x, y, wt in ((q, qo, w[0]), (k, ko, w[1])):
        if x is None:
            assert y is None
            continue
        wd = None if wt is None else wt.double().cpu()
        z = plain(x.double().cpu(), wd, pos, f, ms, 0, pairs, eps)
        ref = plain(x.double().cpu(), wd, pos, f, ms, real, pairs, eps)
        tol = 4e-6 * ms * pair_norm(z, real, pairs) + 1e-30
        if dtype == BF16:
            tol = tol + 2.0 ** -8 * (ref.abs() + tol)
        assert ((y.double().cpu() - ref).abs() <= tol).all()
    # in place in rows of a wider tensor: the others stay
    wide = randn(n, Hq + 2 * Hkv, D, seed=n, dtype=dtype, scale=3.0)
    before = wide.clone()
    vq, vk = wide[:, :Hq], wide[:, Hq:Hq + Hkv] if Hkv else None
    a, b = ris.ris_norm_rope(vq, vk, pos if kind else None, 200000, rope, w[0], w[1], q_out=vq, k_out=vk, **kw)
    assert a.data_ptr() == wide.data_ptr() and torch.equal(vq, qo) and (vk is None or torch.equal(vk, ko))
    assert torch.equal(wide[:, Hq + Hkv:], before[:, Hq + Hkv:])
    ris.ris_device_status()


@pytest.mark.parametrize("case", CASES)
def test_backward(case):
    n, Hq, Hkv, D, rot, pairs, dtype, kind, _ = case
    q, k, pos, w, rope, real, f, ms = setup(*case)
    eps = 1e-5
    dq, dk = randn(n, Hq, D, seed=n + 7, dtype=dtype), randn(n, Hkv, D, seed=n + 8, dtype=dtype) if Hkv else None
    got = ris.ris_norm_rope_backward(dq, dk, q if w[0] is not None else None, k if w[1] is not None else None,
                                     pos if kind else None, 200000, rope, w[0], w[1], eps=eps, rot_dim=rot, pairs=pairs)
    for x, d, gx, wt, gw in ((q, dq, got[0], w[0], got[2]), (k, dk, got[1], w[1], got[3])):
        if x is None:
            assert gx is None and gw is None
            continue
        xd = x.double().cpu().requires_grad_()
        wd = None if wt is None else wt.double().cpu().requires_grad_()
        plain(xd, wd, pos, f, ms, real, pairs, eps).backward(d.double().cpu())
        back = d.double().cpu()
        if real:  # turned back: the transposed map
            t = back.clone().requires_grad_()
            g, = torch.autograd.grad(plain(t, None, pos, f, ms, real, pairs, eps), t, back)
        else:
            g = back
        r = 1.0 / torch.sqrt((xd.detach() ** 2).mean(-1, keepdim=True) + eps) if wt is not None else torch.ones(1, dtype=torch.float64)
        h = xd.detach() * r
        u = pair_norm(g, real, pairs) * (1 if wt is None else wt.double().cpu().abs())
        tol = 1e-5 * r * (u.amax(-1, keepdim=True) + (0 if wt is None else h.abs() * (u * h.abs()).mean(-1, keepdim=True)))
        if dtype == BF16:
            tol = tol + 2.0 ** -8 * (xd.grad.abs() + tol)
        assert ((gx.double().cpu() - xd.grad).abs() <= tol).all()
        if wt is None:
            assert gw is None
        else:
            assert gw.dtype == F32
            assert ((gw.double().cpu() - wd.grad).abs() <= 2e-5 * (pair_norm(g, real, pairs) * h.abs()).sum((0, 1)) + 1e-30).all()
    # in place over dq, and into rows of a wider tensor; the same bits each time
    wide = torch.zeros(n, Hq + 2 * Hkv, D, dtype=dtype, device="cuda")
    d2 = dq.clone()
    again = ris.ris_norm_rope_backward(d2, dk, q, k, pos if kind else None, 200000, rope, w[0], w[1], eps=eps, rot_dim=rot, pairs=pairs,
                                       gq=d2, gk=wide[:, Hq:Hq + Hkv] if Hkv else None)
    assert torch.equal(d2, got[0]) and (Hkv == 0 or torch.equal(wide[:, Hq:Hq + Hkv], got[1]))
    assert (wide[:, Hq + Hkv:] == 0).all()
    for a, b in zip(again[2:], got[2:]):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_backward_against_differences():
    """<dy, (f(x + h e) - f(x - h e)) / 2h> for both inputs and both weights. f is smooth: the error of a central difference is
    h^2 / 6 of the third derivative, and the calls' own rounding, 4e-6 of the outputs, is divided by 2h = 0.04: within 1e-3 of the
    products of norms."""
    n, Hq, Hkv, D = 40, 3, 2, 64
    pos = torch.randint(0, 9000, (n,), dtype=torch.int32, generator=torch.Generator().manual_seed(1)).cuda()
    rope = ris.rope_cfg(ris.ROPE_YARN, 1e4, 2048)
    x = [randn(n, Hq, D, seed=2), randn(n, Hkv, D, seed=3), 1 + 0.3 * randn(D, seed=4), 1 + 0.3 * randn(D, seed=5)]
    dy = [randn(n, Hq, D, seed=6), randn(n, Hkv, D, seed=7)]
    kw = dict(eps=1e-6, rot_dim=32, pairs=True)
    grads = ris.ris_norm_rope_backward(dy[0], dy[1], x[0], x[1], pos, 9000, rope, x[2], x[3], **kw)
    h = 0.02
    for i in range(4):
        e = randn(*x[i].shape, seed=10 + i)
        up, dn = ([t + sign * h * e if j == i else t for j, t in enumerate(x)] for sign in (1, -1))
        fu, fd = (ris.ris_norm_rope(t[0], t[1], pos, 9000, rope, t[2], t[3], **kw) for t in (up, dn))
        num = sum((d.double() * (a.double() - b.double())).sum() for d, a, b in zip(dy, fu, fd)) / (2 * h)
        size = float(sum(d.norm() ** 2 for d in dy) ** 0.5 * e.norm())
        assert abs(float(num - (grads[i].double() * e.double()).sum())) <= 1e-3 * size


def test_no_tokens_and_zero_rows():
    rope, w = ris.rope_cfg(1, 1e4, 2048), torch.ones(64, device="cuda")
    q = torch.empty(0, 2, 64, device="cuda")
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    qo, ko = ris.ris_norm_rope(q, None, pos, 10, rope, w)
    assert qo.shape == (0, 2, 64) and ko is None
    gq, gk, gw, gkw = ris.ris_norm_rope_backward(q, None, q, None, pos, 10, rope, w)
    assert gq.shape == (0, 2, 64) and (gw == 0).all() and gkw is None
    z = torch.zeros(3, 2, 64, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    assert (ris.ris_norm_rope(z, None, pos, 10, rope, w)[0] == 0).all()
    # a value that is not finite stays in its head
    x = randn(3, 2, 64, seed=1)
    good = ris.ris_norm_rope(x, None, pos, 10, rope, w)[0]
    x[1, 1, 5] = float("nan")
    y = ris.ris_norm_rope(x, None, pos, 10, rope, w)[0]
    assert torch.isnan(y[1, 1]).all()
    y[1, 1] = good[1, 1]
    assert torch.equal(y, good)


def test_on_another_stream():
    n = 500
    q, k = randn(n, 4, 128, seed=1, dtype=BF16), randn(n, 2, 128, seed=2, dtype=BF16)
    w = torch.ones(128, dtype=BF16, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    rope = ris.rope_cfg(1, 1e6, 32768)
    want = ris.ris_norm_rope(q, k, pos, n, rope, w, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = [torch.empty_like(q), torch.empty_like(k)]
    torch.cuda.synchronize()
    ris.ris_norm_rope(q, k, pos, n, rope, w, w, q_out=out[0], k_out=out[1], stream=side)
    side.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_binding_refuses():
    """Weights and forward inputs that do not fit, before anything is launched."""
    q, d, w = randn(5, 4, 64), randn(5, 4, 64), randn(64)
    before = ris.ris_launch_count()
    for bad in (randn(128), w[None], w.to(BF16), randn(128)[::2], w.cpu()):
        with pytest.raises(ValueError):
            ris.ris_norm_rope(q, None, None, 1, None, bad)
        with pytest.raises(ValueError):
            ris.ris_norm_rope_backward(d, None, q, None, None, 1, None, bad)
    for bad in (None, randn(5, 4, 128)[..., :64], randn(6, 4, 64), randn(5, 2, 64), q.to(BF16), q[0]):
        with pytest.raises(ValueError):
            ris.ris_norm_rope_backward(d, None, bad, None, None, 1, None, w)
    with pytest.raises(ValueError):
        ris.ris_norm_rope_backward(d, None, q, q, None, 1, None, w, w)  # k has a weight and no gradient
    assert ris.ris_launch_count() == before
