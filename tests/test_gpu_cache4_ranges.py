"""One token's attention over a 4-bit cache whose values are not finite in places, or differ by many powers of two between
groups of 32 channels, between slots and from the usual: every head and group by itself against 64 bits.

What may be off, per channel, with A = sum_j p_j |v_j| over the slots and S = max_j p_j scale_j of the group:
  fp32 outputs  1e-5 A: scores of magnitude up to 20 good to 2^-22 of themselves, exponentials to 2^-22, weights as two
                fp16 parts (2^-22), the tensor pipe's sums (2e-6);
  bf16 outputs  the output's half ulp (2^-8 |o|) and 2^-10 A for weights of 11 bits;
  both          1e-5 S: what is added in fp16 is off by 2^-25 at most where its largest is 2^4 or more, 2^-29 S a slot, times
                values of up to 6 scales: 7e-6 S over 700 slots of the same sign, less over more of both.
Log-sum-exp within 2e-5 (1 + |lse|), weights within 2e-5: neither depends on the values.
"""
import math

import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, F32, INF, attend_plain, randn

pytestmark = pytest.mark.gpu


def cache_of(k, v, lens):
    """k, v [B, cap, H, D] fp32 as a cache with `lens` slots in use."""
    B, cap, H, D = k.shape
    cache = ris.Cache4.empty(B, H, D, cap)
    assert cache.capacity == cap
    with ris.ris_pack_create([cap] * B) as pack:
        ris.ris_cache4_append(cache, pack, k.flatten(0, 1), v.flatten(0, 1), torch.arange(B * cap, dtype=torch.int32, device="cuda"))
    cache.length.copy_(torch.tensor(lens, dtype=torch.int32))
    return cache


def check(cache, q, lens, out):
    """Outputs, log-sum-exp and weights of a call against 64 bits."""
    B, Hq, D = q.shape
    G = Hq // cache.kv_heads
    w1 = torch.zeros_like(cache.weight)
    got, lse = ris.ris_cache4_attend(cache, q, out_dtype=out, return_lse=True, weight_out=w1)
    ris.ris_device_status()
    got, lse, w1 = got.double().cpu(), lse.double().cpu(), w1.double().cpu()
    _, rl, rw = attend_plain(cache, q, lens)
    assert ((lse == rl) | ((lse - rl).abs() <= 2e-5 * (1 + rl.abs()))).all()  # (-infinity: no slots)
    kk, vv = (x.double().cpu() for x in ris.ris_cache4_read(cache))
    sc = cache.v_scale.double().cpu()
    for b, n in enumerate(lens):
        assert ((w1 - rw)[b, :, :n].abs() <= 2e-5).all()
        for h in range(Hq if n else 0):
            g = h // G
            p = torch.exp(kk[b, g, :n] @ q[b, h].double().cpu() / math.sqrt(D) - rl[b, h])
            v = vv[b, g, :n]
            ref, A = p @ v, p @ v.abs()
            S = (p[:, None] * sc[b, g, :n]).amax(0).repeat_interleave(32)
            bad = ~torch.isfinite(v).all(0)
            assert torch.isnan(got[b, h][bad]).all()
            tol = (1e-5 * A if out == F32 else 2.0 ** -8 * ref.abs() + 2.0 ** -10 * A) + 1e-5 * S
            assert ((got[b, h] - ref).abs()[~bad] <= tol[~bad]).all(), (b, h, float(((got[b, h] - ref).abs() / tol)[~bad].max()))
    return got


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 6, 2), (64, 10, 1)])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("at", [0, 70, 299])
@pytest.mark.parametrize("bad", [INF, float("nan")])
def test_value_that_is_not_finite_stays_in_its_group(D, Hq, Hkv, dtype, out, at, bad):
    lens = [300, 77]
    k, v = randn(2, 304, Hkv, D, seed=1), randn(2, 304, Hkv, D, seed=2)
    q = randn(2, Hq, D, seed=3, dtype=dtype, scale=2.0)
    v[0, at, 0, 40] = bad
    got = check(cache_of(k, v, lens), q, lens, out)
    assert torch.isnan(got[0, :Hq // Hkv, 32:64]).all() and torch.isfinite(got[0, :, :32]).all() and torch.isfinite(got[1]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("out", [F32, BF16])
def test_key_that_is_not_finite_stays_in_its_sequence_and_head(D, out):
    lens = [300, 77]
    k, v = randn(2, 304, 2, D, seed=1), randn(2, 304, 2, D, seed=2)
    q = randn(2, 6, D, seed=3, dtype=BF16, scale=2.0)
    good, gl = ris.ris_cache4_attend(cache_of(k, v, lens), q, out_dtype=out, return_lse=True)
    k[0, 33, 1, 7] = INF
    got, lse = ris.ris_cache4_attend(cache_of(k, v, lens), q, out_dtype=out, return_lse=True)
    assert torch.isnan(got[0, 3:]).all() and torch.isnan(lse[0, 3:]).all()
    assert torch.equal(got[0, :3], good[0, :3]) and torch.equal(got[1], good[1]) and torch.equal(lse[1], gl[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("power", [20, 60, -60])
def test_groups_of_different_size(D, dtype, out, power):
    """One group 2^20 or 2^60 times the others, or as much below them."""
    lens = [700]
    k, v = randn(1, 704, 1, D, seed=1), randn(1, 704, 1, D, seed=2)
    v[..., 32:64] *= 2.0 ** power
    check(cache_of(k, v, lens), randn(1, 4, D, seed=3, dtype=dtype, scale=2.0), lens, out)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("n,at", [(300, [0]), (300, [70]), (300, [299]), (5003, [0, 9, 640, 641, 2500, 5002])])
@pytest.mark.parametrize("size,far", [(40, 2.0), (40, 0.6), (100, 2.0), (12, 0.4)])
def test_slot_of_different_size(out, n, at, size, far):
    """Slots whose values are 2^size times the others', `far` of a query away from it: they add next to nothing, or most."""
    D, cap = 128, (n + 15) // 16 * 16
    k, v = randn(1, cap, 1, D, seed=1, scale=0.3), randn(1, cap, 1, D, seed=2)
    sign = torch.where(randn(D, seed=4) > 0, 1.0, -1.0)
    k[0, at, 0] = -far * sign
    v[0, at] *= 2.0 ** size
    q = (3.0 * sign + randn(1, 4, D, seed=5, scale=0.1)).to(BF16).contiguous()
    check(cache_of(k, v, [n]), q, [n], out)


@pytest.mark.parametrize("scale", [1e-32, 1e34, 1e37])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
def test_values_near_the_ends_of_the_range(scale, out, D):
    """Values around 1e37 (their sums pass fp32's range, their average does not): weights and lse as for any others."""
    n = 4000
    k, v = randn(1, n, 1, D, seed=1), randn(1, n, 1, D, seed=2) * scale
    check(cache_of(k, v, [n]), randn(1, 4, D, seed=3, dtype=BF16, scale=2.0), [n], out)


def test_groups_of_zeros():
    """A group that is zero in every slot, or until a late one."""
    n, D = 900, 128
    k, v = randn(1, 912, 1, D, seed=1), randn(1, 912, 1, D, seed=2)
    v[..., :32] = 0.0
    v[0, :800, 0, 64:96] = 0.0
    for out in (F32, BF16):
        check(cache_of(k, v, [n]), randn(1, 4, D, seed=3, dtype=BF16, scale=2.0), [n], out)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("size", [1e2, 1e4])
def test_scores_of_millions(D, out, size):
    """Each output is its best slot's value: fp32 scores of up to 1e9 stand further apart than they are off."""
    n = 3000
    k, v = randn(1, 3008, 1, D, seed=1) * size, randn(1, 3008, 1, D, seed=2)
    cache, q = cache_of(k, v, [n]), (randn(1, 4, D, seed=3) * size).to(BF16)
    got = ris.ris_cache4_attend(cache, q, out_dtype=out)
    ris.ris_device_status()
    ref, _, _ = attend_plain(cache, q, [n])
    assert ((got.double().cpu() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-6).all()


@pytest.mark.parametrize("dtype,out", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("D,Hq", [(128, 12), (64, 9)])
def test_long_lists_and_more_heads_than_a_block(dtype, out, D, Hq):
    """60,001 slots shared out over every CTA, beside a list of none and one of a single slot; query heads in two blocks."""
    lens = [60001, 0, 1]
    k, v = randn(3, 60016, 1, D, seed=1), randn(3, 60016, 1, D, seed=2)
    cache, q = cache_of(k, v, lens), randn(3, Hq, D, seed=3, dtype=dtype, scale=2.0)
    got = check(cache, q, lens, out)
    assert (got[1] == 0).all()
