"""Packed prompts in bf16 whose values differ by many powers of two: what a row does not see takes no part in it, however large
it is, and no prompt or head takes bits from another.

Rows against 64 bits: the parity bar of the bf16 path (1e-2 and, with bf16 outputs, 2^-8 |o|; relative L2 5e-3), in units of
the largest value that the row sees. Rows of other sequences and of other KV heads: the same bits as without the large value.
"""
import pytest
import torch

from helpers import check_bf16_path, rel_l2, to_np
from paper_2607_21927_gb300 import ris
from test_gpu_serving import BF16, F32, INF, LONG_KEYS, packed_plain, randn

pytestmark = pytest.mark.gpu

# rows, keys, row length of a tile kernel's choice: short prompts (row tiles), prompts behind many keys (pairs of CTAs at 128)
FORMS = [([150, 140], [150, 140]), LONG_KEYS]


def inputs(n, m, Hq, Hkv, D):
    return [randn(sum(x), h, D, seed=i, dtype=BF16) for i, (x, h) in enumerate(((n, Hq), (m, Hkv), (m, Hkv)), 1)]


@pytest.mark.parametrize("n,m", FORMS)
@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("big", [1e12, 1e30, 3e38, INF, float("nan")])
def test_hidden_value_takes_no_part(n, m, Hq, Hkv, D, big):
    """In the last key of the first sequence, KV head 1: only the last row of that head's group sees it."""
    q, k, v = inputs(n, m, Hq, Hkv, D)
    y = v.clone()
    y[m[0] - 1, 1, 5] = big
    with ris.ris_pack_create(n, m) as pack:
        good = ris.ris_attention_packed(pack, q, k, v, return_lse=True, weight_rows=20)
        got = ris.ris_attention_packed(pack, q, k, y, return_lse=True, weight_rows=20)
        ris.ris_device_status()
    assert torch.equal(got[1], good[1]) and torch.equal(got[2], good[2])  # neither depends on the values
    first, G = n[0], Hq // Hkv
    assert torch.equal(got[0][first:], good[0][first:]) and torch.equal(got[0][:, :G], good[0][:, :G])
    ref, _, _ = packed_plain(q, k, v, n, m, 1)
    check_bf16_path(to_np(got[0][:first - 1]), ref[:first - 1].numpy(), out_bf16=True)
    last, lref = got[0][first - 1, G:].double().cpu(), ref[first - 1, G:]
    keep = torch.arange(D) != 5
    check_bf16_path(last[:, keep].numpy(), lref[:, keep].numpy(), out_bf16=True)
    if abs(big) < INF:
        p = torch.exp((q[first - 1, G:].double() @ k[m[0] - 1, 1].double()).cpu() / D ** 0.5 - good[1][G:, first - 1].double().cpu())
        assert ((last[:, 5] - p * float(y[m[0] - 1, 1, 5])).abs() <= 5e-3 * p * big + 1.0).all()
    else:
        assert not torch.isfinite(last[:, 5]).any()


@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("out_dtype", [F32, BF16])
def test_prompts_and_heads_of_different_size(Hq, Hkv, D, out_dtype):
    """Values of 1e-20, 1 and 1e20 in three prompts, and 1e10 times as much in one of the heads."""
    lens, sizes = [200, 300, 77], [1e-20, 1.0, 1e20]
    q, k, v = inputs(lens, lens, Hq, Hkv, D)
    unit = torch.cat([torch.full((m,), s) for m, s in zip(lens, sizes)])[:, None, None] * torch.tensor([1.0, 1e10])[None, :, None]
    v = (v.float().cpu() * unit).to(BF16).cuda()
    with ris.ris_pack_create(lens) as pack:
        got, = ris.ris_attention_packed(pack, q, k, v, out_dtype=out_dtype)
        ris.ris_device_status()
    ref, _, _ = packed_plain(q, k, v, lens, lens, 1)
    per_row = unit.repeat_interleave(Hq // Hkv, 1).numpy()
    check_bf16_path(to_np(got) / per_row, ref.numpy() / per_row, out_bf16=out_dtype == BF16)


@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("power", [-10, -24, -40, -100])
def test_first_keys_of_different_size(Hq, Hkv, D, power):
    """The first three keys' values 2^power of the rest's: rows 0 .. 2 see nothing else."""
    lens = [40, 290]
    q, k, v = inputs(lens, lens, Hq, Hkv, D)
    v[40:43] = (v[40:43].float() * 2.0 ** power).to(BF16)
    with ris.ris_pack_create(lens) as pack:
        got, = ris.ris_attention_packed(pack, q, k, v)
        ris.ris_device_status()
    ref, _, _ = packed_plain(q, k, v, lens, lens, 1)
    check_bf16_path(to_np(got), ref.numpy(), out_bf16=True)
    check_bf16_path(to_np(got[40:43]) * 2.0 ** -power, ref[40:43].numpy() * 2.0 ** -power, out_bf16=True)


def test_values_of_zero():
    """A prompt whose values are all zero, one with some zero keys, one with a single key that is not."""
    lens, Hq, Hkv, D = [130, 200, 60], 4, 2, 128
    q, k, v = inputs(lens, lens, Hq, Hkv, D)
    v[:130], v[140:150], v[330:389] = 0.0, 0.0, 0.0
    with ris.ris_pack_create(lens) as pack:
        got, = ris.ris_attention_packed(pack, q, k, v)
        ris.ris_device_status()
    ref, _, _ = packed_plain(q, k, v, lens, lens, 1)
    assert (got[:130] == 0).all() and (got[330:389] == 0).all()
    check_bf16_path(to_np(got), ref.numpy(), out_bf16=True)


@pytest.mark.parametrize("n,D", [(8192, 128), (2000, 128), (4000, 64)])
def test_long_prompt_with_a_hidden_value(n, D):
    """The rows of one KV head from the values as given, for a whole prompt: as from the tiles, in reasonable time."""
    Hq, Hkv = 4, 2
    q, k, v = inputs([n], [n], Hq, Hkv, D)
    y = v.clone()
    y[n - 1, 0, 3] = 1e12
    with ris.ris_pack_create([n]) as pack:
        good, = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32)
        ris.ris_attention_packed(pack, q, k, y, out_dtype=F32)
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        got, = ris.ris_attention_packed(pack, q, k, y, out_dtype=F32)
        b.record()
        ris.ris_device_status()
    assert torch.equal(got[:, Hq // Hkv:], good[:, Hq // Hkv:])
    check_bf16_path(to_np(got[:n - 1]), to_np(good[:n - 1]))
    # pairs of rows and keys at a tenth of the FP32 pipe's rate, and a tile's own chain of steps (a row by itself took five times as long)
    pairs = n * (n + 1) / 2 * Hq / Hkv
    assert a.elapsed_time(b) <= 5.0 + 1e3 * pairs * 4 * D / 7e12


@pytest.mark.parametrize("n,m", [([1500], [1500]), ([300, 40], [6000, 5000])])
@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("nats", [8.0, 14.0, 17.0])
def test_key_that_takes_nearly_all_weight_with_values_of_zero(n, m, Hq, Hkv, D, nats):
    """The first key of each sequence stands `nats` above the others and holds zeros: the outputs are what the others add, each a
    small part of the row's weight. Outputs by themselves at the bf16 path's bar, whatever their size: relative L2 5e-3."""
    q, k, v = inputs(n, m, Hq, Hkv, D)
    q, k = (q.float() * 0.3).to(BF16), (k.float() * 0.3).to(BF16)
    q[..., 0] = 4.0
    k[..., 0] = 0.0
    at = 0
    for x in m:
        k[at, :, 0] = nats * D ** 0.5 / 4.0
        v[at] = 0.0
        at += x
    with ris.ris_pack_create(n, m) as pack:
        got, lse = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32, return_lse=True)
        ris.ris_device_status()
    ref, rl, _ = packed_plain(q, k, v, n, m, 1)
    at = 0
    for x, y in zip(n, m):
        first = max(0, 64 - (y - x))  # (rows of few keys are all their own)
        for h in range(Hq):
            assert rel_l2(to_np(got[at + first:at + x, h]), ref[at + first:at + x, h].numpy()) <= 5e-3
        at += x
    assert ((lse.double().cpu() - rl).abs() <= 2e-5 * (1 + rl.abs())).all()


@pytest.mark.parametrize("n,m", [([300, 77], [300, 77]), ([300, 40], [6000, 5000])])
@pytest.mark.parametrize("Hq,Hkv,D", [(6, 2, 128), (4, 2, 64)])
@pytest.mark.parametrize("size", [1e2, 1e4])
def test_scores_of_millions(n, m, Hq, Hkv, D, size):
    """Each row is its best key's value, or a mixture of very few: fp32 scores of up to 1e9 stand further apart than they are off. The
    log-sum-exp is off by what fp32 leaves of it and of the products (2^-19), weights by that of a score of magnitude S (sums of
    fp32 additions that cut off, 2^-23 S each, eight of them: 1e-6 S), one at most."""
    q, k, v = inputs(n, m, Hq, Hkv, D)
    q, k = (q.float() * size).to(BF16), (k.float() * size).to(BF16)
    with ris.ris_pack_create(n, m) as pack:
        got, lse, w = ris.ris_attention_packed(pack, q, k, v, out_dtype=F32, return_lse=True, weight_rows=50)
        ris.ris_device_status()
    ref, rl, rw = packed_plain(q, k, v, n, m, 50)
    check_bf16_path(to_np(got), ref.numpy())
    assert ((lse.double().cpu() - rl).abs() <= 2.0 ** -19 * rl.abs()).all()
    off = 2e-5 + 1e-6 * float(rl[rl > -INF].abs().max())
    assert (w.double().cpu() - rw).abs().max() <= min(off, 1e-2) * max(1.0, float(rw.max()))
