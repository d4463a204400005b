"""A cache in pages: rows written into it and attention over it, against plain implementations in 64 bits.

Tolerances. fp32: the parity bar of the fp32 path (relative L2 1e-5), log-sum-exp within 2e-5. bf16: products of queries and
keys are exact and summed in fp32; a weight may be rounded to bf16 once (2^-8 of it: 2^-8 sum_j p_j |v_j| in an output), the
output once (2^-8 of it); 1e-5 of the largest value for the fp32 sums and exponentials. Copies are exact."""
import math

import pytest
import torch

from helpers import rel_l2
from paper_2607_21927_gb300 import ris

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")


def randn(*shape, seed=0, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def pools(layout, pages, H, page, D, dtype, fill):
    """(k, v) [pages, H, page, D] in one of the orders that the descriptor's strides describe."""
    z = dict(dtype=dtype, device="cuda")
    if layout == "heads":
        return tuple(torch.full((pages, H, page, D), fill, **z) for _ in range(2))
    if layout == "tokens":
        return tuple(torch.full((pages, page, H, D), fill, **z).permute(0, 2, 1, 3) for _ in range(2))
    both = torch.full((pages, 2, page, H, D), fill, **z)  # a page's keys, then its values
    return both[:, 0].permute(0, 2, 1, 3), both[:, 1].permute(0, 2, 1, 3)


def make(lengths, H, D, page, dtype, layout="heads", seed=0, scale=1.0, fill=float("nan"), junk=-1, spare=2):
    """A cache that holds `lengths` tokens of each sequence in shuffled pages: (cache, keys, values [length, H, D] of each)."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for n in lengths]
    count, width = sum(need) + spare, max(max(need), 1) + 1
    order = torch.randperm(count, generator=g).tolist()
    k, v = pools(layout, count, H, page, D, dtype, fill)
    table = torch.full((len(lengths), width), junk, dtype=torch.int32)
    keys, values = [], []
    for b, n in enumerate(lengths):
        kb, vb = randn(n, H, D, seed=seed + 2 * b + 1, dtype=dtype, scale=scale), randn(n, H, D, seed=seed + 2 * b + 2, dtype=dtype)
        keys.append(kb), values.append(vb)
        for i in range(need[b]):
            p = order.pop()
            table[b, i] = p
            m = min(page, n - i * page)
            k[p, :, :m] = kb[i * page:i * page + m].transpose(0, 1)
            v[p, :, :m] = vb[i * page:i * page + m].transpose(0, 1)
    cache = ris.PagedCache(k, v, table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    return cache, keys, values


def plain(q, keys, values, q_lens, window=0, anchors=0, lengths=None):
    """(out, log-sum-exp, sum of |p v|) in 64 bits on the CPU."""
    q = q.double().cpu()
    Hq, D = q.shape[1:]
    out, mag = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((Hq, q.shape[0]), -INF, dtype=torch.float64)
    a = 0
    for b, n in enumerate(q_lens):
        m = keys[b].shape[0] if lengths is None else lengths[b]
        k, v = keys[b][:m].double().cpu(), values[b][:m].double().cpu()
        G = Hq // k.shape[1]
        pos, j = (torch.arange(n) + m - n)[:, None], torch.arange(m)
        see = j <= pos
        if window:
            see = see & ((j > pos - window) | (j < anchors))
        for h in range(Hq if m and n else 0):
            s = torch.where(see, q[a:a + n, h] @ k[:, h // G].T / math.sqrt(D), torch.full((), -INF, dtype=torch.float64))
            l = torch.logsumexp(s, -1)
            p = torch.where(see, torch.exp(s - torch.where(l == -INF, torch.zeros_like(l), l)[:, None]), torch.zeros_like(s))
            vv = v[:, h // G]
            if torch.isfinite(vv).all():
                out[a:a + n, h], mag[a:a + n, h] = p @ vv, p @ vv.abs()
            else:
                pv = torch.where(see[..., None], p[..., None] * vv, torch.zeros((), dtype=torch.float64))
                out[a:a + n, h], mag[a:a + n, h] = pv.sum(1), pv.abs().sum(1)
            lse[h, a:a + n] = l
        a += n
    return out, lse, mag


def check(got, lse, ref, dtype):
    out, want, mag = ref
    y = got.double().cpu()
    assert got.dtype == dtype and torch.equal(torch.isfinite(y), torch.isfinite(out))
    there = torch.isfinite(out)
    y, out, mag = y[there], out[there], mag[there]
    if dtype == F32:
        assert rel_l2(y, out) <= 1e-5
    elif out.numel():
        top = 1e-5 * max(1.0, float(mag.max()))
        bad = (y - out).abs() > 2.0 ** -8 * (mag + out.abs()) * (1 + 2.0 ** -7) + top
        assert not bad.any(), (int(bad.sum()), float((y - out).abs().max()))
    if lse is not None:
        lse = lse.double().cpu()
        assert torch.equal(lse == -INF, want == -INF)
        fin = want > -INF
        assert ((lse - want)[fin].abs() <= 2e-5 * (1 + want[fin].abs() / 8)).all()


ATTEND = [
    # new rows, keys before them, Hq, Hkv, D, page, window, anchors, dtype, layout
    ([1], [0], 12, 2, 128, 16, 0, 0, BF16, "heads"),
    ([1], [1499], 32, 4, 64, 16, 0, 0, BF16, "heads"),
    ([1, 1, 1], [700, 0, 63], 12, 2, 128, 64, 0, 0, BF16, "tokens"),
    ([1, 1], [2000, 900], 16, 1, 128, 32, 300, 4, BF16, "joint"),
    ([4, 4, 4, 4], [1200, 3, 0, 511], 12, 2, 128, 32, 256, 4, BF16, "heads"),
    ([300], [0], 12, 2, 128, 128, 0, 0, BF16, "heads"),
    ([129, 0, 7, 1, 260], [100, 50, 0, 1000, 513], 32, 4, 64, 64, 0, 0, BF16, "tokens"),
    ([129, 0, 7, 1, 260], [100, 50, 0, 1000, 513], 32, 4, 64, 16, 200, 70, BF16, "joint"),
    ([500], [777], 8, 8, 128, 256, 0, 0, BF16, "heads"),
    ([500], [777], 8, 8, 64, 256, 129, 3, BF16, "heads"),
    ([33, 65], [31, 500], 7, 1, 128, 16, 0, 0, BF16, "heads"),
    ([20], [300], 40, 1, 64, 32, 50, 0, BF16, "heads"),
    ([5], [200], 130, 1, 128, 16, 0, 0, BF16, "heads"),
    ([3, 2], [200, 90], 300, 2, 64, 16, 17, 1, BF16, "tokens"),
    ([200], [0], 2, 2, 128, 1024, 1, 0, BF16, "heads"),
    ([1], [0], 12, 2, 128, 16, 0, 0, F32, "heads"),
    ([130, 0, 1], [300, 4, 70], 12, 2, 128, 16, 0, 0, F32, "tokens"),
    ([130, 9, 1], [300, 4, 700], 32, 4, 64, 64, 100, 5, F32, "joint"),
    ([6], [90], 70, 1, 64, 16, 0, 0, F32, "heads"),
    ([4, 5], [300, 40], 12, 2, 128, 32, 64, 4, F32, "joint"),
    ([1, 1], [900, 131], 8, 1, 128, 16, 200, 20, F32, "tokens"),
    ([700], [0], 12, 2, 128, 16, 0, 0, BF16, "heads"),      # CTAs with many short row tiles
    ([900], [50], 4, 4, 64, 32, 100, 10, BF16, "tokens"),
    ([1] * 40, [37 * i % 900 for i in range(40)], 8, 8, 64, 32, 0, 0, F32, "heads"),
]


@pytest.mark.parametrize("q_lens,prior,Hq,Hkv,D,page,window,anchors,dtype,layout", ATTEND)
def test_attend(q_lens, prior, Hq, Hkv, D, page, window, anchors, dtype, layout):
    lengths = [n + p for n, p in zip(q_lens, prior)]
    cache, keys, values = make(lengths, Hkv, D, page, dtype, layout, seed=sum(lengths), junk=2 ** 30)
    n = sum(q_lens)
    fused = randn(n, Hq + 2, D, seed=n, dtype=dtype)
    q = fused[:, :Hq]
    with ris.ris_pack_create(q_lens) as pack:
        out, lse = ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)
        again, = ris.ris_paged_attend(cache, pack, q.contiguous(), window, anchors, longest=max(lengths))
    check(out, lse, plain(q, keys, values, q_lens, window, anchors), dtype)
    # (another bound of the lengths may share the work out otherwise: the sums' order differs, nothing else)
    check(again, None, plain(q, keys, values, q_lens, window, anchors), dtype)
    ris.ris_device_status()


@pytest.mark.parametrize("dtype,D,page", [(BF16, 128, 16), (BF16, 64, 64), (F32, 64, 16)])
def test_windows_and_anchors(dtype, D, page):
    """Ends of windows and of the first tokens in all places of a granule and of a tile, apart, side by side and one over the other."""
    q_lens, prior = [70, 1, 5], [330, 401, 3]
    lengths = [n + p for n, p in zip(q_lens, prior)]
    cache, keys, values = make(lengths, 1, D, page, dtype, seed=2)
    q = randn(sum(q_lens), 3, D, seed=3, dtype=dtype)
    with ris.ris_pack_create(q_lens) as pack:
        for window in (1, 31, 33, 100, 128, 300):
            for anchors in (0, 1, 32, 33, 129, 250, 10 ** 9):
                out, lse = ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)
                check(out, lse, plain(q, keys, values, q_lens, window, anchors), dtype)
    ris.ris_device_status()


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 12, 2), (64, 8, 1)])
def test_few_rows_behind_many_keys(D, Hq, Hkv):
    """Several tiles to a CTA, most of a row tile's warps without a row, the last tile cut off anywhere; the same bits each time."""
    q_lens = [1, 4, 1, 2, 1, 1, 7, 1]
    lengths = [9001 + 77 * i for i in range(8)]
    cache, keys, values = make(lengths, Hkv, D, 64, BF16, seed=4, fill=3.0)
    q = randn(sum(q_lens), Hq, D, seed=5, dtype=BF16)
    with ris.ris_pack_create(q_lens) as pack:
        for window, anchors in ((0, 0), (5000, 4)):
            out, lse = ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)
            check(out, lse, plain(q, keys, values, q_lens, window, anchors), BF16)
            for _ in range(20):
                again, = ris.ris_paged_attend(cache, pack, q, window, anchors)
                assert torch.equal(out, again)
    ris.ris_device_status()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_sequences(dtype):
    """More sequences than a CTA has threads, with and without several row tiles, some without rows or keys."""
    for most in (1, 70):
        q_lens = [i % 3 if most == 1 and i % 5 else (i * 7) % (most + 1) for i in range(700)]
        lengths = [n + (i * 13) % 150 for i, n in enumerate(q_lens)]
        cache, keys, values = make(lengths, 1, 64, 16, dtype, seed=5)
        q = randn(sum(q_lens), 2, 64, seed=6, dtype=dtype)
        with ris.ris_pack_create(q_lens) as pack:
            out, lse = ris.ris_paged_attend(cache, pack, q, return_lse=True)
        check(out, lse, plain(q, keys, values, q_lens), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_before_the_first_slot_see_nothing(dtype):
    q_lens, lengths = [300, 40, 2], [100, 0, 1]
    cache, keys, values = make(lengths, 2, 64, 16, dtype, seed=3)
    q = randn(sum(q_lens), 4, 64, seed=4, dtype=dtype)
    with ris.ris_pack_create(q_lens) as pack:
        for w, a in ((0, 0), (7, 2)):
            out, lse = ris.ris_paged_attend(cache, pack, q, w, a, return_lse=True)
            check(out, lse, plain(q, keys, values, q_lens, w, a), dtype)
            assert (out[:200] == 0).all() and (out[300:340] == 0).all() and (lse[:, :200] == -INF).all()


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (F32, 128)])
@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
def test_values_and_keys_that_are_not_finite(dtype, D, bad):
    """In a key that only some of the rows see (the newest ones, or those whose window still holds it), of several kinds of call."""
    for q_lens, prior, window, anchors, at in (([150], [70], 0, 0, 180), ([4], [300], 0, 0, 302), ([200], [500], 64, 4, 520),
                                               ([200], [500], 64, 4, 460), ([1], [300], 100, 4, 150)):
        lengths = [n + p for n, p in zip(q_lens, prior)]
        for which in "kv":
            cache, keys, values = make(lengths, 2, D, 16, dtype, seed=9)
            page, slot = int(cache.table[0, at // 16]), at % 16
            (cache.k if which == "k" else cache.v)[page, 1, slot, 3] = bad
            (keys if which == "k" else values)[0][at, 1, 3] = bad
            q = randn(sum(q_lens), 6, D, seed=10, dtype=dtype)
            with ris.ris_pack_create(q_lens) as pack:
                out, lse = ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)
            ref = plain(q, keys, values, q_lens, window, anchors)
            sees = torch.arange(sum(q_lens)) + prior[0] >= at
            if window:
                sees &= torch.arange(sum(q_lens)) + prior[0] - at < window
            if which == "v":
                check(out, lse, ref, dtype)
                assert not torch.isfinite(out[sees.cuda(), 3:, 3]).any()
            else:  # rows that see it may be anything but must not touch the others
                ok = ~sees
                part = tuple(t[ok] if t.dim() == 3 else t[:, ok] for t in ref)
                check(out[ok.cuda()], lse[:, ok.cuda()], part, dtype)
                first = tuple(t[:, :3] if t.dim() == 3 else t[:3] for t in ref)
                check(out[:, :3], lse[:3], first, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(dtype):
    """Scores of hundreds and of 2^24 and beyond, one key far above the others or all alike."""
    for scale in (30.0, 4096.0):
        cache, keys, values = make([400], 1, 64, 32, dtype, seed=1, scale=scale)
        q = randn(70, 2, 64, seed=2, dtype=dtype, scale=scale)
        with ris.ris_pack_create([70]) as pack:
            out, = ris.ris_paged_attend(cache, pack, q)
        s = (q.double().cpu()[:, 0] @ keys[0][:, 0].double().cpu().T) / 8.0
        s = s.masked_fill(torch.arange(400) > torch.arange(70)[:, None] + 330, -INF)
        # the sums of products are good to 2^-24 of the sum of magnitudes, a few times over: rows whose best key leads by more than that
        lead = s.topk(2, -1).values
        mag = (q.double().cpu()[:, 0].abs() @ keys[0][:, 0].double().cpu().abs().T).amax(-1) / 8.0
        clear = lead[:, 0] - lead[:, 1] > 40.0 + mag * 2.0 ** -18
        assert clear.sum() > 20
        best = values[0][:, 0].double().cpu()[s.argmax(-1)]
        assert torch.equal(out[:, 0].double().cpu()[clear], best[clear])
    cache, keys, values = make([400], 1, 64, 32, dtype, seed=1)
    cache.k.zero_()
    keys[0].zero_()
    with ris.ris_pack_create([70]) as pack:
        out, lse = ris.ris_paged_attend(cache, pack, q, return_lse=True)
    check(out, lse, plain(q, keys, values, [70]), dtype)


@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_grow(D):
    """Keys from the fourth tile on with scores 2^60, 2^90, 2^130 or 2^400 above the first ones': a row's reference stays behind them,
    or the row is computed another way. Many rows, and a few behind many keys."""
    for rows, length in ((70, 700), (3, 9000)):
        cache, _, values = make([length], 1, D, 32, BF16, seed=1, fill=0.0)
        q = randn(rows, 4, D, seed=2, dtype=BF16)
        start = torch.zeros(1, dtype=torch.int32, device="cuda")
        for f in (12.0, 18.0, 26.0, 80.0):
            k = randn(length, 1, D, seed=3)
            k[384:] *= f
            k = k.to(BF16)
            with ris.ris_pack_create([length]) as pack:
                ris.ris_paged_append(cache, pack, k, values[0], start=start)
            with ris.ris_pack_create([rows]) as pack:
                out, lse = ris.ris_paged_attend(cache, pack, q, return_lse=True)
            check(out, lse, plain(q, [k], values, [rows]), BF16)


def test_longest_cuts_the_lengths():
    cache, keys, values = make([500, 90], 2, 64, 16, BF16, seed=1)
    q = randn(8, 4, 64, seed=2, dtype=BF16)
    with ris.ris_pack_create([4, 4]) as pack:
        out, lse = ris.ris_paged_attend(cache, pack, q, longest=200, return_lse=True)
    check(out, lse, plain(q, keys, values, [4, 4], lengths=[200, 90]), BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_entries_that_are_no_page_are_reported(dtype):
    for value in (-1, 10 ** 6):
        cache, keys, values = make([300, 300], 2, 64, 16, dtype, seed=1)
        q = randn(2, 4, 64, seed=2, dtype=dtype)
        cache.table[0, 3] = value  # keys 48 .. 63 of the first sequence
        with ris.ris_pack_create([1, 1]) as pack:
            out, = ris.ris_paged_attend(cache, pack, q, window=200, anchors=20)  # not needed
            ris.ris_device_status()
            check(out, None, plain(q, keys, values, [1, 1], 200, 20), dtype)
            out, = ris.ris_paged_attend(cache, pack, q)
            with pytest.raises(ris.RisError) as e:
                ris.ris_device_status()
            assert e.value.status == ris.RIS_ERR_INVALID
            check(out[1:], None, tuple(t[1:] if t.dim() == 3 else t[:, 1:] for t in plain(q, keys, values, [1, 1])), dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(dtype):
    """Pools of more than 2^31 elements, rows in their last pages."""
    page, H, D = 128, 2, 128
    pages = 2 ** 31 // (page * H * D) + 64
    k, v = (torch.empty(pages, H, page, D, dtype=dtype, device="cuda") for _ in range(2))
    table = (pages - 1 - torch.arange(8, dtype=torch.int32)).view(2, 4).cuda()
    cache = ris.PagedCache(k, v, table, torch.zeros(2, dtype=torch.int32, device="cuda"))
    q_lens = [300, 5]
    kr, vr = randn(305, H, D, seed=1, dtype=dtype), randn(305, H, D, seed=2, dtype=dtype)
    q = randn(305, 4, D, seed=3, dtype=dtype)
    with ris.ris_pack_create(q_lens) as pack:
        ris.ris_paged_append(cache, pack, kr, vr)
        assert cache.length.tolist() == q_lens
        out, lse = ris.ris_paged_attend(cache, pack, q, return_lse=True)
    check(out, lse, plain(q, [kr[:300], kr[300:]], [vr[:300], vr[300:]], q_lens), dtype)


# ---------------------------------------------------------------- writing
@pytest.mark.parametrize("q_lens,before,Hkv,D,page,dtype,layout,given", [
    ([1] * 24, [40 * i for i in range(24)], 2, 128, 16, BF16, "heads", True),
    ([1, 0, 1], [15, 16, 31], 8, 64, 16, F32, "tokens", False),
    ([700, 0, 33, 1], [5, 10, 64, 0], 4, 64, 64, BF16, "joint", False),
    ([700, 0, 33, 1], [5, 10, 64, 0], 4, 64, 64, F32, "heads", True),
    ([0, 0], [3, 9], 2, 128, 16, BF16, "heads", True),
    ([0, 0], [3, 9], 2, 128, 16, BF16, "heads", False),
    ([3], [7], 300, 128, 16, F32, "heads", False),
])
def test_append(q_lens, before, Hkv, D, page, dtype, layout, given):
    lengths = [a + b for a, b in zip(q_lens, before)]
    cache, _, _ = make(lengths, Hkv, D, page, dtype, layout, seed=1, fill=0.0)
    n = sum(q_lens)
    fused = randn(n, 2 * Hkv, D, seed=2, dtype=dtype)
    k, v = fused[:, :Hkv], fused[:, Hkv:]
    want_k, want_v = cache.k.clone(), cache.v.clone()
    table, i = cache.table.tolist(), 0
    for b, m in enumerate(q_lens):
        for t in range(m):
            p, s = table[b][(before[b] + t) // page], (before[b] + t) % page
            want_k[p, :, s], want_v[p, :, s] = k[i], v[i]
            i += 1
    start = torch.tensor(before, dtype=torch.int32, device="cuda")
    if not given:
        cache.length.copy_(start)
    with ris.ris_pack_create(q_lens) as pack:
        ris.ris_paged_append(cache, pack, k, v, start=start if given else None)
    assert torch.equal(cache.k, want_k) and torch.equal(cache.v, want_v) and cache.length.tolist() == lengths
    ris.ris_device_status()


def test_append_outside_the_pages():
    cache, _, _ = make([40, 40], 2, 64, 16, BF16, seed=1, fill=0.0, junk=-5)  # four entries to a sequence, the last is no page
    k = randn(60, 2, 64, seed=2, dtype=BF16)
    before = cache.k.clone()
    start = torch.tensor([-10, 35], dtype=torch.int32, device="cuda")
    with ris.ris_pack_create([30, 30]) as pack:
        ris.ris_paged_append(cache, pack, k, k, start=start)
    with pytest.raises(ris.RisError) as e:
        ris.ris_device_status()
    assert e.value.status == ris.RIS_ERR_INVALID
    assert cache.length.tolist() == [20, 64]
    table, want = cache.table.tolist(), before
    for b, first in enumerate((-10, 35)):
        for t in range(30):
            s = first + t
            if 0 <= s < 48:
                want[table[b][s // 16], :, s % 16] = k[30 * b + t]
    assert torch.equal(cache.k, want)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,window", [(BF16, 0), (BF16, 40), (F32, 0)])
def test_a_prompt_in_chunks_and_generated_tokens(dtype, window):
    """Chunks, then single tokens as replays of one captured graph: norm and turn, append, attend. Every row as in one plain pass."""
    Hq, Hkv, D, page, anchors = 12, 2, 128, 16, 4 if window else 0
    B, chunks, steps = 3, [[70, 33, 0], [9, 40, 130]], 5
    total = [sum(c[b] for c in chunks) + steps for b in range(B)]
    rope = ris.rope_cfg(ris.ROPE_YARN, 1e6, 64)
    wq, wk = (1 + 0.2 * randn(D, seed=s).float() for s in (1, 2))
    wq, wk = wq.to(dtype), wk.to(dtype)
    rows = [randn(total[b], Hq + 2 * Hkv, D, seed=20 + b, dtype=dtype) for b in range(B)]
    cache, _, _ = make(total, Hkv, D, page, dtype, seed=7)
    cache.length.zero_()
    got = [[] for _ in range(B)]
    at = [0] * B

    def layer(x, pack, pos, out):
        q, k = ris.ris_norm_rope(x[:, :Hq], x[:, Hq:Hq + Hkv], pos, 300, rope, wq, wk)
        ris.ris_paged_append(cache, pack, k, x[:, Hq + Hkv:])
        ris.ris_paged_attend(cache, pack, q, window, anchors, out=out)

    for c in chunks:
        x = torch.cat([rows[b][at[b]:at[b] + c[b]] for b in range(B)])
        pos = torch.cat([torch.arange(at[b], at[b] + c[b], dtype=torch.int32) for b in range(B)]).cuda()
        out = torch.empty(x.shape[0], Hq, D, dtype=dtype, device="cuda")
        with ris.ris_pack_create(c) as pack:
            layer(x, pack, pos, out)
        for b, part in enumerate(out.split(c)):
            got[b].append(part)
            at[b] += c[b]
    one = ris.ris_pack_create([1] * B)
    x = torch.empty(B, Hq + 2 * Hkv, D, dtype=dtype, device="cuda")
    out = torch.empty(B, Hq, D, dtype=dtype, device="cuda")
    pos = torch.empty(B, dtype=torch.int32, device="cuda")
    lengths = cache.length.clone()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        x.copy_(torch.stack([rows[b][at[b]] for b in range(B)]))
        pos.copy_(lengths)
        layer(x, one, pos, out)  # (once outside: kernels are loaded)
        cache.length.copy_(lengths)
        graph = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            layer(x, one, pos, out)
            pos.add_(1)
        for t in range(steps):
            x.copy_(torch.stack([rows[b][at[b] + t] for b in range(B)]))
            graph.replay()
            for b in range(B):
                got[b].append(out[b:b + 1].clone())
    stream.synchronize()
    del graph
    one.free()
    assert cache.length.tolist() == total
    for b in range(B):
        p = torch.arange(total[b], dtype=torch.int32, device="cuda")
        q, k = ris.ris_norm_rope(rows[b][:, :Hq], rows[b][:, Hq:Hq + Hkv], p, 300, rope, wq, wk)
        ref = plain(q, [k], [rows[b][:, Hq + Hkv:]], [total[b]], window, anchors)
        check(torch.cat(got[b]), None, ref, dtype)
    ris.ris_device_status()


def test_two_graphs_of_two_caches_and_streams():
    """Captured at the same lengths, replayed at others, at the same time on two streams."""
    state = []
    for i in range(2):
        cache, keys, values = make([900, 40], 2, 128, 32, BF16, seed=i)
        q = randn(2, 12, 128, seed=30 + i, dtype=BF16)
        pack, s = ris.ris_pack_create([1, 1]), torch.cuda.Stream()
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            ris.ris_paged_attend(cache, pack, q, out=out)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                ris.ris_paged_attend(cache, pack, q, out=out)
        state.append((cache, keys, values, q, pack, s, out, g))
    for lens in ([900, 40], [3, 0], [650, 33]):
        for cache, *_ in state:
            cache.length.copy_(torch.tensor(lens, dtype=torch.int32))
        torch.cuda.synchronize()
        for *_, s, out, g in state:
            with torch.cuda.stream(s):
                g.replay()
                g.replay()
        torch.cuda.synchronize()
        for cache, keys, values, q, pack, s, out, g in state:
            check(out, None, plain(q, keys, values, [1, 1], lengths=lens), BF16)
    torch.cuda.synchronize()
    state.clear()


def test_same_bits_each_time():
    cache, _, _ = make([4000, 300, 1900], 2, 128, 64, BF16, seed=1)
    q = randn(203, 12, 128, seed=2, dtype=BF16)
    with ris.ris_pack_create([1, 200, 2]) as pack:
        first = ris.ris_paged_attend(cache, pack, q, return_lse=True)
        for _ in range(5):
            for a, b in zip(first, ris.ris_paged_attend(cache, pack, q, return_lse=True)):
                assert torch.equal(a, b)
