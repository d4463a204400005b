"""Attention over pages of keys that are not finite and of rows whose scores grow without bound: what comes out, and what it costs."""
import pytest
import torch

from paper_2607_21927_gb300 import ris
from test_gpu_paged import BF16, INF, check, make, plain, randn

NAN = float("nan")

pytestmark = pytest.mark.gpu


def _us(fn, n=5):
    fn()
    best = float("inf")
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            fn()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b) / n * 1e3)
    return best


def poison(cache, keys, values, page, seq, at, which, what, channels=slice(None)):
    for name, mine, pool in (("k", keys, cache.k), ("v", values, cache.v)):
        if name in which:
            pool[int(cache.table[seq, at // page]), :, at % page, channels] = what
            mine[seq][at, :, channels] = what


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 12, 2), (64, 32, 4)])
@pytest.mark.parametrize("window,anchors", [(0, 0), (1024, 4)])
def test_a_poisoned_key_costs_little(D, Hq, Hkv, window, anchors):
    """A chunk of a prompt beside single tokens; an early key, one in the middle of the chunk, and a whole stretch of the chunk. Rows that
    see such a key come out as they do, the others are right, and the call takes four times as long at most. (With every row that
    is not finite computed again from its own keys, 2,048 rows behind 6,144 keys took 100 times as long and more.)"""
    page, q_lens, prior = 64, [2048, 1, 1], [6144, 3000, 900]
    lengths = [n + p for n, p in zip(q_lens, prior)]
    q = randn(sum(q_lens), Hq, D, seed=1, dtype=BF16)
    times = []
    with ris.ris_pack_create(q_lens) as pack:
        for where in (None, [10], [7000], list(range(6500, 6800))):
            cache, keys, values = make(lengths, Hkv, D, page, BF16, seed=5)

            def call():
                return ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)

            if where is None:
                clean, lse = call()
                times.append(_us(call))
                continue
            for which, what in (("v", NAN), ("v", INF), ("kv", NAN)):
                for at in where:
                    poison(cache, keys, values, page, 0, at, which, what)
                out, _ = call()
                first, last = min(where), max(where)
                pos = torch.arange(2048) + prior[0]
                hit = (pos >= first) & ((pos - last < window) if window else True)
                if window and first < anchors:
                    hit |= pos >= first
                hit = torch.cat([hit, torch.tensor([False, False])]).cuda()
                assert not torch.isfinite(out[hit]).any()
                assert torch.equal(out[~hit], clean[~hit])
                times.append(_us(call))
    print(f"{D}, {Hq} / {Hkv}, window {window}: " + ", ".join(f"{t:.0f}" for t in times) + " us")
    assert max(times[1:]) <= 4 * times[0] + 20, times


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 12, 2), (64, 32, 4)])
def test_a_row_whose_scores_grow_costs_little(D, Hq, Hkv):
    """Beside a chunk of a prompt, single tokens whose later keys' weights are 2^100 times the first ones' and more."""
    page, q_lens, prior = 64, [2048, 1, 1], [6144, 8000, 900]
    lengths = [n + p for n, p in zip(q_lens, prior)]
    q = randn(sum(q_lens), Hq, D, seed=1, dtype=BF16)
    cache, keys, values = make(lengths, Hkv, D, page, BF16, seed=5)
    with ris.ris_pack_create(q_lens) as pack:
        def call():
            return ris.ris_paged_attend(cache, pack, q)

        call()
        clean = _us(call)
        for i in range(64, 126):  # (key 4,096 on)
            cache.k[int(cache.table[1, i])] *= 64
        call()
        grown = _us(call)
    print(f"{D}, {Hq} / {Hkv}: {clean:.0f}, {grown:.0f} us")
    assert grown <= 4 * clean + 20


# rows of each sequence, keys before them, window, anchors, poisoned keys (sequence, key, what, channel or all)
POISON = [
    ([300, 1], [50, 200], 0, 0, [(0, 120, NAN, 3), (0, 121, INF, 3), (0, 200, -INF, 60), (0, 349, NAN, None), (1, 200, INF, 5)]),
    ([300], [50], 0, 0, [(0, 49, INF, None), (0, 140, -INF, 7), (0, 141, INF, 7), (0, 142, -INF, 9)]),
    ([200, 40, 4], [500, 0, 3000], 64, 4, [(0, 2, NAN, 1), (0, 10, NAN, None), (0, 440, INF, 2), (0, 600, NAN, 3), (1, 30, INF, 4), (2, 2950, NAN, 5)]),
    ([33, 129], [0, 1000], 7, 40, [(0, 5, INF, 0), (0, 32, NAN, 63), (1, 39, NAN, 1), (1, 41, NAN, 2), (1, 1000, INF, None), (1, 1100, -INF, 3)]),
    ([90], [-60], 0, 0, [(0, 0, INF, 1), (0, 20, NAN, 2), (0, 29, NAN, 3)]),  # rows before the first slot
    ([1, 1, 1], [4000, 31, 0], 300, 0, [(0, 3700, NAN, 1), (0, 3701, INF, 2), (0, 3699, NAN, 3), (1, 31, NAN, 4), (2, 0, -INF, 5)]),
    ([700], [0], 100, 10, [(0, 100 * i + 7, NAN if i % 2 else INF, i) for i in range(7)]),
]


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 6, 1), (128, 4, 4), (64, 8, 1), (64, 3, 1)])
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("case", POISON)
def test_values_that_are_not_finite(case, page, D, Hq, Hkv):
    """Every output as the formula has it: infinite, NaN, or as without the keys that the row does not see; the same bits each time."""
    q_lens, prior, window, anchors, bad = case
    lengths = [n + p for n, p in zip(q_lens, prior)]
    cache, keys, values = make(lengths, Hkv, D, page, BF16, "tokens", seed=len(bad), junk=2 ** 30)
    for seq, at, what, channel in bad:
        poison(cache, keys, values, page, seq, at, "v", what, slice(None) if channel is None else channel)
    q = randn(sum(q_lens), Hq, D, seed=11, dtype=BF16)
    with ris.ris_pack_create(q_lens) as pack:
        out, lse = ris.ris_paged_attend(cache, pack, q, window, anchors, return_lse=True)
        again, = ris.ris_paged_attend(cache, pack, q, window, anchors)
    ref = plain(q, keys, values, q_lens, window, anchors)
    y, want = out.double().cpu(), ref[0]
    assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y == INF, want == INF) and torch.equal(y == -INF, want == -INF)
    check(out, lse, ref, BF16)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    ris.ris_device_status()


@pytest.mark.parametrize("D,Hq", [(128, 6), (64, 8)])
@pytest.mark.parametrize("window,anchors", [(0, 0), (150, 4)])
def test_scores_past_all_bounds(D, Hq, window, anchors):
    """Keys of eight patterns of +-2^15, queries of such: scores are whole multiples of 2^31, exact in fp32, and a row's weight goes in equal parts to
    the keys with the largest one (a difference of one multiple is past 2^27 in the exponent). Their values' mean is a sum of n bf16 values
    in fp32, rounded once: 2^-8 of it, and n 2^-24 of the sum of magnitudes, n below 700."""
    q_lens, prior = [150, 1, 4], [400, 600, 90]
    lengths = [n + p for n, p in zip(q_lens, prior)]
    cache, keys, values = make(lengths, 1, D, 32, BF16, seed=3)
    g = torch.Generator().manual_seed(7)
    patterns = (torch.randint(0, 2, (8, D), generator=g) * 2 - 1).float() * 2 ** 15
    for b, n in enumerate(lengths):
        keys[b] = patterns[torch.randint(0, 8, (n,), generator=g)].view(n, 1, D).to(BF16).cuda()
        for at in range(n):
            cache.k[int(cache.table[b, at // 32]), :, at % 32] = keys[b][at]
    q = ((torch.randint(0, 2, (sum(q_lens), Hq, D), generator=g) * 2 - 1).float() * 2 ** 15).to(BF16).cuda()
    with ris.ris_pack_create(q_lens) as pack:
        out, = ris.ris_paged_attend(cache, pack, q, window, anchors)
    y, a = out.double().cpu(), 0
    for b, n in enumerate(q_lens):
        m = lengths[b]
        s = q[a:a + n].double().cpu() @ keys[b][:, 0].double().cpu().T  # [n, Hq, m]
        pos, j = (torch.arange(n) + m - n)[:, None], torch.arange(m)
        see = (j <= pos) & ((j > pos - window) | (j < anchors)) if window else j <= pos
        s = s.masked_fill(~see[:, None], -INF)
        w = (s == s.amax(-1, keepdim=True)).double()
        w /= w.sum(-1, keepdim=True)
        v = values[b][:, 0].double().cpu()
        assert ((y[a:a + n] - w @ v).abs() <= 2.0 ** -8 * (w @ v).abs() + 700 * 2.0 ** -24 * (w @ v.abs())).all()
        a += n
    ris.ris_device_status()


def test_a_captured_call_meets_a_poisoned_key():
    """A graph captured over finite keys, replayed before, with and after a NaN in one of them, twice in a row and beside another stream's."""
    lengths, q_lens = [900, 40, 2000], [130, 1, 4]
    cache, keys, values = make(lengths, 2, 128, 32, BF16, seed=1)
    q = randn(135, 12, 128, seed=2, dtype=BF16)
    packs, streams, outs, graphs = [], [], [], []
    for _ in range(2):
        pack, stream, out = ris.ris_pack_create(q_lens), torch.cuda.Stream(), torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            ris.ris_paged_attend(cache, pack, q, out=out)
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                ris.ris_paged_attend(cache, pack, q, out=out)
        packs.append(pack), streams.append(stream), outs.append(out), graphs.append(graph)
    at = (int(cache.table[0, 850 // 32]), 1, 850 % 32, 7)
    was = cache.v[at].clone()
    for what in (None, NAN, INF, None):
        cache.v[at] = was if what is None else what
        values[0][850, 1, 7] = was if what is None else what
        torch.cuda.synchronize()
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
                graph.replay()
        torch.cuda.synchronize()
        ref = plain(q, keys, values, q_lens)
        for out in outs:
            y = out.double().cpu()
            assert torch.equal(y.isnan(), ref[0].isnan()) and torch.equal(y == INF, ref[0] == INF)
            check(out, None, ref, BF16)
    ris.ris_device_status()
    graphs.clear()
