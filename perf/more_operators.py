"""Performance cases of the operators around a cache held in pages: queries and keys normed per head
and turned to their positions in one pass, with the gradient; new keys and values written into
pages; attention of new tokens (one, a few, or a chunk of a prompt) over pages, whole or through a
sliding window with a few first tokens that stay visible.

A case is a dict of plain values. Its ``kind`` says which call it makes:

  norm     RMS norm of every head of q and k with a weight per channel, then the rotation of the first
           ``rot`` channels, in halves or in neighbouring pairs, out of a fused projection's rows
           (``ris_norm_rope``).
  grad     the gradient of that: of q, k and both weights (``ris_norm_rope_backward``).
  append   the rows of a batch into the pages of their sequences (``ris_paged_append``).
  attend   the batch's new rows over the keys in their sequences' pages (``ris_paged_attend``). Row i of
           a sequence that has n new rows and holds m tokens is at p = m - n + i and sees the keys
           j <= p with j > p - window (window 0: all) or j < anchors.

Shapes: 12 / 2 heads of 128 and 32 / 4 heads of 64 are the two grouped-query layers the benchmark
runs; 8 / 8 and 16 / 1 heads of 128 are plain multi-head and multi-query attention. A window of 1024
tokens with 4 anchors is the framework's preset geometry.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(kind="attend", n=0, seqs=1, mix=0, hq=12, hkv=2, d=128, dtype="bf16")
_EPS = 1e-6


def _case(name=None, **kw):
    c = dict(_DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the heads of one decode step of a batch: latency only
        _case("norm-24-tokens", kind="norm", n=24, rot=128, pairs=False, far=40000, rope="yarn"),
        # a long prompt's queries and keys
        _case("norm-30k", kind="norm", n=30011, rot=128, pairs=False, far=30011, rope="plain"),
        # training on a short text in fp32, the precision that gradient checks run in
        _case("grad-900-fp32", kind="grad", n=900, dtype="f32", rot=128, pairs=False, far=900, rope="plain"),
        # a training batch of a model with many small heads that turns half of each, pair by pair
        _case("grad-30k-pairs-hd64", kind="grad", n=30011, hq=32, hkv=4, d=64, rot=32, pairs=True, far=4096, rope="linear"),
        # a decode step's new tokens: latency only
        _case("append-24-tokens", kind="append", n=24, seqs=24, low=30, high=9000, page=16),
        # the keys and values of a batch of prompts, into pages of which each sequence has some
        _case("append-32k-ragged", kind="append", n=32100, seqs=7, mix=3, low=0, high=3000, page=64),
        # a single user's short conversation, many small heads
        _case("attend-1x1500-hd64", n=1, low=1499, high=1499, hq=32, hkv=4, d=64, page=16, window=0, anchors=0, lse=True),
        # a batch in long contexts, past the size of L2
        _case("attend-16x64k", n=16, seqs=16, mix=6, low=48000, high=65535, page=64, window=0, anchors=0, lse=False),
        # drafted tokens, four a sequence, checked through the window and the first tokens
        _case("attend-24x4-window", n=96, seqs=24, mix=4, low=700, high=40000, page=32, window=4096, anchors=4, lse=False),
        # one short chunk behind the keys that its prompt already has, in fp32, as the precision
        # checks of a deployment run it
        _case("chunk-900-fp32", n=900, low=301, high=301, dtype="f32", page=16, window=0, anchors=0, lse=True),
        # a batch of chunks of very different lengths behind their prompts' earlier keys, one of them
        # empty, many small heads, in the preset geometry
        _case("chunk-9-ragged-16k-hd64-window", n=16233, seqs=9, mix=5, empty=True, low=0, high=9000, hq=32, hkv=4, d=64, page=64,
              window=1024, anchors=4, lse=True),
        # the last chunk of a long prompt
        _case("chunk-8k-of-32k", n=8192, low=24576, high=24576, page=128, window=0, anchors=0, lse=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["norm", "grad", "append", "attend", "chunk"], [2, 2, 2, 4, 4])[0]
    hq, hkv, d = rng.choices([(12, 2, 128), (32, 4, 64), (8, 8, 128), (16, 1, 128)], [6, 3, 1, 1])[0]
    c = _case(kind="attend" if kind == "chunk" else kind, hq=hq, hkv=hkv, d=d, mix=rng.randint(1, 10 ** 6))
    if rng.random() < 0.2:
        c["dtype"] = "f32"
    if kind in ("norm", "grad"):
        c.update(n=_log_int(rng, 1, 30011), far=_log_int(rng, 1000, 100000), rope=rng.choice(["plain", "linear", "yarn"]),
                 rot=rng.choice([d, d, d // 2, d // 4]), pairs=rng.random() < 0.4)
        return c
    c["page"] = rng.choice([16, 32, 64, 128, 256])
    c["seqs"] = _log_int(rng, 1, 48)
    if kind == "append":
        c["n"] = max(c["seqs"], _log_int(rng, 1, 32100))
        c["low"], c["high"] = 0, _log_int(rng, 1, 9000)
        return c
    c["window"], c["anchors"] = rng.choice([(0, 0), (0, 0), (_log_int(rng, 1, 8192), rng.choice([0, 4, 64]))])
    c["lse"] = rng.random() < 0.5
    if kind == "attend":
        c["n"] = c["seqs"] * rng.choice([1, 1, 1, 2, 4, 7])
        c["mix"] = -c["mix"]  # as many rows in every sequence
        # keys of all sequences within those of the listed long contexts
        c["high"] = _log_int(rng, 1, min(65535, 2 ** 20 // c["seqs"] * 256 // (hkv * d) + 1))
        c["low"] = rng.randint(0, c["high"])
        if c["dtype"] == "f32":
            c["high"] = min(c["high"], 8000)
            c["low"] = min(c["low"], c["high"])
    else:
        # the products of all heads stay within those of the listed chunk (fp32: of 1,500 rows)
        most = int((1500 if c["dtype"] == "f32" else 12000) * math.sqrt(1536 / (hq * d)))
        c["n"] = _log_int(rng, 1, most)
        c["high"] = _log_int(rng, 1, most)
        c["low"] = rng.randint(0, c["high"])
        c["seqs"] = min(c["seqs"], 16)
        c["empty"] = rng.random() < 0.2
    return c


# ---------------------------------------------------------------- sizes and inputs
def _row_lengths(c):
    """New rows of each sequence, n in all: equal numbers, or shares over a factor of about twenty."""
    if c["mix"] <= 0 or c["n"] == c["seqs"] or c["n"] % c["seqs"] == 0 and c["n"] <= 16 * c["seqs"]:
        return [c["n"] // c["seqs"]] * c["seqs"]
    rng = random.Random(c["mix"])
    share = [math.exp(rng.uniform(0.0, 3.0)) for _ in range(c["seqs"])]
    if c.get("empty") and c["seqs"] > 1:
        share[rng.randrange(c["seqs"])] = 0.0
    ends = [int(round(c["n"] * sum(share[:i + 1]) / sum(share))) for i in range(c["seqs"])]
    return [b - a for a, b in zip([0] + ends, ends)]


def _prior_lengths(c):
    rng = random.Random(c["mix"] + 1)
    return [rng.randint(c["low"], c["high"]) for _ in range(c["seqs"])]


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _rows(gen, n, h, d):
    """n rows of h heads: a hundredth of the channels carries activations six times as large."""
    x = torch.randn(n, h * d, generator=gen, device="cuda")
    m = max(1, round(0.01 * h * d))
    x[:, torch.randperm(h * d, generator=gen, device="cuda")[:m]] *= 6.0
    return x.view(n, h, d)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class _State:
    pass


def _library():
    from paper_2607_21927_gb300 import ris
    return ris


def _base(c):
    """(theta, native context length) of the model that the shape belongs to."""
    return (1e4, 2048) if c["d"] == 64 else (1e6, 32768)


def _frequencies(c):
    """(frequencies in 64 bits, factor on the turned channels) for a context of ``far`` positions."""
    theta, native = _base(c)
    f = theta ** (-2.0 * torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda") / c["rot"])
    s = max(1.0, c["far"] / native)
    if c["rope"] == "linear":
        return f / s, 1.0
    if c["rope"] == "yarn":
        ramp = ((native * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return (1.0 - ramp) * f / s + ramp * f, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _library_rope(c):
    ris = _library()
    return ris.rope_cfg({"plain": ris.ROPE_PLAIN, "linear": ris.ROPE_LINEAR, "yarn": ris.ROPE_YARN}[c["rope"]], *_base(c))


class _Pages:
    """What a program allocates once and keeps: the pools, the page table, the lengths."""

    def __init__(self, c, gen, lengths):
        page, hkv, d = c["page"], c["hkv"], c["d"]
        need = [(n + page - 1) // page for n in lengths]
        count, width = sum(need) + 3, max(max(need), 1) + 1
        # pages in the order that a server with finished sequences hands them out: none
        order = torch.randperm(count, generator=gen, device="cuda").int()
        self.table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        # (slots that no sequence uses hold what earlier sequences left there)
        self.k = _rows(gen, count * hkv * page, 1, d).to(_dtype(c)).view(count, hkv, page, d)
        self.v = _rows(gen, count * hkv * page, 1, d).to(_dtype(c)).view(count, hkv, page, d)
        self.length = _ints(lengths)


def prepare(case, seed):
    c, s = case, _State()
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s.case, dt = c, _dtype(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] in ("norm", "grad"):
        x = _rows(gen, c["n"], hq + 2 * hkv, d).to(dt)
        s.q, s.k = x[:, :hq], x[:, hq:hq + hkv]
        s.wq, s.wk = ((1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2))
        s.positions = torch.randint(0, c["far"], (c["n"],), generator=gen, device="cuda", dtype=torch.int32)
        if c["kind"] == "grad":
            s.dq = torch.randn(c["n"], hq, d, generator=gen, device="cuda").to(dt)
            s.dk = torch.randn(c["n"], hkv, d, generator=gen, device="cuda").to(dt)
        if own:
            s.rope = _library_rope(c)
        return s
    s.lengths, prior = _row_lengths(c), _prior_lengths(c)
    s.key_lengths = [n + p for n, p in zip(s.lengths, prior)]
    s.pages = _Pages(c, gen, s.key_lengths)
    n = sum(s.lengths)
    if c["kind"] == "append":
        s.k, s.v = (_rows(gen, n, hkv, d).to(dt) for _ in range(2))
        s.start = _ints(prior)
    else:
        s.q = _rows(gen, n, hq, d).to(dt)
    if own:
        ris = _library()
        s.cache = ris.PagedCache(s.pages.k, s.pages.v, s.pages.table, s.pages.length)
        s.pack = ris.ris_pack_create(s.lengths)
    else:
        s.rows = _ints(s.lengths)
        seq = torch.arange(c["seqs"], device="cuda").repeat_interleave(s.rows.long())
        s.seq, s.at = seq, torch.arange(n, device="cuda") - _ints(_offsets(s.lengths)[:-1]).long()[seq]
    return s


# ---------------------------------------------------------------- the plain form
def _turn(x, c, cos, sin):
    """x [n, H, d] in 32 bits with its first ``rot`` channels turned."""
    y, rot = x.clone(), c["rot"]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    u, v = a * cos - b * sin, b * cos + a * sin
    if c["pairs"]:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    else:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    return y


def _angles(s):
    # the angles alone in 64 bits: at a position of 30,000 a 32-bit product is off by 1e-3
    f, m = _frequencies(s.case)
    ang = s.positions[:, None].double() * f
    return (ang.cos() * m).float()[:, None], (ang.sin() * m).float()[:, None]


def _run_norm(s):
    cos, sin = _angles(s)

    def one(x, w):
        x32 = x.float()
        r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + _EPS)
        return _turn(x32 * r * w.float(), s.case, cos, sin).to(x.dtype)

    return one(s.q, s.wq), one(s.k, s.wk)


def _run_grad(s):
    cos, sin = _angles(s)

    def one(dy, x, w):
        g = _turn(dy.float(), s.case, cos, -sin)  # turned back
        x32 = x.float()
        r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + _EPS)
        h = x32 * r
        gw = (g * h).sum((0, 1), dtype=torch.float64).float()  # up to a million terms
        g = g * w.float()
        return (r * (g - h * (g * h).mean(-1, keepdim=True))).to(x.dtype), gw

    (gq, gwq), (gk, gwk) = one(s.dq, s.q, s.wq), one(s.dk, s.k, s.wk)
    return gq, gk, gwq, gwk


def _run_append(s):
    c, p = s.case, s.pages
    slot = s.start.long()[s.seq] + s.at
    page = p.table[s.seq, slot // c["page"]].long()
    p.k[page, :, slot % c["page"]] = s.k
    p.v[page, :, slot % c["page"]] = s.v
    p.length.copy_(s.start + s.rows)
    return p.k, p.v, p.length


def _visible(c, pos, j):
    seen = j <= pos
    if c["window"]:
        seen = seen & ((j > pos - c["window"]) | (j < c["anchors"]))
    return seen


def _attend_rows(c, q, k, v, hidden):
    """q [.., hkv, group n, d] over k, v [.., hkv, m, d]: (out, log-sum-exp), hidden [.., n, m]."""
    group = c["hq"] // c["hkv"]
    sc = (q @ k.transpose(-1, -2)).unflatten(-2, (group, -1))
    sc *= 1.0 / math.sqrt(c["d"])
    sc.masked_fill_(hidden, float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top.masked_fill_(top == float("-inf"), 0.0)
    sc.sub_(top).exp_()
    total = sc.sum(-1, keepdim=True)
    out = (sc.flatten(-3, -2) @ v).unflatten(-2, (group, -1)) / total.clamp(min=1e-30)
    return out, (top + total.log())[..., 0]


def _run_attend(s):
    c, p = s.case, s.pages
    group, hkv, d, dt = c["hq"] // c["hkv"], c["hkv"], c["d"], s.q.dtype
    out = torch.zeros(s.q.shape, dtype=dt, device="cuda")
    lse = torch.full((c["hq"], s.q.shape[0]), float("-inf"), device="cuda")
    n = s.lengths[0]
    if 0 < n <= 16 and all(x == n for x in s.lengths):  # a few rows of every sequence: all at once
        j = torch.arange(max(s.key_lengths), device="cuda")
        page = p.table[:, j // c["page"]].clamp(min=0).long()  # [B, m]
        k, v = (x[page, :, j % c["page"]].float().transpose(1, 2) for x in (p.k, p.v))  # [B, hkv, m, d]
        q = s.q.float().unflatten(0, (-1, n)).unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)
        pos = (p.length[:, None] - n + torch.arange(n, device="cuda"))[..., None]
        o, l = _attend_rows(c, q, k, v, ~_visible(c, pos, j)[:, None, None])  # [B, hkv, group, n, d]
        out.copy_(o.permute(0, 3, 1, 2, 4).reshape(s.q.shape))
        lse.copy_(l.permute(1, 2, 0, 3).reshape(lse.shape))
    else:
        q0 = _offsets(s.lengths)
        for b, (n, m) in enumerate(zip(s.lengths, s.key_lengths)):
            if n == 0:
                continue
            j = torch.arange(m, device="cuda")
            page = p.table[b, j // c["page"]].long()
            k, v = (x[page, :, j % c["page"]].float().transpose(0, 1) for x in (p.k, p.v))  # [hkv, m, d]
            q = s.q[q0[b]:q0[b + 1]].float().unflatten(1, (hkv, group)).permute(1, 2, 0, 3).flatten(1, 2)
            pos = torch.arange(m - n, m, device="cuda")[:, None]
            o, l = _attend_rows(c, q, k, v, ~_visible(c, pos, j))  # [hkv, group, n, d]
            out[q0[b]:q0[b + 1]] = o.permute(2, 0, 1, 3).flatten(1, 2).to(dt)
            lse[:, q0[b]:q0[b + 1]] = l.flatten(0, 1)
    return (out, lse) if c["lse"] else (out,)


_PLAIN = {"norm": _run_norm, "grad": _run_grad, "append": _run_append, "attend": _run_attend}


def run(s):
    c = s.case
    if not own:
        return _PLAIN[c["kind"]](s)
    ris = _library()
    if c["kind"] == "norm":
        return ris.ris_norm_rope(s.q, s.k, s.positions, c["far"], s.rope, s.wq, s.wk, eps=_EPS, rot_dim=c["rot"], pairs=c["pairs"])
    if c["kind"] == "grad":
        return ris.ris_norm_rope_backward(s.dq, s.dk, s.q, s.k, s.positions, c["far"], s.rope, s.wq, s.wk, eps=_EPS,
                                          rot_dim=c["rot"], pairs=c["pairs"])
    if c["kind"] == "append":
        ris.ris_paged_append(s.cache, s.pack, s.k, s.v, start=s.start)
        return s.cache.k, s.cache.v, s.cache.length
    return ris.ris_paged_attend(s.cache, s.pack, s.q, window=c["window"], anchors=c["anchors"], longest=max(s.key_lengths),
                                return_lse=c["lse"])


# ---------------------------------------------------------------- work
def _pairs(c):
    """(row, key) pairs that are visible, and keys that some row of their sequence sees."""
    pairs, keys = 0, 0
    for n, prior in zip(_row_lengths(c), _prior_lengths(c)):
        if n == 0:
            continue
        w, a = c["window"], c["anchors"]
        for i in range(n):
            p = prior + i
            pairs += p + 1 if w == 0 else min(p + 1, w) + min(a, max(0, p + 1 - w))
        first = 0 if w == 0 else max(0, prior + 1 - w)
        keys += prior + n - first + (min(a, first) if w else 0)
    return pairs, keys


def work(case):
    c = case
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    esz = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] in ("norm", "grad"):
        elements = c["n"] * (hq + hkv) * d
        moved = 2 if c["kind"] == "norm" else 3
        return {"bytes": float(moved * elements * esz + 4 * c["n"] + 2 * d * (esz + 4 * (moved - 2))),
                "flops": (7.0 if c["kind"] == "norm" else 14.0) * elements}
    n = sum(_row_lengths(c))
    if c["kind"] == "append":
        return {"bytes": 4.0 * n * hkv * d * esz + 8.0 * c["seqs"], "flops": 0.0}
    pairs, keys = _pairs(c)
    b = 2.0 * n * hq * d * esz + 2.0 * keys * hkv * d * esz + 4.0 * n * hq * c["lse"]
    return {"bytes": b, "flops": 4.0 * d * hq * pairs}


# ---------------------------------------------------------------- the same results in 64 bits
def _exact_forward(c, x, w, turn):
    y = x * (x.square().mean(-1, keepdim=True) + _EPS).rsqrt() * w
    head, rest = y[..., :c["rot"]], y[..., c["rot"]:]
    z = head.unflatten(-1, (-1, 2)) if c["pairs"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
    return torch.cat([z.flatten(-2) if c["pairs"] else z.transpose(-1, -2).flatten(-2), rest], -1)


def _exact_norm(c, s):
    f, m = _frequencies(c)
    ang = s.positions.double()[:, None] * f
    turn = torch.polar(torch.full_like(ang, m), ang)[:, None]
    leaves = [x.double().contiguous() for x in (s.q, s.k, s.wq, s.wk)]
    if c["kind"] == "norm":
        return _exact_forward(c, leaves[0], leaves[2], turn), _exact_forward(c, leaves[1], leaves[3], turn)
    leaves = [x.requires_grad_() for x in leaves]
    with torch.enable_grad():
        y = [_exact_forward(c, leaves[i], leaves[i + 2], turn) for i in range(2)]
        return torch.autograd.grad(y, leaves, [s.dq.double(), s.dk.double()])


def _exact_attend(c, s):
    p, group, page = s.pages, c["hq"] // c["hkv"], c["page"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full((c["hq"], s.q.shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    base = 0
    for b, (n, m) in enumerate(zip(s.lengths, s.key_lengths)):
        ids = p.table[b].tolist()[:(m + page - 1) // page]
        for g in range(c["hkv"]):
            k, v = (torch.cat([x[i, g] for i in ids])[:m].double() if ids else None for x in (p.k, p.v))
            for h in range(g * group, (g + 1) * group):
                for r in range(0, n, 4096):
                    rows = torch.arange(r, min(n, r + 4096), device="cuda")
                    dist = (rows + m - n)[:, None] - torch.arange(m, device="cuda")
                    drop = dist < 0
                    if c["window"]:
                        old = dist >= c["window"]
                        old[:, :c["anchors"]] = False
                        drop |= old
                    x = (s.q[base + rows, h].double() @ k.T / math.sqrt(c["d"])).masked_fill(drop, -math.inf)
                    lse[h, base + rows] = torch.logsumexp(x, -1)
                    out[base + rows, h] = torch.softmax(x, -1) @ v
        base += n
    return (out, lse) if c["lse"] else (out,)


def exact(case, seed):
    c = case
    if c["kind"] == "append" or (c["kind"] == "attend" and work(c)["flops"] > 4e12):
        return None  # copies; too long in 64 bits
    s = prepare(c, seed)
    return _exact_attend(c, s) if c["kind"] == "attend" else _exact_norm(c, s)
