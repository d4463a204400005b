"""Performance cases of the serving operators: prompts of several lengths in one call, and a cache
held in 4 bits that is written, read by single tokens and cut back by attention weight.

A case is a dict of plain values. Its ``kind`` says which call it makes:

  rope     rotary positions of q and k, given per token on one axis or on three (time, height,
           width), out of a fused projection's rows (``ris_rope_axes``).
  prompt   causal attention over packed prompts, keys of an earlier chunk before them or not, with
           the attention weight that each key got from the last rows (``ris_attention_packed``).
  append   new keys and values into the 4-bit cache, and the appended rows as the values they now
           stand for (``ris_cache4_append``, ``ris_cache4_read``).
  attend   one token per sequence against the 4-bit cache, with or without the weights added up
           per slot (``ris_cache4_attend``).
  evict    the cache cut back to a budget by accumulated weight, the newest tokens kept
           (``ris_cache4_evict``).

Shapes: 12 / 2 heads of 128 and 32 / 4 heads of 64 are the two grouped-query layers the benchmark
runs; 8 / 8 and 16 / 1 heads of 128 are plain multi-head and multi-query attention.

The 4-bit format: a row (token, head) of D values is cut into groups of 32. A group's scale is
bf16(max |x| * fl32(1/6)); a value is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even
code, sign in bit 3) to x / scale in 32 bits, 6 at most. Two codes to a byte, the first in the low
half; the bytes of a row lie in the order that the kernels' loads take them (``_byte_order``).
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DEFAULTS = dict(kind="prompt", n=0, seqs=1, mix=1, hq=12, hkv=2, d=128, dtype="bf16", out="bf16", lse=False)


def _case(name=None, **kw):
    c = dict(_DEFAULTS, **kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the positions of one decode step of a batch: latency only
        _case("rope-24-tokens", kind="rope", n=24, axes=1, far=40000, rope="yarn"),
        # image and text tokens of a long prompt, three axes, q and k out of fused rows
        _case("rope-30k-3axes", kind="rope", n=30011, axes=3, far=30011, rope="plain"),
        # one short chunk behind the keys that its prompt already has, in fp32, as the precision
        # checks of a deployment run it
        _case("prompt-chunk-900-fp32", n=900, dtype="f32", out="f32", lse=True, prior=301, weight_rows=0),
        # a batch of prompts of very different lengths, one of them empty, many small heads, and the
        # weights of the last 64 rows, by which the cache is cut back afterwards
        _case("prompt-9-ragged-16k-hd64", n=16233, seqs=9, mix=5, empty=True, hq=32, hkv=4, d=64, lse=True, prior=0,
              weight_rows=64),
        # the longest single prompt: the dense layer of the benchmark
        _case("prompt-32k", n=32768, lse=True, prior=0, weight_rows=0),
        # a decode step's new tokens: latency only
        _case("append-24-tokens", kind="append", n=24, seqs=24, mix=0, cap=4096, used=4000, weight=False),
        # the keys and values of a batch of prompts, with their weights
        _case("append-32k-ragged", kind="append", n=32100, seqs=7, mix=3, cap=16384, used=100, weight=True),
        # a single user's short conversation, many small heads, results in fp32
        _case("attend-1x1500-hd64", kind="attend", seqs=1, cap=1504, low=1500, hq=32, hkv=4, d=64, out="f32",
              lse=True, weight=False),
        # a batch in the middle of its generation, each at its own length, weights added up
        _case("attend-24x9k-weights", kind="attend", seqs=24, mix=4, cap=9216, low=700, lse=True, weight=True),
        # long contexts, past the size of L2
        _case("attend-16x64k", kind="attend", seqs=16, mix=6, cap=65536, low=48000, weight=False),
        # a conversation that has outgrown its budget
        _case("evict-1x2100-hd64", kind="evict", seqs=1, cap=2112, low=2100, hq=32, hkv=4, d=64, budget=2048, recent=512),
        # a batch of long prompts cut to a quarter after the prefill
        _case("evict-16x32k", kind="evict", seqs=16, mix=7, cap=32768, low=20000, budget=8192, recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["rope", "prompt", "append", "attend", "evict"], [2, 4, 2, 4, 2])[0]
    hq, hkv, d = rng.choices([(12, 2, 128), (32, 4, 64), (8, 8, 128), (16, 1, 128)], [6, 3, 1, 1])[0]
    c = _case(kind=kind, hq=hq, hkv=hkv, d=d, mix=rng.randint(1, 10 ** 6))
    if rng.random() < 0.2:
        c["dtype"] = c["out"] = "f32"
    c["lse"] = rng.random() < 0.5
    if kind == "rope":
        c.update(axes=rng.choice([1, 3]), n=_log_int(rng, 1, 30011), far=_log_int(rng, 1000, 100000),
                 rope=rng.choice(["plain", "linear", "yarn"]))
    elif kind == "prompt":
        # the products of all heads stay within those of the listed 32k prompt (fp32: of 3,000 tokens)
        most = int((3000 if c["dtype"] == "f32" else 32768) * math.sqrt(1536 / (hq * d)))
        c["seqs"] = _log_int(rng, 1, 24)
        c["n"] = _log_int(rng, 1, most)
        c["prior"] = _log_int(rng, 1, max(2, (most - c["n"]) // 4)) if rng.random() < 0.25 else 0
        c["weight_rows"] = rng.choice([0, 0, 16, 64, 200])
        c["empty"] = rng.random() < 0.2
        if c["seqs"] > 1:  # padding to the longest must fit the plain form's memory
            c["n"] = min(c["n"], 12000)
    elif kind == "append":
        c["seqs"] = _log_int(rng, 1, 48)
        c["n"] = max(c["seqs"], _log_int(rng, 1, 32100))
        c["used"] = _log_int(rng, 1, 5000)
        c["weight"] = rng.random() < 0.5
        c["cap"] = (c["used"] + c["n"] + 15) // 16 * 16
        if c["seqs"] * c["cap"] * hkv * d > 2 ** 25:
            c["seqs"] = max(1, 2 ** 25 // (c["cap"] * hkv * d))
    elif kind == "attend":
        c["out"] = rng.choice([c["out"], "f32"])
        c["weight"] = rng.random() < 0.4
        c["seqs"] = _log_int(rng, 1, 64)
        c["cap"] = (_log_int(rng, 1, 65536) + 15) // 16 * 16
        c["cap"] = max(16, min(c["cap"], 2 ** 20 // c["seqs"] * 256 // (hkv * d) // 16 * 16))
        c["low"] = rng.randint(1, c["cap"])
    else:
        c["seqs"] = _log_int(rng, 1, 32)
        c["cap"] = (_log_int(rng, 200, 65536) + 15) // 16 * 16
        c["cap"] = max(64, min(c["cap"], 2 ** 19 // c["seqs"] * 256 // (hkv * d) // 16 * 16))
        c["low"] = rng.randint(1, c["cap"])
        c["budget"] = rng.randint(2, c["cap"])
        c["recent"] = rng.randint(0, min(1024, c["budget"] - 1))
    return c


# ---------------------------------------------------------------- sizes and inputs
def _prompt_lengths(c):
    """Tokens of each of a call's sequences, n in all: shares over a factor of about twenty."""
    rng = random.Random(c["mix"])
    if c["mix"] == 0:
        return [c["n"] // c["seqs"]] * c["seqs"]
    share = [math.exp(rng.uniform(0.0, 3.0)) for _ in range(c["seqs"])]
    if c.get("empty") and c["seqs"] > 1:
        share[rng.randrange(c["seqs"])] = 0.0
    ends = [int(round(c["n"] * sum(share[:i + 1]) / sum(share))) for i in range(c["seqs"])]
    return [b - a for a, b in zip([0] + ends, ends)]


def _cache_lengths(c):
    rng = random.Random(c["mix"])
    return [rng.randint(c["low"], c["cap"]) for _ in range(c["seqs"])]


def _dtype(s):
    return torch.bfloat16 if s == "bf16" else torch.float32


def _rows(gen, n, h, d, outliers=True):
    """n rows of h heads: a hundredth of the channels carries activations six times as large."""
    x = torch.randn(n, h * d, generator=gen, device="cuda")
    if outliers:
        m = max(1, round(0.01 * h * d))
        x[:, torch.randperm(h * d, generator=gen, device="cuda")[:m]] *= 6.0
    return x.view(n, h, d)


def _offsets(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths) + 1)]


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class _State:
    pass


def _library():
    from paper_2607_21927_gb300 import ris
    return ris


def _axis_sections(c):
    """Frequencies of each axis: all of one, or a quarter and twice three eighths."""
    half = c["d"] // 2
    return [half] if c["axes"] == 1 else [half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8]


def _frequencies(c):
    """(frequencies in 64 bits, factor on the rotated vectors) for a context of ``far`` positions."""
    theta, native = (1e4, 2048) if c["d"] == 64 else (1e6, 32768)
    f = theta ** (-2.0 * torch.arange(c["d"] // 2, dtype=torch.float64, device="cuda") / c["d"])
    s = max(1.0, c["far"] / native)
    if c["rope"] == "linear":
        return f / s, 1.0
    if c["rope"] == "yarn":
        ramp = ((native * f / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        return (1.0 - ramp) * f / s + ramp * f, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _positions(c, gen):
    """[axes][n]: a batch's next positions (one axis), or text runs and image grids (three)."""
    n = c["n"]
    if c["axes"] == 1:
        return torch.randint(0, c["far"], (1, n), generator=gen, device="cuda", dtype=torch.int32)
    i = torch.arange(n, device="cuda")
    grid = i % 1400  # images of 32 x 32 patches between runs of 376 text tokens
    image = grid < 1024
    base = i // 1400 * 408
    t = torch.where(image, base, base + 32 + grid - 1024)
    h = torch.where(image, base + grid // 32, t)
    w = torch.where(image, base + grid % 32, t)
    return torch.stack([t, h, w]).to(torch.int32)


# ---------------------------------------------------------------- the 4-bit format
def _byte_order(d, values):
    """Where byte b of a row in natural order lies: the keys' words of 8 elements as (quarter of a
    group, group), the values' bytes as (column of a 16-element tile, tile)."""
    b = torch.arange(d // 2, device="cuda")
    if values:
        return b % 8 * (d // 16) + b // 8
    return (b // 4 % 4 * (d // 32) + b // 16) * 4 + b % 4


_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_LIMITS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)


def _quantise(x, values):
    """x [..., d] in 32 bits -> (bytes [..., d / 2], scales [..., d / 32])."""
    d = x.shape[-1]
    g = x.float().unflatten(-1, (d // 32, 32))
    sixth = torch.tensor(1.0 / 6.0, dtype=torch.float32, device=x.device)
    scale = (g.abs().amax(-1) * sixth).to(torch.bfloat16)
    s = scale.float().unsqueeze(-1)
    y = torch.where(s > 0, g / torch.where(s > 0, s, torch.ones_like(s)), torch.zeros_like(g))
    a, limits = y.abs(), torch.tensor(_LIMITS, device=x.device)
    code = torch.bucketize(a, limits, right=False)  # a limit itself goes down
    up = (a == 0.75) | (a == 1.75) | (a == 3.5)  # ties go to the even code
    code = (code + up + 8 * (y < 0)).flatten(-2).to(torch.uint8)
    packed = code[..., 0::2] | (code[..., 1::2] << 4)
    out = torch.empty_like(packed)
    out[..., _byte_order(d, values)] = packed
    return out, scale


def _values(packed, scale, values, dtype=torch.float32):
    """The values that bytes [..., d / 2] and scales [..., d / 32] stand for."""
    d = packed.shape[-1] * 2
    b = packed[..., _byte_order(d, values)]
    code = torch.stack([b & 15, b >> 4], -1).flatten(-2).long()
    levels = torch.tensor(_LEVELS, dtype=dtype, device=packed.device)
    y = levels[code & 7] * (1.0 - 2.0 * (code >> 3).to(dtype))
    return (y.unflatten(-1, (d // 32, 32)) * scale.to(dtype).unsqueeze(-1)).flatten(-2)


class _Cache:
    """The tensors of a 4-bit cache: what a program allocates once and keeps."""

    def __init__(self, batch, heads, d, cap):
        z = dict(device="cuda")
        self.k = torch.zeros(batch, heads, cap, d // 2, dtype=torch.uint8, **z)
        self.v = torch.zeros_like(self.k)
        self.k_scale = torch.zeros(batch, heads, cap, d // 32, dtype=torch.bfloat16, **z)
        self.v_scale = torch.zeros_like(self.k_scale)
        self.pos = torch.zeros(batch, heads, cap, dtype=torch.int32, **z)
        self.weight = torch.zeros(batch, heads, cap, dtype=torch.float32, **z)
        self.length = torch.zeros(batch, dtype=torch.int32, **z)


_TENSORS = ("k", "v", "k_scale", "v_scale", "pos", "weight", "length")


def _handle(cache):
    """The library's handle on the same tensors."""
    return _library().Cache4(**{name: getattr(cache, name) for name in _TENSORS})


def _filled(c, gen, lengths):
    """A cache that holds `lengths` tokens of each sequence."""
    cache = _Cache(c["seqs"], c["hkv"], c["d"], c["cap"])
    n = c["seqs"] * c["hkv"] * c["cap"]
    for name, values in (("k", False), ("v", True)):
        x = _rows(gen, n, 1, c["d"]).view(c["seqs"], c["hkv"], c["cap"], c["d"])
        packed, scale = _quantise(x, values)
        getattr(cache, name).copy_(packed)
        getattr(cache, name + "_scale").copy_(scale)
    cache.length.copy_(_ints(lengths))
    # positions of a cache that was cut back before: they grow, with gaps
    gaps = torch.randint(1, 4, cache.pos.shape, generator=gen, device="cuda", dtype=torch.int32)
    cache.pos.copy_(gaps.cumsum(-1, dtype=torch.int32))
    # accumulated weights: a few heavy tokens and a long tail
    u = torch.rand(cache.weight.shape, generator=gen, device="cuda")
    cache.weight.copy_(0.01 / (u + 1e-4))
    return cache


def prepare(case, seed):
    c, s = case, _State()
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s.case, dt = c, _dtype(c["dtype"])
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    if c["kind"] == "rope":
        x = _rows(gen, c["n"], hq + 2 * hkv, d).to(dt)
        s.q, s.k = x[:, :hq], x[:, hq:hq + hkv]
        s.positions = _positions(c, gen)
        if own:
            ris = _library()
            theta, native = (1e4, 2048) if d == 64 else (1e6, 32768)
            kind = {"plain": ris.ROPE_PLAIN, "linear": ris.ROPE_LINEAR, "yarn": ris.ROPE_YARN}[c["rope"]]
            s.rope = ris.rope_cfg(kind, theta, native)
    elif c["kind"] == "prompt":
        s.lengths = _prompt_lengths(c)
        s.key_lengths = [n + (c["prior"] if n else 0) for n in s.lengths]
        s.q = _rows(gen, sum(s.lengths), hq, d).to(dt)
        s.k = _rows(gen, sum(s.key_lengths), hkv, d).to(dt)
        s.v = _rows(gen, sum(s.key_lengths), hkv, d).to(dt)
        if own:
            s.pack = _library().ris_pack_create(s.lengths, s.key_lengths)
        else:
            s.plan = _padding(s.lengths, s.key_lengths)
    elif c["kind"] == "append":
        s.lengths = _prompt_lengths(c)
        s.start = _ints([c["used"] - i % 3 if c["used"] > 2 else c["used"] for i in range(c["seqs"])])
        s.k = _rows(gen, sum(s.lengths), hkv, d).to(dt)
        s.v = _rows(gen, sum(s.lengths), hkv, d).to(dt)
        s.positions = torch.randint(0, 1 << 20, (sum(s.lengths),), generator=gen, device="cuda", dtype=torch.int32)
        s.weight = torch.rand(hkv, sum(s.lengths), generator=gen, device="cuda") if c["weight"] else None
        s.cache = _Cache(c["seqs"], hkv, d, c["cap"])
        if own:
            s.pack = _library().ris_pack_create(s.lengths)
            s.cache = _handle(s.cache)
        else:
            s.plan = _padding(s.lengths, s.lengths)
    else:
        s.lengths = _cache_lengths(c)
        s.cache = _filled(c, gen, s.lengths)
        if c["kind"] == "attend":
            s.q = _rows(gen, c["seqs"], hq, d).to(dt)
            s.sums = torch.zeros_like(s.cache.weight) if c["weight"] else None
        else:
            s.small = _Cache(c["seqs"], hkv, d, (c["budget"] + 63) // 16 * 16)
        if own:
            s.cache = _handle(s.cache)
            if c["kind"] == "evict":
                s.small = _handle(s.small)
    return s


# ---------------------------------------------------------------- the plain form
def _padding(lengths, key_lengths):
    """Index tensors that lay packed rows out as [sequences, longest], and back."""
    p, (q0, k0) = _State(), (_offsets(lengths), _offsets(key_lengths))
    p.mq, p.mk = max(max(lengths), 1), max(max(key_lengths), 1)
    nq, nk = _ints(lengths).long(), _ints(key_lengths).long()
    p.nq, p.nk = nq, nk
    p.q_rows = (_ints(q0[:-1]).long()[:, None] + torch.arange(p.mq, device="cuda")).clamp(max=max(q0[-1] - 1, 0))
    p.k_rows = (_ints(k0[:-1]).long()[:, None] + torch.arange(p.mk, device="cuda")).clamp(max=max(k0[-1] - 1, 0))
    seq = torch.arange(len(lengths), device="cuda")
    sq, sk = seq.repeat_interleave(nq), seq.repeat_interleave(nk)
    p.q_seq, p.q_at = sq, torch.arange(q0[-1], device="cuda") - _ints(q0[:-1]).long()[sq]
    p.k_seq, p.k_at = sk, torch.arange(k0[-1], device="cuda") - _ints(k0[:-1]).long()[sk]
    return p


def _run_rope(s):
    c = s.case
    f, m = _frequencies(c)
    sections = _axis_sections(c)
    axis = torch.arange(len(sections), device="cuda").repeat_interleave(torch.tensor(sections, device="cuda"))
    # the angles alone in 64 bits: at a position of 30,000 a 32-bit product is off by 1e-3
    ang = s.positions[axis].T.double() * f
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    half = c["d"] // 2

    def rotate(x):
        a, b = x[..., :half].float(), x[..., half:].float()
        return (torch.cat([a * cos - b * sin, b * cos + a * sin], -1) * m).to(x.dtype)

    return rotate(s.q), rotate(s.k)


def _run_prompt(s):
    c, p = s.case, s.plan
    hkv, group = c["hkv"], c["hq"] // c["hkv"]
    q = s.q.float()[p.q_rows].unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).flatten(2, 3)  # [S, hkv, group mq, d]
    k, v = s.k.float()[p.k_rows].transpose(1, 2), s.v.float()[p.k_rows].transpose(1, 2)
    sc = (q @ k.transpose(-1, -2)).unflatten(2, (group, p.mq))  # [S, hkv, group, mq, mk]
    sc *= 1.0 / math.sqrt(c["d"])
    i, j = torch.arange(p.mq, device="cuda")[:, None], torch.arange(p.mk, device="cuda")
    hidden = (j > i + (p.nk - p.nq)[:, None, None]) | (j >= p.nk[:, None, None])
    sc.masked_fill_(hidden[:, None, None], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top.masked_fill_(top == float("-inf"), 0.0)
    sc.sub_(top).exp_()
    total = sc.sum(-1, keepdim=True).clamp(min=1e-30)
    out = (sc.flatten(2, 3) @ v).unflatten(2, (group, p.mq)) / total
    res = [out.permute(0, 3, 1, 2, 4).flatten(2, 3)[p.q_seq, p.q_at].to(_dtype(c["out"]))]
    if c["lse"]:
        res.append((top + total.log())[..., 0].flatten(1, 2)[p.q_seq, :, p.q_at].T.contiguous())
    if c["weight_rows"]:
        seen = (i >= (p.nq - c["weight_rows"])[:, None, None]) & (i < p.nq[:, None, None])
        w = (sc * (seen[:, None, None] / total)).sum((2, 3))  # [S, hkv, mk]
        res.append(w[p.k_seq, :, p.k_at].T.contiguous())
    return tuple(res)


def _run_append(s):
    p, cache = s.plan, s.cache
    (k, ks), (v, vs) = _quantise(s.k, False), _quantise(s.v, True)
    slot = s.start.long()[p.q_seq] + p.q_at
    for name, x in (("k", k), ("v", v), ("k_scale", ks), ("v_scale", vs)):
        getattr(cache, name)[p.q_seq, :, slot] = x
    cache.pos[p.q_seq, :, slot] = s.positions[:, None]
    cache.weight[p.q_seq, :, slot] = 0.0 if s.weight is None else s.weight.T
    cache.length.copy_(s.start + p.nq)
    at = torch.arange(p.mq, device="cuda")
    there = (at < p.nq[:, None])[:, None, :, None]
    rows = (s.start.long()[:, None] + at).clamp(max=s.case["cap"] - 1)
    seq = torch.arange(s.case["seqs"], device="cuda")[:, None]
    read = [getattr(cache, name)[seq, :, rows].transpose(1, 2) for name in ("k", "k_scale", "v", "v_scale")]
    return (_values(read[0], read[1], False) * there, _values(read[2], read[3], True) * there, cache.pos, cache.weight,
            cache.length)


def _run_attend(s):
    c, cache = s.case, s.cache
    k, v = _values(cache.k, cache.k_scale, False), _values(cache.v, cache.v_scale, True)
    q = s.q.float().unflatten(1, (c["hkv"], -1))
    sc = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(c["d"]))  # [S, hkv, group, cap]
    there = torch.arange(c["cap"], device="cuda") < cache.length[:, None]
    sc = sc.masked_fill(~there[:, None, None], float("-inf"))
    lse = torch.logsumexp(sc, -1)
    p = torch.exp(sc - lse[..., None])
    res = [(p @ v).flatten(1, 2).to(_dtype(c["out"]))]
    if c["lse"]:
        res.append(lse.flatten(1, 2))
    if c["weight"]:
        res.append(torch.where(there[:, None], cache.weight + p.sum(2), torch.zeros_like(cache.weight)))
    return tuple(res)


def _run_evict(s):
    c, a, b = s.case, s.cache, s.small
    budget, cap = c["budget"], c["cap"]
    slot = torch.arange(cap, device="cuda")
    there = (slot < a.length[:, None])[:, None].expand(-1, c["hkv"], -1)
    newest = torch.where(there, a.pos, torch.full_like(a.pos, -2 ** 31)).amax(-1, keepdim=True)
    # the order of the slots: those of the newest tokens, then by weight, then by slot; what is not there last
    w = torch.where(there, a.weight, torch.full_like(a.weight, float("-inf")))
    by_weight = w.sort(dim=-1, descending=True, stable=True).indices
    recent = there & (a.pos > newest - c["recent"])
    order = by_weight.gather(-1, (~recent).gather(-1, by_weight).to(torch.uint8).sort(dim=-1, stable=True).indices)
    keep = torch.zeros_like(there)
    keep = keep.scatter(-1, order[..., :budget], True) & there
    # kept slots below the budget stay; the i-th kept one above it goes to the i-th freed slot below it
    left = a.length.clamp(max=budget)[:, None, None]
    freed, moved = ~keep & (slot < left), keep & (slot >= left)
    holes = torch.where(freed, slot, slot + cap).sort(-1).values[..., :budget]
    movers = torch.where(moved, slot, slot + cap).sort(-1).values[..., :budget]
    kept = torch.where(slot < left, slot, torch.full_like(slot, -1)).expand(keep.shape)[..., :budget].contiguous()
    kept = torch.cat([kept, kept.new_full((*kept.shape[:-1], 1), -1)], -1)  # (one place for what is no hole)
    to = torch.where(holes < cap, holes, torch.full_like(holes, kept.shape[-1] - 1))
    kept.scatter_(-1, to, torch.where(holes < cap, movers, torch.full_like(movers, -1)))
    kept = kept[..., :-1]
    src, have = kept.clamp(min=0), kept >= 0
    for name in ("k", "v", "k_scale", "v_scale"):
        x, wide = getattr(a, name), have[..., None]
        y = x.gather(2, src[..., None].expand(-1, -1, -1, x.shape[-1]))
        getattr(b, name)[:, :, :budget] = torch.where(wide, y, torch.zeros_like(y))
    for name in ("pos", "weight"):
        y = getattr(a, name).gather(2, src)
        getattr(b, name)[:, :, :budget] = torch.where(have, y, torch.zeros_like(y))
    b.length.copy_(a.length.clamp(max=budget))
    return kept.to(torch.int32), b.k, b.v, b.k_scale, b.v_scale, b.pos, b.weight, b.length


_PLAIN = {"rope": _run_rope, "prompt": _run_prompt, "append": _run_append, "attend": _run_attend, "evict": _run_evict}


def run(s):
    c = s.case
    if not own:
        return _PLAIN[c["kind"]](s)
    ris = _library()
    if c["kind"] == "rope":
        return ris.ris_rope_axes(s.q, s.k, s.positions, _axis_sections(c), c["far"], s.rope)
    if c["kind"] == "prompt":
        return ris.ris_attention_packed(s.pack, s.q, s.k, s.v, out_dtype=_dtype(c["out"]), return_lse=c["lse"],
                                        weight_rows=c["weight_rows"])
    if c["kind"] == "append":
        ris.ris_cache4_append(s.cache, s.pack, s.k, s.v, s.positions, weight=s.weight, start=s.start)
        k, v = ris.ris_cache4_read(s.cache, first=s.start, count=max(s.lengths))
        return k, v, s.cache.pos, s.cache.weight, s.cache.length
    if c["kind"] == "attend":
        res = ris.ris_cache4_attend(s.cache, s.q, out_dtype=_dtype(c["out"]), return_lse=c["lse"],
                                    weight_in=s.cache.weight if c["weight"] else None, weight_out=s.sums)
        res = res if isinstance(res, tuple) else (res,)
        return res + ((s.sums,) if c["weight"] else ())
    kept = ris.ris_cache4_evict(s.cache, s.small, c["budget"], c["recent"])
    b = s.small
    return kept, b.k, b.v, b.k_scale, b.v_scale, b.pos, b.weight, b.length


# ---------------------------------------------------------------- work
def work(case):
    c = case
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    esz, osz = (2 if c["dtype"] == "bf16" else 4), (2 if c["out"] == "bf16" else 4)
    row4 = d + d // 8  # bytes of a token and head: codes and scales of its key and value
    if c["kind"] == "rope":
        pairs = c["n"] * (hq + hkv) * d // 2
        return {"bytes": 4.0 * pairs * esz + 4.0 * c["axes"] * c["n"], "flops": 6.0 * pairs}
    if c["kind"] == "prompt":
        nq = _prompt_lengths(c)
        nk = [n + (c["prior"] if n else 0) for n in nq]
        pairs = sum(n * m - n * (n - 1) / 2.0 for n, m in zip(nq, nk))
        b = sum(nq) * hq * d * (esz + osz) + 2.0 * sum(nk) * hkv * d * esz
        b += 4.0 * sum(nq) * hq * c["lse"] + 4.0 * sum(nk) * hkv * (c["weight_rows"] > 0)
        return {"bytes": b, "flops": 4.0 * d * hq * pairs}
    if c["kind"] == "append":
        rows = sum(_prompt_lengths(c)) * hkv
        longest = max(_prompt_lengths(c)) * c["seqs"] * hkv
        b = rows * (2.0 * d * esz + 8.0 + 4.0 * c["weight"] + 2.0 * row4) + 8.0 * longest * d
        return {"bytes": b, "flops": 6.0 * rows * d}
    slots = sum(_cache_lengths(c)) * hkv
    if c["kind"] == "attend":
        b = slots * (row4 + 8.0 * c["weight"]) + c["seqs"] * hq * (d * (esz + osz) + 4.0 * c["lse"])
        return {"bytes": b, "flops": 4.0 * d * slots * (hq // hkv)}
    left = sum(min(n, c["budget"]) for n in _cache_lengths(c)) * hkv
    return {"bytes": 8.0 * slots + left * (2.0 * row4 + 8.0 + 4.0), "flops": 4.0 * slots}


# ---------------------------------------------------------------- the same results in 64 bits
def _exact_rope(c, s):
    f, m = _frequencies(c)
    edges = _offsets(_axis_sections(c))
    ang = torch.cat([s.positions[a, :, None].double() * f[edges[a]:edges[a + 1]] for a in range(c["axes"])], -1)
    turn = torch.polar(torch.full_like(ang, m), ang)[:, None]

    def rotate(x):
        a, b = x.double().chunk(2, -1)
        z = torch.complex(a, b) * turn
        return torch.cat([z.real, z.imag], -1)

    return rotate(s.q), rotate(s.k)


def _exact_prompt(c, s):
    group = c["hq"] // c["hkv"]
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["hq"], s.q.shape[0], dtype=torch.float64, device="cuda")
    weight = torch.zeros(c["hkv"], s.k.shape[0], dtype=torch.float64, device="cuda")
    q0, k0 = _offsets(s.lengths), _offsets(s.key_lengths)
    for b, (n, m) in enumerate(zip(s.lengths, s.key_lengths)):
        for h in range(c["hq"]):
            g = h // group
            k, v = s.k[k0[b]:k0[b + 1], g].double(), s.v[k0[b]:k0[b + 1], g].double()
            for r in range(0, n, 8192):
                rows = torch.arange(r, min(n, r + 8192), device="cuda")
                x = s.q[q0[b] + rows, h].double() @ k.T / math.sqrt(c["d"])
                x.masked_fill_(torch.arange(m, device="cuda") > (rows + m - n)[:, None], float("-inf"))
                lse[h, q0[b] + rows] = torch.logsumexp(x, -1)
                p = torch.softmax(x, -1)
                out[q0[b] + rows, h] = p @ v
                if c["weight_rows"]:
                    weight[g, k0[b]:k0[b + 1]] += p[rows >= n - c["weight_rows"]].sum(0)
    return (out,) + ((lse,) if c["lse"] else ()) + ((weight,) if c["weight_rows"] else ())


def _exact_attend(c, s):
    group = c["hq"] // c["hkv"]
    out = torch.zeros(c["seqs"], c["hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["seqs"], c["hq"], dtype=torch.float64, device="cuda")
    sums = torch.zeros(s.cache.weight.shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s.lengths):
        for g in range(c["hkv"]):
            k = _values(s.cache.k[b, g, :n], s.cache.k_scale[b, g, :n], False, torch.float64)
            v = _values(s.cache.v[b, g, :n], s.cache.v_scale[b, g, :n], True, torch.float64)
            hs = slice(g * group, (g + 1) * group)
            x = s.q[b, hs].double() @ k.T / math.sqrt(c["d"])
            p = torch.softmax(x, -1)
            out[b, hs], lse[b, hs] = p @ v, torch.logsumexp(x, -1)
            sums[b, g, :n] = s.cache.weight[b, g, :n].double() + p.sum(0)
    return (out,) + ((lse,) if c["lse"] else ()) + ((sums,) if c["weight"] else ())


def exact(case, seed):
    c = case
    if c["kind"] in ("append", "evict"):
        return None  # codes, copies and whole numbers: equal or not
    if c["kind"] == "prompt" and work(c)["flops"] > 4e12:
        return None  # too long in 64 bits
    s = prepare(c, seed)
    return {"rope": _exact_rope, "prompt": _exact_prompt, "attend": _exact_attend}[c["kind"]](c, s)
