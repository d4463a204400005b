"""A batch of prompts answered through the serving operators, on random weights.

    python examples/serve_prompts.py --prompts 9000 700 16000 40 --layers 8 --tokens 256

The model is a stack of attention layers (normalise, one fused q / k / v projection, attention, output
projection, residual): the projections are the program's own matrix products, everything between them is the
library's. The prefill runs all prompts in one call per layer, however their lengths differ:

  ris_rope_axes        positions out of the fused projection's rows; the first prompt opens with an image, whose
                       tokens have a height and a width besides their time
  ris_attention_packed causal attention of every prompt, and the attention weight that each key got from the last rows
  ris_cache4_append    keys and values into the layer's 4-bit cache, with those weights
  ris_cache4_evict     each head's slots cut back to the budget by weight, the newest ones kept

Then one token per sequence and step, a step of all layers being one replayed CUDA graph (ris_rope_axes, ris_cache4_append of
one token each, ris_cache4_attend with the weights added up in the cache); whenever the caches have grown by
--slack tokens over the budget they are cut back again. What is "generated" is each sequence's last hidden state, fed back.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_21927_gb300 import ris  # noqa: E402

BF16 = torch.bfloat16


def prompt_positions(lens, image):
    """[3, tokens] time, height and width of every token, and the time of each sequence's next token.

    An image of h x w tokens at the start of the first prompt is one moment of time; text counts on from the largest
    of its positions, with the same number on each axis.
    """
    cols, after = [], []
    for s, n in enumerate(lens):
        h, w = image if s == 0 and image[0] * image[1] <= n else (0, 0)
        grid = torch.stack([torch.zeros(h, w), torch.arange(h)[:, None].expand(h, w), torch.arange(w).expand(h, w)])
        first = max(h, w)
        text = torch.arange(first, first + n - h * w).expand(3, -1)
        cols.append(torch.cat([grid.reshape(3, -1), text], 1))
        after.append(first + n - h * w)
    return torch.cat(cols, 1).to(torch.int32).cuda(), torch.tensor(after, dtype=torch.int32, device="cuda")


class Layer:
    def __init__(self, width, heads, kv_heads, head_dim, gen):
        rows = (heads + 2 * kv_heads) * head_dim
        self.w_in = (torch.randn(width, rows, generator=gen, device="cuda") * width ** -0.5).to(BF16)
        self.w_out = (torch.randn(heads * head_dim, width, generator=gen, device="cuda") * (heads * head_dim) ** -0.5).to(BF16)
        self.cache = None


class Server:
    def __init__(self, layers, heads, kv_heads, head_dim, budget, recent, slack, max_ctx, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.width = heads * head_dim
        self.budget, self.recent, self.slack, self.max_ctx = budget, recent, slack, max_ctx
        self.rope = ris.rope_cfg(ris.ROPE_YARN, 1e6, 32768)
        quarter = head_dim // 8
        self.sections = [quarter, 3 * quarter // 2, 3 * quarter // 2]
        self.layers = [Layer(self.width, heads, kv_heads, head_dim, gen) for _ in range(layers)]

    def _project(self, layer, x):
        y = torch.nn.functional.rms_norm(x.float(), (self.width,)).to(BF16) @ layer.w_in
        y = y.view(-1, self.heads + 2 * self.kv_heads, self.head_dim)
        return y[:, :self.heads], y[:, self.heads:self.heads + self.kv_heads], y[:, self.heads + self.kv_heads:]

    def prefill(self, x, lens, image=(0, 0), weight_rows=64):
        """x [tokens, width]: hidden states of every prompt's tokens, one prompt after another; returns the last ones."""
        at, self.time = prompt_positions(lens, image)
        order = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).cuda()
        self.token = torch.tensor(lens, dtype=torch.int32, device="cuda")
        full = max(max(lens), self.budget)
        whole = ris.Cache4.empty(len(lens), self.kv_heads, self.head_dim, full)  # one layer's prompt keys, used again by the next
        with ris.ris_pack_create(lens) as pack:
            for layer in self.layers:
                q, k, v = self._project(layer, x)
                q, k = ris.ris_rope_axes(q, k, at, self.sections, self.max_ctx, self.rope)
                o, weight = ris.ris_attention_packed(pack, q, k, v, weight_rows=weight_rows)
                whole.length.zero_()
                ris.ris_cache4_append(whole, pack, k, v, order, weight=weight)
                layer.cache = ris.Cache4.empty(len(lens), self.kv_heads, self.head_dim, self.budget + self.slack)
                ris.ris_cache4_evict(whole, layer.cache, self.budget, self.recent)
                x = x + o.view(-1, self.width) @ layer.w_out
        ris.ris_device_status()
        last = torch.tensor(lens).cumsum(0) - 1
        return x[last.cuda()]

    def _step(self):
        x = self.state
        at = self.time.expand(3, -1).contiguous()
        for layer in self.layers:
            q, k, v = self._project(layer, x)
            q, k = ris.ris_rope_axes(q, k, at, self.sections, self.max_ctx, self.rope)
            ris.ris_cache4_append(layer.cache, self.ones, k, v, self.token)
            c = layer.cache
            o = ris.ris_cache4_attend(c, q, weight_in=c.weight, weight_out=c.weight)
            x = x + o.view(-1, self.width) @ layer.w_out
        self.state.copy_(x)
        self.time.add_(1)
        self.token.add_(1)

    def generate(self, state, tokens):
        """`tokens` steps of every sequence from hidden states [sequences, width]; returns the states after each."""
        self.state, self.ones = state.clone(), ris.ris_pack_create([1] * len(state))
        out, grown, graph = [], 0, None
        for t in range(tokens):
            if grown == self.slack:  # every cache that was at its budget is full
                for layer in self.layers:
                    ris.ris_cache4_evict(layer.cache, layer.cache, self.budget, self.recent)
                grown = 0
            if t == 0:
                self._step()  # on its own once: the library loads, the matrix products pick their forms
            else:
                if graph is None:
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        self._step()
                graph.replay()
            grown += 1
            out.append(self.state.clone())
        ris.ris_device_status()
        return torch.stack(out)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--prompts", type=int, nargs="+", default=[9000, 700, 16000, 40], help="tokens of each prompt")
    ap.add_argument("--image", type=int, nargs=2, default=[24, 32], help="height and width of the first prompt's image, in tokens")
    ap.add_argument("--layers", type=int, default=8)
    ap.add_argument("--heads", type=int, nargs=2, default=[12, 2], help="query heads and KV heads")
    ap.add_argument("--head-dim", type=int, choices=(64, 128), default=128)
    ap.add_argument("--tokens", type=int, default=256, help="tokens to generate per sequence")
    ap.add_argument("--budget", type=int, default=4096, help="slots of a sequence and head after a cut")
    ap.add_argument("--recent", type=int, default=512, help="newest slots that a cut always keeps")
    ap.add_argument("--slack", type=int, default=128, help="tokens between two cuts")
    a = ap.parse_args(argv)
    server = Server(a.layers, *a.heads, a.head_dim, a.budget, a.recent, a.slack, max(a.prompts) + a.tokens)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(sum(a.prompts), server.width, generator=gen, device="cuda").to(BF16)
    server.generate(server.prefill(x, a.prompts, a.image), min(2, a.tokens))  # warm
    mark = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    mark[0].record()
    state = server.prefill(x, a.prompts, a.image)
    mark[1].record()
    states = server.generate(state, a.tokens)
    mark[2].record()
    torch.cuda.synchronize()
    pre, dec = mark[0].elapsed_time(mark[1]), mark[1].elapsed_time(mark[2])
    held = sum(t.numel() * t.element_size() for t in (server.layers[0].cache.k, server.layers[0].cache.k_scale)) * 2 * a.layers
    print(f"prefill  {sum(a.prompts)} tokens of {len(a.prompts)} prompts, {a.layers} layers: {pre:.2f} ms")
    print(f"generate {a.tokens} x {len(a.prompts)} tokens: {dec:.2f} ms, {dec / max(1, a.tokens):.3f} ms a step")
    print(f"caches   {held / 2 ** 20:.1f} MiB of keys and values, slots in use {server.layers[0].cache.length.tolist()}")
    return server, states


if __name__ == "__main__":
    main()
