"""A small decoder served with packed ternary projections, a 4-bit K/V cache and
a 4-bit output head: a prompt, a few tokens, several continuations of it.

    python examples/serve_4bit_cache.py [--layers 4] [--tokens 16]

Weights are random (the shapes' scale of a transformer), so the text is noise;
what the example shows is how the calls go together:

  * tq_kv4_extend makes room for a step's tokens (once for all layers) and says
    where they go and which queries are whose;
  * in each layer tq_linear gives q, k, v (one fused projection; k and v are
    columns of its output), tq_kv4_append stores k and v, tq_kv4_attention
    reads the cache;
  * tq_w4_linear turns the last hidden state into logits;
  * tq_kv4_fork starts continuations that share the prompt's pages,
    tq_kv4_free and tq_kv4_compact give pages back.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_09240_gb300 import tq  # noqa: E402


def norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).half()


class Model:
    """Random weights: ternarized projections, an fp16 embedding, a 4-bit head."""

    def __init__(self, layers=4, hidden=1024, q_heads=8, kv_heads=2, dim=128, ffn=2816, vocab=8192, seed=0):
        self.layers, self.q_heads, self.kv_heads, self.dim = layers, q_heads, kv_heads, dim
        g = torch.Generator(device="cuda").manual_seed(seed)

        def dense(n, k):
            return (torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)).half()

        def ternary(n, k):
            return tq.ternarize(dense(n, k), round(0.1 * n * k / tq.TQ_GROUP))
        wide = q_heads * dim
        self.embedding = torch.randn((vocab, hidden), generator=g, device="cuda").half()
        self.blocks = [dict(qkv=ternary(wide + 2 * kv_heads * dim, hidden), o=ternary(hidden, wide),
                            up=ternary(2 * ffn, hidden), down=ternary(hidden, ffn)) for _ in range(layers)]
        self.head = tq.quantize_w4(dense(vocab, hidden))
        self.ffn = ffn

    def rotate(self, x, pos):
        """Rotary positions on [tokens][heads][dim]."""
        half = self.dim // 2
        f = 10000.0 ** (-torch.arange(half, device=x.device) / half)
        a = pos[:, None, None] * f
        lo, hi = x.float().split(half, -1)
        return torch.cat([lo * a.cos() - hi * a.sin(), lo * a.sin() + hi * a.cos()], -1).half()

    def step(self, cache, slots, counts, tokens, max_q):
        """tokens: the new tokens of sequences slots, counts[i] of each.  Returns
        the logits after each sequence's last one."""
        T, wide = tokens.shape[0], self.q_heads * self.dim
        before = cache.length[slots.long()]
        indptr, where = tq.tq_kv4_extend(cache, slots, counts, T)
        seq = torch.repeat_interleave(torch.arange(slots.shape[0], device="cuda"), counts, output_size=T)
        pos = before[seq] + torch.arange(T, device="cuda") - indptr[seq]
        x = self.embedding[tokens]
        for layer, b in enumerate(self.blocks):
            qkv = tq.tq_linear(norm(x), b["qkv"])
            q, k, v = qkv.split([wide, self.kv_heads * self.dim, self.kv_heads * self.dim], 1)
            q, k = (self.rotate(t.unflatten(1, (-1, self.dim)), pos) for t in (q, k))
            tq.tq_kv4_append(k, v.unflatten(1, (-1, self.dim)), cache, layer, where)
            o = tq.tq_kv4_attention(q, cache, layer, slots, indptr, max_q=max_q)
            x = x + tq.tq_linear(o.flatten(1), b["o"])
            gate, up = tq.tq_linear(norm(x), b["up"]).split(self.ffn, 1)
            x = x + tq.tq_linear((torch.nn.functional.silu(gate.float()) * up.float()).half(), b["down"])
        return tq.tq_w4_linear(norm(x[indptr[1:].long() - 1]), self.head, f32=True)


def int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def run(layers=4, prompts=(150, 37), tokens=16, continuations=3, seed=0):
    """Two prompts, `tokens` greedy tokens each, then continuations of the first
    one.  Returns the model, the cache and what was said."""
    model = Model(layers=layers, seed=seed)
    cache = tq.Kv4Cache.empty(layers, 64, model.kv_heads, model.dim, slots=8, max_pages=16)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    text = [torch.randint(0, model.embedding.shape[0], (n,), generator=g, device="cuda") for n in prompts]
    slots = int32(list(range(len(prompts))))
    logits = model.step(cache, slots, int32(list(prompts)), torch.cat(text), max(prompts))
    one = int32([1] * len(prompts))
    for _ in range(tokens):
        new = logits.argmax(-1)
        text = [torch.cat([t, n[None]]) for t, n in zip(text, new)]
        logits = model.step(cache, slots, one, new, 1)
    # continuations of the first sequence: they share its pages until they write
    children = list(range(len(prompts), len(prompts) + continuations))
    tq.tq_kv4_fork(cache, int32([0] * continuations), int32(children))
    new = torch.topk(logits[0], continuations).indices
    said = [[int(t)] for t in new]
    for _ in range(tokens):
        new = model.step(cache, int32(children), int32([1] * continuations), new, 1).argmax(-1)
        for s, t in zip(said, new.tolist()):
            s.append(t)
    # the second prompt and all continuations but one are done
    tq.tq_kv4_free(cache, int32([1] + children[1:]))
    _, live = tq.tq_kv4_compact(cache)
    cache.check()
    return model, cache, text, said, int(live.item())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=16)
    a = ap.parse_args()
    model, cache, text, said, live = run(a.layers, tokens=a.tokens)
    for i, t in enumerate(text):
        print(f"sequence {i}: {t.shape[0]} tokens, the last ones {t[-a.tokens:].tolist()}")
    for i, t in enumerate(said):
        print(f"continuation {i}: {t}")
    print(f"{live} pages in use, {cache.length.tolist()} tokens by slot")


if __name__ == "__main__":
    main()
