#!/usr/bin/env python3
"""A small model taught to compress its cache, then served from the compressed cache.

    python examples/retrofit.py [--steps 200] [--ratio 4]

Two DMC attention layers over packed sequences of different lengths, with the
operators of paper_2403_09636_gb300.retrofit for everything but the plain matrix
products: relaxed states and attention (`attention`), cross entropy (`cross_entropy`).
The task: a sequence repeats a short random phrase, so that a token follows from the
one a phrase earlier. Beside the loss the one-sided penalty of the paper pushes the
number of slots kept, the sum of 1 - alpha, towards 1 / ratio of the tokens, a ratio
that grows over the first half of the steps.

At the end the decisions are made binary (no noise, the sign of k[0] - offset) and a
sequence is served by DmcCache: its prompt by prefill_attention, the rest token by
token. Printed are the loss as trained and as served, and the slots per token.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2403_09636_gb300 import DmcCache  # noqa: E402
from paper_2403_09636_gb300.retrofit import DmcRetrofit, attention, cross_entropy  # noqa: E402

LAYERS, HEADS, KV_HEADS, HEAD_DIM, HIDDEN, VOCAB, PHRASE = 2, 4, 2, 128, 256, 61, 11
OFFSET, TEMPERATURE = 5.0, 0.1


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        def matrix(rows, cols, scale=1.0):
            return torch.nn.Parameter(torch.randn(rows, cols) * scale * cols ** -0.5)
        self.words = matrix(VOCAB, HIDDEN, HIDDEN ** 0.5)
        self.places = matrix(512, HIDDEN, HIDDEN ** 0.5)
        self.qkv = torch.nn.ParameterList(matrix((HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN) for _ in range(LAYERS))
        self.out = torch.nn.ParameterList(matrix(HIDDEN, HEADS * HEAD_DIM, 0.5) for _ in range(LAYERS))
        self.head = matrix(VOCAB, HIDDEN)

    def project(self, layer, x):
        y = (torch.nn.functional.layer_norm(x, (HIDDEN,)) @ self.qkv[layer].t()).to(torch.bfloat16)
        q, k, v = y.view(len(x), -1, HEAD_DIM).split([HEADS, KV_HEADS, KV_HEADS], 1)
        # the gate's neuron is one of the key's; it starts where a fraction of the tokens merges
        k = torch.cat([k[..., :1] + OFFSET - 0.5, k[..., 1:]], -1)
        return q.contiguous(), k.contiguous(), v.contiguous()

    def join(self, layer, x, o):
        return x + o.reshape(len(x), -1).float() @ self.out[layer].t()

    def embed(self, tokens, places):
        return self.words[tokens] + self.places[places]


def batch(lens, dev, g):
    """Packed tokens, their places, targets (the last of a sequence has none) and cu_seqlens."""
    tokens, targets, places = [], [], []
    for n in lens:
        phrase = torch.randint(0, VOCAB, (PHRASE,), generator=g)
        t = phrase.repeat(-(-(n + 1) // PHRASE))[:n + 1]
        tokens.append(t[:-1])
        targets.append(torch.where(torch.arange(n) < PHRASE - 1, -100, t[1:]))  # the first phrase cannot be known
        places.append(torch.arange(n))
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    return (torch.cat(tokens).to(dev), torch.cat(places).to(dev), torch.cat(targets).to(torch.int32).to(dev), cu.to(dev))


def train(steps, ratio, dev, seed=0, quiet=False):
    torch.manual_seed(seed)
    g = torch.Generator().manual_seed(seed)
    model = Model().to(dev)
    opt = torch.optim.AdamW(model.parameters(), lr=2e-3)
    most = 16 * 200
    dmc = DmcRetrofit(HEADS, KV_HEADS, HEAD_DIM, torch.bfloat16, max_tokens=most, max_seqs=16, hidden=HIDDEN, vocab=VOCAB,
                      device=dev)
    first = loss = kept = None
    for step in range(steps):
        lens = torch.randint(40, 201, (16,), generator=g).tolist()
        tokens, places, targets, cu = batch(lens, dev, g)
        T, x, alphas = len(tokens), model.embed(tokens, places), []
        for layer in range(LAYERS):
            q, k, v = model.project(layer, x)
            u = torch.rand(KV_HEADS, T, device=dev).clamp(1e-6, 1 - 1e-6)
            o, alpha = attention(dmc, q, k, v, cu, max(lens), noise=torch.log(u) - torch.log1p(-u), offset=OFFSET,
                                 temperature=TEMPERATURE)
            alphas.append(alpha)
            x = model.join(layer, x, o)
        x = torch.nn.functional.layer_norm(x, (HIDDEN,))
        losses = cross_entropy(dmc, x.to(torch.bfloat16), model.head.to(torch.bfloat16), targets)
        loss = losses.sum() / (targets >= 0).sum()
        kept = 1.0 - torch.stack(alphas).mean()
        goal = 1.0 / (1.0 + (ratio - 1.0) * min(1.0, 2.0 * step / steps))
        total = loss + 5.0 * torch.relu(kept - goal)
        opt.zero_grad()
        total.backward()
        opt.step()
        first = float(loss.detach()) if first is None else first
        if not quiet and step % max(1, steps // 10) == 0:
            print(f"step {step:4d}  loss {float(loss.detach()):.3f}  slots per token {float(kept.detach()):.3f}")
    status, bits = dmc.status()
    if status:
        raise RuntimeError(f"device fault {bits:#x}")
    return model, first, float(loss.detach()), float(kept.detach())


@torch.no_grad()
def serve(model, dev, n=176, prompt=128, seed=1):
    """One sequence from the compressed cache: loss over its repeated part, slots per token."""
    tokens, places, targets, _ = batch([n], dev, torch.Generator().manual_seed(seed))
    cache = DmcCache(LAYERS, 1, HEADS, KV_HEADS, HEAD_DIM, torch.bfloat16, n, LAYERS * KV_HEADS * (n // 32 + 1), prompt,
                     device=dev)
    cu = torch.tensor([0, prompt], dtype=torch.int32, device=dev)

    def keys(k):  # at inference the decision is the sign of k[0]
        return torch.cat([k[..., :1] - OFFSET, k[..., 1:]], -1).contiguous()

    x = model.embed(tokens, places)
    done = []
    for start, end in [(0, prompt)] + [(i, i + 1) for i in range(prompt, n)]:
        y = x[start:end]
        for layer in range(LAYERS):
            q, k, v = model.project(layer, y)
            o = torch.empty_like(q)
            if end - start > 1:
                cache.prefill_attention(layer, q, keys(k), v, cu, prompt, o)
            else:
                cache.decode(layer, q, keys(k), v, o)
            y = model.join(layer, y, o)
        done.append(y)
    y = torch.nn.functional.layer_norm(torch.cat(done), (HIDDEN,))
    logits = y.to(torch.bfloat16).float() @ model.head.to(torch.bfloat16).float().t()
    loss = torch.nn.functional.cross_entropy(logits, targets.long(), ignore_index=-100)
    status, bits, _ = cache.status()
    if status:
        raise RuntimeError(f"device fault {bits:#x}")
    slots = sum(float(cache.lengths(layer).sum()) for layer in range(LAYERS))
    return float(loss), slots / (LAYERS * KV_HEADS * n)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--ratio", type=float, default=4.0)
    a = ap.parse_args()
    dev = torch.device("cuda", torch.cuda.current_device())
    model, first, last, kept = train(a.steps, a.ratio, dev)
    loss, slots = serve(model, dev)
    print(f"trained: loss {first:.3f} -> {last:.3f}, slots per token {kept:.3f}")
    print(f"served:  loss {loss:.3f}, slots per token {slots:.3f}")


if __name__ == "__main__":
    main()
