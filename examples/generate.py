#!/usr/bin/env python3
"""A small rotary model taught to compress its cache, then continued with beams from the compressed cache.

    python examples/generate.py [--steps 200] [--ratio 3] [--beams 4]

As examples/retrofit.py, with positions that are rotations of queries and keys (rotary.apply while it is taught) and a
search at the end: prompts are rotated, attended and compressed by one call per layer, every beam starts from its
prompt's cache (DmcCache.reorder, which shares the pages), and each step appends the beams' tokens with the rotation on the
way (append), attends (attend), selects (BeamSelect) and lets the caches follow their beams. Printed are
the loss, how many of the continued tokens repeat the phrase, slots per token, and the pages that sharing saves.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2403_09636_gb300 import DmcCache  # noqa: E402
from paper_2403_09636_gb300 import rotary as R  # noqa: E402
from paper_2403_09636_gb300.beam import BeamSelect  # noqa: E402
from paper_2403_09636_gb300.retrofit import DmcRetrofit, attention, cross_entropy  # noqa: E402

LAYERS, HEADS, KV_HEADS, HEAD_DIM, HIDDEN, VOCAB, PHRASE = 2, 4, 2, 128, 256, 61, 11
OFFSET, TEMPERATURE = 5.0, 0.1
BF16 = torch.bfloat16


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        def matrix(rows, cols, scale=1.0):
            return torch.nn.Parameter(torch.randn(rows, cols) * scale * cols ** -0.5)
        self.words = matrix(VOCAB, HIDDEN, HIDDEN ** 0.5)
        self.qkv = torch.nn.ParameterList(matrix((HEADS + 2 * KV_HEADS) * HEAD_DIM, HIDDEN) for _ in range(LAYERS))
        self.out = torch.nn.ParameterList(matrix(HIDDEN, HEADS * HEAD_DIM, 0.5) for _ in range(LAYERS))
        self.head = matrix(VOCAB, HIDDEN)

    def project(self, layer, x):
        """q, k, v, not rotated. The gate's neuron, one of the key's, starts where a fraction of the tokens merges."""
        y = (torch.nn.functional.layer_norm(x, (HIDDEN,)) @ self.qkv[layer].t()).to(BF16)
        q, k, v = y.view(len(x), -1, HEAD_DIM).split([HEADS, KV_HEADS, KV_HEADS], 1)
        return q.contiguous(), torch.cat([k[..., :1] + OFFSET - 0.5, k[..., 1:]], -1), v.contiguous()

    def join(self, layer, x, o):
        return x + o.reshape(len(x), -1).float() @ self.out[layer].t()

    def last(self, x):
        return torch.nn.functional.layer_norm(x, (HIDDEN,)).to(BF16)


def texts(lens, g):
    """Texts that repeat a short random phrase."""
    return [torch.randint(0, VOCAB, (PHRASE,), generator=g).repeat(-(-n // PHRASE))[:n] for n in lens]


def loss_of(model, dmc, rotary, lens, g, noisy=True, turn=R.apply):
    """Mean loss of a batch of packed texts, and the share of tokens that keep a slot."""
    dev = model.words.device
    t = texts([n + 1 for n in lens], g)
    tokens = torch.cat([x[:-1] for x in t]).to(dev)
    targets = torch.cat([torch.where(torch.arange(len(x) - 1) < PHRASE - 1, -100, x[1:]) for x in t]).to(torch.int32).to(dev)
    places = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).to(dev)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(dev)
    x, alphas = model.words[tokens], []
    for layer in range(LAYERS):
        q, k, v = model.project(layer, x)
        q, k = turn(rotary, q, k, places)
        noise = None
        if noisy:
            u = torch.rand(KV_HEADS, len(tokens), device=dev).clamp(1e-6, 1 - 1e-6)
            noise = torch.log(u) - torch.log1p(-u)
        o, alpha = attention(dmc, q, k, v, cu, max(lens), noise=noise, offset=OFFSET, temperature=TEMPERATURE)
        alphas.append(alpha)
        x = model.join(layer, x, o)
    losses = cross_entropy(dmc, model.last(x), model.head.to(BF16), targets)
    return losses.sum() / (targets >= 0).sum(), 1.0 - torch.stack(alphas).mean()


def train(steps, ratio, dev, seed=0, quiet=False):
    torch.manual_seed(seed)
    g = torch.Generator().manual_seed(seed)
    model = Model().to(dev)
    rotary = R.Rotary(HEAD_DIM, device=dev)
    opt = torch.optim.AdamW(model.parameters(), lr=2e-3)
    dmc = DmcRetrofit(HEADS, KV_HEADS, HEAD_DIM, BF16, max_tokens=16 * 200, max_seqs=16, hidden=HIDDEN, vocab=VOCAB, device=dev)
    loss = math.nan
    for step in range(steps):
        lens = torch.randint(40, 201, (16,), generator=g).tolist()
        loss, kept = loss_of(model, dmc, rotary, lens, g)
        goal = 1.0 / (1.0 + (ratio - 1.0) * min(1.0, 2.0 * step / steps))
        opt.zero_grad()
        (loss + 5.0 * torch.relu(kept - goal)).backward()
        opt.step()
        if not quiet and step % max(1, steps // 10) == 0:
            print(f"step {step:4d}  loss {float(loss.detach()):.3f}  slots per token {float(kept.detach()):.3f}")
    if dmc.status()[0]:
        raise RuntimeError("device fault")
    return model, rotary, float(loss.detach())


@torch.no_grad()
def search(model, rotary, dev, beams=4, prompts=(77, 130, 45), steps=44, seed=1):
    """Continues prompts with beams; the best beam's tokens, what they should be, slots per token, pages with and without
    sharing."""
    G, n = len(prompts), len(prompts) * beams
    whole = texts([p + steps for p in prompts], torch.Generator().manual_seed(seed))
    most = max(prompts) + steps
    cache = DmcCache(LAYERS, n, HEADS, KV_HEADS, HEAD_DIM, BF16, most, LAYERS * n * KV_HEADS * (most // 32 + 1), max(prompts),
                     device=dev)

    def heads(layer, x):  # at inference the decision is the sign of k[0]
        q, k, v = model.project(layer, x)
        return q, torch.cat([k[..., :1] - OFFSET, k[..., 1:]], -1).contiguous(), v

    def words(x):
        return model.last(x).float() @ model.head.to(BF16).float().t()

    first = torch.zeros(n, VOCAB, device=dev)
    for g, m in enumerate(prompts):  # each prompt into its group's first sequence
        x = model.words[whole[g][:m].to(dev)]
        cu = torch.tensor([0, m], dtype=torch.int32, device=dev)
        places = torch.arange(m, dtype=torch.int32, device=dev)
        for layer in range(LAYERS):
            q, k, v = heads(layer, x)
            q, k = R.rotate(rotary, q, k, places)
            o = torch.empty_like(q)
            cache.prefill_attention(layer, q, k, v, cu, m, o, first_seq=g * beams)
            x = model.join(layer, x, o)
        first[g * beams] = words(x[-1:])[0]
    rows = torch.arange(n, dtype=torch.int32, device=dev)
    cache.reorder(rows // beams * beams)  # every beam continues its group's prompt
    logits = first[(rows // beams * beams).long()]
    scores = torch.full((G, beams), -math.inf, device=dev)
    scores[:, 0] = 0.0
    select = BeamSelect(G, beams, VOCAB, dtype=torch.float32, device=dev)
    place = torch.tensor(prompts, dtype=torch.int32, device=dev).repeat_interleave(beams)
    said = torch.zeros(n, 0, dtype=torch.int32, device=dev)
    for _ in range(steps):
        scores, tokens, parents, _ = select.select(logits, scores)
        parents, tokens = parents.view(-1), tokens.view(-1)
        cache.reorder(parents)
        said = torch.cat([said[parents.long()], tokens[:, None]], 1)
        x = model.words[tokens.long()]
        for layer in range(LAYERS):
            q, k, v = heads(layer, x)
            q = cache.append(layer, q, k, v, place, rotary)
            x = model.join(layer, x, cache.attend(layer, q))
        logits = words(x)
        place += 1
    status, bits, pages = cache.status()
    if status:
        raise RuntimeError(f"device fault {bits:#x}")
    counts = torch.stack([cache.lengths(layer) for layer in range(LAYERS)])
    slots = float(counts.sum()) / (LAYERS * KV_HEADS * beams * (sum(prompts) + G * steps))
    want = torch.stack([t[-steps:] for t in whole])
    return said.view(G, beams, -1)[:, 0].cpu(), want, slots, pages, int(((counts + 31) // 32).sum())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--ratio", type=float, default=3.0)
    ap.add_argument("--beams", type=int, default=4)
    a = ap.parse_args()
    dev = torch.device("cuda", torch.cuda.current_device())
    model, rotary, loss = train(a.steps, a.ratio, dev)
    said, want, slots, pages, apart = search(model, rotary, dev, a.beams)
    print(f"taught: loss {loss:.3f}")
    print(f"continued: {float((said == want).float().mean()):.1%} of the tokens repeat the phrase, slots per token {slots:.3f}, "
          f"{pages} pages of {apart}")


if __name__ == "__main__":
    main()
