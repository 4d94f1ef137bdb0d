"""What reordered sequences hold after many rounds of pages given back and taken again, against tokens kept apart (GPU).

Every token opens a slot, which is then its key (without the gate) and value as they are, with z = omega: sigmoid of a mean,
off by some 12 steps of 2^-24."""
import pytest
import torch

from generate_harness import cache_of, exported, near, tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


class Kept:
    """The tokens of each sequence, copied in whole where a sequence continues another."""

    def __init__(self, batch, hq, hkv):
        self.rows, self.G, self.H = [[] for _ in range(batch)], hq // hkv, hkv

    def append(self, q, k, v):
        k = k.clone()
        k[..., 0] = 0
        omega = torch.sigmoid(q[..., 0].double().view(len(q), self.H, self.G).mean(2))
        for s in range(len(self.rows)):
            self.rows[s].append((k[s], v[s], omega[s]))

    def reorder(self, parents):
        self.rows = [list(self.rows[p]) for p in parents]

    def check(self, cache, cap):
        k, v, z, n = exported(cache, 0, cap)
        for s, rows in enumerate(self.rows):
            for i, (got, at) in enumerate(((k, 0), (v, 1), (z, 2))):
                here = got[s * self.H:(s + 1) * self.H, :len(rows)]
                want = torch.stack([r[at] for r in rows], 1)
                if i < 2:
                    assert torch.equal(here, want), (s, i)
                else:
                    near(here, want, 12 * 2.0 ** -24 * want)
            assert n[s * self.H:(s + 1) * self.H].tolist() == [len(rows)] * self.H


@pytest.mark.parametrize("dt,heads,B", [(BF16, (2, 2), 8), (F32, (4, 1), 5), (BF16, (8, 2), 3)])
@pytest.mark.parametrize("one", [True, False])
def test_pages_that_come_back_hold_what_is_written_next(cuda_dev, dt, heads, B, one):
    """Single tokens for 400 steps, a reordering at every 20th (all continue one, or anyone) and at some others. The pool
    holds what is shared and little more, so that pages go round many times; every sequence is compared after
    each reordering and after the steps that follow it."""
    hq, hkv = heads
    g = torch.Generator().manual_seed(B)
    steps = 400
    pages = hkv * ((steps // 32 + 2) + 3 * B) if one else hkv * B * (steps // 32 + 2)
    cache, kept = cache_of(B, hq, hkv, 64, dt, steps + 1, pages=pages), Kept(B, hq, hkv)
    for i in range(steps):
        q, k, v = tokens(g, B, hq, hkv, 64, dt, 1.0)
        cache.append(0, q.cuda(), k.cuda(), v.cuda())
        kept.append(q, k, v)
        if i % 20 == 19 or i % 33 == 0:
            kept.check(cache, steps + 1)
            parents = ([int(torch.randint(0, B, (1,), generator=g))] * B if one
                       else torch.randint(0, B, (B,), generator=g).tolist())
            cache.reorder(torch.tensor(parents, dtype=torch.int32).cuda())
            kept.reorder(parents)
            kept.check(cache, steps + 1)
    kept.check(cache, steps + 1)
    assert cache.status()[:2] == (0, 0)


def test_all_copies_are_the_continued_one(cuda_dev):
    """Eight sequences of 925 tokens of which the last 600 came one by one, all continuing one of them every 20 steps, last
    after the last token: they hold the same keys, values and sums, and those are the continued one's own."""
    hkv, B, T = 2, 8, 325
    g = torch.Generator().manual_seed(7)
    pages = hkv * (11 + (B - 1) + B * 4)
    cache, kept = cache_of(B, 2, hkv, 64, BF16, 1000, pages=pages, prompt=T), Kept(B, 2, hkv)
    q, k, v = tokens(g, T, 2, hkv, 64, BF16, 1.0)
    cache.prefill(0, q[..., 0].cuda(), k.cuda(), v.cuda(), torch.tensor([0, T], dtype=torch.int32).cuda(), T)
    for t in range(T):
        kept.append(*(x[t:t + 1].expand(B, -1, -1) for x in (q, k, v)))
    cache.reorder(torch.zeros(B, dtype=torch.int32).cuda())
    for i in range(600):
        q, k, v = tokens(g, B, 2, hkv, 64, BF16, 1.0)
        cache.append(0, q.cuda(), k.cuda(), v.cuda())
        kept.append(q, k, v)
        if i % 20 == 19:
            p = int(torch.randint(0, B, (1,), generator=g))
            cache.reorder(torch.tensor([p] * B, dtype=torch.int32).cuda())
            kept.reorder([p] * B)
    kept.check(cache, 1000)
    k, v, z, n = exported(cache, 0, 1000)
    for t in (k, v, z, n):
        for i in range(1, B):
            assert torch.equal(t[:hkv], t[hkv * i:hkv * (i + 1)])
    assert cache.status()[:2] == (0, 0)
