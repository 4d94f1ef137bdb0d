"""Sequences of a cache that continue from one another's, against plain copies (GPU)."""
import pytest
import torch

import paper_2403_09636_gb300 as P
from generate_harness import EPS, Plain, cache_of, exported, near, tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def ids_of(n, parents, first, total, hkv):
    """Which head each head's content comes from."""
    src = list(range(total))
    for j, p in enumerate(parents):
        src[first + j] = first + p
    return torch.tensor([s * hkv + h for s in src for h in range(hkv)])


def same(cache, layer, cap, want):
    for got, w in zip(exported(cache, layer, cap), want):
        assert torch.equal(got, w)


def reorder(cache, parents, first=0, **kw):
    cache.reorder(torch.tensor(parents, dtype=torch.int32).cuda(), first_seq=first, **kw)


def step(cache, g, layers=1, opens=0.7):
    c = cache.cfg
    for layer in range(layers):
        x = tokens(g, c.batch, c.num_q_heads, c.num_kv_heads, c.head_dim, cache.dtype, opens)
        cache.append(layer, *(t.cuda() for t in x))


@pytest.mark.parametrize("dt,heads,D,window", [(BF16, (2, 2), 128, 0), (F32, (3, 1), 64, 0), (BF16, (8, 2), 64, 0),
                                               (BF16, (2, 2), 64, 7), (F32, (2, 2), 128, 32)])
def test_any_parents_between_steps(cuda_dev, dt, heads, D, window):
    """Random parents and single tokens in turn, over page borders: after each, every slot is a plain copy's, bit for
    bit, and a cache that was never reordered but holds the same gives the same from then on."""
    B, layers, steps = 6, 2, 110
    g = torch.Generator().manual_seed(3)
    cache = cache_of(B, *heads, D, dt, steps + 2, layers=layers, window=window)
    for i in range(steps):
        step(cache, g, layers, 0.85)
        if i % 3 == 0:
            before = [exported(cache, layer, steps + 2) for layer in range(layers)]
            kind = i // 3 % 4
            if kind == 0:
                parents = torch.randint(0, B, (B,), generator=g).tolist()
            elif kind == 1:
                parents = torch.randperm(B, generator=g).tolist()
            elif kind == 2:
                parents = [int(torch.randint(0, B, (1,), generator=g))] * B
            else:
                parents = [p if p != 2 else 0 for p in range(B)]
            reorder(cache, parents)
            src = ids_of(B, parents, 0, B, heads[1])
            for layer in range(layers):
                same(cache, layer, steps + 2, [t[src] for t in before[layer]])
    assert cache.status()[:2] == (0, 0)


def test_copies_go_their_own_ways(cuda_dev):
    """Four continuations of one prompt, each with tokens of its own, merges into the shared last slot among them: against
    plain copies."""
    hq, hkv, D, dt = 4, 2, 64, F32
    g = torch.Generator().manual_seed(5)
    T, n = 95, 4
    cache, plain = cache_of(n, hq, hkv, D, dt, T + 50, prompt=T), Plain(n, hq, hkv, D, dt)
    q, k, v = tokens(g, T, hq, hkv, D, dt, 0.7)
    cu = torch.tensor([0, T], dtype=torch.int32).cuda()
    cache.prefill(0, q[..., 0].cuda(), k.cuda(), v.cuda(), cu, T, first_seq=1)
    plain.append(1, q, k, v)
    reorder(cache, [1, 1, 1, 1])
    plain.reorder([1, 1, 1, 1])
    for i in range(40):
        q, k, v = tokens(g, n, hq, hkv, D, dt, 0.5)
        cache.append(0, q.cuda(), k.cuda(), v.cuda())
        for s in range(n):
            plain.append(s, q[s:s + 1], k[s:s + 1], v[s:s + 1])
        if i % 7 == 6:
            parents = torch.randint(0, n, (n,), generator=g).tolist()
            reorder(cache, parents)
            plain.reorder(parents)
    got, want = exported(cache, 0, T + 50), plain.dense(T + 50)
    assert torch.equal(got[3], want[3])
    for a, b in zip(got[:3], want[:3]):
        near(a, b, 512 * 2.0 ** -24 * b.abs().max())
    out = cache.attend(0, q.cuda())
    w, size = plain.attend(q)
    near(out.cpu(), w, 2.0 ** -12 * size[..., None])


def test_a_long_prompt_continues_on_every_copy(cuda_dev):
    """Prompts in parts after a reordering: a continued prompt writes its own pages alone."""
    hq, hkv, D, dt, T = 2, 2, 128, BF16, 200
    g = torch.Generator().manual_seed(6)
    cache = cache_of(3, hq, hkv, D, dt, 3 * T, prompt=3 * T)
    plain = Plain(3, hq, hkv, D, dt)
    cu = torch.tensor([0, T, 2 * T, 3 * T], dtype=torch.int32).cuda()
    for i in range(2):
        q, k, v = tokens(g, 3 * T, hq, hkv, D, dt, 0.5)
        cache.prefill(0, q[..., 0].cuda(), k.cuda(), v.cuda(), cu, T)
        for s in range(3):
            plain.append(s, *(t[s * T:(s + 1) * T] for t in (q, k, v)))
        if i == 0:
            reorder(cache, [2, 1, 2])
            plain.reorder([2, 1, 2])
    got, want = exported(cache, 0, 3 * T), plain.dense(3 * T)
    assert torch.equal(got[3], want[3])
    for a, b in zip(got[:2], want[:2]):
        near(a, b, 4 * EPS[dt] * b.abs().max())


def distinct_pages(cap_pages, lengths):
    return int(((lengths + 31) // 32).sum())


def test_pages_are_shared_and_come_back(cuda_dev):
    """Eight copies of a prompt hold its pages once (and a last page each); when one of them is continued by all, the
    pages of the others come back, and the pool, which holds less than eight prompts, never runs out."""
    hkv, D, B, T = 2, 64, 8, 32 * 10 + 5
    g = torch.Generator().manual_seed(7)
    pages = hkv * (11 + (B - 1) + B * 4)  # the prompt, last pages, four pages for each sequence beyond them
    cache = cache_of(B, 2, hkv, D, BF16, T + 3000, pages=pages, prompt=T)
    q, k, v = (t.cuda() for t in tokens(g, T, 2, hkv, D, BF16, 1.0))
    cache.prefill(0, q[..., 0], k, v, torch.tensor([0, T], dtype=torch.int32).cuda(), T)
    assert cache.status() == (0, 0, hkv * 11)
    reorder(cache, [0] * B)
    assert cache.status() == (0, 0, hkv * (11 + B - 1))
    n = T
    for i in range(600):
        step(cache, g, opens=1.0)
        n += 1
        if i % 20 == 19:
            p = int(torch.randint(0, B, (1,), generator=g))
            reorder(cache, [p] * B)
            st, bits, used = cache.status()
            assert (st, bits) == (0, 0)
            if n % 32:
                assert used == hkv * ((n - 1) // 32 + B), (i, used)
    assert torch.equal(cache.lengths(0).cpu(), torch.full((B, hkv), n, dtype=torch.int32))
    k, v, z, ln = exported(cache, 0, n)  # every copy holds what the last continued one holds
    for i in range(1, B):
        assert torch.equal(k[:hkv], k[hkv * i:hkv * (i + 1)]) or n % 20
    cache.reset()
    assert cache.status() == (0, 0, 0)
    step(cache, g)
    assert cache.status() == (0, 0, B * hkv)


def test_emptied_after_sharing(cuda_dev):
    """A cache that is emptied while its sequences share pages begins anew: the same steps give the same, over and over."""
    cache = cache_of(4, 2, 2, 64, F32, 200, prompt=200, pages=40)
    first = None
    for _ in range(3):
        g = torch.Generator().manual_seed(14)
        q, k, v = (t.cuda() for t in tokens(g, 100, 2, 2, 64, F32, 0.9))
        cache.prefill(0, q[..., 0], k, v, torch.tensor([0, 100], dtype=torch.int32).cuda(), 100)
        reorder(cache, [0] * 4)
        for i in range(60):
            step(cache, g, opens=0.8)
            if i % 9 == 8:
                reorder(cache, torch.randint(0, 4, (4,), generator=g).tolist())
        assert cache.status()[:2] == (0, 0)
        got = exported(cache, 0, 200)
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))
        cache.reset()


def test_sequences_outside_the_call_stay(cuda_dev):
    cache = cache_of(7, 2, 2, 64, BF16, 80, layers=2)
    g = torch.Generator().manual_seed(8)
    for _ in range(40):
        step(cache, g, 2)
    before = [exported(cache, layer, 80) for layer in range(2)]
    reorder(cache, [1, 1, 0], first=3)
    src = ids_of(3, [1, 1, 0], 3, 7, 2)
    for layer in range(2):
        same(cache, layer, 80, [t[src] for t in before[layer]])
    # and a second call that reaches into the first one's sequences
    before = [exported(cache, layer, 80) for layer in range(2)]
    reorder(cache, [3, 0, 0, 1], first=2)
    src = ids_of(4, [3, 0, 0, 1], 2, 7, 2)
    for layer in range(2):
        same(cache, layer, 80, [t[src] for t in before[layer]])


def test_empty_sequences(cuda_dev):
    """Copies of empty sequences are empty and give their pages back; copies into empty ones take pages of the pool."""
    cache = cache_of(4, 2, 1, 64, F32, 100, prompt=100)
    g = torch.Generator().manual_seed(9)
    q, k, v = (t.cuda() for t in tokens(g, 70, 2, 1, 64, F32, 1.0))
    cache.prefill(0, q[..., 0], k, v, torch.tensor([0, 70], dtype=torch.int32).cuda(), 70, first_seq=2)
    assert cache.status() == (0, 0, 3)
    reorder(cache, [0, 2, 3, 2])
    assert cache.lengths(0)[:, 0].tolist() == [0, 70, 0, 70]
    assert cache.status() == (0, 0, 4)
    reorder(cache, [0, 0, 0, 0])
    assert cache.lengths(0)[:, 0].tolist() == [0, 0, 0, 0]
    assert cache.status() == (0, 0, 0)


def test_no_page_left_for_a_copy(cuda_dev):
    cache = cache_of(2, 1, 1, 64, BF16, 64, pages=1)
    g = torch.Generator().manual_seed(10)
    x = [t.cuda() for t in tokens(g, 1, 1, 1, 64, BF16, 1.0)]
    cache.append(0, *x, first_seq=0)
    reorder(cache, [0, 0])
    st, bits, _ = cache.status()
    assert st == P.DMC_ERR_PAGES_EXHAUSTED and bits == P.DMC_FAULT_PAGES_EXHAUSTED
    assert cache.lengths(0)[:, 0].tolist() == [1, 0]


def test_parents_outside_the_call(cuda_dev):
    cache = cache_of(3, 1, 1, 64, BF16, 64)
    g = torch.Generator().manual_seed(11)
    for _ in range(3):
        step(cache, g)
    before = exported(cache, 0, 8)
    reorder(cache, [3, -1, 0])
    assert cache.status()[1] == P.DMC_FAULT_BAD_PARENT
    same(cache, 0, 8, [t[torch.tensor([0, 1, 0])] for t in before])


def test_the_most_sequences_of_a_call(cuda_dev):
    B = 512
    cache = cache_of(B, 1, 1, 64, BF16, 100, window=3)
    g = torch.Generator().manual_seed(12)
    for i in range(70):
        step(cache, g, opens=0.9)
        if i % 23 == 22:
            before = exported(cache, 0, 100)
            parents = torch.randint(0, B, (B,), generator=g).tolist()
            reorder(cache, parents)
            same(cache, 0, 100, [t[torch.tensor(parents)] for t in before])
    assert cache.status()[:2] == (0, 0)


def test_captured_and_replayed(cuda_dev):
    """A graph of a step and a reordering with parents that the program changes."""
    hq, hkv, D, B = 2, 2, 64, 3
    g = torch.Generator().manual_seed(13)
    cache, plain = cache_of(B, hq, hkv, D, F32, 60), Plain(B, hq, hkv, D, F32)
    q, k, v = (t.cuda() for t in tokens(g, B, hq, hkv, D, F32))
    parents = torch.zeros(B, dtype=torch.int32).cuda()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.append(0, q, k, v)
        cache.reorder(parents)
    for _ in range(50):
        x = tokens(g, B, hq, hkv, D, F32, 0.9)
        p = torch.randint(0, B, (B,), generator=g)
        for to, t in zip((q, k, v, parents), (*x, p.to(torch.int32))):
            to.copy_(t)
        graph.replay()
        for s in range(B):
            plain.append(s, *(t[s:s + 1] for t in x))
        plain.reorder(p.tolist())
    torch.cuda.synchronize()
    got, want = exported(cache, 0, 60), plain.dense(60)
    assert torch.equal(got[3], want[3])
    for a, b in zip(got[:3], want[:3]):
        near(a, b, 512 * 2.0 ** -24 * b.abs().max())


def test_refusals(cuda_dev):
    cache = cache_of(3, 1, 1, 64, BF16, 64)
    ok = torch.zeros(3, dtype=torch.int32).cuda()
    for bad in (ok.long(), ok.cpu(), ok.float(), torch.zeros(6, dtype=torch.int32).cuda()[::2], [0, 0, 0]):
        with pytest.raises(ValueError):
            cache.reorder(bad)
    for first in (-1, 1):
        with pytest.raises(P.DmcError):
            cache.reorder(ok, first_seq=first)
    many = cache_of(600, 1, 1, 64, BF16, 32)
    with pytest.raises(P.DmcError):
        many.reorder(torch.zeros(513, dtype=torch.int32).cuda())
    cache.reorder(ok[:0])
    assert cache.status() == (0, 0, 0)
