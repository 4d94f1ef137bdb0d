"""The pool of pages after requests that it could not serve (GPU)."""
import pytest
import torch

import paper_2403_09636_gb300 as P
from generate_harness import cache_of, tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def prompt(cache, g, slots, seq, layer=0):
    """A text that takes `slots` slots of every head of a sequence; its keys and values."""
    c = cache.cfg
    q, k, v = (t.cuda() for t in tokens(g, slots, c.num_q_heads, c.num_kv_heads, c.head_dim, cache.dtype, 1.0))
    cache.prefill(layer, q[..., 0], k, v, torch.tensor([0, slots], dtype=torch.int32).cuda(), slots, first_seq=seq)
    return k, v


def reorder(cache, parents):
    cache.reorder(torch.tensor(parents, dtype=torch.int32).cuda())


def holds(cache, seq, k, v):
    """A slot of one token is omega k / omega: two products and a reciprocal (or a quotient), each off by 2^-24 of it at
    most; a value of bf16 comes back as it was."""
    n, H = k.shape[0], k.shape[1]
    got = cache.export_heads(0, [seq * H + h for h in range(H)], n)
    k = k.clone()
    k[..., 0] = 0
    for x, y in zip(got, (k, v)):
        y = y.transpose(0, 1).double()
        if not bool(((x.double() - y).abs() <= 4 * 2.0 ** -24 * y.abs() * (cache.dtype is F32)).all()):
            return False
    return bool((got[3] == n).all())


def test_a_prompt_that_does_not_fit_takes_nothing(cuda_dev):
    """Ten pages, six of them held: a prompt of eight is refused, and is not counted. When the six come back, all ten can
    be had."""
    g = torch.Generator().manual_seed(1)
    cache = cache_of(2, 1, 1, 64, F32, 400, pages=10, prompt=400)
    prompt(cache, g, 6 * 32, 0)
    assert cache.status() == (0, 0, 6)
    prompt(cache, g, 8 * 32, 1)
    prompt(cache, g, 5 * 32, 1)
    assert cache.status() == (P.DMC_ERR_PAGES_EXHAUSTED, P.DMC_FAULT_PAGES_EXHAUSTED, 6)
    assert cache.lengths(0)[:, 0].tolist() == [192, 0]
    reorder(cache, [1, 1])  # both empty
    assert cache.status()[2] == 0
    k, v = prompt(cache, g, 10 * 32, 0)
    assert cache.status()[2] == 10 and holds(cache, 0, k, v)


def test_single_tokens_that_find_no_page_take_nothing(cuda_dev):
    """Tokens that open slots go on while the pool is empty: what they ask for is not counted, and pages that come back are
    there for others."""
    g = torch.Generator().manual_seed(2)
    cache = cache_of(3, 2, 2, 64, BF16, 200, pages=4, prompt=200)
    prompt(cache, g, 64, 0)  # all four pages
    for _ in range(9):
        q, k, v = (t.cuda() for t in tokens(g, 3, 2, 2, 64, BF16, 1.0))
        cache.append(0, q, k, v)
        cache.decode(0, q, k, v, torch.empty_like(q))
    assert cache.status()[1:] == (P.DMC_FAULT_PAGES_EXHAUSTED, 4)
    assert cache.lengths(0).tolist() == [[64, 64], [0, 0], [0, 0]]
    reorder(cache, [1, 1, 1])
    assert cache.status()[2] == 0
    k, v = prompt(cache, g, 64, 2)
    assert cache.status()[2] == 4 and holds(cache, 2, k, v)


def test_no_page_is_lost_or_given_twice(cuda_dev):
    """Many rounds of prompts that fit and prompts that do not, on four sequences that hold pages and give them back: the
    count is that of the pages held, whatever fits is served, and every sequence keeps its own content."""
    g = torch.Generator().manual_seed(3)
    H, total = 2, 37
    cache = cache_of(4, H, H, 64, F32, 1200, pages=total, prompt=1200)
    held, texts = [0] * 4, [None] * 4
    refused = 0
    for i in range(120):
        drop = [s for s in range(4) if held[s] and float(torch.rand(1, generator=g)) < 0.4]
        free = [s for s in range(4) if not held[s]]
        if free:  # (sequences that are dropped continue an empty one)
            reorder(cache, [free[0] if s in drop else s for s in range(4)])
            for s in drop:
                held[s], texts[s] = 0, None
        else:
            reorder(cache, [0, 1, 2, 3])
        room = total - sum(held)  # (nothing is asked for after a refusal before the next reordering)
        for s in range(4):
            if held[s]:
                continue
            pages = int(torch.randint(1, 9, (1,), generator=g))
            if float(torch.rand(1, generator=g)) < 0.3:  # more than there is, for either head
                pages = room + pages
                if pages * 32 > 1200:
                    continue
                prompt(cache, g, pages * 32, s)
                refused += 1
                break
            if pages * H > room:
                continue
            texts[s], held[s] = prompt(cache, g, pages * 32, s), pages * H
            room -= held[s]
        want = [held[s] // H * 32 for s in range(4)]
        assert cache.lengths(0)[:, 0].tolist() == want, i
        assert cache.status()[2] == sum(held), i
        for s in range(4):
            assert texts[s] is None or holds(cache, s, *texts[s]), (i, s)
    assert refused >= 10
