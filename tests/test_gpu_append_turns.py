"""The turns of appended prompts' keys in fp32, against 64 bits (GPU).

A slot of one token is its key turned, times omega, over omega. A turn that is computed from its phase is off by 4 steps of
2^-24 (tests/test_gpu_rotate.py); omega's products with its cosine and sine, the two multiply-adds, the reciprocal of z and
the product with it round once each: 4 + 1 + 2 + 2 = 9 steps of (|x| + |y|) in all, 10 with their products. A slot of n
tokens adds a step for each of its sums."""
import pytest
import torch

from generate_harness import Plain, cache_of, exported, inv_freq, near, tokens
from paper_2403_09636_gb300 import rotary as R

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("window", [0, 4])
def test_every_token_has_its_own_turn(cuda_dev, D, pairs, window):
    hq, hkv, T, at = 4, 2, 517, 70001
    g = torch.Generator().manual_seed(D + pairs)
    q, k, v = tokens(g, T, hq, hkv, D, F32, 1.0)
    freq = inv_freq(D)
    cache, plain = cache_of(1, hq, hkv, D, F32, T, prompt=T, window=window), Plain(1, hq, hkv, D, F32, window)
    cache.append(0, q.cuda(), k.cuda(), v.cuda(), torch.tensor([at], dtype=torch.int32).cuda(),
                 R.Rotary(D, inv_freq=freq, interleaved=pairs), cu_seqlens=torch.tensor([0, T], dtype=torch.int32).cuda(),
                 max_seqlen=T)
    plain.append(0, q, k, v, at, freq, pairs)
    got, want = exported(cache, 0, T), plain.dense(T)
    assert torch.equal(got[3], want[3])
    x = k.clone()
    x[..., 0] = 0
    a = x.abs().double().transpose(0, 1)  # [heads, T, D]
    other = a.unflatten(-1, (-1, 2)).flip(-1).flatten(-2) if pairs else torch.cat(a.chunk(2, -1)[::-1], -1)
    near(got[0], want[0], 10 * 2.0 ** -24 * (a + other))


@pytest.mark.parametrize("pairs", [False, True])
def test_slots_of_many_tokens(cuda_dev, pairs):
    """Segments of some 30 tokens, which cross the rows' groups."""
    hq, hkv, D, T, at = 2, 2, 128, 400, 123
    g = torch.Generator().manual_seed(5)
    q, k, v = tokens(g, T, hq, hkv, D, F32, 0.03)
    freq = inv_freq(D)
    cache, plain = cache_of(1, hq, hkv, D, F32, T, prompt=T), Plain(1, hq, hkv, D, F32)
    cache.append(0, q.cuda(), k.cuda(), v.cuda(), torch.tensor([at], dtype=torch.int32).cuda(),
                 R.Rotary(D, inv_freq=freq, interleaved=pairs), cu_seqlens=torch.tensor([0, T], dtype=torch.int32).cuda(),
                 max_seqlen=T)
    plain.append(0, q, k, v, at, freq, pairs)
    got, want = exported(cache, 0, T), plain.dense(T)
    assert torch.equal(got[3], want[3])
    longest = 0
    for h in range(hkv):
        opens = (k[:, h, 0] < 0).nonzero()[:, 0].tolist() + [T]
        longest = max([longest, opens[0]] + [b - a for a, b in zip(opens, opens[1:])])
    near(got[0], want[0], (12 + longest) * 2.0 ** -24 * 2 * float(k[..., 1:].abs().max()))
