"""Offsets that pass 32 bits: rotations, caches and logits of more than 4 GB (GPU)."""
import pytest
import torch

from generate_harness import EPS, inv_freq, near, picked, turned
from paper_2403_09636_gb300 import DmcCache
from paper_2403_09636_gb300 import rotary as R
from paper_2403_09636_gb300.beam import BeamSelect

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_rotation(cuda_dev):
    T, H, D = 150_001, 128, 128  # 4.9 GB in and out
    r = R.Rotary(D, inv_freq=inv_freq(D))
    q = torch.full((T, H, D), 0.5, dtype=BF16, device=cuda_dev)
    at = torch.arange(T, dtype=torch.int32, device=cuda_dev)
    R.rotate(r, q, None, at, out=(q, None))
    for t in (0, 70_000, 140_000, T - 1):
        want = turned(torch.full((1, 1, D), 0.5), torch.tensor([t]), inv_freq(D), False)
        near(q[t, [0, H - 1]].cpu(), want[0].expand(2, D), 2.0 ** -20 + 1.01 * EPS[BF16] * want[0].abs())
    del q
    torch.cuda.empty_cache()


def test_a_cache_whose_pages_pass_4_gb(cuda_dev):
    """Tokens appended to, attended in and copied from pages beyond the pool's first 4 GB."""
    hq, hkv, D, B = 8, 8, 128, 16
    T = 40_000  # slots of each sequence and head: 20 MB a head, 2.6 GB a layer
    cache = DmcCache(2, B, hq, hkv, D, BF16, T + 40, 2 * B * hkv * (T // 32 + 3), T * B, device=cuda_dev)
    g = torch.Generator(device=cuda_dev).manual_seed(1)
    cu = torch.arange(0, B * T + 1, T, dtype=torch.int32, device=cuda_dev)
    k = torch.randn(B * T, hkv, D, generator=g, device=cuda_dev, dtype=BF16).mul_(0.5)
    v = torch.randn(B * T, hkv, D, generator=g, device=cuda_dev, dtype=BF16).mul_(0.5)
    k[..., 0] = -1.0
    q = torch.randn(B, hq, D, generator=g, device=cuda_dev, dtype=BF16)
    r = R.Rotary(D, inv_freq=inv_freq(D))
    big = torch.randn(B * T, hq, D, generator=g, device=cuda_dev, dtype=BF16)
    for layer in range(2):
        cache.append(layer, big, k, v, torch.zeros(B, dtype=torch.int32, device=cuda_dev), r, cu_seqlens=cu, max_seqlen=T)
    assert cache.status()[:2] == (0, 0) and cache.status()[2] * 16384 > 4 << 30
    cache.reorder(torch.tensor([15] + list(range(1, 16)), dtype=torch.int32, device=cuda_dev))
    at = torch.full((B,), T, dtype=torch.int32, device=cuda_dev)
    k1, v1 = k[:B].contiguous(), v[:B].contiguous()
    out = cache.attend(1, cache.append(1, q, k1, v1, at, r))
    heads = [0 * hkv + 3, 15 * hkv + 3, 14 * hkv + 7]
    ks, vs, _, ln = cache.export_heads(1, heads, T + 1)
    assert ln.tolist() == [T + 1] * 3
    assert torch.equal(ks[0, :T], ks[1, :T]) and torch.equal(vs[0, :T], vs[1, :T])
    for i, h in enumerate(heads):
        b, hh = divmod(h, hkv)
        at1 = torch.tensor([T])
        qr = turned(q[b:b + 1, hh:hh + 1].cpu(), at1, inv_freq(D), False).to(BF16).double()
        score = ks[i, :, 1:].double() @ qr[0, 0, 1:].to(cuda_dev) / D ** 0.5
        want = torch.softmax(score, 0) @ vs[i].double()
        near(out[b, hh].cpu(), want.cpu(), 2.0 ** -13 * float(vs[i].float().abs().max()) + 1.01 * EPS[BF16] * want.cpu().abs())
    del cache, k, v, big, ks, vs
    torch.cuda.empty_cache()


def test_logits(cuda_dev):
    V, B, G = 4_000_003, 4, 150  # 600 rows of 8 MB
    logits = torch.zeros(G * B, V, dtype=BF16, device=cuda_dev)
    scores = -torch.rand(G, B, generator=torch.Generator().manual_seed(2))
    words = torch.randint(0, V, (G * B, 3), generator=torch.Generator().manual_seed(3))
    words[-1, 0] = V - 1
    for i in range(3):
        logits[torch.arange(G * B), words[:, i].cuda()] = 20.0 + i
    got = BeamSelect(G, B, V, keep=6, dtype=BF16, device=cuda_dev).select(logits, scores.cuda())
    for g in (0, 70, G - 1):
        want = picked(logits[g * B:(g + 1) * B].float().cpu(), scores[g:g + 1], None, -1, 6)
        assert torch.equal(got[1][g].cpu().long(), want[1][0]) and torch.equal(got[2][g].cpu().long() - g * B, want[2][0])
        near(got[0][g].cpu(), want[0][0], 2.0 ** -18)
    del logits
    torch.cuda.empty_cache()
