"""A whole generation: a small model with rotary positions taught nothing, whose prompt is attended and compressed, and
whose continuation is searched with beams over the compressed caches, against the same in 64 bits with plain copies (GPU).

The model: two layers of attention (grouped queries) with a residual, fp32, random weights; tokens and beams of every step
are compared as whole numbers, so the weights are drawn such that the best scores lie apart; scores at the end within
2^-10 (about 600 roundings of 2^-24 of numbers up to 40 in a row)."""
import math

import pytest
import torch

from generate_harness import Plain, inv_freq, near, picked, turned
from paper_2403_09636_gb300 import DmcCache
from paper_2403_09636_gb300 import rotary as R
from paper_2403_09636_gb300.beam import BeamSelect

pytestmark = pytest.mark.gpu
F32 = torch.float32
LAYERS, HQ, H, D, V, E = 2, 4, 2, 64, 97, 48


class Model:
    def __init__(self, seed, dtype, device):
        g = torch.Generator().manual_seed(seed)
        def w(*shape):
            return (torch.randn(*shape, generator=g) / math.sqrt(shape[0])).to(device=device, dtype=dtype)
        self.embed = torch.randn(V, E, generator=g).to(device=device, dtype=dtype)
        self.qkv = [(w(E, HQ * D), w(E, H * D), w(E, H * D)) for _ in range(LAYERS)]
        self.out = [w(HQ * D, E) for _ in range(LAYERS)]
        self.head = 3.0 * w(E, V)

    def heads(self, layer, x):
        q, k, v = (x @ w for w in self.qkv[layer])
        return q.view(-1, HQ, D), k.view(-1, H, D), v.view(-1, H, D)


def plain_prompt(m, cache, rows, tokens, freq, pairs):
    """Token by token, as decoding."""
    for t, token in enumerate(tokens):
        x = m.embed[token][None]
        for layer in range(LAYERS):
            q, k, v = m.heads(layer, x)
            qr = cache[layer].append(rows, q, k, v, t, freq, pairs)
            whole = torch.zeros(len(cache[layer].heads), HQ, D, dtype=torch.float64)
            whole[rows] = qr[0]
            x = x + cache[layer].attend(whole)[0][rows].reshape(1, -1) @ m.out[layer]
    return x @ m.head


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("group,beams", [(2, 3), (1, 5)])
def test_beam_search_over_compressed_caches(cuda_dev, pairs, group, beams):
    steps, eos, n = 40, 5, group * beams
    freq = inv_freq(D)
    m, ref = Model(3, F32, cuda_dev), Model(3, torch.float64, "cpu")
    g = torch.Generator().manual_seed(group)
    lens = [23 + 40 * i for i in range(group)]
    prompts = [torch.randint(0, V, (t,), generator=g) for t in lens]
    rotary = R.Rotary(D, inv_freq=freq, interleaved=pairs)
    pages = LAYERS * n * H * 5
    cache = DmcCache(LAYERS, n, HQ, H, D, F32, 200, pages, sum(lens), device=cuda_dev)
    plain = [Plain(n, HQ, H, D, F32) for _ in range(LAYERS)]

    # the prompt, one token after the other (its layers need each token's attention): all groups' first beams
    logits = torch.zeros(n, V, device=cuda_dev)
    want_logits = torch.zeros(n, V, dtype=torch.float64)
    for i, p in enumerate(prompts):
        row = i * beams
        for t in range(lens[i]):
            x = m.embed[p[t]][None]
            at = torch.tensor([t], dtype=torch.int32, device=cuda_dev)
            for layer in range(LAYERS):
                q, k, v = (y.contiguous() for y in m.heads(layer, x))
                qr = cache.append(layer, q, k, v, at, rotary, first_seq=row)
                whole = torch.zeros(n, HQ, D, device=cuda_dev)
                whole[row] = qr[0]
                x = x + cache.attend(layer, whole)[row].reshape(1, -1) @ m.out[layer]
        logits[row] = (x @ m.head)[0]
        want_logits[row] = plain_prompt(ref, plain, row, p, freq, pairs)[0]
    near(logits.cpu(), want_logits, 2.0 ** -12 * want_logits.abs().max())

    # every beam continues its group's first one
    start = torch.arange(n, dtype=torch.int32, device=cuda_dev) // beams * beams
    cache.reorder(start)
    for p in plain:
        p.reorder(start.tolist())
    logits, want_logits = logits[start.long()].contiguous(), want_logits[start.cpu().long()]
    scores = torch.full((group, beams), -math.inf)
    scores[:, 0] = 0.0
    done = torch.zeros(group, beams, dtype=torch.bool)
    want = [scores.double(), None, None, done]
    scores, done = scores.to(cuda_dev), done.to(cuda_dev)
    position = torch.tensor(lens).repeat_interleave(beams)
    select = BeamSelect(group, beams, V, dtype=F32, device=cuda_dev)
    for step in range(steps):
        scores, tokens, parents, done = select.select(logits, scores, done, eos)
        want = picked(want_logits, want[0], want[3], eos, beams)
        assert torch.equal(tokens.cpu().long(), want[1]), step
        assert torch.equal(parents.cpu().long(), want[2]), step
        assert torch.equal(done.cpu(), want[3]), step
        cache.reorder(parents.view(-1))
        for p in plain:
            p.reorder(want[2].view(-1).tolist())
        x, y = m.embed[tokens.view(-1).long()], ref.embed[want[1].view(-1)]
        at = position.to(torch.int32).to(cuda_dev)
        for layer in range(LAYERS):
            q, k, v = (t.contiguous() for t in m.heads(layer, x))
            x = x + cache.attend(layer, cache.append(layer, q, k, v, at, rotary)).view(n, -1) @ m.out[layer]
            q, k, v = ref.heads(layer, y)
            qr = torch.stack([plain[layer].append(i, q[i:i + 1], k[i:i + 1], v[i:i + 1], int(position[i]), freq, pairs)[0]
                              for i in range(n)])
            y = y + plain[layer].attend(qr)[0].view(n, -1) @ ref.out[layer]
        logits, want_logits = x @ m.head, y @ ref.head
        position += 1
    near(scores.cpu(), want[0], 2.0 ** -10)
    assert cache.status()[:2] == (0, 0)
    slots = sum(int(cache.lengths(layer).sum()) for layer in range(LAYERS))
    assert slots == sum(int(p.dense(200)[3].sum()) for p in plain)


def test_prompt_attention_reads_what_rotation_and_append_leave(cuda_dev):
    """A prompt in one go: rotated queries and keys through prompt attention fill a cache and attend; appending the raw
    ones fills another alike; the next token, appended and attended, gives the same from both, and the outputs are those
    of the rotated model in 64 bits."""
    hq, hkv, Dh, T, bf = 8, 2, 128, 300, torch.bfloat16
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(T, n, Dh, generator=g).mul_(0.5).to(bf) for n in (hq, hkv, hkv))
    freq = inv_freq(Dh)
    rotary = R.Rotary(Dh, inv_freq=freq)
    at = torch.arange(T, dtype=torch.int32, device=cuda_dev) + 1000
    qr, kr = R.rotate(rotary, q.cuda(), k.cuda(), at)
    cu = torch.tensor([0, T], dtype=torch.int32, device=cuda_dev)
    a, b = (DmcCache(1, 1, hq, hkv, Dh, bf, T + 2, 40, T, device=cuda_dev) for _ in range(2))
    out = torch.empty_like(qr)
    a.prefill_attention(0, qr, kr, v.cuda(), cu, T, out)
    got = b.append(0, q.cuda(), k.cuda(), v.cuda(), at[:1].contiguous(), rotary, cu_seqlens=cu, max_seqlen=T)
    assert torch.equal(got, qr)
    ids = list(range(hkv))
    x, y = a.export_heads(0, ids, T), b.export_heads(0, ids, T)
    assert torch.equal(x[3], y[3])
    # a's keys were rounded once more, before they were merged
    near(x[0].cpu(), y[0].cpu().double(), 3 * 2.0 ** -8 * float(kr.float().abs().max()))
    near(x[1].cpu(), y[1].cpu().double(), 2 * 2.0 ** -8 * float(v.float().abs().max()))
    plain = Plain(1, hq, hkv, Dh, F32)
    worst = 0.0
    for t in range(T):
        w = plain.append(0, q[t:t + 1], k[t:t + 1], v[t:t + 1], 1000 + t, freq)
        o, size = plain.attend(w)
        worst = max(worst, float((out[t].cpu().double() - o[0]).abs().max()))
    assert worst <= 2e-2  # bf16 slots, keys and weights: as the tests of prompt attention
    q1, k1, v1 = (torch.randn(1, n, Dh, generator=g).to(bf) for n in (hq, hkv, hkv))
    p = torch.tensor([1000 + T], dtype=torch.int32, device=cuda_dev)
    outs = [c.attend(0, c.append(0, q1.cuda(), k1.cuda(), v1.cuda(), p, rotary)) for c in (a, b)]
    near(outs[0].cpu(), outs[1].cpu().double(), 2e-2)
    w = plain.append(0, q1, k1, v1, 1000 + T, freq)
    near(outs[1].cpu(), plain.attend(w)[0], 2e-2)


def test_a_step_in_one_graph(cuda_dev):
    """Selection, reordering, appending and attending of one step captured together and replayed, positions moved on by
    the graph itself: as the same steps called one by one."""
    G, B, hq, hkv, Dh, bf, vocab = 2, 3, 4, 4, 64, torch.bfloat16, 50
    n = G * B
    g = torch.Generator().manual_seed(11)
    table = torch.randn(vocab, 3, hq, Dh, generator=g).to(bf).cuda()
    head = torch.randn(hq * Dh, vocab, generator=g).to(bf).cuda() * 0.3
    rotary = R.Rotary(Dh)

    def make():
        return dict(cache=DmcCache(1, n, hq, hkv, Dh, bf, 80, n * hkv * 4, 0, device=cuda_dev),
                    select=BeamSelect(G, B, vocab, dtype=bf, device=cuda_dev),
                    logits=torch.randn(n, vocab, generator=torch.Generator().manual_seed(5)).to(bf).cuda(),
                    scores=torch.zeros(G, B, device=cuda_dev), done=torch.zeros(G, B, dtype=torch.bool, device=cuda_dev),
                    tokens=torch.zeros(G, B, dtype=torch.int32, device=cuda_dev),
                    parents=torch.zeros(G, B, dtype=torch.int32, device=cuda_dev),
                    at=torch.zeros(n, dtype=torch.int32, device=cuda_dev))

    def step(s):
        s["select"].select(s["logits"], s["scores"], s["done"], 7, out=(s["scores"], s["tokens"], s["parents"], s["done"]))
        s["cache"].reorder(s["parents"].view(-1))
        q, k, v = table[s["tokens"].view(-1).long()].unbind(1)
        qr = s["cache"].append(0, q.contiguous(), k.contiguous(), v.contiguous(), s["at"], rotary)
        s["logits"].copy_(s["cache"].attend(0, qr).view(n, -1) @ head)
        s["at"].add_(1)

    a, b = make(), make()
    step(a)
    step(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for _ in range(60):
        step(a)
        graph.replay()
    torch.cuda.synchronize()
    for name in ("scores", "tokens", "parents", "done", "logits", "at"):
        assert torch.equal(a[name], b[name]), name
    assert a["cache"].status()[:2] == (0, 0) and b["cache"].status()[:2] == (0, 0)
    ids = list(range(n * hkv))
    for x, y in zip(a["cache"].export_heads(0, ids, 80), b["cache"].export_heads(0, ids, 80)):
        assert torch.equal(x, y)
