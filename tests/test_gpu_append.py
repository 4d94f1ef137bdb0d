"""Appending to the cache with the rotation on the way, against 64 bits (GPU).

Bounds, for segments of up to 128 tokens. Keys: a token's turn is off by 4 steps of 2^-24 at its group's start and by 3 more
for each of up to 31 tokens after it, omega by 12, sums by a step for each token: 256 2^-24 of the largest value in
all; with each call the slot is rounded to its type, and a value near a border may be rounded to the other side, one step
(two EPS), which later calls only make smaller: so 2 EPS of the largest value for each call. z: 12 and a step for each
token, 160 2^-24 of it."""
import pytest
import torch

import paper_2403_09636_gb300 as P
from generate_harness import EPS, Plain, cache_of, exported, inv_freq, near, tokens, turned
from paper_2403_09636_gb300 import rotary as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def compare(cache, layer, plain, cap, calls, top):
    k, v, z, ln = exported(cache, layer, cap)
    wk, wv, wz, wl = plain.dense(cap)
    assert torch.equal(ln, wl)
    for got, want in ((k, wk), (v, wv)):
        near(got, want, top * (256 * 2.0 ** -24 + (2 * EPS[plain.dt] * calls if plain.dt == BF16 else 0)))
    near(z, wz, 160 * 2.0 ** -24 * wz)
    assert bool((k[..., 0] == 0).all())


def run(cuda_dev, hq, hkv, D, dt, pairs, prompts, steps, opens, window=0, layers=1, far=70000):
    """Prompts (a list of calls, each a list of the sequences' token counts), then single tokens."""
    g = torch.Generator().manual_seed(hash((hq, hkv, D, pairs, steps, window)) % 2 ** 31)
    n = len(prompts[0]) if prompts else 3
    most = sum(max(p) for p in prompts) + steps + 1
    cache = cache_of(n, hq, hkv, D, dt, most, layers=layers, prompt=max([sum(p) for p in prompts] + [0]), window=window)
    plain = Plain(n, hq, hkv, D, dt, window)
    freq = inv_freq(D)
    r = R.Rotary(D, inv_freq=freq, interleaved=pairs)
    at = [int(x) for x in torch.randint(0, far, (n,), generator=g)]
    calls, top, layer = 0, 0.0, layers - 1
    for lens in prompts + [[1] * n] * steps:
        T = sum(lens)
        q, k, v = tokens(g, T, hq, hkv, D, dt, opens)
        top = max(top, float(k[..., 1:].abs().max()) * 1.5, float(v.abs().max()))
        pos = torch.tensor(at, dtype=torch.int32).cuda()
        dev = [t.cuda() for t in (q, k, v)]
        if lens == [1] * n:
            qr = cache.append(layer, *dev, pos, r)
        else:
            cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
            qr = cache.append(layer, *dev, pos, r, cu_seqlens=cu, max_seqlen=max(lens))
        b = 0
        for i, m in enumerate(lens):
            if m:
                want = plain.append(i, q[b:b + m], k[b:b + m], v[b:b + m], at[i], freq, pairs)
                x = q[b:b + m].double().abs()
                near(qr[b:b + m].cpu(), want, 8 * 2.0 ** -24 * (x + x.amax(-1, keepdim=True)) + 1.01 * EPS[dt] * want.abs())
            b, at[i] = b + m, at[i] + m
        calls += 1
    compare(cache, layer, plain, most, calls, top)
    assert cache.status()[:2] == (0, 0)
    return cache, plain


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("heads", [(2, 2), (6, 2), (32, 1)])
def test_single_tokens(cuda_dev, dt, D, pairs, heads):
    run(cuda_dev, *heads, D, dt, pairs, [], 37, 0.9)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("opens", [0.03, 0.4, 1.0])
def test_prompts_then_tokens(cuda_dev, dt, D, pairs, opens):
    """Ragged prompts, empty ones among them, in two calls (the second continues open segments), then single tokens."""
    run(cuda_dev, 4, 2, D, dt, pairs, [[1, 130, 0, 259], [33, 0, 2, 128]], 3, opens)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("window", [1, 3, 12, 32])
def test_windows(cuda_dev, dt, pairs, window):
    run(cuda_dev, 2, 2, 64, dt, pairs, [[60, 7], [5, 40]], 5, 0.1, window=window)


def test_all_tokens_in_one_slot(cuda_dev):
    """No token but the first opens: one segment of a prompt that ends inside its second chunk, and steps."""
    run(cuda_dev, 2, 1, 128, F32, False, [[127]], 2, 0.0)


def test_another_layer_and_some_sequences(cuda_dev):
    """A call writes its layer and its sequences alone."""
    hq, hkv, D, dt = 4, 2, 64, BF16
    cache = cache_of(5, hq, hkv, D, dt, 40, layers=3)
    g = torch.Generator().manual_seed(1)
    q, k, v = (t.cuda() for t in tokens(g, 2, hq, hkv, D, dt, 1.0))
    at = torch.tensor([4, 9], dtype=torch.int32).cuda()
    cache.append(1, q, k, v, at, R.Rotary(D), first_seq=2)
    for layer in range(3):
        n = cache.lengths(layer).cpu()
        want = torch.zeros(5, hkv, dtype=torch.int32)
        if layer == 1:
            want[2:4] = 1
        assert torch.equal(n, want)


def test_tokens_for_some_by_cu_seqlens(cuda_dev):
    """max_seqlen 1 with sequences that have no token in this call: rows of others are left as they are."""
    hq, hkv, D, dt = 2, 1, 64, F32
    cache = cache_of(4, hq, hkv, D, dt, 8)
    g = torch.Generator().manual_seed(2)
    q, k, v = tokens(g, 2, hq, hkv, D, dt, 1.0)
    cu = torch.tensor([0, 0, 1, 1, 2], dtype=torch.int32).cuda()
    at = torch.tensor([7, 8, 9, 10], dtype=torch.int32).cuda()
    out = torch.full((2, hq, D), 5.0).cuda()
    qr = cache.append(0, q.cuda(), k.cuda(), v.cuda(), at, R.Rotary(D), cu_seqlens=cu, max_seqlen=1, q_out=out)
    assert qr is out
    assert cache.lengths(0)[:, 0].tolist() == [0, 1, 0, 1]
    want = turned(q, torch.tensor([8, 10]), inv_freq(D), False)
    near(qr.cpu(), want, 16 * 2.0 ** -24 * q.abs().max().double())


@pytest.mark.parametrize("G", [1, 2])
def test_rows_of_no_sequence_are_left_as_they_are(cuda_dev, G):
    """cu_seqlens that end before the tokens do: queries behind the last sequence are not rotated, keys join nothing."""
    hq, hkv, D, dt, T = 2 * G, 2, 128, BF16, 300
    cache, plain = cache_of(3, hq, hkv, D, dt, T, prompt=T), Plain(3, hq, hkv, D, dt)
    g = torch.Generator().manual_seed(9)
    q, k, v = tokens(g, T, hq, hkv, D, dt, 0.5)
    cu = torch.tensor([0, 100, 100, 260], dtype=torch.int32).cuda()
    at = torch.tensor([5, 6, 7], dtype=torch.int32).cuda()
    out = torch.full((T, hq, D), 3.0, dtype=dt).cuda()
    freq = inv_freq(D)
    cache.append(0, q.cuda(), k.cuda(), v.cuda(), at, R.Rotary(D, inv_freq=freq), cu_seqlens=cu, max_seqlen=160, q_out=out)
    assert bool((out[260:] == 3.0).all()) and not bool((out[:260] == 3.0).all())
    plain.append(0, q[:100], k[:100], v[:100], 5, freq)
    plain.append(2, q[100:260], k[100:260], v[100:260], 7, freq)
    compare(cache, 0, plain, T, 1, 4.0)
    assert cache.status()[:2] == (0, 0)


def test_sequences_that_contradict_one_another(cuda_dev):
    """cu_seqlens that go back or begin late: the fault bit, and the caches of sequences that are whole."""
    hq, hkv, D, dt, T = 2, 2, 128, BF16, 300
    g = torch.Generator().manual_seed(10)
    q, k, v = (t.cuda() for t in tokens(g, T, hq, hkv, D, dt, 0.5))
    at = torch.zeros(3, dtype=torch.int32).cuda()
    for cu in ([0, 200, 100, 300], [40, 90, 200, 300], [0, 100, 200, 301], [-9, 100, 200, 300]):
        cache = cache_of(3, hq, hkv, D, dt, T, prompt=T)
        cache.append(0, q, k, v, at, R.Rotary(D), cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), max_seqlen=200)
        faulty = cu[2] < cu[1] or cu[0] < 0 or cu[3] > T
        assert cache.status()[1] == (P.DMC_FAULT_BAD_SEQLENS if faulty else 0), cu
        assert int(cache.lengths(0).max()) <= T


@pytest.mark.parametrize("T", [1, 70])
def test_in_place_queries_and_no_rotation(cuda_dev, T):
    hq, hkv, D, dt = 4, 4, 128, BF16
    g = torch.Generator().manual_seed(3)
    q, k, v = (t.cuda() for t in tokens(g, 2 * T, hq, hkv, D, dt, 0.5))
    cu = torch.tensor([0, T, 2 * T], dtype=torch.int32).cuda()
    at = torch.tensor([0, 100], dtype=torch.int32).cuda()
    r = R.Rotary(D)
    a, b, c = (cache_of(2, hq, hkv, D, dt, T + 2, prompt=2 * T) for _ in range(3))
    want = a.append(0, q, k, v, at, r, cu_seqlens=cu, max_seqlen=T)
    same = q.clone()
    assert b.append(0, same, k, v, at, r, cu_seqlens=cu, max_seqlen=T, q_out=same) is same
    assert torch.equal(want, same)
    assert all(torch.equal(x, y) for x, y in zip(exported(a, 0, T), exported(b, 0, T)))
    # without a rotation: as the calls that were there
    assert c.append(0, q, k, v, cu_seqlens=cu, max_seqlen=T) is None
    d = cache_of(2, hq, hkv, D, dt, T + 2, prompt=2 * T)
    d.prefill(0, q[..., 0], k, v, cu, T)
    for x, y in zip(exported(c, 0, T), exported(d, 0, T)):
        near(x, y.double(), 2.0 ** -20 * y.double().abs() + (0 if T > 1 else 2.0 ** -20))


def test_follows_decoding_and_is_followed_by_it(cuda_dev):
    """append and dmc_decode_step on one cache in turn: the same slots as by either alone."""
    hq, hkv, D, dt = 4, 2, 64, F32
    g = torch.Generator().manual_seed(4)
    a, b = cache_of(3, hq, hkv, D, dt, 70), cache_of(3, hq, hkv, D, dt, 70)
    for i in range(66):
        q, k, v = (t.cuda() for t in tokens(g, 3, hq, hkv, D, dt, 0.8))
        b.decode(0, q, k, v, torch.empty_like(q))
        if i % 3:
            a.append(0, q, k, v)
        else:
            a.decode(0, q, k, v, torch.empty_like(q))
    x, y = exported(a, 0, 70), exported(b, 0, 70)
    assert torch.equal(x[3], y[3])
    for s, t in zip(x[:3], y[:3]):
        near(s, t.double(), 64 * 2.0 ** -24 * t.double().abs().max())


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T", [1, 40])
def test_gates_of_any_size(cuda_dev, pairs, T):
    """Infinite gates decide and weigh, and reach nothing else: neither their partners nor the slots' first dimension."""
    hq, hkv, D, dt = 2, 2, 64, F32
    g = torch.Generator().manual_seed(8)
    q, k, v = tokens(g, T, hq, hkv, D, dt, 0.5)
    k[:, 0, 0], k[:, 1, 0] = float("inf"), float("-inf")  # one segment; a slot for each
    q[:, :, 0] = float("inf")  # omega 1
    cache, plain = cache_of(1, hq, hkv, D, dt, T + 1, prompt=T), Plain(1, hq, hkv, D, dt)
    at = torch.tensor([11], dtype=torch.int32).cuda()
    cu = torch.tensor([0, T], dtype=torch.int32).cuda()
    freq = inv_freq(D)
    qr = cache.append(0, q.cuda(), k.cuda(), v.cuda(), at, R.Rotary(D, inv_freq=freq, interleaved=pairs), cu_seqlens=cu,
                      max_seqlen=T).cpu()
    partner = 1 if pairs else D // 2
    assert torch.equal(qr[..., 0], q[..., 0]) and torch.equal(qr[..., partner], q[..., partner])
    assert bool(torch.isfinite(qr[..., 1:]).all())
    kz = k.clone()
    kz[..., 0] = torch.where(k[..., 0] < 0, -1.0, 1.0)
    q[:, :, 0] = 100.0  # omega 1 in 64 bits, too
    plain.append(0, q, kz, v, 11, freq, pairs)
    compare(cache, 0, plain, T + 1, 1, 4.0)


def test_faults_of_the_device(cuda_dev):
    """A gate that is not a number, a full head, an empty pool, bad cu_seqlens: a bit each, and nothing out of place."""
    hq, hkv, D, dt = 2, 2, 64, BF16
    g = torch.Generator().manual_seed(5)
    r = R.Rotary(D)
    at = torch.zeros(1, dtype=torch.int32).cuda()
    q, k, v = (t.cuda() for t in tokens(g, 1, hq, hkv, D, dt, 1.0))
    c = cache_of(1, hq, hkv, D, dt, 2)
    bad = k.clone()
    bad[0, 1, 0] = float("nan")
    c.append(0, q, bad, v, at, r)
    assert c.status()[1] == P.DMC_FAULT_NAN_GATE and c.lengths(0).tolist() == [[1, 1]]
    c.reset()
    for _ in range(3):
        c.append(0, q, k, v, at, r)
    assert c.status()[1] == P.DMC_FAULT_SLOT_CAPACITY and c.lengths(0).tolist() == [[2, 2]]
    c = cache_of(1, hq, hkv, D, dt, 40, pages=1)
    c.append(0, q, k, v, at, r)
    assert c.status()[1] == P.DMC_FAULT_PAGES_EXHAUSTED and sorted(c.lengths(0)[0].tolist()) == [0, 1]
    c = cache_of(2, hq, hkv, D, dt, 4)
    q2, k2, v2 = (torch.cat([t, t]) for t in (q, k, v))
    cu = torch.tensor([0, 2, 1], dtype=torch.int32).cuda()
    c.append(0, q2, k2, v2, at.expand(2).contiguous(), r, cu_seqlens=cu, max_seqlen=1)
    assert c.status()[1] == P.DMC_FAULT_BAD_SEQLENS and int(c.lengths(0).sum()) == 0


def test_refusals(cuda_dev):
    hq, hkv, D, dt = 4, 2, 64, BF16
    g = torch.Generator().manual_seed(6)
    c = cache_of(3, hq, hkv, D, dt, 50, prompt=20)
    q, k, v = (t.cuda() for t in tokens(g, 3, hq, hkv, D, dt))
    at, r = torch.zeros(3, dtype=torch.int32).cuda(), R.Rotary(D)
    ok = dict(q=q, k=k, v=v, positions=at, rotary=r)
    for bad in (dict(q=q.float()), dict(k=k[:2]), dict(v=v[..., :32]), dict(positions=at.long()), dict(positions=at[:2]),
                dict(positions=None), dict(rotary=None), dict(rotary=R.Rotary(128)), dict(rotary=R.Rotary(D, device="cpu")),
                dict(q_out=q[:2]), dict(q_out=q.float()), dict(q=q.transpose(0, 1)), dict(cu_seqlens=at.long()),
                dict(q=q.cpu())):
        with pytest.raises(ValueError):
            c.append(0, **{**ok, **bad})
    cu = torch.tensor([0, 3], dtype=torch.int32).cuda()
    for bad in (dict(layer=1), dict(layer=-1), dict(first_seq=1), dict(first_seq=-1)):
        with pytest.raises(P.DmcError):
            c.append(bad.pop("layer", 0), **ok, **bad)
    with pytest.raises(P.DmcError):  # three tokens of one sequence, said to be one
        c.append(0, q, k, v, at[:1], r, cu_seqlens=cu, max_seqlen=1)
    big = [t.cuda() for t in tokens(g, 21, hq, hkv, D, dt)]
    with pytest.raises(P.DmcError):  # more than max_prefill_tokens
        c.append(0, *big, at[:1], r, cu_seqlens=torch.tensor([0, 21], dtype=torch.int32).cuda(), max_seqlen=21)
    s = torch.cuda.current_stream().cuda_stream
    p = [t.data_ptr() for t in (q, k, v)]
    call = lambda *a: P.dmc_cache_append(c.handle, 0, 0, 3, *a, s)  # noqa: E731
    assert call(p[0] + 8, p[1], p[2], None, 3, 1, None, None, 0, None) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 3, 2, None, None, 0, None) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 2, 1, None, None, 0, None) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 3, 1, at.data_ptr(), None, 0, None) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 3, 1, at.data_ptr(), r.turns.data_ptr(), 0, None) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 3, 1, at.data_ptr(), r.turns.data_ptr() + 4, 0, p[0]) == P.DMC_ERR_INVALID_ARG
    assert call(*p, None, 3, 0, None, None, 0, None) == P.DMC_ERR_INVALID_ARG
    assert c.status() == (0, 0, 0) and int(c.lengths(0).sum()) == 0


def test_a_prompt_captured_and_replayed(cuda_dev):
    hq, hkv, D, dt, T = 8, 2, 128, BF16, 500
    g = torch.Generator().manual_seed(11)
    x = [tokens(g, T, hq, hkv, D, dt, 0.4) for _ in range(3)]
    q, k, v = (t.cuda() for t in x[0])
    cu = torch.tensor([0, 13, T], dtype=torch.int32).cuda()
    at = torch.tensor([0, 90], dtype=torch.int32).cuda()
    r, a, b = R.Rotary(D), cache_of(2, hq, hkv, D, dt, 2 * T, prompt=T), cache_of(2, hq, hkv, D, dt, 2 * T, prompt=T)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.append(0, q, k, v, at, r, cu_seqlens=cu, max_seqlen=T, q_out=out)
    for y in x[1:]:
        for to, t in zip((q, k, v), y):
            to.copy_(t)
        graph.replay()
        want = b.append(0, *(t.cuda() for t in y), at, r, cu_seqlens=cu, max_seqlen=T)
        assert torch.equal(out, want)
    for s, t in zip(exported(a, 0, 2 * T), exported(b, 0, 2 * T)):
        assert torch.equal(s, t)


def test_captured_and_replayed(cuda_dev):
    """A graph of one step, replayed: positions are read on the device, so the program moves them on."""
    hq, hkv, D, dt = 4, 2, 64, F32
    g = torch.Generator().manual_seed(7)
    r, freq = R.Rotary(D, inv_freq=inv_freq(D)), inv_freq(D)
    c, plain = cache_of(2, hq, hkv, D, dt, 40), Plain(2, hq, hkv, D, dt)
    q, k, v = (t.cuda() for t in tokens(g, 2, hq, hkv, D, dt))
    at = torch.tensor([3, 9], dtype=torch.int32).cuda()
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        c.append(0, q, k, v, at, r, q_out=out)
        at.add_(1)
    for i in range(36):
        x = tokens(g, 2, hq, hkv, D, dt, 0.9)
        for to, t in zip((q, k, v), x):
            to.copy_(t)
        graph.replay()
        for s in range(2):
            plain.append(s, *(t[s:s + 1] for t in x), (3, 9)[s] + i, freq)
    torch.cuda.synchronize()
    assert at.tolist() == [39, 45]
    compare(c, 0, plain, 40, 36, 4.0)
