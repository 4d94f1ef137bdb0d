"""Attention of one token's queries over the cache as it stands, against 64 bits (GPU).

Bounds: a score is off by some 43 steps of 2^-24 at these scales, a weight by 64, an output by twice that of the largest
value, 2^-17 of it; weights of grouped bf16 queries enter their product as two bf16 numbers, which leaves 2^-17 of each
in turn: 2^-14 in all. Then the one rounding to the type."""
import pytest
import torch

import paper_2403_09636_gb300 as P
from generate_harness import EPS, Plain, cache_of, exported, near, tokens

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def over(cache, layer, q, hkv):
    """Plain attention over the slots the cache holds."""
    B, Hq, D = q.shape
    plain = Plain(B, Hq, hkv, D, q.dtype)
    k, v, z, ln = exported(cache, layer, int(cache.lengths(layer).max().clamp(min=1)))
    for i in range(B * hkv):
        plain.heads[i // hkv][i % hkv] = [(k[i, j].double(), v[i, j].double(), z[i, j]) for j in range(int(ln[i]))]
    return plain.attend(q)


def check(cache, layer, q, hkv):
    got = cache.attend(layer, q.cuda())
    want, size = over(cache, layer, q, hkv)
    near(got.cpu(), want, 1.01 * EPS[q.dtype] * want.abs() + 2.0 ** -14 * size[..., None])
    return got


def filled(lens, hq, hkv, D, dt, opens, seed=0, layers=1, window=0):
    g = torch.Generator().manual_seed(seed)
    cache = cache_of(len(lens), hq, hkv, D, dt, max(lens) + 2, layers=layers, prompt=max(1, sum(lens)), window=window)
    q, k, v = (t.cuda() for t in tokens(g, sum(lens), hq, hkv, D, dt, opens))
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    for layer in range(layers):
        if sum(lens):
            cache.prefill(layer, q[..., 0], k, v, cu, max(lens))
    return cache, g


HEADS = [(2, 2), (4, 2), (6, 2), (16, 2), (18, 2), (32, 1)]


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", [[1], [0, 31, 32, 33, 0], [300, 5, 0, 1000]])
def test_against_64_bits(cuda_dev, dt, D, heads, lens):
    """Heads of many lengths, empty ones (which give zeros) before, between and after them."""
    cache, g = filled(lens, *heads, D, dt, 0.6)
    q = torch.randn(len(lens), heads[0], D, generator=g).to(dt)
    got = check(cache, 0, q, heads[1])
    for i, n in enumerate(lens):
        if n == 0:
            assert not bool(got[i].any())
    before = cache.lengths(0)
    again = cache.attend(0, q.cuda())
    assert torch.equal(got, again) and torch.equal(before, cache.lengths(0))
    assert cache.status()[:2] == (0, 0)


@pytest.mark.parametrize("dt,heads", [(BF16, (4, 4)), (F32, (4, 4)), (BF16, (16, 2)), (F32, (6, 2))])
def test_an_empty_cache(cuda_dev, dt, heads):
    cache = cache_of(3, *heads, 64, dt, 40)
    out = torch.full((3, heads[0], 64), 7.0, dtype=dt).cuda()
    assert cache.attend(0, torch.ones(3, heads[0], 64, dtype=dt).cuda(), out) is out
    assert not bool(out.any())


@pytest.mark.parametrize("dt,heads", [(BF16, (2, 2)), (BF16, (8, 1)), (F32, (2, 1))])
def test_one_long_head_split_over_the_gpu(cuda_dev, dt, heads):
    cache, g = filled([20011], *heads, 128, dt, 1.0)
    check(cache, 0, torch.randn(1, heads[0], 128, generator=g).to(dt), heads[1])


@pytest.mark.parametrize("dt,heads", [(BF16, (1, 1)), (BF16, (2, 1)), (F32, (1, 1))])
def test_many_short_heads(cuda_dev, dt, heads):
    """More heads than warps, every third one empty."""
    lens = [0 if i % 3 == 1 else 1 + i % 40 for i in range(1500)]
    cache, g = filled(lens, *heads, 64, dt, 0.7)
    check(cache, 0, torch.randn(len(lens), heads[0], 64, generator=g).to(dt), heads[1])


@pytest.mark.parametrize("dt,heads", [(BF16, (2, 2)), (BF16, (8, 2)), (F32, (4, 2))])
def test_decoding_is_appending_and_attending(cuda_dev, dt, heads):
    """dmc_decode_step's outputs and slots against append + attend of the same tokens."""
    D = 128
    a, _ = filled([70, 3], *heads, D, dt, 0.5)
    b, g = filled([70, 3], *heads, D, dt, 0.5)
    for _ in range(5):
        x = tokens(g, 2, *heads, D, dt)
        q, k, v = (t.cuda() for t in x)
        out = torch.empty_like(q)
        a.decode(0, q, k, v, out)
        b.append(0, q, k, v)
        got = b.attend(0, q)
        size = float(v.abs().max()) + 4.0
        near(got.cpu(), out.cpu().double(), 4 * EPS[dt] * size)
    for s, t in zip(exported(a, 0, 75), exported(b, 0, 75)):
        near(s, t.double(), 2.0 ** -7 * t.double().abs().max() if dt == BF16 else 64 * 2.0 ** -24 * t.double().abs().max())


def test_the_gate_takes_no_part(cuda_dev):
    for dt, heads in ((BF16, (2, 2)), (BF16, (4, 2)), (F32, (2, 2))):
        cache, g = filled([50], *heads, 64, dt, 0.5)
        q = torch.randn(1, heads[0], 64, generator=g).to(dt)
        other = q.clone()
        other[..., 0] = 1000.0
        assert torch.equal(cache.attend(0, q.cuda()), cache.attend(0, other.cuda()))


def test_layers_windows_streams_and_decoding_between(cuda_dev):
    """Two layers in turn on another stream with decodes between them; a cache with window grouping."""
    hq, hkv, D, dt = 4, 4, 64, BF16
    cache, g = filled([90, 41], hq, hkv, D, dt, 0.5, layers=2, window=5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for i in range(4):
        x = tokens(g, 2, hq, hkv, D, dt)
        q, k, v = (t.cuda() for t in x)
        s.wait_stream(torch.cuda.current_stream())
        cache.decode(i % 2, q, k, v, torch.empty_like(q), stream=s)
        a = cache.attend(i % 2, q, stream=s)
        b = cache.attend(1 - i % 2, q, stream=s)
        cache.decode(1 - i % 2, q, k, v, torch.empty_like(q), stream=s)
        s.synchronize()
        assert torch.isfinite(a.float()).all() and torch.isfinite(b.float()).all()
    for layer in range(2):
        check(cache, layer, torch.randn(2, hq, D, generator=g).to(dt), hkv)
    assert cache.status()[:2] == (0, 0)


def test_captured_and_replayed(cuda_dev):
    hq, hkv, D, dt = 8, 2, 128, BF16
    cache, g = filled([300, 7], hq, hkv, D, dt, 0.5)
    q = torch.randn(2, hq, D, generator=g).to(dt).cuda()
    out = torch.empty_like(q)
    cache.attend(0, q, out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.attend(0, q, out)
    for _ in range(3):
        x = tokens(g, 2, hq, hkv, D, dt)
        cache.append(0, *(t.cuda() for t in x))  # the replay sees the cache as it is then
        q.copy_(x[0])
        graph.replay()
        want, size = over(cache, 0, x[0], hkv)
        near(out.cpu(), want, 1.01 * EPS[dt] * want.abs() + 2.0 ** -14 * size[..., None])


def test_values_that_are_not_finite_stay_in_their_head(cuda_dev):
    for heads in ((3, 3), (6, 3)):
        cache = cache_of(1, *heads, 64, BF16, 40)
        g = torch.Generator().manual_seed(1)
        for _ in range(35):
            q, k, v = tokens(g, 1, *heads, 64, BF16, 1.0)
            v[0, 1, 5] = float("nan")
            cache.append(0, q.cuda(), k.cuda(), v.cuda())
        out = cache.attend(0, torch.ones(1, heads[0], 64, dtype=BF16).cuda())
        bad = torch.isnan(out[0]).cpu()
        G = heads[0] // 3
        want = torch.zeros_like(bad)
        want[G:2 * G, 5] = True
        assert torch.equal(bad, want)


def test_refusals(cuda_dev):
    cache, g = filled([5], 2, 2, 64, BF16, 0.5)
    q = torch.zeros(1, 2, 64, dtype=BF16).cuda()
    for bad in (q.float(), q[:, :1], q.cpu(), torch.zeros(2, 2, 64, dtype=BF16).cuda(), q.transpose(0, 1)):
        with pytest.raises(ValueError):
            cache.attend(0, bad)
    with pytest.raises(ValueError):
        cache.attend(0, q, q.float())
    for layer in (-1, 1):
        with pytest.raises(P.DmcError):
            cache.attend(layer, q)
    with pytest.raises(P.DmcError):
        cache.attend(0, q, q)  # in place: heads would read what others wrote
