"""The position rotation of queries and keys, and its gradient, against 64 bits (GPU).

Bound of an element x c - y s: cos and sin are off by 4 steps of 2^-24 (their argument's rounding to fp32, pi 2^-25, and
the functions' own two), the two products and the sum by one each, so 7 (|x| + |y|) 2^-24; then the one rounding to the
type."""
import math
from fractions import Fraction

import pytest
import torch

from generate_harness import EPS, inv_freq, near, turned
from paper_2403_09636_gb300 import rotary as R

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bound(x, want, dt):
    return 8 * 2.0 ** -24 * (x.double().abs() + x.double().abs().amax(-1, keepdim=True)) + EPS[dt] * 1.01 * want.abs()


def made(T, hq, hk, D, dt, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, hq, D, generator=g).to(dt), torch.randn(T, hk, D, generator=g).to(dt),
            torch.randint(-1000, 100000, (T,), generator=g, dtype=torch.int32))


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,hq,hk", [(1, 1, 1), (1, 40, 40), (3, 5, 2), (257, 8, 1), (1025, 4, 4), (4099, 1, 2)])
def test_against_64_bits(cuda_dev, dt, D, pairs, T, hq, hk):
    q, k, at = made(T, hq, hk, D, dt)
    r = R.Rotary(D, inv_freq=inv_freq(D), interleaved=pairs)
    for back in (False, True):
        got = R.rotate(r, q.cuda(), k.cuda(), at.cuda(), inverse=back)
        for x, y in zip((q, k), got):
            want = turned(x, at, inv_freq(D), pairs, back)
            assert y.dtype == dt and y.shape == x.shape
            near(y.cpu(), want, bound(x, want, dt))
            gate = [0, 1] if pairs else [0, D // 2]
            assert torch.equal(y.cpu()[..., gate], x[..., gate])


def test_positions_at_the_ends_of_their_range(cuda_dev):
    """Phases of far positions are exact: against angles from exact fractions."""
    D, at = 128, [0, -1, (1 << 31) - 1, -(1 << 31), 123456789]
    pi = 2 * Fraction(0xC90FDAA22168C234C4C6628B80DC1CD129024E088A67CC74, 1 << 191)
    freq = inv_freq(D)
    turns = torch.tensor([[float(Fraction(float(f)) * a / (2 * pi) % 1) for f in freq] for a in at], dtype=torch.float64)
    angle = turns * 2 * math.pi
    angle[:, 0] = 0.0
    q = torch.randn(len(at), 3, D, generator=torch.Generator().manual_seed(1))
    x, y = q.double().chunk(2, -1)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    want = torch.cat([x * c - y * s, y * c + x * s], -1)
    got, none = R.rotate(R.Rotary(D, inv_freq=freq), q.cuda(), None, torch.tensor(at, dtype=torch.int32).cuda())
    assert none is None
    near(got.cpu(), want, bound(q, want, F32))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_slices_of_a_joint_projection_and_in_place(cuda_dev, dt):
    T, hq, hk, D = 77, 6, 2, 64
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(T, hq + 2 * hk, D, generator=g).to(dt)
    at = torch.arange(T, dtype=torch.int32)
    dev = qkv.cuda()
    r = R.Rotary(D)
    want = [t.clone() for t in R.rotate(r, dev[:, :hq].contiguous(), dev[:, hq:hq + hk].contiguous(), at.cuda())]
    got = R.rotate(r, dev[:, :hq], dev[:, hq:hq + hk], at.cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    R.rotate(r, dev[:, :hq], dev[:, hq:hq + hk], at.cuda(), out=(dev[:, :hq], dev[:, hq:hq + hk]))
    assert torch.equal(dev[:, :hq], want[0]) and torch.equal(dev[:, hq:hq + hk], want[1])
    assert torch.equal(dev[:, hq + hk:].cpu(), qkv[:, hq + hk:])  # v as it was


def test_values_that_are_not_finite_keep_to_their_pair(cuda_dev):
    D = 64
    q = torch.zeros(2, 1, D)
    q[0, 0, 3], q[1, 0, 40] = math.inf, math.nan
    q[..., 0] = math.nan  # a gate
    got = R.rotate(R.Rotary(D), q.cuda(), None, torch.tensor([5, 9], dtype=torch.int32).cuda())[0].cpu()
    finite = torch.isfinite(got)
    bad = torch.zeros(2, 1, D, dtype=torch.bool)
    bad[..., 0] = True
    bad[0, 0, [3, 35]] = True
    bad[1, 0, [8, 40]] = True
    assert torch.equal(~finite, bad)


@pytest.mark.parametrize("pairs", [False, True])
def test_gradients(cuda_dev, pairs):
    """apply()'s gradients against the formula's (the rotation back) and against differences of a loss (the loss is
    linear in q and k, so that a difference of any step is exact but for rounding)."""
    T, hq, hk, D = 33, 4, 2, 64
    q, k, at = made(T, hq, hk, D, F32, 3)
    g = torch.Generator().manual_seed(4)
    dq, dk = torch.randn(T, hq, D, generator=g), torch.randn(T, hk, D, generator=g)
    r = R.Rotary(D, inv_freq=inv_freq(D), interleaved=pairs)
    a, b = q.cuda().requires_grad_(), k.cuda().requires_grad_()
    y, z = R.apply(r, a, b, at.cuda())
    loss = (y * dq.cuda()).sum() + (z * dk.cuda()).sum()
    loss.backward()
    for got, up in ((a.grad, dq), (b.grad, dk)):
        want = turned(up, at, inv_freq(D), pairs, True)
        near(got.cpu(), want, bound(up, want, F32))
    step = torch.randn(T, hq, D, generator=g)
    up = R.apply(r, (q + step).cuda(), b, at.cuda())[0].double() - R.apply(r, (q - step).cuda(), b, at.cuda())[0].double()
    slope = float((up.detach() * dq.cuda().double()).sum()) / 2
    want = float((a.grad.cpu().double() * step.double()).sum())
    size = float((dq.abs().double().sum(-1) * (q.abs() + step.abs()).double().amax(-1)).sum())
    assert abs(slope - want) <= 16 * 2.0 ** -24 * size
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(R.apply(r, a, b, at.cuda())[0].sum(), a, create_graph=True)[0].sum(), a)


def test_gradient_of_one_output_alone(cuda_dev):
    r = R.Rotary(64)
    q, k, at = made(5, 2, 2, 64, BF16, 5)
    a, b = q.cuda().requires_grad_(), k.cuda().requires_grad_()
    R.apply(r, a, b, at.cuda())[0].sum().backward()
    assert bool(a.grad.any()) and not bool(b.grad.any())


def test_gradients_of_what_needs_them(cuda_dev):
    r = R.Rotary(64)
    q, k, at = made(5, 2, 1, 64, F32, 6)
    for which in ("q", "k", "q alone"):
        a, b = q.cuda(), None if which == "q alone" else k.cuda()
        leaf = b if which == "k" else a
        leaf.requires_grad_()
        y, z = R.apply(r, a, b, at.cuda())
        assert (z is None) == (b is None)
        out = z if which == "k" else y
        out.sum().backward()
        up = torch.ones(out.shape)
        want = turned(up, at, inv_freq(64), False, True)
        near(leaf.grad.cpu(), want, bound(up, want, F32))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_gradients_that_begin_anywhere(cuda_dev, dt):
    """What follows the rotation may hand back a piece of a longer gradient, one element off its start, or one that is
    laid out in another order."""
    r = R.Rotary(64)
    q, k, at = made(5, 2, 2, 64, dt, 7)
    a, b = q.cuda().requires_grad_(), k.cuda().requires_grad_()
    y, z = R.apply(r, a, b, at.cuda())
    up = torch.randn(2, 641, generator=torch.Generator().manual_seed(8)).to(dt)
    x = torch.cat((torch.zeros(1, dtype=dt, device=cuda_dev), y.reshape(-1)))
    ((x * up[0].cuda()).sum() + (z.transpose(0, 1) * up[1, 1:].view(2, 5, 64).cuda()).sum()).backward()
    for got, g in ((a.grad, up[0, 1:].view(5, 2, 64)), (b.grad, up[1, 1:].view(2, 5, 64).transpose(0, 1))):
        want = turned(g, at, inv_freq(64), False, True)
        near(got.cpu(), want, bound(g, want, dt))


def test_nothing_to_do(cuda_dev):
    r = R.Rotary(64)
    q, k = R.rotate(r, torch.empty(0, 2, 64, device=cuda_dev), torch.empty(0, 1, 64, device=cuda_dev),
                    torch.empty(0, dtype=torch.int32, device=cuda_dev))
    assert q.shape == (0, 2, 64) and k.shape == (0, 1, 64)


def test_refusals(cuda_dev):
    r = R.Rotary(64)
    q, k, at = (t.cuda() for t in made(4, 2, 1, 64, BF16))
    for bad in (dict(q=q.half()), dict(q=q[..., :32]), dict(k=k.float()), dict(k=k[:3]), dict(at=at.long()), dict(at=at[:3]),
                dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)), dict(q=q.cpu()), dict(out=(q,)), dict(out=(q, None)),
                dict(out=(k, k)), dict(q=q.expand(4, 2, 64)[:1].expand(4, 2, 64))):
        x = {"q": q, "k": k, "at": at, "out": None, **bad}
        with pytest.raises(ValueError):
            R.rotate(r, x["q"], x["k"], x["at"], out=x["out"])


def test_in_a_graph_and_on_another_stream(cuda_dev):
    r = R.Rotary(128)
    q, k, at = (t.cuda() for t in made(65, 4, 4, 128, BF16))
    want = R.rotate(r, q, k, at)
    out = tuple(torch.zeros_like(t) for t in want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rotate(r, q, k, at, out=out)
    for _ in range(2):
        for t in out:
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = R.rotate(r, q, k, at, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
