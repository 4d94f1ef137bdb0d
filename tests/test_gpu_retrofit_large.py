"""The retrofitting operators where element offsets pass 32 bits: the last sequences of a
long pack give the bits that they give alone, and a vocabulary's last words count."""
import pytest
import torch

from retrofit_harness import OFFSET, TEMPERATURE, handle
from paper_2403_09636_gb300.retrofit import DmcRetrofit

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def normal(g, *shape, scale=1.0, dtype=BF16):
    return torch.randn(*shape, generator=g, device=g.device, dtype=dtype).mul_(scale)


def pack(dev, heads, per, n, seed=2):
    Hq, H, D = heads
    g = torch.Generator(device=dev).manual_seed(seed)
    T = per * n
    x = {"q": normal(g, T, Hq, D), "k": normal(g, T, H, D, scale=0.5), "v": normal(g, T, H, D, scale=0.5),
         "bias": -torch.nn.functional.softplus(normal(g, H, T, scale=8.0, dtype=torch.float32)),
         "dout": normal(g, T, Hq, D)}
    return x, torch.arange(0, T + 1, per, dtype=torch.int32, device=dev)


def tail(t, n, dim):
    return t.narrow(dim, t.shape[dim] - n, n).contiguous()


def test_attention_beyond_32_bits(cuda_dev):
    heads, per, n = (64, 8, 128), 300, 900  # 270,000 tokens of 64 x 128: 2.2e9 elements
    x, cu = pack(cuda_dev, heads, per, n)
    assert x["q"].numel() > 2 ** 31

    def run(x, cu):
        h = handle(cuda_dev, *heads, BF16, [per] * (cu.numel() - 1))
        a = (x["q"], x["k"], x["v"])
        o, lse = h.attention(*a, cu, per, x["bias"])
        grads = h.attention_backward(x["dout"], *a, o, lse, cu, per, x["bias"])
        assert h.status() == (0, 0)
        return o, *grads[:3], lse, grads[3]

    few = 2 * per
    small = {i: tail(t, few, 1 if i == "bias" else 0) for i, t in x.items()}
    want = run(small, torch.arange(0, few + 1, per, dtype=torch.int32, device=cuda_dev))
    got = run(x, cu)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(tail(a, few, 1 if i > 3 else 0), b), i


def test_states_beyond_32_bits(cuda_dev):
    heads, per, n = (64, 64, 128), 300, 900
    x, cu = pack(cuda_dev, heads, per, n)
    T = per * n
    g = torch.Generator(device=cuda_dev).manual_seed(5)
    x["k"][..., 0] += OFFSET
    x["q0"] = x.pop("q")[..., 0].contiguous()
    x["dkt"], x["dvt"] = x.pop("dout"), x["v"].flip(0)
    x["dbias"], x["dalpha"] = x["bias"].to(BF16), normal(g, 64, T, dtype=torch.float32)
    x["noise"] = normal(g, 64, T, dtype=torch.float32)

    def run(x, cu):
        h = handle(cuda_dev, *heads, BF16, [per] * (cu.numel() - 1))
        a = (x["q0"], x["k"], x["v"], cu, per)
        kw = {"noise": x["noise"], "offset": OFFSET, "temperature": TEMPERATURE}
        kt, vt, alpha, bias, saved = h.states(*a, **kw)
        grads = h.states_backward(*a, saved, x["dkt"], x["dvt"], x["dbias"], x["dalpha"], **kw)
        assert h.status() == (0, 0)
        return kt, vt, *grads, alpha, bias

    few = 2 * per
    small = {i: tail(t, few, 1 if i in ("bias", "dbias", "dalpha", "noise") else 0) for i, t in x.items()}
    want = run(small, torch.arange(0, few + 1, per, dtype=torch.int32, device=cuda_dev))
    got = run(x, cu)
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(tail(a, few, 1 if i > 4 else 0), b), i


def test_loss_beyond_32_bits(cuda_dev):
    V, H, N = 300000, 8192, 5
    g = torch.Generator(device=cuda_dev).manual_seed(3)
    hidden, weight = normal(g, N, H), normal(g, V, H, scale=2.0 / H ** 0.5)
    assert weight.numel() > 2 ** 31
    targets = torch.tensor([0, V - 1, V - 129, 262200, -1], dtype=torch.int32, device=cuda_dev)
    dloss = torch.ones(N, device=cuda_dev)
    h = DmcRetrofit(dtype=BF16, max_tokens=N, hidden=H, vocab=V, device=cuda_dev)
    loss, lse = h.loss(hidden, weight, targets)
    dh, dw = h.loss_backward(dloss, hidden, weight, targets, lse)
    assert h.status() == (0, 0)
    logits = torch.cat([hidden.double() @ w.double().t() for w in weight.split(50000)], 1)
    want = torch.logsumexp(logits, 1)
    assert float((lse - want).abs().max()) < 1e-4
    hit = logits.gather(1, targets.long().clamp(min=0)[:, None])[:, 0]
    assert float(((want - hit)[:4] - loss[:4]).abs().max()) < 1e-4 and float(loss[4]) == 0.0
    p = torch.exp(logits - want[:, None])
    for i, t in enumerate(targets.tolist()):
        if t < 0:
            p[i] = 0.0
        else:
            p[i, t] -= 1.0
    rows = torch.tensor([0, 1, 131072, 262143, 262144, 262200, V - 129, V - 1], device=cuda_dev)
    ref = p[:, rows].t() @ hidden.double()
    size = p[:, rows].abs().t() @ hidden.double().abs()
    assert bool(((dw[rows].double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + 1.01 * size)).all())
    ref = sum(p[:, a:a + 50000] @ weight[a:a + 50000].double() for a in range(0, V, 50000))
    size = sum(p[:, a:a + 50000].abs() @ weight[a:a + 50000].double().abs() for a in range(0, V, 50000))
    assert bool(((dh.double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + 1.01 * size)).all())
