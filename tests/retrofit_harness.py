"""Inputs and comparisons shared by the tests of the retrofitting operators."""
import math

import numpy as np
import torch

from oracle import retrofit_ref as R
from paper_2403_09636_gb300.retrofit import DmcRetrofit

OFFSET, TEMPERATURE = 5.0, 0.1


def cu_of(lens, dev):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=dev)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def normal(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def noise_of(g, *shape):
    u = torch.rand(*shape, generator=g).clamp(1e-6, 1 - 1e-6)
    return torch.log(u) - torch.log1p(-u)


def handle(dev, Hq, Hkv, D, dtype, lens):
    return DmcRetrofit(Hq, Hkv, D, dtype=dtype, max_tokens=max(1, sum(lens)), max_seqs=max(1, len(lens)), device=dev)


def states_inputs(lens, Hq, Hkv, D, dtype, seed=1, spread=0.5):
    """CPU tensors: q0, k, v, noise and the states' gradients."""
    g, T = gen(seed), sum(lens)
    k = normal(g, T, Hkv, D, scale=0.5, dtype=dtype)
    k[..., 0] = (normal(g, T, Hkv, scale=spread) + OFFSET).to(dtype)
    return {"q0": normal(g, T, Hq, scale=0.5, dtype=dtype), "k": k, "v": normal(g, T, Hkv, D, scale=0.5, dtype=dtype),
            "noise": noise_of(g, Hkv, T), "dkt": normal(g, T, Hkv, D, dtype=dtype),
            "dvt": normal(g, T, Hkv, D, dtype=dtype), "dbias": normal(g, Hkv, T, dtype=dtype),
            "dalpha": normal(g, Hkv, T)}


def attention_inputs(lens, Hq, Hkv, D, dtype, seed=1, bias="soft"):
    g, T = gen(seed), sum(lens)
    x = {"q": normal(g, T, Hq, D, scale=2.0, dtype=dtype), "k": normal(g, T, Hkv, D, scale=0.5, dtype=dtype),
         "v": normal(g, T, Hkv, D, scale=0.5, dtype=dtype), "dout": normal(g, T, Hq, D, dtype=dtype), "bias": None}
    if bias != "none":
        x["bias"] = -torch.nn.functional.softplus(normal(g, Hkv, T, scale=8.0))
    if bias == "hard":
        x["bias"] = torch.where(torch.rand(Hkv, T, generator=g) < 0.5, 0.0, -math.inf)
    return x


def on(x, dev):
    return {n: t.to(dev) if isinstance(t, torch.Tensor) else t for n, t in x.items()}


def spans(lens):
    a = 0
    for n in lens:
        yield a, a + n
        a += n


def close(name, got, want, bound):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), f"{name} is not finite"
    off = (got - want).abs() / bound
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times its bound at {np.unravel_index(int(off.argmax()), off.shape)}"


def check_attention(x, lens, dtype, got):
    """got: out, lse and the gradients over all tokens."""
    for a, b in spans(lens):
        if a == b:
            continue
        part = R.attention_all(x["q"][a:b], x["k"][a:b], x["v"][a:b],
                               None if x["bias"] is None else x["bias"][:, a:b], x["dout"][a:b], dtype)
        for name, (want, bound) in part.items():
            if name in got:
                close(f"{name} [{a}:{b}]", got[name][:, a:b] if name in ("lse", "dbias") else got[name][a:b], want, bound)


def check_states(x, lens, dtype, got, noise=True, dalpha=True):
    for a, b in spans(lens):
        if a == b:
            continue
        part = R.states_all(x["q0"][a:b], x["k"][a:b], x["v"][a:b], x["noise"][:, a:b] if noise else None, OFFSET,
                            TEMPERATURE, x["dkt"][a:b], x["dvt"][a:b], x["dbias"][:, a:b],
                            x["dalpha"][:, a:b] if dalpha else None, dtype)
        for name, (want, bound) in part.items():
            close(f"{name} [{a}:{b}]", got[name][:, a:b] if name in ("alpha", "bias") else got[name][a:b], want, bound)
