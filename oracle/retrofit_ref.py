"""Plain fp64 statement of the retrofitting operators (torch on the CPU, test
infrastructure only): the relaxed states token by token (Eq. partial-accumulation
with alpha in [0, 1]), attention under the additive training mask (masking appendix),
softmax cross entropy. Written from the definitions with differentiable torch
operations, so that autograd of these functions is the gradient's oracle.

`*_bounds` give, next to each value, how far a correctly rounded computation may be
from it: `u` is the relative rounding of what is stored or fed to a product in the
tensors' type (half a unit in the last of its 8 bits for bf16, 2^-8), `e` that of the fp32 arithmetic between.
"""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def states(q0, k, v, noise, offset, temperature):
    """One sequence: q0 [n, Hq], k and v [n, H, D], noise [H, n] or None.
    Returns k~, v~ [n, H, D], alpha, bias [H, n], z [n, H]."""
    n, H, D = k.shape
    x = k[:, :, 0] - offset
    if noise is not None:
        x = x + noise.t()
    x = x / temperature
    alpha = torch.cat([torch.zeros_like(x[:1]), torch.sigmoid(x[1:])])
    bias = torch.cat([torch.nn.functional.logsigmoid(-x[1:]), torch.zeros_like(x[:1])])
    omega = torch.sigmoid(q0.reshape(n, H, -1).mean(2))
    k = torch.cat([torch.zeros_like(k[:, :, :1]), k[:, :, 1:]], 2)
    kt, vt, zs = [], [], []
    for t in range(n):
        if t == 0:
            z, ks, vs = omega[0], k[0], v[0]
        else:
            old = alpha[t] * z
            z = old + omega[t]
            ks = (old[:, None] * ks + omega[t][:, None] * k[t]) / z[:, None]
            vs = (old[:, None] * vs + omega[t][:, None] * v[t]) / z[:, None]
        kt.append(ks)
        vt.append(vs)
        zs.append(z)
    return torch.stack(kt), torch.stack(vt), alpha.t(), bias.t(), torch.stack(zs)


def attention(q, k, v, bias):
    """One sequence: q [n, Hq, D], k and v [n, H, D], bias [H, n] or None. Returns out [n, Hq, D],
    lse [Hq, n] and the weights [Hq, n, n]."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    kx, vx = (t.permute(1, 0, 2).repeat_interleave(G, 0) for t in (k, v))
    s = q.permute(1, 0, 2) @ kx.transpose(1, 2) / math.sqrt(D)
    i = torch.arange(n)
    if bias is not None:
        b = bias.repeat_interleave(G, 0)[:, None, :].expand(Hq, n, n)
        s = s + torch.where(i[:, None] > i, b, torch.zeros((), dtype=s.dtype))
    s = s.masked_fill(i[:, None] < i, -math.inf)
    lse = torch.logsumexp(s, 2)
    p = torch.exp(s - lse[..., None])
    return (p @ vx).permute(1, 0, 2), lse, p


def attention_all(q, k, v, bias, dout, dtype):
    """One sequence's outputs, gradients and the bounds of both, as {name: (value, bound)}."""
    n, Hq, D = q.shape
    H = k.shape[1]
    G = Hq // H
    u, c = U[dtype], 1.0 / math.sqrt(D)
    leaf = [t.double().requires_grad_() for t in (q, k, v)]
    b = None if bias is None else bias.double().requires_grad_()
    out, lse, p = attention(*leaf, b)
    out.backward(dout.double())
    with torch.no_grad():
        q, k, v = leaf
        # fp32 arithmetic: a score's error is a multiple of the sum of its terms' sizes, a
        # weight's relative error that of its score and of the exponential
        kx, vx = (t.permute(1, 0, 2).repeat_interleave(G, 0) for t in (k, v))
        qh, doh = q.permute(1, 0, 2), dout.double().permute(1, 0, 2)
        terms = qh.abs() @ kx.abs().transpose(1, 2) * c
        seen = p > 0
        shift = torch.zeros(()) if b is None or not bool((b > -math.inf).any()) else b[b > -math.inf].abs().max()
        e = 2.0 ** -22 * (8 + (terms * seen).amax() + shift.clamp(max=200.0))
        rp = e if dtype == torch.float32 else e + u       # relative, of a weight in a product
        o_sum = p @ vx.abs()
        o_bound = (u * out.permute(1, 0, 2).abs() + (rp + e) * o_sum)
        res = {"out": (out, o_bound.permute(1, 0, 2)),
               "lse": (lse, e + 2.0 ** -22 * lse.abs())}
        # a row's delta = dO . out comes from the rounded out
        d_delta = (doh.abs() * o_bound).sum(-1, keepdim=True) + e * (doh.abs() * out.permute(1, 0, 2).abs()).sum(-1, keepdim=True)
        dp = doh @ vx.transpose(1, 2)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        size = p * (doh.abs() @ vx.abs().transpose(1, 2) + (doh.abs() * o_sum).sum(-1, keepdim=True))
        d_ds = p * d_delta + 4 * e * size
        group = lambda t: t.reshape(H, G, *t.shape[1:]).sum(1)  # noqa: E731
        dq = q.grad
        res["dq"] = (dq, (c * ((d_ds + u * ds.abs()) @ kx.abs()).permute(1, 0, 2) + u * dq.abs()))
        res["dk"] = (k.grad, (c * group((d_ds + u * ds.abs()).transpose(1, 2) @ qh.abs()).permute(1, 0, 2)
                              + u * k.grad.abs()))
        res["dv"] = (v.grad, (group(((rp + e) * p).transpose(1, 2) @ doh.abs()).permute(1, 0, 2) + u * v.grad.abs()))
        if b is not None:
            i = torch.arange(n)
            below = (i[:, None] > i).double()
            res["dbias"] = (b.grad, group((d_ds * below).sum(1)) + u * b.grad.abs())
    return {name: (x.detach(), y + 1e-30) for name, (x, y) in res.items()}


def states_all(q0, k, v, noise, offset, temperature, dkt, dvt, dbias, dalpha, dtype):
    """One sequence's states, their gradients and the bounds of both, as {name: (value, bound)}."""
    u = U[dtype]
    leaf = [t.double().requires_grad_() for t in (q0, k, v)]
    kt, vt, alpha, bias, z = states(*leaf, None if noise is None else noise.double(), offset, temperature)
    loss = (kt * dkt.double()).sum() + (vt * dvt.double()).sum() + (bias * dbias.double()).sum()
    if dalpha is not None:
        loss = loss + (alpha * dalpha.double()).sum()
    loss.backward()
    for t in leaf:  # a single token's state does not depend on its weight
        t.grad = torch.zeros_like(t) if t.grad is None else t.grad
    with torch.no_grad():
        # Rounding errors of fp32 sums in the order of the definition (or of a scan of it): `B` are the
        # sums of the terms' sizes, `E` the errors; `d` is the relative error that a step
        # adds, roundings and that of alpha, whose logit is off by `dx`.
        n, H, D = k.shape
        q0, k, v = leaf
        kin = k[:, :, 0].abs() + abs(offset) + (0 if noise is None else noise.double().abs().t())
        eps = 2.0 ** -23
        dx = eps * 4 * kin / temperature
        a = alpha.t()
        d = 8 * eps + (1 - a) * dx
        omega = torch.sigmoid(q0.reshape(n, H, -1).mean(2))
        row = torch.cat([k, v], 2)
        row[:, :, 0] = 0.0
        y = torch.cat([kt, vt], 2)
        g = torch.cat([dkt.double(), dvt.double()], 2)
        g[:, :, 0] = 0.0
        zero = torch.zeros_like(row[0])
        B, E, Ez = [], [], []
        b_, e_, ez_, z_ = zero, zero, torch.zeros_like(omega[0]), torch.zeros_like(omega[0])
        for t in range(n):
            at, dt = a[t][:, None], d[t][:, None]
            own = omega[t][:, None] * row[t].abs()
            b_, e_ = at * b_ + own, at * (e_ + dt * b_) + dt * (at * b_ + own)
            ez_ = a[t] * (ez_ + d[t] * z_) + d[t] * z[t]
            z_ = z[t]
            B.append(b_)
            E.append(e_)
            Ez.append(ez_)
        B, E, Ez = torch.stack(B), torch.stack(E), torch.stack(Ez)
        zx = z[..., None]
        Ey = E / zx + B / zx * (Ez / z + eps)[..., None]
        # the way back
        gL, gE, gZ, gEz = [None] * n, [None] * n, [None] * n, [None] * n
        up = g.abs() / zx
        dup = up * (Ez / z + 4 * eps)[..., None]
        W = (g.abs() * B / zx).sum(2) / z
        dW = (g.abs() * Ey).sum(2) / z + W * (Ez / z + 2 * D ** 0.5 * eps)
        l_, le_, s_, se_ = zero, zero, torch.zeros_like(omega[0]), torch.zeros_like(omega[0])
        for t in range(n - 1, -1, -1):  # l_ .. arrive with the alpha of the next token
            l_, le_, s_, se_ = l_ + up[t], le_ + dup[t], s_ + W[t], se_ + dW[t]
            gL[t], gE[t], gZ[t], gEz[t] = l_, le_, s_, se_
            at, dt = a[t][:, None], d[t][:, None]
            l_, le_ = at * l_, at * (le_ + dt * l_)
            s_, se_ = a[t] * s_, a[t] * (se_ + d[t] * s_)
        gL, gE, gZ, gEz = (torch.stack(t) for t in (gL, gE, gZ, gEz))
        before = lambda t: torch.cat([torch.zeros_like(t[:1]), t[:-1]])  # noqa: E731
        many = 2 * D ** 0.5 * eps
        dwb = (gE * row.abs() + many * gL * row.abs()).sum(2) + gEz + many * gZ
        dab = (gE * before(B) + gL * before(E) + many * gL * before(B)).sum(2) + gEz * before(z) + gZ * before(Ez + many * z)
        da = (gL * before(B)).sum(2) + gZ * before(z)  # its size
        if dalpha is not None:
            da = da + dalpha.double().abs().t()
        db = torch.cat([torch.zeros_like(bias[:, :1]), dbias.double().abs()[:, :-1]], 1).t()
        gate = a * (1 - a)
        rows = omega[..., None] * (gE + 8 * eps * gL)
        gatew = (omega * (1 - omega))
        G = q0.shape[1] // H
        dk_bound = u * k.grad.abs() + rows[:, :, :D]
        dk_bound[:, :, 0] = u * k.grad[:, :, 0].abs() + (
            gate * (dab + da * (dx + 16 * eps)) + db * a * (d + 8 * eps)) / temperature
        dq_bound = (gatew * (dwb + 32 * eps * ((gL * row.abs()).sum(2) + gZ)) / G)[:, :, None].expand(n, H, G).reshape(n, H * G)
        res = {"kt": (kt, u * kt.abs() + Ey[:, :, :D]), "vt": (vt, u * vt.abs() + Ey[:, :, D:]),
               "alpha": (alpha, ((d + 8 * eps) * a).t()), "bias": (bias, torch.cat(
                   [(a * dx + 8 * eps * (1 + bias.t().abs().max()))[1:], torch.zeros_like(dx[:1])]).t()),
               "dk": (k.grad, dk_bound), "dv": (v.grad, u * v.grad.abs() + rows[:, :, D:]),
               "dq0": (q0.grad, u * q0.grad.abs() + dq_bound)}
    return {name: (x.detach(), y + 1e-30) for name, (x, y) in res.items()}


def loss_all(hidden, weight, targets, dloss, dtype):
    """Losses, gradients and their bounds, as {name: (value, bound)}."""
    u = U[dtype]
    h, w = (t.detach().double().requires_grad_() for t in (hidden, weight))
    logits = h @ w.t()
    lse = torch.logsumexp(logits, 1)
    counts = targets >= 0
    at = targets.long().clamp(min=0)[:, None]
    loss = torch.where(counts, lse - logits.gather(1, at)[:, 0], torch.zeros((), dtype=torch.float64))
    (loss * torch.where(counts, dloss.double(), torch.zeros((), dtype=torch.float64))).sum().backward()
    with torch.no_grad():
        e = 2.0 ** -22 * (8 + (h.abs() @ w.abs().t()).max())
        g = (torch.exp(logits - lse[:, None]) + torch.nn.functional.one_hot(at[:, 0], w.shape[0])).abs()
        g = g * torch.where(counts, dloss.double().abs(), torch.zeros((), dtype=torch.float64))[:, None]
        return {name: (x.detach(), y + 1e-30) for name, (x, y) in {
            "loss": (loss, e + 2.0 ** -23 * lse.abs()), "lse": (lse, e + 2.0 ** -23 * lse.abs()),
            "dhidden": (h.grad, u * h.grad.abs() + (u + 2 * e) * (g @ w.abs())),
            "dweight": (w.grad, u * w.grad.abs() + (u + 2 * e) * (g.t() @ h.abs()))}.items()}
