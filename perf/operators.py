"""The operators of a retrofitting step as cases that can be timed.

Teaching a model to compress its cache takes, per layer and step, three pieces of
work beside the plain matrix products:

  states     the relaxed compression: gates from k[0], q[0] and logistic noise,
             alpha = sigmoid((k[0] - offset + noise) / temperature), omega =
             sigmoid(mean of the group's q[0]), and the running states
               z_t = alpha_t z_{t-1} + omega_t
               k~_t = (alpha_t z_{t-1} k~_{t-1} + omega_t k_t) / z_t, v~_t alike,
             of every token (k_t[0] = 0; a sequence's first token has alpha = 0),
             with bias_j = log(1 - alpha_{j+1}) (0 for a sequence's last token).
             Its gradient goes to k, v and the queries' first components.
  attention  query i over the states j <= i of its sequence, score
             q_i . k~_j / sqrt(d) + bias_j for j < i, without bias for j = i;
             packed sequences, grouped queries. Its gradient goes to q, k~, v~ and
             the bias.
  loss       softmax cross entropy of hidden states against a vocabulary, the logits
             hidden weight^T never kept; its gradient goes to both. A target below
             zero is an ignored position.

A case with "train" is one forward and one backward pass, given the gradients of
the forward's outputs; without it the forward alone (evaluation).

Distributions: k and v at scale 0.5, queries at scale 2, so that scores spread by
about one; k[0] on either side of the offset, so that a fraction of the tokens
merges, with logistic noise at the temperature 0.1, which makes most decisions
nearly binary; logits of standard deviation 2.
"""
import math

import torch

own = False

_GOLDEN = 0.6180339887498949
_OFFSET, _TEMPERATURE = 5.0, 0.1


# ---------------------------------------------------------------- cases

def _tokens(name, kind, **kw):
    """A case of packed sequences: `seqs` of them, lengths between lo and hi."""
    c = {"name": name, "kind": kind, "train": True, "dtype": "bf16", "q_heads": 32, "kv_heads": 32, "head_dim": 128,
         "seqs": 1, "lo": 2048, "hi": 2048}
    c.update(kw)
    return c


def _loss(name, **kw):
    c = {"name": name, "kind": "loss", "train": True, "dtype": "bf16", "tokens": 4096, "hidden": 4096,
         "vocab": 32000, "ignored": 0.0}
    c.update(kw)
    return c


def listed():
    return [
        # the smallest configuration, one short sequence in fp32: launches and latency
        _tokens("states_tiny_f32", "states", dtype="f32", q_heads=4, kv_heads=4, head_dim=64, lo=256, hi=256),
        # a training batch of the 7B shape: four sequences of 2048 tokens
        _tokens("states_7b", "states", seqs=4),
        # sequences of very different lengths packed together, 70B shape: eight queries per KV head
        _tokens("states_70b_ragged", "states", q_heads=64, kv_heads=8, seqs=6, lo=19, hi=4099),
        # the smallest configuration in fp32, forward and backward
        _tokens("attention_tiny_f32", "attention", dtype="f32", q_heads=4, kv_heads=4, head_dim=64, lo=256, hi=256),
        # evaluation of many short texts: forward alone, from one token upwards
        _tokens("attention_short", "attention", train=False, q_heads=32, kv_heads=8, seqs=24, lo=1, hi=211),
        # a training batch of the 7B shape
        _tokens("attention_7b", "attention", seqs=4),
        # one long sequence of the 70B shape, the gradients of a KV head summed over its eight queries
        _tokens("attention_70b", "attention", q_heads=64, kv_heads=8, lo=8192, hi=8192),
        # packed sequences of odd lengths, heads of 64, five queries per KV head
        _tokens("attention_ragged_d64", "attention", q_heads=40, kv_heads=8, head_dim=64, seqs=7, lo=101, hi=2999),
        # a small model's loss in fp32, a vocabulary of odd size
        _loss("loss_tiny_f32", dtype="f32", tokens=257, hidden=256, vocab=1009, ignored=0.1),
        # the perplexity of a short text: forward alone
        _loss("loss_forward_7b", train=False, tokens=1000),
        # a training batch of the 7B shape
        _loss("loss_7b", tokens=8192),
        # the 70B shape, with masked positions, odd numbers of tokens and words
        _loss("loss_70b_odd", tokens=6001, hidden=8192, vocab=32003, ignored=0.3),
    ]


def draw(rng):
    def spread(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return n - 1 if n == 3072 else n

    kind = rng.choice(["states", "attention", "attention", "loss"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    train = rng.random() < 0.75
    if kind == "loss":
        c = _loss("", train=train, dtype=dtype, tokens=spread(1, 8192), hidden=8 * spread(8, 1024),
                  vocab=spread(100, 130000), ignored=rng.choice([0.0, 0.1, 0.5]))
        while c["tokens"] * c["hidden"] * c["vocab"] > (1.0e12 if dtype == "bf16" else 1.0e11):
            c["tokens"], c["vocab"] = c["tokens"] // 2 + 1, c["vocab"] * 3 // 4
        if c["hidden"] == 3072:
            c["hidden"] += 8
    else:
        hq, hkv = rng.choice([(32, 32), (40, 40), (64, 8), (32, 8), (40, 8), (16, 8), (8, 8), (4, 4)])
        hi = spread(2, 8192)
        c = _tokens("", kind, train=train, dtype=dtype, q_heads=hq, kv_heads=hkv, head_dim=rng.choice([128, 128, 64]),
                    seqs=spread(1, 64), hi=hi, lo=hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 0.9))))
        # the plain form holds matrices of seqs x heads x hi x hi
        heads = hq if kind == "attention" else hkv
        most = (3.5e9 if kind == "attention" else 8e8) * (1.0 if dtype == "bf16" else 0.25)
        while c["seqs"] * heads * c["hi"] ** 2 > most or c["seqs"] * c["hi"] > 32768:
            if c["seqs"] > 1:
                c["seqs"] = (c["seqs"] + 1) // 2
            else:
                c["hi"] = c["hi"] * 3 // 4
                c["lo"] = min(c["lo"], c["hi"])
    del c["name"]
    return c


def _lengths(c):
    """Tokens of every sequence, between lo and hi."""
    lo, hi = c["lo"], c["hi"]
    return [lo + int((hi - lo + 1) * ((0.5 + i * _GOLDEN) % 1.0)) for i in range(c["seqs"])]


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "loss":
        n, h, v = c["tokens"], c["hidden"], c["vocab"]
        nbytes, flops = (n + v) * h * es + n * (4 + 8), 2.0 * n * h * v  # matrices, targets, loss and its log-sum
        if c["train"]:
            nbytes, flops = nbytes + (n + v) * h * es + n * 4, 3 * flops
        return {"bytes": nbytes, "flops": flops}
    lens, D, Hq, H = _lengths(c), c["head_dim"], c["q_heads"], c["kv_heads"]
    T, row = sum(lens), D * es
    if c["kind"] == "states":
        nbytes = T * (4.0 * H * row + Hq * es + H * 12)  # k, v, the states, q[0]; noise, alpha, bias
        flops = T * H * (2 * D * 3.0)
        if c["train"]:  # the states' gradients, those of k and v, of q[0]; of alpha and bias
            nbytes, flops = nbytes + T * (4.0 * H * row + Hq * es + H * (4 + es)), 4 * flops
        return {"bytes": nbytes, "flops": flops}
    pairs = sum(n * (n + 1) / 2.0 for n in lens)
    nbytes, flops = T * ((2.0 * Hq + 2 * H) * row + 4 * Hq + 4 * H), 4.0 * pairs * Hq * D
    if c["train"]:
        nbytes, flops = nbytes + T * ((2.0 * Hq + 2 * H) * row + es * H), flops + 10.0 * pairs * Hq * D
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------- inputs

def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    if c["kind"] == "loss":
        n, h, v = c["tokens"], c["hidden"], c["vocab"]
        x = {"hidden": normal(n, h), "weight": normal(v, h, scale=2.0 / math.sqrt(h))}
        targets = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
        skip = torch.rand(n, generator=g, device="cuda") < c["ignored"]
        x["targets"] = torch.where(skip, -100, targets).to(torch.int32)
        if c["train"]:  # the mean's gradient, with a weight for each position
            x["dloss"] = torch.rand(n, generator=g, device="cuda").add_(0.5).div_(n)
        return x
    lens, D, Hq, H = _lengths(c), c["head_dim"], c["q_heads"], c["kv_heads"]
    T = sum(lens)
    x = {"cu": torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32).cuda(), "longest": max(lens)}
    u = torch.rand(H, T, generator=g, device="cuda").clamp_(1e-6, 1 - 1e-6)
    noise = torch.log(u) - torch.log1p(-u)
    gate = normal(T, H, dtype=torch.float32).abs_().add_(0.1).mul_(0.5)
    gate *= torch.where(torch.rand(T, H, generator=g, device="cuda") < 0.5, -1.0, 1.0)
    x["k"], x["v"] = normal(T, H, D, scale=0.5), normal(T, H, D, scale=0.5)
    if c["kind"] == "states":
        x["q0"] = normal(T, Hq, scale=0.5)
        x["k"][..., 0] = (gate + _OFFSET).to(dt)
        x["noise"] = noise
        if c["train"]:
            x["dkt"], x["dvt"] = normal(T, H, D), normal(T, H, D)
            x["dbias"] = normal(H, T)
            x["dalpha"] = normal(H, T, dtype=torch.float32)
        return x
    x["q"] = normal(T, Hq, D, scale=2.0)
    x["k"][..., 0] = 0.0
    x["bias"] = -torch.nn.functional.softplus((gate.t() + noise * _TEMPERATURE) / _TEMPERATURE).contiguous()
    if c["train"]:
        x["dout"] = normal(T, Hq, D)
    return x


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    if own:
        from paper_2403_09636_gb300.retrofit import DmcRetrofit

        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        if c["kind"] == "loss":
            s["dmc"] = DmcRetrofit(dtype=dt, max_tokens=c["tokens"], hidden=c["hidden"], vocab=c["vocab"])
        else:
            s["dmc"] = DmcRetrofit(c["q_heads"], c["kv_heads"], c["head_dim"], dtype=dt, max_tokens=sum(_lengths(c)),
                                   max_seqs=c["seqs"])
    else:
        s["at"] = _positions(c) if c["kind"] != "loss" else None
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    return globals()["_own_" + c["kind"] if own else "_plain_" + c["kind"]](c, s)


def _own_states(c, s):
    seqs = (s["cu"], s["longest"])
    gates = {"noise": s["noise"], "offset": _OFFSET, "temperature": _TEMPERATURE}
    kt, vt, alpha, bias, saved = s["dmc"].states(s["q0"], s["k"], s["v"], *seqs, **gates)
    out = {"kt": kt, "vt": vt, "alpha": alpha, "bias": bias}
    if c["train"]:
        out["dq0"], out["dk"], out["dv"] = s["dmc"].states_backward(
            s["q0"], s["k"], s["v"], *seqs, saved, s["dkt"], s["dvt"], s["dbias"], s["dalpha"], **gates)
    return out


def _own_attention(c, s):
    a = (s["q"], s["k"], s["v"])
    o, lse = s["dmc"].attention(*a, s["cu"], s["longest"], s["bias"])
    out = {"out": o, "lse": lse}
    if c["train"]:
        out["dq"], out["dk"], out["dv"], out["dbias"] = s["dmc"].attention_backward(
            s["dout"], *a, o, lse, s["cu"], s["longest"], s["bias"])
    return out


def _own_loss(c, s):
    a = (s["hidden"], s["weight"], s["targets"])
    loss, lse = s["dmc"].loss(*a)
    out = {"loss": loss, "lse": lse}
    if c["train"]:
        out["dhidden"], out["dweight"] = s["dmc"].loss_backward(s["dloss"], *a, lse)
    return out


# ---- the plain form: 32 bits, padded sequences

def _positions(c):
    """Where each position of the padded sequences is among the packed tokens [seqs, hi], which of them are
    tokens, and those in packed order."""
    lens = torch.tensor(_lengths(c), device="cuda")
    cu = lens.cumsum(0) - lens
    t = torch.arange(int(lens.max()), device="cuda")
    valid = t < lens[:, None]
    return torch.where(valid, cu[:, None] + t, 0), valid, valid.reshape(-1).nonzero()[:, 0]


def _pad(x, at):
    """Packed [T, heads, ...] as [seqs, heads, hi, ...] in 32 bits, zero beyond a sequence's end."""
    y = x.float()[at[0]]
    y = torch.where(at[1].reshape(at[1].shape + (1,) * (y.dim() - 2)), y, 0.0)
    return y.transpose(1, 2).contiguous()


def _pack(y, at, dtype):
    """[seqs, heads, hi, ...] back as [T, heads, ...], rounded once."""
    y = y.transpose(1, 2)
    return y.reshape(-1, *y.shape[2:])[at[2]].to(dtype)


def _pack_heads(y, at, dtype):
    """[seqs, heads, hi] as [heads, T]."""
    return _pack(y, at, dtype).t().contiguous()


def _log_sigmoid(x):
    return torch.clamp(x, max=0.0) - torch.log1p(torch.exp(-x.abs()))


def _plain_states(c, s):
    at, dt, H = s["at"], s["k"].dtype, c["kv_heads"]
    B, L = at[0].shape
    k, v, noise = _pad(s["k"], at), _pad(s["v"], at), _pad(s["noise"].t(), at)
    x = (k[..., 0] - _OFFSET + noise) / _TEMPERATURE                       # [B, H, L]
    first = (torch.arange(L, device="cuda") == 0).expand(x.shape)
    last = at[1] & ~torch.cat([at[1][:, 1:], torch.zeros_like(at[1][:, :1])], 1)
    alpha = torch.where(first, 0.0, 1.0 / (1.0 + torch.exp(-x)))
    log_keep = _log_sigmoid(-x)                                            # log(1 - alpha)
    bias = torch.where(last[:, None], 0.0, torch.cat([log_keep[..., 1:], torch.zeros_like(x[..., :1])], -1))
    omega = 1.0 / (1.0 + torch.exp(-_pad(s["q0"], at).reshape(B, H, -1, L).mean(2)))
    # decay[t, j] = alpha_{j+1} ... alpha_t
    i = torch.arange(L, device="cuda")
    below = i[:, None] > i
    decay = torch.where(below, torch.where(first, -math.inf, _log_sigmoid(x))[..., None], 0.0).cumsum_(-2).exp_()
    decay.mul_(i[:, None] >= i)
    kv = torch.cat([k, v], -1)
    kv[..., 0] = 0.0
    total = decay @ (omega[..., None] * kv)
    z = (decay @ omega[..., None])
    y = total / z
    D = c["head_dim"]
    out = {"kt": _pack(y[..., :D], at, dt), "vt": _pack(y[..., D:], at, dt), "alpha": _pack_heads(alpha, at, torch.float32),
           "bias": _pack_heads(bias, at, torch.float32)}
    if c["train"]:
        dy = torch.cat([_pad(s["dkt"], at), _pad(s["dvt"], at)], -1)
        dy[..., 0] = 0.0
        dbias, dalpha = _pad(s["dbias"].t(), at), _pad(s["dalpha"].t(), at)
        up = decay.transpose(-1, -2)
        lam = up @ (dy / z)                                                # gradient of the sums
        zeta = up @ (-(dy * y).sum(-1, keepdim=True) / z)                  # gradient of z
        domega = (lam * kv).sum(-1) + zeta[..., 0]
        before = torch.cat([torch.zeros_like(total[..., :1, :]), total[..., :-1, :]], -2)
        zbefore = torch.cat([torch.zeros_like(z[..., :1, :]), z[..., :-1, :]], -2)
        da = dalpha + (lam * before).sum(-1) + (zeta * zbefore)[..., 0]
        dlog = torch.cat([torch.zeros_like(x[..., :1]), dbias[..., :-1]], -1)  # of log(1 - alpha) at its own token
        dx = torch.where(first, 0.0, da * alpha / (1.0 + torch.exp(x)) - dlog * alpha)
        dkv = omega[..., None] * lam
        dkv[..., 0] = dx / _TEMPERATURE
        G = c["q_heads"] // H
        dq0 = (domega * omega * (1.0 - omega) / G)[:, :, None].expand(B, H, G, L).reshape(B, H * G, L)
        out |= {"dq0": _pack(dq0, at, dt), "dk": _pack(dkv[..., :D], at, dt), "dv": _pack(dkv[..., D:], at, dt)}
    return out


def _plain_attention(c, s):
    at, dt, D, H, G = s["at"], s["q"].dtype, c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    B, L = at[0].shape
    scale = 1.0 / math.sqrt(D)
    q, k, v, bias = _pad(s["q"], at), _pad(s["k"], at), _pad(s["v"], at), _pad(s["bias"].t(), at)
    q = q.view(B, H, G * L, D)
    i = torch.arange(L, device="cuda")
    mask = torch.where(i[:, None] > i, bias[..., None, :], torch.where(i[:, None] == i, 0.0, -math.inf))
    p = (q @ k.transpose(-1, -2)).view(B, H, G, L, L).mul_(scale).add_(mask[:, :, None])
    m = p.amax(-1, keepdim=True)
    p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    p.div_(l)
    o = p.view(B, H, G * L, L) @ v
    lse = (m + torch.log(l)).view(B, H * G, L)
    out = {"out": _pack(o.view(B, H * G, L, D), at, dt), "lse": _pack_heads(lse, at, torch.float32)}
    if c["train"]:
        do = _pad(s["dout"], at).view(B, H, G * L, D)
        dv = p.view(B, H, G * L, L).transpose(-1, -2) @ do
        ds = (do @ v.transpose(-1, -2)).view(B, H, G, L, L)
        ds.sub_((do * o).sum(-1).view(B, H, G, L, 1)).mul_(p)
        db = ds.sum((2, 3)) - ds.diagonal(dim1=-2, dim2=-1).sum(2)
        ds = ds.view(B, H, G * L, L)
        dq = (ds @ k).mul_(scale)
        dk = (ds.transpose(-1, -2) @ q).mul_(scale)
        out |= {"dq": _pack(dq.view(B, H * G, L, D), at, dt), "dk": _pack(dk, at, dt), "dv": _pack(dv, at, dt),
                "dbias": _pack_heads(db, at, dt)}
    return out


def _plain_loss(c, s):
    dt, targets = s["hidden"].dtype, s["targets"].long()
    h, w = s["hidden"].float(), s["weight"].float()
    logits = h @ w.t()
    m = logits.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(logits - m).sum(1, keepdim=True)))[:, 0]
    counts = targets >= 0
    at = targets.clamp(min=0)[:, None]
    loss = torch.where(counts, lse - logits.gather(1, at)[:, 0], 0.0)
    out = {"loss": loss, "lse": lse}
    if c["train"]:
        p = logits.sub_(lse[:, None]).exp_()
        p.scatter_add_(1, at, torch.full_like(lse, -1.0)[:, None])
        p.mul_(torch.where(counts, s["dloss"], 0.0)[:, None])
        out |= {"dhidden": (p @ w).to(dt), "dweight": (p.t() @ h).to(dt)}
    return out


# ---------------------------------------------------------------- the same in 64 bits, one sequence or block at a time

def exact(case, seed):
    c = case
    if work(c)["flops"] > 1.3e13:
        return None
    return globals()["_exact_" + c["kind"]](c, _inputs(c, seed))


def _spans(c):
    b = 0
    for n in _lengths(c):
        yield b, b + n
        b += n


def _exact_states(c, x):
    H, D = c["kv_heads"], c["head_dim"]
    names = ["kt", "vt", "alpha", "bias"] + (["dq0", "dk", "dv"] if c["train"] else [])
    parts = {n: [] for n in names}
    for a, b in _spans(c):
        n = b - a
        leaf = [x[i][a:b].double() for i in ("q0", "k", "v")]
        q0, k, v = leaf
        logit = (k[:, :, 0] - _OFFSET + x["noise"][:, a:b].double().t()) / _TEMPERATURE   # [n, H]
        alpha = torch.sigmoid(logit)
        alpha[0] = 0.0
        bias = torch.zeros_like(logit)
        bias[:-1] = torch.nn.functional.logsigmoid(-logit[1:])
        omega = torch.sigmoid(q0.view(n, H, -1).mean(2))
        row = torch.cat([k, v], 2)
        row[:, :, 0] = 0.0
        ys, zs = [], []
        y, z = torch.zeros_like(row[0]), torch.zeros_like(omega[0])
        for t in range(n):  # the definition, token by token
            old = alpha[t] * z
            z = old + omega[t]
            y = (old[:, None] * y + omega[t][:, None] * row[t]) / z[:, None]
            ys.append(y)
            zs.append(z)
        y, z = torch.stack(ys), torch.stack(zs)
        got = {"kt": y[:, :, :D], "vt": y[:, :, D:], "alpha": alpha.t(), "bias": bias.t()}
        if c["train"]:
            # its chain rule, token by token from the last
            g = torch.cat([x["dkt"][a:b], x["dvt"][a:b]], 2).double()
            g[:, :, 0] = 0.0
            drow, domega, dalpha = torch.zeros_like(row), torch.zeros_like(omega), x["dalpha"][:, a:b].double().t().clone()
            gy, gz = torch.zeros_like(y[0]), torch.zeros_like(z[0])
            for t in range(n - 1, -1, -1):
                gy = gy + g[t]
                zp = z[t - 1] if t else torch.zeros_like(gz)
                yp = y[t - 1] if t else torch.zeros_like(gy)
                share, old = gy / z[t][:, None], alpha[t] * zp       # y_t = (old yp + omega row) / (old + omega)
                drow[t] = share * omega[t][:, None]
                domega[t] = (share * (row[t] - y[t])).sum(1) + gz
                dold = (share * (yp - y[t])).sum(1) + gz
                dalpha[t] += dold * zp
                gz = dold * alpha[t]
                gy = share * old[:, None]
            # z_t's own gradient has gone into domega and dold: z_t = old + omega
            dl = dalpha * torch.sigmoid(logit) * torch.sigmoid(-logit)
            dl[1:] -= x["dbias"][:, a:b].double().t()[:-1] * alpha[1:]
            dl[0] = 0.0
            drow[:, :, 0] = dl / _TEMPERATURE
            G = c["q_heads"] // H
            dq0 = (domega * omega * (1 - omega) / G)[:, :, None].expand(n, H, G).reshape(n, H * G)
            got |= {"dq0": dq0, "dk": drow[:, :, :D], "dv": drow[:, :, D:]}
        for name in names:
            parts[name].append(got[name])
    return {n: torch.cat(p, 1 if n in ("alpha", "bias") else 0) for n, p in parts.items()}


def _exact_attention(c, x):
    H, G, D = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    names = ["out", "lse"] + (["dq", "dk", "dv", "dbias"] if c["train"] else [])
    T = x["q"].shape[0]
    res = {n: torch.zeros(x["k" if n in ("dk", "dv") else "q"].shape, dtype=torch.float64, device="cuda") for n in names}
    for n, h in (("lse", H * G), ("dbias", H)):
        if n in names:
            res[n] = torch.zeros(h, T, dtype=torch.float64, device="cuda")
    for a, b in _spans(c):
        step = max(1, min(b - a, int(2e8 // (H * G * (b - a)))))
        for i0 in range(a, b, step):  # rows i0 .. i1 see the tokens a .. i1
            i1 = min(b, i0 + step)
            q = x["q"][i0:i1].double().view(i1 - i0, H, G, D).permute(1, 2, 0, 3)       # [H, G, i, D]
            k, v = (x[n][a:i1].double().permute(1, 0, 2)[:, None] for n in ("k", "v"))  # [H, 1, j, D]
            at = torch.arange(i0 - a, i1 - a, device="cuda")[:, None] - torch.arange(i1 - a, device="cuda")
            score = q @ k.transpose(-1, -2) / math.sqrt(D)
            score = score + x["bias"][:, None, None, a:i1].double() * (at > 0)
            score = score.masked_fill(at < 0, -math.inf)
            lse = torch.logsumexp(score, -1)
            p = torch.exp(score - lse[..., None])
            o = p @ v
            res["out"][i0:i1] = o.permute(2, 0, 1, 3).reshape(i1 - i0, H * G, D)
            res["lse"][:, i0:i1] = lse.reshape(H * G, -1)
            if c["train"]:
                do = x["dout"][i0:i1].double().view(i1 - i0, H, G, D).permute(1, 2, 0, 3)
                dp = do @ v.transpose(-1, -2)
                ds = p * (dp - (p * dp).sum(-1, keepdim=True))
                res["dq"][i0:i1] = (ds @ k / math.sqrt(D)).permute(2, 0, 1, 3).reshape(i1 - i0, H * G, D)
                res["dk"][a:i1] += (ds.transpose(-1, -2) @ q / math.sqrt(D)).sum(1).permute(1, 0, 2)
                res["dv"][a:i1] += (p.transpose(-1, -2) @ do).sum(1).permute(1, 0, 2)
                res["dbias"][:, a:i1] += (ds * (at > 0)).sum((1, 2))
    return res


def _exact_loss(c, x):
    h, w = x["hidden"].double(), x["weight"].double()
    t = x["targets"].long()
    n, v = c["tokens"], c["vocab"]
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    step = max(1, int(5e8 // v))
    for a in range(0, n, step):
        b = min(n, a + step)
        logits = h[a:b] @ w.t()
        lse[a:b] = torch.logsumexp(logits, 1)
        word = torch.arange(v, device="cuda") == t[a:b, None]
        loss[a:b] = torch.where(t[a:b] < 0, 0.0, lse[a:b] - (logits * word).sum(1))
        if c["train"]:
            g = (torch.softmax(logits, 1) - word.double()) * torch.where(t[a:b] < 0, 0.0, x["dloss"][a:b].double())[:, None]
            dh[a:b] = g @ w
            dw += g.t() @ h[a:b]
    return {"loss": loss, "lse": lse} | ({"dhidden": dh, "dweight": dw} if c["train"] else {})
