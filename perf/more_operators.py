"""Generating text from a compressed cache, as cases that can be timed.

A program that serves a model with rotary positions, with beams, does five things
beside the model's own matrix products:

  rotate   the position rotation of queries and keys: pair i of a head (dims i and
           i + D/2, or 2i and 2i + 1) turns by position * frequency_i. Dimension 0
           is the gate of the compression, so its pair stays as it is. Its gradient
           is the rotation back.
  append   new tokens join the compressed cache, rotated on the way: a token with
           k[0] >= 0 merges into the head's last slot, another opens one; a slot is
           the omega-weighted mean of its tokens, omega = sigmoid(mean of the
           group's q[0]), z the sum of its omegas. The rotated queries come back.
           Prompts of any lengths, then single tokens.
  attend   one new token's queries over every slot of their KV head, score
           q . k / sqrt(D) without dimension 0 (k[0] is 0 in the cache).
  select   the `keep` best continuations of each group of beams: score of beam b and
           word w: scores[b] + logits[b, w] - logsumexp(logits[b]); a finished beam
           has one continuation, the end word at an unchanged score. Ties go to the
           lower b * vocab + w.
  reorder  the caches follow their beams: sequence j continues from the cache of
           sequence parents[j]. The state comes back whole, as padded tensors.

Distributions: k and v at scale 0.5; queries at scale 2, so that scores spread by
about one; a token opens a slot with probability 1 / ratio; logits of standard
deviation 2.5, sums of log probabilities between -40 and 0.
"""
import math

import torch

own = False

_BASE = 10000.0
_GOLDEN = 0.6180339887498949


# ---------------------------------------------------------------- cases

def _heads(name, kind, **kw):
    c = {"name": name, "kind": kind, "dtype": "bf16", "q_heads": 32, "kv_heads": 32, "head_dim": 128}
    c.update(kw)
    return c


def _rotate(name, **kw):
    return _heads(name, "rotate", **{"tokens": 8192, "train": True, "interleaved": False, "far": 8192, **kw})


def _append(name, **kw):
    """`seqs` prompts of lengths between lo and hi, then `steps` single tokens for each."""
    return _heads(name, "append", **{"seqs": 1, "lo": 2048, "hi": 2048, "steps": 1, "ratio": 4.0, "interleaved": False,
                                     "far": 0, **kw})


def _attend(name, **kw):
    return _heads(name, "attend", **{"seqs": 1, "lo": 2048, "hi": 2048, "ratio": 4.0, **kw})


def _select(name, **kw):
    c = {"name": name, "kind": "select", "dtype": "bf16", "groups": 1, "beams": 4, "keep": 4, "vocab": 32000,
         "finished": 0.0}
    c.update(kw)
    return c


def _reorder(name, **kw):
    return _heads(name, "reorder", **{"layers": 4, "groups": 1, "beams": 4, "lo": 2048, "hi": 2048, "ratio": 4.0, **kw})


def listed():
    return [
        # one step's queries and keys of a few sequences: launches and latency
        _rotate("rotate_step", tokens=4, train=False, far=32000),
        # a training batch of the 7B shape, forward and backward
        _rotate("rotate_7b"),
        # a short chat turn: a prompt of 59 tokens, then sixteen single tokens
        _append("append_chat", lo=59, hi=59, steps=16),
        # prompts of the 7B shape handed over at once
        _append("append_7b", seqs=8),
        # ragged prompts of the 70B shape that continue far texts, interleaved pairs
        _append("append_70b_ragged", q_heads=64, kv_heads=8, seqs=6, lo=19, hi=4099, ratio=2.0, interleaved=True,
                far=100000),
        # the smallest configuration in fp32: launches and latency
        _attend("attend_tiny_f32", dtype="f32", q_heads=4, kv_heads=4, head_dim=64, lo=256, hi=256, ratio=2.0),
        # a serving batch of the 7B shape
        _attend("attend_7b", seqs=32),
        # one long text, eight queries per KV head: split over the cache's length
        _attend("attend_long", q_heads=64, kv_heads=8, lo=65536, hi=65536, ratio=1.5),
        # four beams of one text: latency
        _select("select_4_beams"),
        # a batch of groups in fp32 over a large vocabulary of odd size, more kept than beams, some beams at their end
        _select("select_batch_f32", dtype="f32", groups=32, beams=8, keep=16, vocab=130003, finished=0.1),
        # four beams of one text, two places taken by copies of the others
        _reorder("reorder_4_beams"),
        # groups of beams of ragged texts, grouped queries
        _reorder("reorder_batch", q_heads=64, kv_heads=8, layers=8, groups=8, beams=8, lo=101, hi=2999, ratio=2.0),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rotate", "append", "append", "attend", "attend", "select", "select", "reorder"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "select":
        beams = rng.randint(1, 16)
        c = _select("", dtype=dtype, groups=spread(1, 64), beams=beams, keep=rng.choice([beams, min(2 * beams, 32), 1]),
                    vocab=spread(50, 130003), finished=rng.choice([0.0, 0.1, 0.5]))
        while c["groups"] * c["beams"] * c["vocab"] > 32 * 8 * 130003:
            c["groups"] = c["groups"] // 2
        del c["name"]
        return c
    hq, hkv = rng.choice([(32, 32), (40, 40), (64, 8), (32, 8), (40, 8), (16, 8), (8, 8), (4, 4)])
    shape = {"dtype": dtype, "q_heads": hq, "kv_heads": hkv, "head_dim": rng.choice([128, 128, 64])}
    ratio = rng.choice([1.0, 1.5, 2.0, 4.0, 8.0])
    if kind == "rotate":
        c = _rotate("", tokens=spread(1, 8192), train=rng.random() < 0.6, interleaved=rng.random() < 0.4,
                    far=spread(1, 1000000), **shape)
        while c["tokens"] * (hq + hkv) * c["head_dim"] * (4 if dtype == "f32" else 2) > 8192 * 64 * 256:
            c["tokens"] //= 2
    else:
        hi = spread(2, 4099)
        lo = hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.02, 0.9)))
        row = hkv * shape["head_dim"] * (4 if dtype == "f32" else 2)
        if kind == "append":
            c = _append("", seqs=spread(1, 32), lo=lo, hi=hi, steps=rng.choice([0, 1, 1, 3, 16]), ratio=ratio,
                        interleaved=rng.random() < 0.4, far=rng.choice([0, 0, 5000, 300000]), **shape)
            row, most = row + hq * row // hkv, 8 * 2048 * 64 * 256
            while c["seqs"] * c["hi"] * row > most:
                c["seqs"], c["hi"] = (c["seqs"] + 1) // 2, c["hi"] * 3 // 4
        elif kind == "attend":
            c = _attend("", seqs=spread(1, 64), lo=lo, hi=hi, ratio=ratio, **shape)
            while c["seqs"] * c["hi"] * row > 32 * 2048 * 32 * 256:
                c["seqs"], c["hi"] = (c["seqs"] + 1) // 2, c["hi"] * 3 // 4
        else:
            c = _reorder("", layers=rng.randint(1, 8), groups=spread(1, 16), beams=rng.randint(2, 8), lo=lo, hi=hi,
                         ratio=ratio, **shape)
            while c["layers"] * c["groups"] * c["beams"] * c["hi"] * row / ratio > 8 * 64 * 2999 * 8 * 128:
                c["groups"], c["hi"] = (c["groups"] + 1) // 2, c["hi"] * 3 // 4
        c["hi"] = max(1, c["hi"])
        c["lo"] = min(c["lo"], c["hi"])
    del c["name"]
    return c


def _lengths(c):
    """Tokens of every text, between lo and hi."""
    lo, hi = c["lo"], c["hi"]
    n = c["groups"] if c["kind"] == "reorder" else c["seqs"]
    return [lo + int((hi - lo + 1) * ((0.5 + i * _GOLDEN) % 1.0)) for i in range(n)]


def _cap(c):
    """Slots that no head of a case passes: six standard deviations above the most tokens over the ratio."""
    n, p = max(_lengths(c)) + c.get("steps", 0), 1.0 / c["ratio"]
    return min(n, int(n * p + 6.0 * math.sqrt(n * p * (1.0 - p))) + 8)


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        return {"bytes": rows * (c["vocab"] * es + 5.0) + c["groups"] * c["keep"] * 13.0, "flops": 4.0 * rows * c["vocab"]}
    Hq, H, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    row = D * es
    if c["kind"] == "rotate":
        n = c["tokens"] * (2 if c["train"] else 1)
        return {"bytes": 2.0 * n * (Hq + H) * row + 4.0 * c["tokens"], "flops": 3.0 * n * (Hq + H) * D}
    T = float(sum(_lengths(c)))
    if c["kind"] == "attend":
        slots = T / c["ratio"] * H
        return {"bytes": slots * 2 * row + 2.0 * c["seqs"] * Hq * row, "flops": 4.0 * slots * (Hq // H) * D}
    if c["kind"] == "append":
        T += c["steps"] * c["seqs"]
        slots = T / c["ratio"] * H
        return {"bytes": T * (2.0 * Hq + 2 * H) * row + slots * (2 * row + 4), "flops": T * (3.0 * Hq + 7.0 * H) * D}
    slots = c["layers"] * c["beams"] * T / c["ratio"] * H
    return {"bytes": 2.0 * slots * (2 * row + 4), "flops": 0.0}


# ---------------------------------------------------------------- inputs

def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _inv_freq(D):
    """Radians per token of each pair."""
    return (_BASE ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float()


class _Draw:
    def __init__(self, c, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))
        self.dt = _type(c)

    def normal(self, *shape, scale=1.0, dtype=None):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=dtype or self.dt).mul_(scale)

    def rand(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def gate(self, T, H, ratio):
        """k[0] of tokens that open a slot with probability 1 / ratio: below zero where they do."""
        size = self.normal(T, H, dtype=torch.float32).abs_().add_(0.1).mul_(0.5)
        return torch.where(self.rand(T, H) * ratio < 1.0, -size, size).to(self.dt)


def _cu(lens):
    return torch.tensor([0] + lens, dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _inputs(c, seed):
    d, x = _Draw(c, seed), {}
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        x["logits"] = d.normal(rows, c["vocab"], scale=2.5)
        x["scores"] = (d.rand(c["groups"], c["beams"]) * -40.0).contiguous()
        x["finished"] = d.rand(c["groups"], c["beams"]) < c["finished"]
        x["end"] = c["vocab"] // 7
        return x
    H, Hq, D = c["kv_heads"], c["q_heads"], c["head_dim"]
    if c["kind"] == "rotate":
        T = c["tokens"]
        x["q"], x["k"] = d.normal(T, Hq, D, scale=2.0), d.normal(T, H, D, scale=0.5)
        x["at"] = (d.rand(T) * c["far"]).to(torch.int32)
        if c["train"]:
            x["dq"], x["dk"] = d.normal(T, Hq, D), d.normal(T, H, D)
        return x
    lens = _lengths(c)
    T = sum(lens)
    x["cu"], x["longest"] = _cu(lens), max(lens)
    if c["kind"] == "append":
        n = T + c["steps"] * len(lens)  # the prompts' tokens, then every step's
        q, k, v = d.normal(n, Hq, D, scale=2.0), d.normal(n, H, D, scale=0.5), d.normal(n, H, D, scale=0.5)
        k[..., 0] = d.gate(n, H, c["ratio"])
        cut = lambda t: [t[:T]] + list(t[T:].view(c["steps"], len(lens), *t.shape[1:]).unbind(0))  # noqa: E731
        x["q"], x["k"], x["v"] = cut(q), cut(k), cut(v)
        start = (d.rand(len(lens)) * c["far"]).to(torch.int32)
        x["start"] = [start] + [start + (x["cu"][1:] - x["cu"][:-1]) + i for i in range(c["steps"])]
        return x
    # a cache whose slots are known: the tokens of a segment are alike, so that their mean is their value
    layers = c.get("layers", 1)
    x["q"] = d.normal(len(lens), Hq, D, scale=2.0)
    first = torch.zeros(T, dtype=torch.bool, device="cuda")
    first[x["cu"][:-1].long()] = True
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
    x["k"], x["v"], x["slots"], x["lens"] = [], [], [], []
    for _ in range(layers):
        gate = d.gate(T, H, c["ratio"])
        opens = (gate < 0) | first[:, None]
        run = opens.cumsum(0)  # [T, H]
        before = (run - opens.long())[x["cu"][:-1].long()]
        slot = run - 1 - before[seq]
        n, cap = run[x["cu"][1:].long() - 1] - before, _cap(c)  # [seqs, H]
        k, v = d.normal(len(lens), H, cap, D, scale=0.5), d.normal(len(lens), H, cap, D, scale=0.5)
        h = torch.arange(H, device="cuda")
        kt, vt = k[seq[:, None], h, slot], v[seq[:, None], h, slot]
        kt[..., 0] = gate
        k[..., 0] = 0.0
        past = torch.arange(cap, device="cuda") >= n[..., None]
        k.masked_fill_(past[..., None], 0.0)
        v.masked_fill_(past[..., None], 0.0)
        z = torch.zeros(len(lens), H, cap, device="cuda")
        z.index_put_((seq[:, None].expand(T, H), h.expand(T, H), slot), torch.full((T, H), 0.5, device="cuda"), accumulate=True)
        x["k"].append(kt)
        x["v"].append(vt)
        x["slots"].append((k, v, z))
        x["lens"].append(n.to(torch.int32))
    if c["kind"] == "reorder":
        # half of a group's beams or so stay, the others' places are taken by copies of those
        G, B = c["groups"], c["beams"]
        keep = torch.rand(G, B, generator=d.g, device="cuda") < 0.5
        keep[:, 0] |= ~keep.any(1)
        pick = torch.multinomial(keep.float(), B, replacement=True, generator=d.g)
        b = torch.arange(B, device="cuda")
        local = torch.where(keep, b, pick)
        x["parents"] = (local + torch.arange(G, device="cuda")[:, None] * B).reshape(-1).to(torch.int32)
    return x


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    s["case"] = c
    dt = _type(c)
    if c["kind"] == "select":
        if own:
            from paper_2403_09636_gb300.beam import BeamSelect

            s["beam"] = BeamSelect(c["groups"], c["beams"], c["vocab"], keep=c["keep"], dtype=dt)
        return s
    D, H, Hq = c["head_dim"], c["kv_heads"], c["q_heads"]
    if c["kind"] in ("rotate", "append"):
        if own:
            from paper_2403_09636_gb300.rotary import Rotary

            s["rotary"] = Rotary(D, inv_freq=_inv_freq(D), interleaved=c["interleaved"])
        else:
            s["freq"] = _inv_freq(D).cuda()
    if c["kind"] == "rotate":
        return s
    if c["kind"] == "append":
        n = len(_lengths(c))
        s["order"], s["cu_all"], s["cap"] = *_order(c, s), _cap(c)
        if own:
            from paper_2403_09636_gb300 import DmcCache

            pages = n * H * (-(-s["cap"] // 32) + 1)
            s["cache"] = DmcCache(1, n, Hq, H, D, dt, s["cap"], pages, s["k"][0].shape[0])
            s["ids"] = torch.arange(n * H, dtype=torch.int32, device="cuda")
        return s
    beams = c.get("beams", 1)
    s["cap"] = _cap(c)
    if own:
        from paper_2403_09636_gb300 import DmcCache

        n, lens = len(_lengths(c)) * beams, _lengths(c)
        pages = n * H * len(s["k"]) * (-(-s["cap"] // 32) + 1)
        s["cache"] = DmcCache(len(s["k"]), n, Hq, H, D, dt, s["cap"], pages, sum(lens))
        q0 = torch.zeros(sum(lens), Hq, dtype=dt, device="cuda")  # omega 1/2 everywhere
        for layer in range(len(s["k"])):
            if beams == 1:
                s["cache"].prefill(layer, q0, s["k"][layer], s["v"][layer], s["cu"], s["longest"])
            else:  # every beam begins with its group's text
                at = 0
                for i, m in enumerate(lens):
                    one = torch.tensor([0, m], dtype=torch.int32, device="cuda")
                    for b in range(beams):
                        s["cache"].prefill(layer, q0[:m], s["k"][layer][at:at + m], s["v"][layer][at:at + m], one, m,
                                           first_seq=i * beams + b)
                    at += m
        s["ids"] = torch.arange(n * H, dtype=torch.int32, device="cuda")
    else:
        s["slots"] = [tuple(t.repeat_interleave(beams, 0) for t in x) for x in s["slots"]]
        s["lens"] = [t.repeat_interleave(beams, 0) for t in s["lens"]]
        if c["kind"] == "reorder":
            s["slots"] = tuple(torch.stack(t) for t in zip(*s["slots"]))
            s["lens"] = torch.stack(s["lens"])
    del s["k"], s["v"]
    return s


def _order(c, s):
    """Where the tokens of each text are among the prompts' and the steps', text after text; and where the texts begin."""
    n, S, lens = len(s["cu"]) - 1, c["steps"], _lengths(c)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.tensor(lens, device="cuda"))
    seq = torch.cat([seq, torch.arange(n, device="cuda").repeat(S)])
    return torch.argsort(seq, stable=True), s["cu"].long() + S * torch.arange(n + 1, device="cuda")


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    return globals()["_own_" + c["kind"] if own else "_plain_" + c["kind"]](c, s)


def _own_rotate(c, s):
    from paper_2403_09636_gb300 import rotary

    q, k = rotary.rotate(s["rotary"], s["q"], s["k"], s["at"])
    out = {"q": q, "k": k}
    if c["train"]:
        out["dq"], out["dk"] = rotary.rotate(s["rotary"], s["dq"], s["dk"], s["at"], inverse=True)
    return out


def _own_append(c, s):
    cache = s["cache"]
    cache.reset()
    q = [cache.append(0, s["q"][0], s["k"][0], s["v"][0], s["start"][0], s["rotary"], cu_seqlens=s["cu"],
                      max_seqlen=s["longest"])]
    q += [cache.append(0, *x, s["rotary"]) for x in zip(s["q"][1:], s["k"][1:], s["v"][1:], s["start"][1:])]
    k, v, z, n = cache.export_heads(0, s["ids"], s["cap"])
    return {"q": q, "k": k, "v": v, "z": z, "len": n}


def _own_attend(c, s):
    return s["cache"].attend(0, s["q"])


def _own_select(c, s):
    scores, tokens, parents, done = s["beam"].select(s["logits"], s["scores"], s["finished"], s["end"])
    return {"scores": scores, "tokens": tokens, "parents": parents, "done": done}


def _own_reorder(c, s):
    s["cache"].reorder(s["parents"])
    return [s["cache"].export_heads(layer, s["ids"], s["cap"]) for layer in range(c["layers"])]


# ---- the plain form: 32 bits, angles, log-sums and what is ordered in 64

def _turned(x, at, freq, interleaved, back=False):
    """x [T, H, D] rotated to the positions at [T], in 32 bits; the pair of dimension 0 stays."""
    angle = at.double()[:, None] * freq.double()
    angle[:, 0] = 0.0
    c, s = torch.cos(angle).float()[:, None], torch.sin(-angle if back else angle).float()[:, None]
    x = x.float()
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else x.chunk(2, -1)
    a, b = a * c - b * s, b * c + a * s
    return torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)


def _plain_rotate(c, s):
    dt, how = s["q"].dtype, (s["at"], s["freq"], c["interleaved"])
    out = {"q": _turned(s["q"], *how).to(dt), "k": _turned(s["k"], *how).to(dt)}
    if c["train"]:
        out |= {"dq": _turned(s["dq"], *how, back=True).to(dt), "dk": _turned(s["dk"], *how, back=True).to(dt)}
    return out


def _plain_append(c, s):
    H, D, cap, n, dt = c["kv_heads"], c["head_dim"], s["cap"], len(s["cu"]) - 1, s["k"][0].dtype
    q, k, v = (torch.cat(s[i])[s["order"]].float() for i in ("q", "k", "v"))
    cu = s["cu_all"]
    t = torch.arange(k.shape[0], device="cuda")
    seq = torch.searchsorted(cu, t, right=True) - 1
    at = s["start"][0].long()[seq] + t - cu[seq]
    how = (at, s["freq"], c["interleaved"])
    opens = (k[..., 0] < 0) | (t == cu[seq])[:, None]
    run = opens.cumsum(0)
    before = (run - opens.long())[cu[:-1]]
    place = ((seq[:, None] * H + torch.arange(H, device="cuda")) * cap + run - 1 - before[seq]).reshape(-1)
    w = 1.0 / (1.0 + torch.exp(-q[..., 0].view(len(t), H, -1).mean(2)))
    z = torch.zeros(n * H * cap, device="cuda").index_add_(0, place, w.reshape(-1))
    kr = _turned(k, *how)
    kr[..., 0] = 0.0
    over = torch.where(z > 0, 1.0 / z, 0.0)[:, None]
    mean = lambda x: (torch.zeros(n * H * cap, D, device="cuda").index_add_(  # noqa: E731
        0, place, (x * w[..., None]).reshape(-1, D)) * over).to(dt).view(n * H, cap, D)
    turned = _turned(q, *how).to(dt)
    back = torch.empty_like(turned)
    back[s["order"]] = turned
    T = s["q"][0].shape[0]
    counts = torch.zeros(n * H * cap, dtype=torch.int32, device="cuda").index_fill_(0, place, 1)
    return {"q": [back[:T]] + list(back[T:].view(c["steps"], n, *back.shape[1:]).unbind(0)), "k": mean(kr), "v": mean(v),
            "z": z.view(n * H, cap), "len": counts.view(n * H, cap).sum(1, dtype=torch.int32)}


def _plain_attend(c, s):
    (k, v, _), n, q = s["slots"][0], s["lens"][0], s["q"]
    B, H, cap, D = k.shape
    qf = q.float().view(B, H, -1, D)
    p = (qf @ k.float().transpose(-1, -2)) / math.sqrt(D)
    there = torch.arange(cap, device="cuda") < n[:, :, None, None]
    p = torch.where(there, p, -math.inf)
    p = torch.exp(p - p.amax(-1, keepdim=True))
    return ((p / p.sum(-1, keepdim=True)) @ v.float()).view(q.shape).to(q.dtype)


def _plain_select(c, s):
    G, B, V = c["groups"], c["beams"], c["vocab"]
    x = s["logits"].double().view(G, B, V)
    m = x.amax(-1, keepdim=True)
    score = s["scores"].double()[..., None] + x - (m + torch.log(torch.exp(x - m).sum(-1, keepdim=True)))
    ends = torch.where(torch.arange(V, device="cuda") == s["end"], s["scores"].double()[..., None], -math.inf)
    score = torch.where(s["finished"][..., None], ends, score).view(G, B * V)
    best, at = torch.sort(score, stable=True, dim=1, descending=True)
    best, at = best[:, :c["keep"]], at[:, :c["keep"]]
    beam, token = at // V, at % V
    done = s["finished"].gather(1, beam) | (token == s["end"])
    return {"scores": best.float(), "tokens": token.to(torch.int32),
            "parents": (beam + torch.arange(G, device="cuda")[:, None] * B).to(torch.int32), "done": done}


def _plain_reorder(c, s):
    at = s["parents"].long()
    s["slots"] = tuple(t[:, at] for t in s["slots"])  # [layers, sequences, heads, ...]
    s["lens"] = s["lens"][:, at]
    return [tuple(t) for t in zip(*(t.flatten(1, 2).unbind(0) for t in (*s["slots"], s["lens"])))]


# ---------------------------------------------------------------- the same in 64 bits, from the definitions

def exact(case, seed):
    return globals()["_exact_" + case["kind"]](case, _inputs(case, seed))


def _complex(x, interleaved):
    x = x.double()
    return torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) if interleaved else torch.complex(*x.chunk(2, -1))


def _real(y, interleaved):
    return torch.view_as_real(y).flatten(-2) if interleaved else torch.cat([y.real, y.imag], -1)


def _turn(c, x, at, sign=1.0):
    """x times e^(i angle), the pairs as complex numbers."""
    angle = sign * at.double()[:, None] * _inv_freq(c["head_dim"]).double().cuda()
    angle[:, 0] = 0.0
    return _real(_complex(x, c["interleaved"]) * torch.polar(torch.ones_like(angle), angle)[:, None], c["interleaved"])


def _exact_rotate(c, x):
    out = {"q": _turn(c, x["q"], x["at"]), "k": _turn(c, x["k"], x["at"])}
    if c["train"]:
        out |= {"dq": _turn(c, x["dq"], x["at"], -1.0), "dk": _turn(c, x["dk"], x["at"], -1.0)}
    return out


def _exact_append(c, x):
    H, D, S, lens = c["kv_heads"], c["head_dim"], c["steps"], _lengths(c)
    n, cap = len(lens), _cap(c)
    k_out, v_out = (torch.zeros(n, H, cap, D, dtype=torch.float64, device="cuda") for _ in range(2))
    z_out = torch.zeros(n, H, cap, dtype=torch.float64, device="cuda")
    turned = [torch.zeros(q.shape, dtype=torch.float64, device="cuda") for q in x["q"]]
    a = 0
    for i, m in enumerate(lens):
        q, k, v = (torch.cat([t[0][a:a + m]] + [u[i:i + 1] for u in t[1:]]) for t in (x["q"], x["k"], x["v"]))
        at = int(x["start"][0][i]) + torch.arange(m + S, device="cuda")
        qr, kr = _turn(c, q, at), _turn(c, k, at)
        turned[0][a:a + m] = qr[:m]
        for j in range(S):
            turned[1 + j][i] = qr[m + j]
        kr[..., 0] = 0.0
        w = torch.sigmoid(q[..., 0].double().view(m + S, H, -1).mean(2))
        rows = torch.cat([kr, v.double(), torch.ones_like(kr[..., :1])], -1) * w[..., None]
        sums = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)])
        for h in range(H):  # a slot's sums are the difference of the running sums at its ends
            opens = k[:, h, 0] < 0
            opens[0] = True
            first = opens.nonzero()[:, 0]
            last = torch.cat([first[1:], first.new_tensor([m + S])])
            total = sums[last, h] - sums[first, h]
            k_out[i, h, :len(first)] = total[:, :D] / total[:, -1:]
            v_out[i, h, :len(first)] = total[:, D:2 * D] / total[:, -1:]
            z_out[i, h, :len(first)] = total[:, -1]
        a += m
    flat = lambda t: t.flatten(0, 1)  # noqa: E731
    return {"q": turned, "k": flat(k_out), "v": flat(v_out), "z": flat(z_out), "len": None}


def _exact_attend(c, x):
    k, v, _ = x["slots"][0]
    B, H, cap, D = k.shape
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda").view(B, H, -1, D)
    for b in range(B):
        for h in range(H):
            n = int(x["lens"][0][b, h])
            score = x["q"].view(B, H, -1, D)[b, h].double() @ k[b, h, :n].double().t() * D ** -0.5
            out[b, h] = torch.softmax(score, -1) @ v[b, h, :n].double()
    return out.view(x["q"].shape)


def _exact_select(c, x):
    G, B, V, keep = c["groups"], c["beams"], c["vocab"], c["keep"]
    best = []
    for g in range(G):
        rows = []
        for b in range(B):
            logp = torch.log_softmax(x["logits"][g * B + b].double(), 0) + x["scores"][g, b].double()
            rows.append(x["scores"][g, b:b + 1].double() if x["finished"][g, b] else logp)
        every = torch.cat(rows + [torch.full((keep,), -math.inf, dtype=torch.float64, device="cuda")])
        best.append(torch.topk(every, keep)[0])
    return {"scores": torch.stack(best), "tokens": None, "parents": None, "done": None}


def _exact_reorder(c, x):
    B, at = c["beams"], x["parents"].long()
    return [tuple(t.double()[at // B].flatten(0, 1) for t in slots) + (None,) for slots in x["slots"]]  # a group's beams begin alike
