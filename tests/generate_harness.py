"""Plain 64-bit forms of what generating text takes (rotation, appending, attention of one token, selection), for the
tests of the kernels. CPU, one loop per definition."""
import math

import torch

from paper_2403_09636_gb300 import DmcCache

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # the most one rounding is off, relative to the value


def inv_freq(D, base=10000.0):
    return base ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)


def turned(x, at, freq, pairs, back=False):
    """x [T, H, D] rotated to the positions at [T]; the pair of dimension 0 stays."""
    angle = at.double()[:, None] * freq.double()
    angle[:, 0] = 0.0
    c, s = angle.cos()[:, None], (-angle if back else angle).sin()[:, None]
    x, y = x.double(), torch.empty(x.shape, dtype=torch.float64)
    D = x.shape[2]
    i = torch.arange(D // 2)
    a, b = (2 * i, 2 * i + 1) if pairs else (i, i + D // 2)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Plain:
    """A cache in 64 bits: for every sequence and KV head, the slots (k, v, z), rounded to the cache's type where a call
    of the real one ends; with window grouping also the open segment's tokens."""

    def __init__(self, batch, hq, hkv, D, dtype, window=0):
        self.G, self.H, self.D, self.dt, self.W = hq // hkv, hkv, D, dtype, window
        self.heads = [[[] for _ in range(hkv)] for _ in range(batch)]
        self.open = [[[] for _ in range(hkv)] for _ in range(batch)]

    def append(self, seq, q, k, v, at=None, freq=None, pairs=False):
        """Tokens q [T, Hq, D], k, v [T, H, D] of one sequence, the first at position `at`; returns the rotated queries."""
        T = k.shape[0]
        q, k, v = q.double(), k.double(), v.double()
        kr, qr = k, q
        if freq is not None:
            pos = at + torch.arange(T)
            kr, qr = turned(k, pos, freq, pairs), turned(q, pos, freq, pairs)
        for h in range(self.H):
            slots, tokens = self.heads[seq][h], self.open[seq][h]
            touched = set()
            for t in range(T):
                w = torch.sigmoid(q[t, h * self.G:(h + 1) * self.G, 0].mean())
                row = kr[t, h].clone()
                row[0] = 0.0
                if slots and k[t, h, 0] >= 0:
                    tokens.append((row, v[t, h], w))
                    if self.W:
                        last = tokens[-self.W:]
                        z = sum(x[2] for x in last)
                        slots[-1] = (sum(x[0] * x[2] for x in last) / z, sum(x[1] * x[2] for x in last) / z, z)
                    else:
                        ko, vo, zo = slots[-1]
                        slots[-1] = ((ko * zo + row * w) / (zo + w), (vo * zo + v[t, h] * w) / (zo + w), zo + w)
                else:
                    tokens[:] = [(row, v[t, h], w)]
                    slots.append((row, v[t, h], w))
                touched.add(len(slots) - 1)
            for i in touched:
                ko, vo, zo = slots[i]
                slots[i] = (ko.to(self.dt).double(), vo.to(self.dt).double(), zo)
            if self.W:  # the window's tokens are kept in the cache's type
                tokens[:] = [(x[0].to(self.dt).double(), x[1].to(self.dt).double(), x[2]) for x in tokens]
        return qr

    def reorder(self, parents, first=0):
        heads = [self.heads[first + p] for p in parents]
        tokens = [self.open[first + p] for p in parents]
        for j in range(len(parents)):
            self.heads[first + j] = [list(x) for x in heads[j]]
            self.open[first + j] = [list(x) for x in tokens[j]]

    def attend(self, q):
        """q [batch, Hq, D] over every head's slots; and the largest |v| of each output's head."""
        out, size = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
        for b, heads in enumerate(self.heads):
            for h, slots in enumerate(heads):
                if not slots:
                    continue
                K, V = torch.stack([x[0] for x in slots]), torch.stack([x[1] for x in slots])
                for g in range(h * self.G, (h + 1) * self.G):
                    p = torch.softmax(K[:, 1:] @ q[b, g, 1:].double() / math.sqrt(self.D), 0)
                    out[b, g], size[b, g] = p @ V, V.abs().max()
        return out, size

    def dense(self, cap):
        """(k, v, z, len) as DmcCache.export_heads of every head."""
        n = len(self.heads) * self.H
        k, v = torch.zeros(n, cap, self.D, dtype=torch.float64), torch.zeros(n, cap, self.D, dtype=torch.float64)
        z, ln = torch.zeros(n, cap, dtype=torch.float64), torch.zeros(n, dtype=torch.int32)
        for b, heads in enumerate(self.heads):
            for h, slots in enumerate(heads):
                for i, (a, c, w) in enumerate(slots):
                    k[b * self.H + h, i], v[b * self.H + h, i], z[b * self.H + h, i] = a, c, w
                ln[b * self.H + h] = len(slots)
        return k, v, z, ln


def tokens(g, T, hq, hkv, D, dtype, opens=0.5, scale=0.5):
    """(q, k, v) of T tokens that open a slot with probability `opens`."""
    q, k, v = (torch.randn(T, n, D, generator=g) * scale for n in (hq, hkv, hkv))
    gate = torch.randn(T, hkv, generator=g).abs() + 0.1
    k[..., 0] = torch.where(torch.rand(T, hkv, generator=g) < opens, -gate, gate)
    return q.to(dtype), k.to(dtype), v.to(dtype)


def cache_of(batch, hq, hkv, D, dtype, slots, layers=1, pages=None, prompt=0, window=0, device="cuda"):
    if pages is None:
        pages = layers * batch * hkv * (-(-slots // 32) + 1)
    return DmcCache(layers, batch, hq, hkv, D, dtype, slots, pages, prompt, window=window, device=device)


def exported(cache, layer, cap):
    """export_heads of every head, on the CPU."""
    ids = list(range(cache.cfg.batch * cache.cfg.num_kv_heads))
    return [t.cpu() for t in cache.export_heads(layer, ids, cap)]


def near(got, want, bound, what=""):
    """|got - want| <= bound everywhere (bound: a number or a tensor that broadcasts)."""
    off = (got.double() - want).abs()
    worst = (off - bound).max() if off.numel() else torch.tensor(-1.0)
    assert bool(worst <= 0), (what, float(off.max()), float(worst))


def picked(logits, scores, finished, eos, keep):
    """The selection by its definition, one group after the other: (scores, tokens, parents, done)."""
    G, B = scores.shape
    V = logits.shape[1]
    out = [], [], [], []
    for g in range(G):
        rows = []
        for b in range(B):
            x, base = logits[g * B + b].double(), float(scores[g, b])
            nothing = torch.full((V,), -math.inf, dtype=torch.float64)
            if finished is not None and bool(finished[g, b]):
                row = nothing
                if math.isfinite(base):
                    row[eos] = base
            else:
                lse = torch.logsumexp(x, 0)
                row = base + x - lse if math.isfinite(base) and bool(torch.isfinite(lse)) else nothing
            rows.append(row)
        row = torch.cat(rows)
        best, at = torch.sort(row, dim=0, descending=True, stable=True)
        best, at = best[:keep], at[:keep]
        out[0].append(best)
        out[1].append(at % V)
        out[2].append(g * B + at // V)
        done = at % V == eos
        if finished is not None:
            done = done | finished[g][at // V]
        out[3].append(done)
    return [torch.stack(x) for x in out]
