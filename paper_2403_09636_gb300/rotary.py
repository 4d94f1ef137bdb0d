"""The position rotation of queries and keys (include/dmc.h has the mathematics).

`Rotary` holds a model's frequencies as the kernels take them; `DmcCache.append` rotates with it on the way into the
cache. `rotate` is the rotation alone, `apply` the same with its gradient:

    rotary = Rotary(128, base=10000.0)
    q, k = apply(rotary, q, k, positions)               # a training step, or a prompt before its attention
    q = cache.append(layer, q, k, v, positions, rotary)  # one token of each sequence: raw q and k

The pair that holds dimension 0, the method's gate, is not rotated.
"""
from __future__ import annotations

import math

import torch
from torch.autograd.function import once_differentiable

from . import DMC_BF16, DMC_F32, _check, lib

_CODES = {torch.float32: DMC_F32, torch.bfloat16: DMC_BF16}
# 1 / (2 pi), times 2^140: turns times 2^64 of frequencies from 2^-64 up keep all of their 53 bits
_TURN = 0x28BE60DB9391054A7F09D5F47D4D377036E


def _turns(x):
    """x radians in turns modulo one, times 2^64, rounded, as the int64 with the same bits."""
    n, d = float(x).as_integer_ratio()
    bits = (((n * _TURN << 1) // (d << 76)) + 1 >> 1) % (1 << 64)  # 2^64 / 2^140
    return bits - (1 << 64) if bits >> 63 else bits


class Rotary:
    """Frequencies of a rotation: `inv_freq`, radians per token of each pair (head_dim / 2 numbers; the first is not
    used), or base ** (-2 i / head_dim). Pairs are dims i and i + head_dim / 2, or 2 i and 2 i + 1 if interleaved."""

    def __init__(self, head_dim, base=10000.0, inv_freq=None, interleaved=False, device=None):
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim must be 64 or 128, got {head_dim}")
        if inv_freq is None:
            if not (math.isfinite(base) and base > 0):
                raise ValueError(f"base must be a positive number, got {base}")
            values = [base ** (-2.0 * i / head_dim) for i in range(head_dim // 2)]
        else:
            values = inv_freq.tolist() if isinstance(inv_freq, torch.Tensor) else [float(x) for x in inv_freq]
        if len(values) != head_dim // 2 or not all(math.isfinite(x) for x in values):
            raise ValueError(f"inv_freq must hold {head_dim // 2} finite numbers")
        self.head_dim, self.interleaved = head_dim, bool(interleaved)
        self.turns = torch.tensor([_turns(x) for x in values], dtype=torch.int64,
                                  device=device if device is not None else "cuda")
        self.index, self.pointer, self.pairs = self.turns.get_device(), self.turns.data_ptr(), int(self.interleaved)
        # that the turns' memory waits for when it is given up
        self.streams = {torch._C._cuda_getCurrentRawStream(self.index)} if self.index >= 0 else set()

    def used_on(self, raw):
        """Notes that the stream of this number reads the turns."""
        dev = self.turns.device
        self.turns.record_stream(torch.cuda.ExternalStream(raw, device=dev) if raw else torch.cuda.default_stream(dev))
        self.streams.add(raw)


def _stride(rotary, name, x, tokens, dtype):
    """Token stride of [tokens, heads, head_dim] whose heads are contiguous."""
    D = rotary.head_dim
    try:
        T, H, width = x.shape
        a, b, c = x.stride()
        row = H * D
        if (T == tokens and width == D and x.dtype is dtype and x.get_device() == rotary.index and c == 1
                and (b == D or H <= 1) and (a >= row or T <= 1)):
            return a if T > 1 else row
    except (AttributeError, TypeError, ValueError):
        pass
    what = f"{x.dtype} {tuple(x.shape)}, strides {x.stride()}, on {x.device}" if isinstance(x, torch.Tensor) else type(x).__name__
    raise ValueError(f"{name} must be {dtype} [{tokens}, heads, {D}] on {rotary.turns.device}, its heads contiguous, its "
                     f"tokens apart, got {what}")


def rotate(rotary, q, k, positions, inverse=False, out=None, stream=None):
    """(q', k'): q [T, Hq, D] and k [T, Hkv, D] (or None) rotated to positions, int32 [T], in one launch; inverse rotates
    back. Heads are contiguous, tokens may be apart (a slice of a joint projection). out: (q', k') tensors, which may be
    q and k themselves."""
    dt = getattr(q, "dtype", None)
    if dt not in _CODES or q.dim() != 3:
        raise ValueError("q must be float32 or bfloat16 [tokens, heads, head_dim]")
    T, hq, D = q.shape
    index = rotary.index
    if torch._C._cuda_getDevice() != index:
        raise ValueError(f"the rotation is for {rotary.turns.device}, which is not the current device")
    if (not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32 or positions.shape != (T,)
            or positions.get_device() != index or not positions.is_contiguous()):
        raise ValueError(f"positions must be contiguous int32 ({T},) on {rotary.turns.device}")
    qs = _stride(rotary, "q", q, T, dt)
    hk = ks = kos = 0
    if k is not None:
        ks, hk = _stride(rotary, "k", k, T, dt), k.shape[1]
    raw = torch._C._cuda_getCurrentRawStream(index)
    number = raw if stream is None else stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if out is None:
        if number == raw:
            out = _new(q, k)
        else:
            dev = rotary.turns.device
            with torch.cuda.stream(torch.cuda.ExternalStream(number, device=dev) if number else torch.cuda.default_stream(dev)):
                out = _new(q, k)
        qos, kos = hq * D, hk * D
    else:
        if len(out) != 2 or (out[1] is None) != (k is None):
            raise ValueError("out must hold q' and k'")
        qos = _stride(rotary, "q'", out[0], T, dt)
        if k is not None:
            kos = _stride(rotary, "k'", out[1], T, dt)
        if out[0].shape[1] != hq or (k is not None and out[1].shape[1] != hk):
            raise ValueError("out must have the shapes of q and k")
    qo, ko = out
    if number not in rotary.streams:
        rotary.used_on(number)
    st = lib().dmc_rotate(_CODES[dt], D, T, positions.data_ptr(), rotary.pointer, rotary.pairs, 1 if inverse else 0, hq,
                          q.data_ptr(), qs, qo.data_ptr(), qos, hk, None if k is None else k.data_ptr(), ks,
                          None if k is None else ko.data_ptr(), kos, number)
    if st:
        _check(st, "dmc_rotate")
    return out


def _new(q, k):
    # (empty_like keeps the strides of what is not dense)
    qo = torch.empty_like(q) if q.is_contiguous() else torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is None:
        return qo, None
    return qo, torch.empty_like(k) if k.is_contiguous() else torch.empty(k.shape, dtype=k.dtype, device=k.device)


class _Apply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rotary, q, k, positions):
        ctx.rotary = rotary
        ctx.save_for_backward(positions)
        return rotate(rotary, q, k, positions)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        at, (_, needs_q, needs_k, _) = ctx.saved_tensors[0], ctx.needs_input_grad
        if needs_q:
            dq, dk = rotate(ctx.rotary, _dense(dq), _dense(dk) if needs_k else None, at, inverse=True)
        else:
            dq, dk = None, rotate(ctx.rotary, _dense(dk), None, at, inverse=True)[0]
        return None, dq, dk, None


def _dense(g):
    # (a gradient can be a piece of another one that begins anywhere)
    g = g.contiguous()
    return g if g.data_ptr() % 16 == 0 else g.clone()


def apply(rotary, q, k, positions):
    """(q', k') of `rotate`, differentiable (once) in q and k; k may be None."""
    return _Apply.apply(rotary, q, k, positions)
