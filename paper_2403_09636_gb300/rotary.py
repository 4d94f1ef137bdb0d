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
from fractions import Fraction

import torch
from torch.autograd.function import once_differentiable

from . import DMC_BF16, DMC_F32, _check, lib

_CODES = {torch.float32: DMC_F32, torch.bfloat16: DMC_BF16}
# 1 / (2 pi), to 2^-140: turns times 2^64 of frequencies from 2^-64 up keep all of their 53 bits
_TURN = Fraction(0x28BE60DB9391054A7F09D5F47D4D377036E, 1 << 140)


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
        # turns per token modulo one, times 2^64, as the int64 with the same bits
        bits = [round(Fraction(x) * _TURN * (1 << 64)) % (1 << 64) for x in values]
        self.head_dim, self.interleaved = head_dim, bool(interleaved)
        self.turns = torch.tensor([b - (1 << 64) if b >> 63 else b for b in bits], dtype=torch.int64,
                                  device=device if device is not None else "cuda")


def _rows(rotary, name, x, tokens, dtype):
    """Pointer, heads and token stride of [tokens, heads, head_dim] whose heads are contiguous."""
    D = rotary.head_dim
    if (not isinstance(x, torch.Tensor) or x.dim() != 3 or x.shape[0] != tokens or x.shape[2] != D or x.dtype is not dtype
            or x.device != rotary.turns.device):
        raise ValueError(f"{name} must be {dtype} [{tokens}, heads, {D}] on {rotary.turns.device}")
    H = x.shape[1]
    stride = x.stride(0) if tokens > 1 else H * D
    if x.numel() and ((H > 1 and x.stride(1) != D) or x.stride(2) != 1 or stride < H * D):
        raise ValueError(f"{name}'s heads must be contiguous and its tokens apart, got strides {x.stride()}")
    return H, x.data_ptr(), stride


def rotate(rotary, q, k, positions, inverse=False, out=None, stream=None):
    """(q', k'): q [T, Hq, D] and k [T, Hkv, D] (or None) rotated to positions, int32 [T], in one launch; inverse rotates
    back. Heads are contiguous, tokens may be apart (a slice of a joint projection). out: (q', k') tensors, which may be
    q and k themselves."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or q.dtype not in _CODES:
        raise ValueError("q must be float32 or bfloat16 [tokens, heads, head_dim]")
    T, dt, dev = q.shape[0], q.dtype, rotary.turns.device
    if (not isinstance(positions, torch.Tensor) or positions.dtype is not torch.int32 or positions.shape != (T,)
            or positions.device != dev or not positions.is_contiguous()):
        raise ValueError(f"positions must be contiguous int32 ({T},) on {dev}")
    given = (_rows(rotary, "q", q, T, dt), (0, None, 0) if k is None else _rows(rotary, "k", k, T, dt))
    raw = torch._C._cuda_getCurrentRawStream(dev.index)
    number = raw if stream is None else stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if out is None:
        def new(x):
            return None if x is None else torch.empty(x.shape, dtype=dt, device=dev)
        if number == raw:
            out = (new(q), new(k))
        else:
            other = torch.cuda.ExternalStream(number, device=dev) if number else torch.cuda.default_stream(dev)
            with torch.cuda.stream(other):
                out = (new(q), new(k))
    elif len(out) != 2 or (out[1] is None) != (k is None):
        raise ValueError("out must hold q' and k'")
    to = (_rows(rotary, "q'", out[0], T, dt), (0, None, 0) if k is None else _rows(rotary, "k'", out[1], T, dt))
    if to[0][0] != given[0][0] or to[1][0] != given[1][0]:
        raise ValueError("out must have the shapes of q and k")
    (hq, qp, qs), (hk, kp, ks) = given
    st = lib().dmc_rotate(_CODES[dt], rotary.head_dim, T, positions.data_ptr(), rotary.turns.data_ptr(),
                          int(rotary.interleaved), int(bool(inverse)), hq, qp, qs, to[0][1], to[0][2], hk, kp, ks, to[1][1],
                          to[1][2], number)
    if st:
        _check(st, "dmc_rotate")
    return out


class _Apply(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rotary, q, k, positions):
        ctx.rotary = rotary
        ctx.save_for_backward(positions)
        return rotate(rotary, q, k, positions)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        return None, *rotate(ctx.rotary, dq.contiguous(), dk.contiguous(), *ctx.saved_tensors, inverse=True), None


def apply(rotary, q, k, positions):
    """(q', k') of `rotate`, differentiable (once) in q and k."""
    return _Apply.apply(rotary, q, k, positions)
