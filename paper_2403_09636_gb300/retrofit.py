"""The operators of a retrofitting step (training a model to compress its cache).

`DmcRetrofit` owns a torch uint8 arena and forwards to the dmc_retrofit_* functions
of the C ABI (include/dmc.h has the mathematics): the relaxed compression's states,
attention over packed sequences with the bias that hides merged states, and cross
entropy against a vocabulary whose logits are never kept, each with its gradient.
Arguments are checked (type, shape, device, contiguity) and refused with ValueError;
statuses of the library become DmcError.

`attention` and `cross_entropy` are the same as autograd functions:

    dmc = DmcRetrofit(32, 32, 128, torch.bfloat16, max_tokens=8192, max_seqs=4, hidden=4096, vocab=32000)
    out, alpha = attention(dmc, q, k, v, cu_seqlens, max_seqlen, noise=noise)
    loss = cross_entropy(dmc, hidden, weight, targets).sum() / counted
    loss.backward()
"""
from __future__ import annotations

import torch

from . import (DMC_BF16, DMC_ERR_INVALID_ARG, DMC_F32, DmcError, _check, dmc_retrofit_attention,
               dmc_retrofit_attention_backward, dmc_retrofit_config, dmc_retrofit_create, dmc_retrofit_destroy,
               dmc_retrofit_loss, dmc_retrofit_loss_backward, dmc_retrofit_required_bytes, dmc_retrofit_saved_bytes,
               dmc_retrofit_states, dmc_retrofit_states_backward, dmc_retrofit_status)

_F32, _I32 = torch.float32, torch.int32


class DmcRetrofit:
    """Scratch and entry points of the retrofitting operators for one shape of heads and
    (or) one vocabulary. Calls on one handle must be ordered on the GPU.

    Outputs are new tensors, or those given as `out` (a tuple in the order of the
    results). Tensors must be contiguous and on the handle's device; q0 may be strided."""

    def __init__(self, num_q_heads=0, num_kv_heads=0, head_dim=0, dtype=torch.bfloat16, max_tokens=0, max_seqs=1,
                 hidden=0, vocab=0, device=None, stream=None):
        self.handle = None
        codes = {_F32: DMC_F32, torch.bfloat16: DMC_BF16}
        if dtype not in codes:
            raise ValueError(f"dtype must be float32 or bfloat16, got {dtype}")
        dev = torch.device(device if device is not None else "cuda")
        if dev.type == "cuda" and dev.index is None and torch.cuda.is_available():
            dev = torch.device("cuda", torch.cuda.current_device())
        self.dtype, self.device = dtype, dev
        self.cfg = dmc_retrofit_config(int(num_q_heads), int(num_kv_heads), int(head_dim), codes[dtype],
                                       int(max_tokens), int(max_seqs), int(hidden), int(vocab))
        self.nbytes = dmc_retrofit_required_bytes(self.cfg)
        if self.nbytes == 0:
            raise DmcError(DMC_ERR_INVALID_ARG, "dmc_retrofit_required_bytes")
        self.arena = torch.empty(self.nbytes, dtype=torch.uint8, device=self.device)
        st, self.handle = dmc_retrofit_create(self.cfg, self.arena.data_ptr(), self.nbytes, self._s(stream))
        _check(st, "dmc_retrofit_create")

    def _s(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.device.index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def close(self):
        if getattr(self, "handle", None):
            dmc_retrofit_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- checks

    def _is(self, name, t, shape, dtype):
        if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != self.device or tuple(t.shape) != shape:
            what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
            raise ValueError(f"{name} must be {dtype} {shape} on {self.device}, got {what}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        return t.data_ptr()

    def _may(self, name, t, shape, dtype):
        return None if t is None else self._is(name, t, shape, dtype)

    def _out(self, out, *specs):
        """The call's outputs: new ones of the (name, shape, dtype) given, or the caller's."""
        if out is None:
            return tuple(torch.empty(shape, dtype=dtype, device=self.device) for _, shape, dtype in specs)
        if len(out) != len(specs):
            raise ValueError(f"out must hold {len(specs)} tensors: {', '.join(s[0] for s in specs)}")
        for t, (name, shape, dtype) in zip(out, specs):
            self._is(name, t, shape, dtype)
        return tuple(out)

    def _seqs(self, k, cu_seqlens):
        if not self.cfg.num_q_heads:
            raise ValueError("this handle was made without heads")
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            raise ValueError("k must be [tokens, KV heads, head_dim]")
        if not isinstance(cu_seqlens, torch.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
            raise ValueError("cu_seqlens must be int32 [sequences + 1]")
        n = cu_seqlens.numel() - 1
        return k.shape[0], n, self._is("cu_seqlens", cu_seqlens, (n + 1,), _I32)

    def _first(self, name, q0, T):
        """q's first components: [T, Hq] of any strides."""
        if (not isinstance(q0, torch.Tensor) or q0.dtype != self.dtype or q0.device != self.device
                or tuple(q0.shape) != (T, self.cfg.num_q_heads)):
            raise ValueError(f"{name} must be {self.dtype} {(T, self.cfg.num_q_heads)} on {self.device}")
        return q0.data_ptr(), q0.stride(0), q0.stride(1)

    # ---- states

    def states(self, q0, k, v, cu_seqlens, max_seqlen, noise=None, offset=5.0, temperature=0.1, out=None, stream=None):
        """(k~, v~, alpha, bias, saved) of packed tokens: q0 [T, Hq] (q[..., 0], any strides), k and v
        [T, Hkv, D], noise [Hkv, T] or None; alpha and bias are fp32 [Hkv, T], saved is for the
        backward pass."""
        T, n, cu = self._seqs(k, cu_seqlens)
        H, D = self.cfg.num_kv_heads, self.cfg.head_dim
        q = self._first("q0", q0, T)
        ptrs = [self._is(i, t, (T, H, D), self.dtype) for i, t in (("k", k), ("v", v))]
        ptrs.append(self._may("noise", noise, (H, T), _F32))
        saved = dmc_retrofit_saved_bytes(self.handle, n, T) // 4
        out = self._out(out, ("kt", (T, H, D), self.dtype), ("vt", (T, H, D), self.dtype), ("alpha", (H, T), _F32),
                        ("bias", (H, T), _F32), ("saved", (saved,), _F32))
        _check(dmc_retrofit_states(self.handle, n, *q, *ptrs, float(offset), float(temperature), cu, T,
                                   int(max_seqlen), *(t.data_ptr() for t in out), self._s(stream)),
               "dmc_retrofit_states")
        return out

    def states_backward(self, q0, k, v, cu_seqlens, max_seqlen, saved, dkt, dvt, dbias, dalpha=None, noise=None,
                        offset=5.0, temperature=0.1, out=None, stream=None):
        """(dq0, dk, dv) from the states' gradients: dbias [Hkv, T] in the handle's dtype, dalpha fp32
        [Hkv, T] or None. out's dq0 may be strided (dq[..., 0] of the attention's dq)."""
        T, n, cu = self._seqs(k, cu_seqlens)
        H, D, dt = self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype
        q = self._first("q0", q0, T)
        ptrs = [self._is(i, t, (T, H, D), dt) for i, t in (("k", k), ("v", v))]
        ptrs.append(self._may("noise", noise, (H, T), _F32))
        grads = [self._is("saved", saved, (dmc_retrofit_saved_bytes(self.handle, n, T) // 4,), _F32)]
        grads += [self._is(i, t, (T, H, D), dt) for i, t in (("dkt", dkt), ("dvt", dvt))]
        grads += [self._is("dbias", dbias, (H, T), dt), self._may("dalpha", dalpha, (H, T), _F32)]
        if out is None:
            dq0 = torch.empty((T, self.cfg.num_q_heads), dtype=dt, device=self.device)
            rest = None
        elif len(out) == 3:
            dq0, rest = out[0], out[1:]
        else:
            raise ValueError("out must hold 3 tensors: dq0, dk, dv")
        rest = self._out(rest, ("dk", (T, H, D), dt), ("dv", (T, H, D), dt))
        _check(dmc_retrofit_states_backward(self.handle, n, *q, *ptrs, float(offset), float(temperature), cu, T,
                                            int(max_seqlen), *grads, *self._first("dq0", dq0, T),
                                            *(t.data_ptr() for t in rest), self._s(stream)),
               "dmc_retrofit_states_backward")
        return (dq0, *rest)

    # ---- attention

    def attention(self, q, k, v, cu_seqlens, max_seqlen, bias=None, out=None, stream=None):
        """(out, lse): causal attention of packed sequences, q [T, Hq, D], k and v [T, Hkv, D], bias
        [Hkv, T] added to the scores of earlier rows (None: none); lse fp32 [Hq, T]."""
        T, n, cu = self._seqs(k, cu_seqlens)
        Hq, H, D = self.cfg.num_q_heads, self.cfg.num_kv_heads, self.cfg.head_dim
        ptrs = [self._is("q", q, (T, Hq, D), self.dtype)]
        ptrs += [self._is(i, t, (T, H, D), self.dtype) for i, t in (("k", k), ("v", v))]
        ptrs.append(self._may("bias", bias, (H, T), _F32))
        out = self._out(out, ("out", (T, Hq, D), self.dtype), ("lse", (Hq, T), _F32))
        _check(dmc_retrofit_attention(self.handle, n, *ptrs, cu, T, int(max_seqlen), *(t.data_ptr() for t in out),
                                      self._s(stream)), "dmc_retrofit_attention")
        return out

    def attention_backward(self, dout, q, k, v, o, lse, cu_seqlens, max_seqlen, bias=None, out=None, stream=None):
        """(dq, dk, dv, dbias) of `attention`, given its outputs o and lse; dbias [Hkv, T] in the
        handle's dtype, None without a bias."""
        T, n, cu = self._seqs(k, cu_seqlens)
        Hq, H, D, dt = self.cfg.num_q_heads, self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype
        ptrs = [self._is("q", q, (T, Hq, D), dt)]
        ptrs += [self._is(i, t, (T, H, D), dt) for i, t in (("k", k), ("v", v))]
        ptrs += [self._may("bias", bias, (H, T), _F32), self._is("o", o, (T, Hq, D), dt),
                 self._is("lse", lse, (Hq, T), _F32), self._is("dout", dout, (T, Hq, D), dt)]
        specs = [("dq", (T, Hq, D), dt), ("dk", (T, H, D), dt), ("dv", (T, H, D), dt)]
        if bias is not None:
            specs.append(("dbias", (H, T), dt))
        out = self._out(out, *specs)
        given = [t.data_ptr() for t in out] + [None] * (4 - len(out))
        _check(dmc_retrofit_attention_backward(self.handle, n, *ptrs, cu, T, int(max_seqlen), *given,
                                               self._s(stream)), "dmc_retrofit_attention_backward")
        return out if bias is not None else (*out, None)

    # ---- loss

    def _words(self, hidden, weight, targets):
        if not self.cfg.hidden:
            raise ValueError("this handle was made without a vocabulary")
        if not isinstance(hidden, torch.Tensor) or hidden.dim() != 2:
            raise ValueError("hidden must be [tokens, hidden]")
        N = hidden.shape[0]
        return N, [self._is("hidden", hidden, (N, self.cfg.hidden), self.dtype),
                   self._is("weight", weight, (self.cfg.vocab, self.cfg.hidden), self.dtype),
                   self._is("targets", targets, (N,), _I32)]

    def loss(self, hidden, weight, targets, out=None, stream=None):
        """(loss, lse), fp32 [N]: cross entropy of hidden [N, hidden] against weight [vocab, hidden] at
        int32 targets [N]; below 0 a position is ignored."""
        N, ptrs = self._words(hidden, weight, targets)
        out = self._out(out, ("loss", (N,), _F32), ("lse", (N,), _F32))
        _check(dmc_retrofit_loss(self.handle, N, *ptrs, *(t.data_ptr() for t in out), self._s(stream)),
               "dmc_retrofit_loss")
        return out

    def loss_backward(self, dloss, hidden, weight, targets, lse, out=None, stream=None):
        """(dhidden, dweight) of `loss` from dloss, fp32 [N], and its lse."""
        N, ptrs = self._words(hidden, weight, targets)
        ptrs += [self._is("lse", lse, (N,), _F32), self._is("dloss", dloss, (N,), _F32)]
        out = self._out(out, ("dhidden", (N, self.cfg.hidden), self.dtype),
                        ("dweight", (self.cfg.vocab, self.cfg.hidden), self.dtype))
        _check(dmc_retrofit_loss_backward(self.handle, N, *ptrs, *(t.data_ptr() for t in out), self._s(stream)),
               "dmc_retrofit_loss_backward")
        return out

    def status(self, stream=None):
        """(status, fault bits); synchronizes the stream."""
        return dmc_retrofit_status(self.handle, self._s(stream))


# ---------------------------------------------------------------- autograd

class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, dmc, q, k, v, cu_seqlens, max_seqlen, noise, offset, temperature):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        gates = {"noise": noise, "offset": offset, "temperature": temperature}
        kt, vt, alpha, bias, saved = dmc.states(q[..., 0], k, v, cu_seqlens, max_seqlen, **gates)
        o, lse = dmc.attention(q, kt, vt, cu_seqlens, max_seqlen, bias)
        ctx.save_for_backward(q, k, v, kt, vt, bias, saved, o, lse, cu_seqlens)
        ctx.dmc, ctx.max_seqlen, ctx.gates = dmc, max_seqlen, gates
        return o, alpha

    @staticmethod
    def backward(ctx, do, dalpha):
        q, k, v, kt, vt, bias, saved, o, lse, cu = ctx.saved_tensors
        dmc, longest = ctx.dmc, ctx.max_seqlen
        dq, dkt, dvt, dbias = dmc.attention_backward(do.contiguous(), q, kt, vt, o, lse, cu, longest, bias)
        dk, dv = torch.empty_like(k), torch.empty_like(v)
        dmc.states_backward(q[..., 0], k, v, cu, longest, saved, dkt, dvt, dbias, dalpha.contiguous(), **ctx.gates,
                            out=(dq[..., 0], dk, dv))
        return None, dq, dk, dv, None, None, None, None, None


def attention(dmc, q, k, v, cu_seqlens, max_seqlen, noise=None, offset=5.0, temperature=0.1):
    """DMC's training attention of packed sequences, differentiable in q, k and v: (out [T, Hq, D],
    alpha [Hkv, T]). The first components of q and k are the gates, as at inference."""
    return _Attention.apply(dmc, q, k, v, cu_seqlens, int(max_seqlen), noise, float(offset), float(temperature))


class _CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, dmc, hidden, weight, targets):
        hidden, weight = hidden.contiguous(), weight.contiguous()
        loss, lse = dmc.loss(hidden, weight, targets)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.dmc = dmc
        return loss

    @staticmethod
    def backward(ctx, dloss):
        hidden, weight, targets, lse = ctx.saved_tensors
        return None, *ctx.dmc.loss_backward(dloss.float().contiguous(), hidden, weight, targets, lse), None


def cross_entropy(dmc, hidden, weight, targets):
    """Each position's cross entropy (fp32 [N], 0 where the target is below 0), differentiable in
    hidden and weight."""
    return _CrossEntropy.apply(dmc, hidden, weight, targets)
