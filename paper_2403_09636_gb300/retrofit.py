"""The operators of a retrofitting step (training a model to compress its cache).

`DmcRetrofit` owns a torch uint8 arena and forwards to the dmc_retrofit_* functions
of the C ABI (include/dmc.h has the mathematics): the relaxed compression's states,
attention over packed sequences with the bias that hides merged states, and cross
entropy against a vocabulary whose logits are not kept for the backward pass, each with its gradient.
Arguments are checked (type, shape, device, contiguity) and refused with ValueError;
statuses of the library become DmcError.

`attention` and `cross_entropy` are the same as autograd functions (second derivatives are refused):

    dmc = DmcRetrofit(32, 32, 128, torch.bfloat16, max_tokens=8192, max_seqs=4, hidden=4096, vocab=32000)
    out, alpha = attention(dmc, q, k, v, cu_seqlens, max_seqlen, noise=noise)
    loss = cross_entropy(dmc, hidden, weight, targets).sum() / counted
    loss.backward()
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import (DMC_BF16, DMC_ERR_INVALID_ARG, DMC_F32, DmcError, _check, dmc_retrofit_config, dmc_retrofit_create,
               dmc_retrofit_destroy, dmc_retrofit_required_bytes, dmc_retrofit_saved_bytes, dmc_retrofit_status, lib)

_F32, _I32 = torch.float32, torch.int32


class DmcRetrofit:
    """Scratch and entry points of the retrofitting operators for one shape of heads and
    (or) one vocabulary. Calls on one handle must be ordered on the GPU.

    Outputs are new tensors of the call's stream, the current one unless `stream` names another, or those
    given as `out` (a tuple in the order of the results). Tensors must be contiguous and on the handle's device; q0
    may be strided."""

    def __init__(self, num_q_heads=0, num_kv_heads=0, head_dim=0, dtype=torch.bfloat16, max_tokens=0, max_seqs=1,
                 hidden=0, vocab=0, device=None, stream=None):
        self.handle = None
        codes = {_F32: DMC_F32, torch.bfloat16: DMC_BF16}
        if dtype not in codes:
            raise ValueError(f"dtype must be float32 or bfloat16, got {dtype}")
        dev = torch.device(device if device is not None else "cuda")
        if dev.type == "cuda" and dev.index is None and torch.cuda.is_available():
            dev = torch.device("cuda", torch.cuda.current_device())
        self.dtype, self.device, self.index = dtype, dev, dev.index if dev.type == "cuda" else -1
        self.cfg = dmc_retrofit_config(int(num_q_heads), int(num_kv_heads), int(head_dim), codes[dtype],
                                       int(max_tokens), int(max_seqs), int(hidden), int(vocab))
        self.nbytes = dmc_retrofit_required_bytes(self.cfg)
        if self.nbytes == 0:
            raise DmcError(DMC_ERR_INVALID_ARG, "dmc_retrofit_required_bytes")
        self.arena = self._maker(stream)((self.nbytes,), torch.uint8)
        self._streams = {self._raw(stream)}  # that the arena's memory waits for when it is given up
        st, self.handle = dmc_retrofit_create(self.cfg, self.arena.data_ptr(), self.nbytes, self._s(stream))
        _check(st, "dmc_retrofit_create")
        self.lib = lib()
        self._saved = {}  # floats of `saved` by (sequences, tokens)

    def _raw(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def _stream(self, raw):
        # (an ExternalStream of the number 0 would be another one)
        return torch.cuda.ExternalStream(raw, device=self.device) if raw else torch.cuda.default_stream(self.device)

    def _s(self, stream):
        """The number of the stream of a call."""
        raw = torch._C._cuda_getCurrentRawStream(self.index) if stream is None else self._raw(stream)
        if raw not in self._streams:
            self.arena.record_stream(self._stream(raw))
            self._streams.add(raw)
        return raw

    def close(self):
        if getattr(self, "handle", None):
            dmc_retrofit_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- checks, of one expression each: 3 of the 10 us that a call with its outputs given takes on the host

    def _is(self, name, t, shape, dtype):
        if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == self.index
                and t.is_contiguous()):
            return t.data_ptr()
        what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} must be contiguous {dtype} {shape} on {self.device}, got {what}")

    def _new(self, shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def _maker(self, stream):
        """`_new`, of memory that belongs to the stream of a call: work of the current one that still uses what was
        freed there does not run beside the call."""
        if self._raw(stream) == self._raw(None):
            return self._new
        other = self._stream(self._raw(stream))

        def new(shape, dtype):
            with torch.cuda.stream(other):
                return self._new(shape, dtype)

        return new

    def _seqs(self, k, cu_seqlens):
        """Tokens, sequences and the pointer of cu_seqlens."""
        if not self.cfg.num_q_heads:
            raise ValueError("this handle was made without heads")
        if not isinstance(k, torch.Tensor) or k.dim() != 3:
            raise ValueError("k must be [tokens, KV heads, head_dim]")
        if not isinstance(cu_seqlens, torch.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
            raise ValueError("cu_seqlens must be int32 [sequences + 1]")
        n = cu_seqlens.numel()
        if n == 1 and k.shape[0]:
            raise ValueError(f"cu_seqlens has no sequence for {k.shape[0]} tokens")
        return k.shape[0], n - 1, self._is("cu_seqlens", cu_seqlens, (n,), _I32)

    def _first(self, name, q0, T):
        """q's first components, [T, Hq] of any strides: pointer and strides."""
        if (not isinstance(q0, torch.Tensor) or q0.dtype is not self.dtype or q0.get_device() != self.index
                or q0.shape != (T, self.cfg.num_q_heads)):
            raise ValueError(f"{name} must be {self.dtype} {(T, self.cfg.num_q_heads)} on {self.device}")
        return q0.data_ptr(), *q0.stride()

    def _saved_floats(self, n, T):
        floats = self._saved.get((n, T))
        if floats is None:
            floats = self._saved[(n, T)] = dmc_retrofit_saved_bytes(self.handle, n, T) // 4
        return floats

    @staticmethod
    def _given(out, names):
        if len(out) != len(names):
            raise ValueError(f"out must hold {len(names)} tensors: {', '.join(names)}")
        return out

    # ---- states

    def states(self, q0, k, v, cu_seqlens, max_seqlen, noise=None, offset=5.0, temperature=0.1, out=None, stream=None):
        """(k~, v~, alpha, bias, saved) of packed tokens: q0 [T, Hq] (q[..., 0], any strides), k and v
        [T, Hkv, D], noise [Hkv, T] or None; alpha and bias are fp32 [Hkv, T], saved is for the
        backward pass."""
        T, n, cu = self._seqs(k, cu_seqlens)
        H, D, dt, check = self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype, self._is
        rows, scalars, saved = (T, H, D), (H, T), self._saved_floats(n, T)
        q = self._first("q0", q0, T)
        kp, vp = check("k", k, rows, dt), check("v", v, rows, dt)
        np_ = None if noise is None else check("noise", noise, scalars, _F32)
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new(rows, dt), new(rows, dt), new(scalars, _F32), new(scalars, _F32), new((saved,), _F32))
            ptrs = [t.data_ptr() for t in out]
        else:
            kt, vt, alpha, bias, keep = out = self._given(out, ("kt", "vt", "alpha", "bias", "saved"))
            ptrs = (check("kt", kt, rows, dt), check("vt", vt, rows, dt), check("alpha", alpha, scalars, _F32),
                    check("bias", bias, scalars, _F32), check("saved", keep, (saved,), _F32))
        st = self.lib.dmc_retrofit_states(self.handle, n, *q, kp, vp, np_, offset, temperature, cu, T, max_seqlen, *ptrs,
                                          self._s(stream))
        if st:
            _check(st, "dmc_retrofit_states")
        return out

    def states_backward(self, q0, k, v, cu_seqlens, max_seqlen, saved, dkt, dvt, dbias, dalpha=None, noise=None,
                        offset=5.0, temperature=0.1, out=None, stream=None):
        """(dq0, dk, dv) from the states' gradients: dbias [Hkv, T] in the handle's dtype, dalpha fp32
        [Hkv, T] or None. out's dq0 may be strided (dq[..., 0] of the attention's dq)."""
        T, n, cu = self._seqs(k, cu_seqlens)
        H, D, dt, check = self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype, self._is
        rows, scalars = (T, H, D), (H, T)
        q = self._first("q0", q0, T)
        ptrs = (check("k", k, rows, dt), check("v", v, rows, dt),
                None if noise is None else check("noise", noise, scalars, _F32))
        grads = (check("saved", saved, (self._saved_floats(n, T),), _F32), check("dkt", dkt, rows, dt),
                 check("dvt", dvt, rows, dt), check("dbias", dbias, scalars, dt),
                 None if dalpha is None else check("dalpha", dalpha, scalars, _F32))
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new((T, self.cfg.num_q_heads), dt), new(rows, dt), new(rows, dt))
        dq0, dk, dv = out = self._given(out, ("dq0", "dk", "dv"))
        st = self.lib.dmc_retrofit_states_backward(
            self.handle, n, *q, *ptrs, offset, temperature, cu, T, max_seqlen, *grads, *self._first("dq0", dq0, T),
            check("dk", dk, rows, dt), check("dv", dv, rows, dt), self._s(stream))
        if st:
            _check(st, "dmc_retrofit_states_backward")
        return out

    # ---- attention

    def attention(self, q, k, v, cu_seqlens, max_seqlen, bias=None, out=None, stream=None):
        """(out, lse): causal attention of packed sequences, q [T, Hq, D], k and v [T, Hkv, D], bias
        [Hkv, T] added to the scores of earlier rows (None: none); lse fp32 [Hq, T]."""
        T, n, cu = self._seqs(k, cu_seqlens)
        Hq, H, D, dt, check = self.cfg.num_q_heads, self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype, self._is
        queries, rows = (T, Hq, D), (T, H, D)
        ptrs = (check("q", q, queries, dt), check("k", k, rows, dt), check("v", v, rows, dt),
                None if bias is None else check("bias", bias, (H, T), _F32))
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new(queries, dt), new((Hq, T), _F32))
        o, lse = out = self._given(out, ("out", "lse"))
        st = self.lib.dmc_retrofit_attention(self.handle, n, *ptrs, cu, T, max_seqlen, check("out", o, queries, dt),
                                             check("lse", lse, (Hq, T), _F32), self._s(stream))
        if st:
            _check(st, "dmc_retrofit_attention")
        return out

    def attention_backward(self, dout, q, k, v, o, lse, cu_seqlens, max_seqlen, bias=None, out=None, stream=None):
        """(dq, dk, dv, dbias) of `attention`, given its outputs o and lse; dbias [Hkv, T] in the
        handle's dtype, None without a bias."""
        T, n, cu = self._seqs(k, cu_seqlens)
        Hq, H, D, dt, check = self.cfg.num_q_heads, self.cfg.num_kv_heads, self.cfg.head_dim, self.dtype, self._is
        queries, rows, scalars = (T, Hq, D), (T, H, D), (H, T)
        ptrs = (check("q", q, queries, dt), check("k", k, rows, dt), check("v", v, rows, dt),
                None if bias is None else check("bias", bias, scalars, _F32), check("o", o, queries, dt),
                check("lse", lse, (Hq, T), _F32), check("dout", dout, queries, dt))
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new(queries, dt), new(rows, dt), new(rows, dt)) + (() if bias is None else (new(scalars, dt),))
        self._given(out, ("dq", "dk", "dv") if bias is None else ("dq", "dk", "dv", "dbias"))
        grads = (check("dq", out[0], queries, dt), check("dk", out[1], rows, dt), check("dv", out[2], rows, dt),
                 None if bias is None else check("dbias", out[3], scalars, dt))
        st = self.lib.dmc_retrofit_attention_backward(self.handle, n, *ptrs, cu, T, max_seqlen, *grads, self._s(stream))
        if st:
            _check(st, "dmc_retrofit_attention_backward")
        return out if bias is not None else (*out, None)

    # ---- loss

    def _words(self, hidden, weight, targets):
        if not self.cfg.hidden:
            raise ValueError("this handle was made without a vocabulary")
        if not isinstance(hidden, torch.Tensor) or hidden.dim() != 2:
            raise ValueError("hidden must be [tokens, hidden]")
        N, H, dt = hidden.shape[0], self.cfg.hidden, self.dtype
        return N, (self._is("hidden", hidden, (N, H), dt), self._is("weight", weight, (self.cfg.vocab, H), dt),
                   self._is("targets", targets, (N,), _I32))

    def loss(self, hidden, weight, targets, out=None, stream=None):
        """(loss, lse), fp32 [N]: cross entropy of hidden [N, hidden] against weight [vocab, hidden] at
        int32 targets [N]; below 0 a position is ignored."""
        N, ptrs = self._words(hidden, weight, targets)
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new((N,), _F32), new((N,), _F32))
        loss, lse = out = self._given(out, ("loss", "lse"))
        st = self.lib.dmc_retrofit_loss(self.handle, N, *ptrs, self._is("loss", loss, (N,), _F32),
                                        self._is("lse", lse, (N,), _F32), self._s(stream))
        if st:
            _check(st, "dmc_retrofit_loss")
        return out

    def loss_backward(self, dloss, hidden, weight, targets, lse, out=None, stream=None):
        """(dhidden, dweight) of `loss` from dloss, fp32 [N], and its lse."""
        N, ptrs = self._words(hidden, weight, targets)
        given = (self._is("lse", lse, (N,), _F32), self._is("dloss", dloss, (N,), _F32))
        shapes = (N, self.cfg.hidden), (self.cfg.vocab, self.cfg.hidden)
        if out is None:
            new = self._new if stream is None else self._maker(stream)
            out = (new(shapes[0], self.dtype), new(shapes[1], self.dtype))
        dh, dw = out = self._given(out, ("dhidden", "dweight"))
        st = self.lib.dmc_retrofit_loss_backward(self.handle, N, *ptrs, *given, self._is("dhidden", dh, shapes[0], self.dtype),
                                                 self._is("dweight", dw, shapes[1], self.dtype), self._s(stream))
        if st:
            _check(st, "dmc_retrofit_loss_backward")
        return out

    def status(self, stream=None):
        """(status, fault bits); synchronizes the stream."""
        return dmc_retrofit_status(self.handle, self._s(stream))


# ---------------------------------------------------------------- autograd

class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, dmc, q, k, v, cu_seqlens, max_seqlen, noise, offset, temperature):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        gates = {"offset": offset, "temperature": temperature}
        kt, vt, alpha, bias, saved = dmc.states(q[..., 0], k, v, cu_seqlens, max_seqlen, noise, **gates)
        o, lse = dmc.attention(q, kt, vt, cu_seqlens, max_seqlen, bias)
        ctx.save_for_backward(q, k, v, kt, vt, bias, saved, o, lse, cu_seqlens, noise)
        ctx.dmc, ctx.max_seqlen, ctx.gates = dmc, max_seqlen, gates
        return o, alpha

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dalpha):
        q, k, v, kt, vt, bias, saved, o, lse, cu, noise = ctx.saved_tensors
        dmc, longest = ctx.dmc, ctx.max_seqlen
        dq, dkt, dvt, dbias = dmc.attention_backward(do.contiguous(), q, kt, vt, o, lse, cu, longest, bias)
        dk, dv = torch.empty_like(k), torch.empty_like(v)
        dmc.states_backward(q[..., 0], k, v, cu, longest, saved, dkt, dvt, dbias, dalpha.contiguous(), noise, **ctx.gates,
                            out=(dq[..., 0], dk, dv))
        # the noise is added to k's first component
        dnoise = dk[..., 0].t().float() if ctx.needs_input_grad[6] else None
        return None, dq, dk, dv, None, None, dnoise, None, None


def attention(dmc, q, k, v, cu_seqlens, max_seqlen, noise=None, offset=5.0, temperature=0.1):
    """DMC's training attention of packed sequences, differentiable (once) in q, k, v and noise: (out
    [T, Hq, D], alpha [Hkv, T]). The first components of q and k are the gates, as at inference."""
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
    @once_differentiable
    def backward(ctx, dloss):
        hidden, weight, targets, lse = ctx.saved_tensors
        return None, *ctx.dmc.loss_backward(dloss.float().contiguous(), hidden, weight, targets, lse), None


def cross_entropy(dmc, hidden, weight, targets):
    """Each position's cross entropy (fp32 [N], 0 where the target is below 0), differentiable (once) in
    hidden and weight."""
    return _CrossEntropy.apply(dmc, hidden, weight, targets)
