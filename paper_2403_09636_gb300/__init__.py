"""Dynamic Memory Compression hot path on one GB300 (sm_103a): Python binding.

A thin ctypes layer over libdmc.so (include/dmc.h). Every function named
dmc_* forwards its arguments unchanged to the C function of the same name:
pointers are plain integers (e.g. tensor.data_ptr()), streams are raw
cudaStream_t handles (torch.cuda.current_stream().cuda_stream). All compute
runs in the library's CUDA kernels; there is no fallback of any kind, and a
missing library raises.

`DmcCache` is a convenience wrapper that owns a torch uint8 arena tensor and
turns non-OK statuses into exceptions. `paper_2403_09636_gb300.retrofit` wraps the
operators of a training step in the same way. The synthetic input generator lives in
`paper_2403_09636_gb300.synthetic` and is imported separately.
"""
from __future__ import annotations

import ctypes as C
import os

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdmc.so")

DMC_OK, DMC_ERR_INVALID_ARG, DMC_ERR_ARENA_TOO_SMALL = 0, 1, 2
DMC_ERR_PAGES_EXHAUSTED, DMC_ERR_CUDA, DMC_ERR_DEVICE_FAULT = 3, 4, 5
DMC_F32, DMC_BF16 = 0, 1
DMC_FAULT_PAGES_EXHAUSTED = 0x1
DMC_FAULT_SLOT_CAPACITY = 0x2
DMC_FAULT_NAN_GATE = 0x4
DMC_FAULT_BAD_SEQLENS = 0x8
DMC_FAULT_WAIT_TIMEOUT = 0x10
DMC_FAULT_BAD_TARGET = 0x20
DMC_FAULT_BAD_PARENT = 0x40
PAGE_SIZE = 32

EXPORTED = ("dmc_cache_required_bytes", "dmc_cache_create", "dmc_cache_destroy",
            "dmc_cache_reset", "dmc_prefill_compress", "dmc_prefill_attention", "dmc_decode_step",
            "dmc_decode_step_layers", "dmc_decode_step_static_scratch", "dmc_cache_lengths",
            "dmc_cache_export_heads", "dmc_cache_export_heads_padded", "dmc_cache_status", "dmc_status_string",
            "dmc_retrofit_required_bytes", "dmc_retrofit_create", "dmc_retrofit_destroy",
            "dmc_retrofit_saved_bytes", "dmc_retrofit_states", "dmc_retrofit_states_backward",
            "dmc_retrofit_attention", "dmc_retrofit_attention_backward", "dmc_retrofit_loss",
            "dmc_retrofit_loss_backward", "dmc_retrofit_status",
            "dmc_rotate", "dmc_cache_append", "dmc_cache_attend", "dmc_cache_reorder",
            "dmc_beam_required_bytes", "dmc_beam_create", "dmc_beam_destroy", "dmc_beam_select")


class dmc_cache_config(C.Structure):
    _fields_ = [("num_layers", C.c_int32), ("batch", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("page_size", C.c_int32), ("max_slots_per_head", C.c_int32),
                ("num_pages", C.c_int64), ("max_prefill_tokens", C.c_int32),
                ("window", C.c_int32)]


class dmc_retrofit_config(C.Structure):
    _fields_ = [("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("max_tokens", C.c_int32), ("max_seqs", C.c_int32),
                ("hidden", C.c_int32), ("vocab", C.c_int32)]


class dmc_beam_config(C.Structure):
    _fields_ = [("groups", C.c_int32), ("beams", C.c_int32), ("keep", C.c_int32), ("vocab", C.c_int32),
                ("dtype", C.c_int32)]


class DmcError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        super().__init__(f"{what}: {dmc_status_string(status)} ({status})" if what else
                         dmc_status_string(status))


_lib = None


def lib():
    """The loaded libdmc.so. Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2403_09636_gb300.build` (nvcc, sm_103a)")
        l = C.CDLL(LIB_PATH)
        vp, i32, i64, sz, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t, C.c_float
        cfgp = C.POINTER(dmc_cache_config)
        rcfgp = C.POINTER(dmc_retrofit_config)
        bcfgp = C.POINTER(dmc_beam_config)
        sig = {
            "dmc_cache_required_bytes": (sz, [cfgp]),
            "dmc_cache_create": (C.c_int, [cfgp, vp, sz, vp, C.POINTER(vp)]),
            "dmc_cache_destroy": (C.c_int, [vp]),
            "dmc_cache_reset": (C.c_int, [vp, vp]),
            "dmc_prefill_compress": (C.c_int, [vp, i32, i32, i32, vp, i64, i64, vp, vp, vp, i32,
                                               i32, vp]),
            "dmc_prefill_attention": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, i32, i32, vp, vp]),
            "dmc_decode_step": (C.c_int, [vp, i32, vp, vp, vp, vp, vp]),
            "dmc_decode_step_layers": (C.c_int, [vp, i32, i32, vp, vp, vp, vp, vp]),
            "dmc_decode_step_static_scratch": (C.c_int, [vp, i32, vp, vp, vp, vp, vp]),
            "dmc_cache_lengths": (C.c_int, [vp, i32, vp, vp]),
            "dmc_cache_export_heads": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp]),
            "dmc_cache_export_heads_padded": (C.c_int, [vp, i32, i32, vp, i32, vp, vp, vp, vp, vp]),
            "dmc_cache_status": (C.c_int, [vp, vp, C.POINTER(C.c_uint32), C.POINTER(i64)]),
            "dmc_status_string": (C.c_char_p, [C.c_int]),
            "dmc_retrofit_required_bytes": (sz, [rcfgp]),
            "dmc_retrofit_create": (C.c_int, [rcfgp, vp, sz, vp, C.POINTER(vp)]),
            "dmc_retrofit_destroy": (C.c_int, [vp]),
            "dmc_retrofit_saved_bytes": (sz, [vp, i32, i32]),
            "dmc_retrofit_states": (C.c_int, [vp, i32, vp, i64, i64, vp, vp, vp, f32, f32, vp, i32, i32, vp, vp,
                                              vp, vp, vp, vp]),
            "dmc_retrofit_states_backward": (C.c_int, [vp, i32, vp, i64, i64, vp, vp, vp, f32, f32, vp, i32, i32,
                                                       vp, vp, vp, vp, vp, vp, i64, i64, vp, vp, vp]),
            "dmc_retrofit_attention": (C.c_int, [vp, i32, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]),
            "dmc_retrofit_attention_backward": (C.c_int, [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp,
                                                          vp, vp, vp]),
            "dmc_retrofit_loss": (C.c_int, [vp, i32, vp, vp, vp, vp, vp, vp]),
            "dmc_retrofit_loss_backward": (C.c_int, [vp, i32, vp, vp, vp, vp, vp, vp, vp, vp]),
            "dmc_retrofit_status": (C.c_int, [vp, vp, C.POINTER(C.c_uint32)]),
            "dmc_rotate": (C.c_int, [i32, i32, i32, vp, vp, i32, i32, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, vp]),
            "dmc_cache_append": (C.c_int, [vp, i32, i32, i32, vp, vp, vp, vp, i32, i32, vp, vp, i32, vp, vp]),
            "dmc_cache_attend": (C.c_int, [vp, i32, vp, vp, vp]),
            "dmc_cache_reorder": (C.c_int, [vp, i32, i32, vp, vp]),
            "dmc_beam_required_bytes": (sz, [bcfgp]),
            "dmc_beam_create": (C.c_int, [bcfgp, vp, sz, vp, C.POINTER(vp)]),
            "dmc_beam_destroy": (C.c_int, [vp]),
            "dmc_beam_select": (C.c_int, [vp, vp, i64, vp, vp, i32, vp, vp, vp, vp, vp]),
        }
        for name, (res, args) in sig.items():
            f = getattr(l, name)
            f.restype, f.argtypes = res, args
        _lib = l
    return _lib


# ---------------------------------------------------------------- same-name forwarders

def dmc_cache_required_bytes(cfg: dmc_cache_config) -> int:
    return int(lib().dmc_cache_required_bytes(C.byref(cfg)))


def dmc_cache_create(cfg: dmc_cache_config, arena_ptr: int, arena_bytes: int, stream: int):
    """Returns (status, handle)."""
    h = C.c_void_p()
    st = lib().dmc_cache_create(C.byref(cfg), arena_ptr, arena_bytes, stream, C.byref(h))
    return st, h.value


def dmc_cache_destroy(handle) -> int:
    return lib().dmc_cache_destroy(handle)


def dmc_cache_reset(handle, stream: int) -> int:
    return lib().dmc_cache_reset(handle, stream)


def dmc_prefill_compress(handle, layer, first_seq, num_seqs, q_ptr, q_token_stride,
                         q_head_stride, k_ptr, v_ptr, cu_seqlens_ptr, total_tokens, max_seqlen,
                         stream) -> int:
    return lib().dmc_prefill_compress(handle, layer, first_seq, num_seqs, q_ptr, q_token_stride,
                                      q_head_stride, k_ptr, v_ptr, cu_seqlens_ptr, total_tokens,
                                      max_seqlen, stream)


def dmc_prefill_attention(handle, layer, first_seq, num_seqs, q_ptr, k_ptr, v_ptr, cu_seqlens_ptr,
                          total_tokens, max_seqlen, out_ptr, stream) -> int:
    return lib().dmc_prefill_attention(handle, layer, first_seq, num_seqs, q_ptr, k_ptr, v_ptr,
                                       cu_seqlens_ptr, total_tokens, max_seqlen, out_ptr, stream)


def dmc_decode_step(handle, layer, q_ptr, k_ptr, v_ptr, out_ptr, stream) -> int:
    return lib().dmc_decode_step(handle, layer, q_ptr, k_ptr, v_ptr, out_ptr, stream)


def dmc_decode_step_layers(handle, first_layer, num_layers, q_ptr, k_ptr, v_ptr, out_ptr,
                           stream) -> int:
    return lib().dmc_decode_step_layers(handle, first_layer, num_layers, q_ptr, k_ptr, v_ptr,
                                        out_ptr, stream)


def dmc_decode_step_static_scratch(handle, layer, q_ptr, k_ptr, v_ptr, out_ptr, stream) -> int:
    """dmc_decode_step for callers that cannot allocate device memory: its
    scratch lives in the library's static device array (see include/dmc.h)."""
    return lib().dmc_decode_step_static_scratch(handle, layer, q_ptr, k_ptr, v_ptr, out_ptr, stream)


def dmc_cache_lengths(handle, layer, out_ptr, stream) -> int:
    return lib().dmc_cache_lengths(handle, layer, out_ptr, stream)


def dmc_cache_export_heads(handle, layer, n, head_ids_ptr, cap, k_out_ptr, v_out_ptr, z_out_ptr,
                           len_out_ptr, stream) -> int:
    return lib().dmc_cache_export_heads(handle, layer, n, head_ids_ptr, cap, k_out_ptr, v_out_ptr,
                                        z_out_ptr, len_out_ptr, stream)


def dmc_cache_export_heads_padded(handle, layer, n, head_ids_ptr, cap, k_out_ptr, v_out_ptr,
                                  z_out_ptr, len_out_ptr, stream) -> int:
    return lib().dmc_cache_export_heads_padded(handle, layer, n, head_ids_ptr, cap, k_out_ptr,
                                               v_out_ptr, z_out_ptr, len_out_ptr, stream)


def dmc_cache_status(handle, stream):
    """Returns (status, fault_bits, pages_used). Synchronizes the stream."""
    bits = C.c_uint32()
    used = C.c_int64()
    st = lib().dmc_cache_status(handle, stream, C.byref(bits), C.byref(used))
    return st, int(bits.value), int(used.value)


def dmc_status_string(status: int) -> str:
    return lib().dmc_status_string(int(status)).decode()


def dmc_retrofit_required_bytes(cfg: dmc_retrofit_config) -> int:
    return int(lib().dmc_retrofit_required_bytes(C.byref(cfg)))


def dmc_retrofit_create(cfg: dmc_retrofit_config, arena_ptr: int, arena_bytes: int, stream: int):
    """Returns (status, handle)."""
    h = C.c_void_p()
    st = lib().dmc_retrofit_create(C.byref(cfg), arena_ptr, arena_bytes, stream, C.byref(h))
    return st, h.value


def dmc_retrofit_destroy(handle) -> int:
    return lib().dmc_retrofit_destroy(handle)


def dmc_retrofit_saved_bytes(handle, num_seqs, total_tokens) -> int:
    return int(lib().dmc_retrofit_saved_bytes(handle, num_seqs, total_tokens))


def dmc_retrofit_states(handle, num_seqs, q_ptr, q_token_stride, q_head_stride, k_ptr, v_ptr, noise_ptr, offset,
                        temperature, cu_seqlens_ptr, total_tokens, max_seqlen, kt_ptr, vt_ptr, alpha_ptr, bias_ptr,
                        saved_ptr, stream) -> int:
    return lib().dmc_retrofit_states(handle, num_seqs, q_ptr, q_token_stride, q_head_stride, k_ptr, v_ptr, noise_ptr,
                                     offset, temperature, cu_seqlens_ptr, total_tokens, max_seqlen, kt_ptr, vt_ptr,
                                     alpha_ptr, bias_ptr, saved_ptr, stream)


def dmc_retrofit_states_backward(handle, num_seqs, q_ptr, q_token_stride, q_head_stride, k_ptr, v_ptr, noise_ptr,
                                 offset, temperature, cu_seqlens_ptr, total_tokens, max_seqlen, saved_ptr, dkt_ptr,
                                 dvt_ptr, dbias_ptr, dalpha_ptr, dq_ptr, dq_token_stride, dq_head_stride, dk_ptr,
                                 dv_ptr, stream) -> int:
    return lib().dmc_retrofit_states_backward(handle, num_seqs, q_ptr, q_token_stride, q_head_stride, k_ptr, v_ptr,
                                              noise_ptr, offset, temperature, cu_seqlens_ptr, total_tokens,
                                              max_seqlen, saved_ptr, dkt_ptr, dvt_ptr, dbias_ptr, dalpha_ptr, dq_ptr,
                                              dq_token_stride, dq_head_stride, dk_ptr, dv_ptr, stream)


def dmc_retrofit_attention(handle, num_seqs, q_ptr, k_ptr, v_ptr, bias_ptr, cu_seqlens_ptr, total_tokens, max_seqlen,
                           out_ptr, lse_ptr, stream) -> int:
    return lib().dmc_retrofit_attention(handle, num_seqs, q_ptr, k_ptr, v_ptr, bias_ptr, cu_seqlens_ptr,
                                        total_tokens, max_seqlen, out_ptr, lse_ptr, stream)


def dmc_retrofit_attention_backward(handle, num_seqs, q_ptr, k_ptr, v_ptr, bias_ptr, out_ptr, lse_ptr, dout_ptr,
                                    cu_seqlens_ptr, total_tokens, max_seqlen, dq_ptr, dk_ptr, dv_ptr, dbias_ptr,
                                    stream) -> int:
    return lib().dmc_retrofit_attention_backward(handle, num_seqs, q_ptr, k_ptr, v_ptr, bias_ptr, out_ptr, lse_ptr,
                                                 dout_ptr, cu_seqlens_ptr, total_tokens, max_seqlen, dq_ptr, dk_ptr,
                                                 dv_ptr, dbias_ptr, stream)


def dmc_retrofit_loss(handle, num_tokens, hidden_ptr, weight_ptr, targets_ptr, loss_ptr, lse_ptr, stream) -> int:
    return lib().dmc_retrofit_loss(handle, num_tokens, hidden_ptr, weight_ptr, targets_ptr, loss_ptr, lse_ptr, stream)


def dmc_retrofit_loss_backward(handle, num_tokens, hidden_ptr, weight_ptr, targets_ptr, lse_ptr, dloss_ptr,
                               dhidden_ptr, dweight_ptr, stream) -> int:
    return lib().dmc_retrofit_loss_backward(handle, num_tokens, hidden_ptr, weight_ptr, targets_ptr, lse_ptr,
                                            dloss_ptr, dhidden_ptr, dweight_ptr, stream)


def dmc_retrofit_status(handle, stream):
    """Returns (status, fault_bits). Synchronizes the stream."""
    bits = C.c_uint32()
    st = lib().dmc_retrofit_status(handle, stream, C.byref(bits))
    return st, int(bits.value)


def dmc_rotate(dtype, head_dim, num_tokens, positions_ptr, turns_ptr, interleaved, inverse, num_q_heads, q_ptr,
               q_token_stride, q_out_ptr, q_out_token_stride, num_k_heads, k_ptr, k_token_stride, k_out_ptr,
               k_out_token_stride, stream) -> int:
    return lib().dmc_rotate(dtype, head_dim, num_tokens, positions_ptr, turns_ptr, interleaved, inverse, num_q_heads,
                            q_ptr, q_token_stride, q_out_ptr, q_out_token_stride, num_k_heads, k_ptr, k_token_stride,
                            k_out_ptr, k_out_token_stride, stream)


def dmc_cache_append(handle, layer, first_seq, num_seqs, q_ptr, k_ptr, v_ptr, cu_seqlens_ptr, total_tokens, max_seqlen,
                     positions_ptr, turns_ptr, interleaved, q_out_ptr, stream) -> int:
    return lib().dmc_cache_append(handle, layer, first_seq, num_seqs, q_ptr, k_ptr, v_ptr, cu_seqlens_ptr, total_tokens,
                                  max_seqlen, positions_ptr, turns_ptr, interleaved, q_out_ptr, stream)


def dmc_cache_attend(handle, layer, q_ptr, out_ptr, stream) -> int:
    return lib().dmc_cache_attend(handle, layer, q_ptr, out_ptr, stream)


def dmc_cache_reorder(handle, first_seq, num_seqs, parents_ptr, stream) -> int:
    return lib().dmc_cache_reorder(handle, first_seq, num_seqs, parents_ptr, stream)


def dmc_beam_required_bytes(cfg: dmc_beam_config) -> int:
    return int(lib().dmc_beam_required_bytes(C.byref(cfg)))


def dmc_beam_create(cfg: dmc_beam_config, arena_ptr: int, arena_bytes: int, stream: int):
    """Returns (status, handle)."""
    h = C.c_void_p()
    st = lib().dmc_beam_create(C.byref(cfg), arena_ptr, arena_bytes, stream, C.byref(h))
    return st, h.value


def dmc_beam_destroy(handle) -> int:
    return lib().dmc_beam_destroy(handle)


def dmc_beam_select(handle, logits_ptr, logits_row_stride, scores_ptr, finished_ptr, eos, out_scores_ptr, out_tokens_ptr,
                    out_parents_ptr, out_done_ptr, stream) -> int:
    return lib().dmc_beam_select(handle, logits_ptr, logits_row_stride, scores_ptr, finished_ptr, eos, out_scores_ptr,
                                 out_tokens_ptr, out_parents_ptr, out_done_ptr, stream)


def _check(st: int, what: str):
    if st != DMC_OK:
        raise DmcError(st, what)


# ---------------------------------------------------------------- convenience wrapper

class DmcCache:
    """A cache living in a torch-allocated device arena. Tensors passed to the
    methods must be contiguous, on the cache's device, in the cache dtype. The arena is memory of the constructor's
    stream, and waits for every stream that a method used when the cache is dropped: streams must outlive it."""

    def __init__(self, num_layers, batch, num_q_heads, num_kv_heads, head_dim, dtype,
                 max_slots_per_head, num_pages, max_prefill_tokens=0, device=None, stream=None,
                 window=0):
        import torch
        self.torch = torch
        self.device = torch.device(device if device is not None else "cuda")
        cuda = self.device.type == "cuda" and torch.cuda.is_available()
        self.index = (torch.cuda.current_device() if self.device.index is None else self.device.index) if cuda else -1
        tdt = {torch.float32: DMC_F32, torch.bfloat16: DMC_BF16}[dtype]
        self.dtype = dtype
        self.cfg = dmc_cache_config(num_layers, batch, num_q_heads, num_kv_heads, head_dim, tdt,
                                    PAGE_SIZE, max_slots_per_head, int(num_pages),
                                    int(max_prefill_tokens), int(window))
        self.nbytes = dmc_cache_required_bytes(self.cfg)
        if self.nbytes == 0:
            raise DmcError(DMC_ERR_INVALID_ARG, "dmc_cache_required_bytes")
        raw = self._s(stream)
        self.arena = self._on(raw, lambda: torch.empty(self.nbytes, dtype=torch.uint8, device=self.device))
        self._streams = {raw}  # that the arena's memory waits for when it is given up (_used_on)
        st, self.handle = dmc_cache_create(self.cfg, self.arena.data_ptr(), self.nbytes, raw)
        _check(st, "dmc_cache_create")
        self.lib = lib()
        self.num_q_heads, self.num_kv_heads, self.head_dim = int(num_q_heads), int(num_kv_heads), int(head_dim)
        self.queries = (int(batch), self.num_q_heads, self.head_dim)
        self._raw, self._empty_like, self._int32 = torch._C._cuda_getCurrentRawStream, torch.empty_like, torch.int32
        self._export = None

    def _s(self, stream):
        if stream is None:
            # the current stream's handle without a Stream object: 0.1 us instead of
            # 3.5, of the 8 that the host spent on a decode call
            c = self.torch._C
            index = self.device.index
            return c._cuda_getCurrentRawStream(c._cuda_getDevice() if index is None else index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def _stream(self, raw):
        # (an ExternalStream of the number 0 would be another one)
        cuda = self.torch.cuda
        return cuda.ExternalStream(raw, device=self.device) if raw else cuda.default_stream(self.device)

    def _used_on(self, raw):
        self.arena.record_stream(self._stream(raw))
        self._streams.add(raw)

    def _call(self, stream):
        """The number of a call's stream, which the arena's memory waits for when it is given up."""
        raw = self._s(stream)
        if raw not in self._streams:
            self._used_on(raw)
        return raw

    def _on(self, raw, make):
        """make(), its memory that of the stream of this number."""
        if self.device.type != "cuda" or raw == self._s(None):
            return make()
        with self.torch.cuda.stream(self._stream(raw)):
            return make()

    def close(self):
        if getattr(self, "handle", None):
            dmc_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self, stream=None):
        _check(dmc_cache_reset(self.handle, self._call(stream)), "dmc_cache_reset")

    def prefill(self, layer, q0, k, v, cu_seqlens, max_seqlen, first_seq=0, stream=None):
        """q0: [total, Hq] (or any tensor whose element (t, j, 0) sits at
        t*stride(0) + j*stride(1)); k, v: [total, Hkv, D]; cu_seqlens int32."""
        n = cu_seqlens.numel() - 1
        total = k.shape[0]
        _check(dmc_prefill_compress(self.handle, layer, first_seq, n, q0.data_ptr(),
                                    q0.stride(0), q0.stride(1), k.data_ptr(), v.data_ptr(),
                                    cu_seqlens.data_ptr(), total, int(max_seqlen),
                                    self._call(stream)), "dmc_prefill_compress")

    def prefill_attention(self, layer, q, k, v, cu_seqlens, max_seqlen, out, first_seq=0,
                          stream=None):
        """q, out: [total, Hq, D]; k, v: [total, Hkv, D]; cu_seqlens int32."""
        n = cu_seqlens.numel() - 1
        _check(dmc_prefill_attention(self.handle, layer, first_seq, n, q.data_ptr(), k.data_ptr(),
                                     v.data_ptr(), cu_seqlens.data_ptr(), k.shape[0],
                                     int(max_seqlen), out.data_ptr(), self._call(stream)),
               "dmc_prefill_attention")

    def decode(self, layer, q, k, v, out, stream=None):
        _check(dmc_decode_step(self.handle, layer, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                               out.data_ptr(), self._call(stream)), "dmc_decode_step")

    def decode_layers(self, first_layer, q, k, v, out, stream=None):
        """q, out: [n, B, Hq, D]; k, v: [n, B, Hkv, D] for layers first_layer .. + n - 1."""
        _check(dmc_decode_step_layers(self.handle, first_layer, q.shape[0], q.data_ptr(),
                                      k.data_ptr(), v.data_ptr(), out.data_ptr(), self._call(stream)),
               "dmc_decode_step_layers")

    # ---- calls that check their tensors (what does not fit is refused with ValueError). The check is one expression,
    # and only where it fails is the tensor looked for that does not fit: with a check for each tensor an append took the
    # host 11.9 us, 6.9 so

    def _is(self, name, t, shape, dtype):
        torch = self.torch
        if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == self.index
                and t.is_contiguous()):
            return t.data_ptr()
        what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} must be contiguous {dtype} {tuple(shape)} on {self.device}, got {what}")

    def _new(self, like, stream):
        """A tensor as `like`, of memory that belongs to the call's stream."""
        return self._on(self._s(stream), lambda: self.torch.empty_like(like))

    def _append_is_wrong(self, q, k, v, positions, rotary, cu_seqlens, n, q_out):
        c, t = self.cfg, self.torch
        if not isinstance(k, t.Tensor) or k.dim() != 3:
            raise ValueError("k must be [tokens, KV heads, head_dim]")
        T, D, dt = k.shape[0], c.head_dim, self.dtype
        self._is("q", q, (T, c.num_q_heads, D), dt)
        self._is("k", k, (T, c.num_kv_heads, D), dt)
        self._is("v", v, (T, c.num_kv_heads, D), dt)
        if cu_seqlens is not None:
            if not isinstance(cu_seqlens, t.Tensor) or cu_seqlens.dim() != 1 or cu_seqlens.numel() < 1:
                raise ValueError("cu_seqlens must be int32 [sequences + 1]")
            n = cu_seqlens.numel() - 1
            self._is("cu_seqlens", cu_seqlens, (n + 1,), t.int32)
        if rotary is None:
            raise ValueError("positions and q_out are for a rotation")
        if rotary.head_dim != D or rotary.index != self.index:
            raise ValueError(f"the rotation is for heads of {rotary.head_dim} on {rotary.turns.device}")
        self._is("positions", positions, (n,), t.int32)
        self._is("q_out", q_out, (T, c.num_q_heads, D), dt)
        raise ValueError("the tensors do not fit")

    def append(self, layer, q, k, v, positions=None, rotary=None, cu_seqlens=None, max_seqlen=1, first_seq=0, q_out=None,
               stream=None):
        """New tokens join the cache, rotated on the way; returns the rotated queries (None without a rotation).
        q: [T, Hq, D]; k, v: [T, Hkv, D], of one token for each of T sequences from first_seq on, or packed
        by cu_seqlens (int32 [sequences + 1]); positions: int32, one for each sequence's first token; rotary: a
        `rotary.Rotary`; q_out may be q. Rows of no sequence (cu_seqlens that end before T) are left as they are: in a
        tensor that this call makes, as its memory came."""
        i32, dt, index = self._int32, self.dtype, self.index
        try:
            T, H, D = rows = k.shape
            queries = (T, self.num_q_heads, D)
            n = T if cu_seqlens is None else cu_seqlens.numel() - 1
            fits = (H == self.num_kv_heads and D == self.head_dim and q.shape == queries and v.shape == rows
                    and q.dtype is dt and k.dtype is dt and v.dtype is dt and q.get_device() == index
                    and k.get_device() == index and v.get_device() == index and q.is_contiguous() and k.is_contiguous()
                    and v.is_contiguous())
            if cu_seqlens is not None:
                fits = (fits and cu_seqlens.dim() == 1 and cu_seqlens.dtype is i32 and cu_seqlens.get_device() == index
                        and cu_seqlens.is_contiguous())
            if rotary is None:
                fits = fits and positions is None and q_out is None
            else:
                fits = (fits and rotary.head_dim == D and rotary.index == index and positions.shape == (n,)
                        and positions.dtype is i32 and positions.get_device() == index and positions.is_contiguous())
                if q_out is not None:
                    fits = (fits and q_out.shape == queries and q_out.dtype is dt and q_out.get_device() == index
                            and q_out.is_contiguous())
        except (AttributeError, TypeError, ValueError):
            fits, n = False, 0
        if not fits:
            self._append_is_wrong(q, k, v, positions, rotary, cu_seqlens, n, q_out)
        raw = self._raw(index) if stream is None else self._s(stream)
        if raw not in self._streams:
            self._used_on(raw)
        at = turns = to = None
        pairs = 0
        if rotary is not None:
            if q_out is None:
                q_out = self._empty_like(q) if stream is None else self._new(q, stream)
            if raw not in rotary.streams:
                rotary.used_on(raw)
            at, turns, pairs, to = positions.data_ptr(), rotary.pointer, rotary.pairs, q_out.data_ptr()
        st = self.lib.dmc_cache_append(self.handle, layer, first_seq, n, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                       None if cu_seqlens is None else cu_seqlens.data_ptr(), T,
                                       max_seqlen if max_seqlen < T else T, at, turns, pairs, to, raw)
        if st:
            _check(st, "dmc_cache_append")
        return q_out

    def attend(self, layer, q, out=None, stream=None):
        """Attention of q [batch, Hq, D] over the cache as it stands; the cache is not changed."""
        try:
            fits = (q.shape == self.queries and q.dtype is self.dtype and q.get_device() == self.index and q.is_contiguous())
        except AttributeError:
            fits = False
        p = q.data_ptr() if fits else self._is("q", q, self.queries, self.dtype)
        if out is None:
            out = self._empty_like(q) if stream is None else self._new(q, stream)
            to = out.data_ptr()
        else:
            to = self._is("out", out, self.queries, self.dtype)
        raw = self._raw(self.index) if stream is None else self._s(stream)
        if raw not in self._streams:
            self._used_on(raw)
        st = self.lib.dmc_cache_attend(self.handle, layer, p, to, raw)
        if st:
            _check(st, "dmc_cache_attend")
        return out

    def reorder(self, parents, first_seq=0, stream=None):
        """Sequence first_seq + j continues from the cache of sequence first_seq + parents[j] (int32 on the cache's
        device), in every layer. What they have in common is shared."""
        if not isinstance(parents, self.torch.Tensor) or parents.dim() < 1:
            raise ValueError("parents must be int32, one for each sequence")
        p = self._is("parents", parents, parents.shape, self.torch.int32)
        st = self.lib.dmc_cache_reorder(self.handle, first_seq, parents.numel(), p, self._call(stream))
        if st:
            _check(st, "dmc_cache_reorder")

    def lengths(self, layer, stream=None):
        raw = self._call(stream)
        out = self._counts() if stream is None else self._on(raw, self._counts)
        _check(dmc_cache_lengths(self.handle, layer, out.data_ptr(), raw), "dmc_cache_lengths")
        return out

    def _counts(self):
        t = self.torch
        return t.empty((self.cfg.batch, self.cfg.num_kv_heads), dtype=t.int32, device=self.device)

    def export_heads(self, layer, head_ids, cap, stream=None):
        """(k, v, z, len) of the heads head_ids (int32 on the cache's device, or a list), padded to cap slots with zeros:
        new tensors of the call's stream."""
        raw = self._call(stream)
        if stream is not None and self.device.type == "cuda" and raw != self._s(None):
            with self.torch.cuda.stream(self._stream(raw)):
                return self._export_heads(layer, head_ids, cap, raw)
        return self._export_heads(layer, head_ids, cap, raw)

    def _export_heads(self, layer, head_ids, cap, raw):
        t = self.torch
        ids = head_ids
        if not (isinstance(ids, t.Tensor) and ids.dtype is t.int32 and ids.get_device() == self.index and ids.is_contiguous()):
            ids = t.as_tensor(head_ids, dtype=t.int32, device=self.device).contiguous()
        n = ids.numel()
        # (an element each: the host makes a tensor like another sooner than anew. Shapes and tensors are one attribute, read
        # once: another thread may export other shapes meanwhile)
        kept = self._export
        if kept is None or kept[0] != (n, cap):
            kept = self._export = (n, cap), *(t.empty(1, dtype=d, device=self.device).expand(shape) for d, shape in (
                (self.dtype, (n, cap, self.head_dim)), (t.float32, (n, cap)), (t.int32, (n,))))
        _, rows, sums, counts = kept
        new = self._empty_like
        k, v, z, ln = new(rows), new(rows), new(sums), new(counts)  # padded: every row is written
        st = self.lib.dmc_cache_export_heads_padded(self.handle, layer, n, ids.data_ptr(), cap, k.data_ptr(), v.data_ptr(),
                                                    z.data_ptr(), ln.data_ptr(), raw)
        if st:
            _check(st, "dmc_cache_export_heads")
        return k, v, z, ln

    def status(self, stream=None):
        """(status, fault bits, pages used); synchronizes the stream."""
        return dmc_cache_status(self.handle, self._s(stream))
