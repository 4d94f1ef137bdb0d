"""Beam search over a compressed cache: the selection among beams and words (include/dmc.h has the rules).

One step of a search over `groups` texts with `beams` beams each, whose caches are the sequences g * beams + b:

    select = BeamSelect(groups, beams, vocab, dtype=logits.dtype)
    scores, tokens, parents, done = select.select(logits, scores, done, eos)
    cache.reorder(parents.view(-1))
"""
from __future__ import annotations

import torch

from . import (DMC_BF16, DMC_ERR_INVALID_ARG, DMC_F32, DmcError, _check, dmc_beam_config, dmc_beam_create,
               dmc_beam_destroy, dmc_beam_required_bytes, lib)


class BeamSelect:
    """Scratch and entry point of the selection for one shape. Calls on one handle must be ordered on the GPU.

    Outputs are new tensors of the call's stream, the current one unless `stream` names another, or those given as
    `out`, (scores, tokens, parents, done)."""

    def __init__(self, groups, beams, vocab, keep=None, dtype=torch.bfloat16, device=None, stream=None):
        self.handle = None
        codes = {torch.float32: DMC_F32, torch.bfloat16: DMC_BF16}
        if dtype not in codes:
            raise ValueError(f"dtype must be float32 or bfloat16, got {dtype}")
        dev = torch.device(device if device is not None else "cuda")
        if dev.type == "cuda" and dev.index is None and torch.cuda.is_available():
            dev = torch.device("cuda", torch.cuda.current_device())
        self.dtype, self.device, self.index = dtype, dev, dev.index if dev.type == "cuda" else -1
        self.groups, self.beams, self.vocab = int(groups), int(beams), int(vocab)
        self.keep = self.beams if keep is None else int(keep)
        self.cfg = dmc_beam_config(self.groups, self.beams, self.keep, self.vocab, codes[dtype])
        self.nbytes = dmc_beam_required_bytes(self.cfg)
        if self.nbytes == 0:
            raise DmcError(DMC_ERR_INVALID_ARG, "dmc_beam_required_bytes")
        self.arena = self._on(stream, lambda: torch.empty(self.nbytes, dtype=torch.uint8, device=dev))
        self._streams = {self._raw(stream)}  # that the arena's memory waits for when it is given up
        st, self.handle = dmc_beam_create(self.cfg, self.arena.data_ptr(), self.nbytes, self._raw(stream))
        _check(st, "dmc_beam_create")
        self.lib = lib()
        self._shape = (self.groups, self.beams)
        self._rows = (self.groups * self.beams, self.vocab)
        shape = (self.groups, self.keep)
        self._kinds = tuple(zip(("scores", "tokens", "parents", "done"), (torch.float32, torch.int32, torch.int32, torch.bool)))
        self._like = [torch.empty(shape, dtype=t, device=dev) for _, t in self._kinds]  # of the results

    def _raw(self, stream):
        if stream is None:
            return torch._C._cuda_getCurrentRawStream(self.index)
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    def _stream(self, raw):
        # (an ExternalStream of the number 0 would be another one)
        return torch.cuda.ExternalStream(raw, device=self.device) if raw else torch.cuda.default_stream(self.device)

    def _on(self, stream, make):
        """make(), its memory that of the call's stream."""
        raw = self._raw(stream)
        if stream is None or raw == self._raw(None):
            return make()
        with torch.cuda.stream(self._stream(raw)):
            return make()

    def close(self):
        if getattr(self, "handle", None):
            dmc_beam_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _is(self, name, t, shape, dtype):
        if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == self.index
                and t.is_contiguous()):
            return t.data_ptr()
        what = f"{t.dtype} {tuple(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} must be contiguous {dtype} {shape} on {self.device}, got {what}")

    def select(self, logits, scores, finished=None, eos=-1, out=None, stream=None):
        """(scores fp32, tokens int32, parents int32, done bool), [groups, keep]: the best continuations, best first.
        logits: [groups * beams, vocab], rows may be apart; scores: fp32 [groups, beams]; finished: bool
        [groups, beams] or None; eos: the end word, -1 for none. parents are rows of logits."""
        rows, index = self._rows, self.index
        if (not isinstance(logits, torch.Tensor) or logits.dtype is not self.dtype or logits.shape != rows
                or logits.get_device() != index):
            raise ValueError(f"logits must be {self.dtype} {rows} on {self.device}")
        apart, step = logits.stride()
        if rows[0] == 1:
            apart = rows[1]
        if apart < rows[1] or (step != 1 and rows[1] > 1):
            raise ValueError(f"logits' words must be contiguous and its rows apart, got strides {logits.stride()}")
        shape = self._shape
        if (isinstance(scores, torch.Tensor) and scores.dtype is torch.float32 and scores.shape == shape
                and scores.get_device() == index and scores.is_contiguous()):
            sp = scores.data_ptr()
        else:
            sp = self._is("scores", scores, shape, torch.float32)
        fp = None if finished is None else self._is("finished", finished, shape, torch.bool)
        raw = torch._C._cuda_getCurrentRawStream(index) if stream is None else self._raw(stream)
        like = self._like
        if out is None:
            out = s, t, p, d = (tuple(map(torch.empty_like, like)) if stream is None
                                else self._on(stream, lambda: tuple(map(torch.empty_like, like))))
            ptrs = (s.data_ptr(), t.data_ptr(), p.data_ptr(), d.data_ptr())
        else:
            if len(out) != 4:
                raise ValueError("out must hold 4 tensors: scores, tokens, parents, done")
            ptrs = [self._is(name, t, x.shape, kind) for (name, kind), t, x in zip(self._kinds, out, like)]
        if raw not in self._streams:
            self.arena.record_stream(self._stream(raw))
            self._streams.add(raw)
        st = self.lib.dmc_beam_select(self.handle, logits.data_ptr(), apart, sp, fp, eos, *ptrs, raw)
        if st:
            _check(st, "dmc_beam_select")
        return out
