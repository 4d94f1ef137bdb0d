"""Exports of one cache by two host threads (CPU; the call of the library is replaced)."""
import ctypes
import sys
import threading

import pytest
import torch

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300 import build as B


class Library:
    @staticmethod
    def dmc_cache_export_heads_padded(handle, layer, n, ids, cap, k, v, z, counts, stream):
        return P.DMC_OK


@pytest.fixture
def cache(monkeypatch):
    B.build()
    monkeypatch.setattr(P, "dmc_cache_create", lambda *a: (P.DMC_OK, 1))
    c = P.DmcCache(1, 8, 2, 2, 64, torch.bfloat16, 64, 32, device="cpu", stream=0)
    c.lib = Library
    yield c
    c.handle = None


def test_each_call_gets_buffers_of_its_own_shape(cache):
    """The library writes n x cap rows: buffers of another call's shape would be written past their end."""
    wrong, start = [], threading.Barrier(2)

    def work(n, cap):
        ids = list(range(n))
        start.wait()
        for _ in range(8000):
            k, v, z, ln = cache.export_heads(0, ids, cap, stream=0)
            got = tuple(k.shape), tuple(v.shape), tuple(z.shape), tuple(ln.shape)
            if got != ((n, cap, 64), (n, cap, 64), (n, cap), (n,)):
                wrong.append(got)

    was = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)
    try:
        threads = [threading.Thread(target=work, args=a) for a in ((4, 8), (2, 3))]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(was)
    assert not wrong, (len(wrong), wrong[:3])


def test_results_are_dense_and_of_the_call(cache):
    for n, cap in ((3, 5), (1, 5), (3, 1), (1, 1), (3, 0), (0, 4)):
        k, v, z, ln = cache.export_heads(0, list(range(n)), cap, stream=0)
        assert (k.shape, z.shape, ln.shape) == ((n, cap, 64), (n, cap), (n,)) and v.shape == k.shape
        assert all(t.is_contiguous() for t in (k, v, z, ln))
        assert (k.dtype, v.dtype, z.dtype, ln.dtype) == (torch.bfloat16, torch.bfloat16, torch.float32, torch.int32)


def test_heads_named_by_every_other_element(cache):
    """Ids of a tensor with a stride are those of its elements, not of its memory."""
    seen = []

    class Reads(Library):
        @staticmethod
        def dmc_cache_export_heads_padded(handle, layer, n, ids, *rest):
            seen.append(list((ctypes.c_int32 * n).from_address(ids)))
            return P.DMC_OK

    cache.lib = Reads
    for ids in (torch.arange(12, dtype=torch.int32)[::2], torch.arange(12)[1::3], [7, 1]):
        cache.export_heads(0, ids, 4, stream=0)
    assert seen == [[0, 2, 4, 6, 8, 10], [1, 4, 7, 10], [7, 1]]
