"""A cache's memory and the streams that its methods name (GPU)."""
import pytest
import torch

from generate_harness import cache_of, tokens
from paper_2403_09636_gb300 import DmcCache

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def stream_of(t):
    at = t.data_ptr()
    return [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]


@pytest.fixture
def inputs(cuda_dev):
    """Tokens of two sequences; a call of every method that launches something, as f(cache, stream)."""
    q, k, v = (t.cuda() for t in tokens(torch.Generator().manual_seed(1), 2, 2, 2, 128, BF16, 1.0))
    cu, out = torch.tensor([0, 1, 2], dtype=torch.int32).cuda(), torch.empty_like(q)
    parents = torch.tensor([0, 0], dtype=torch.int32).cuda()
    ids = torch.arange(4, dtype=torch.int32).cuda()
    calls = {
        "reset": lambda c, s: c.reset(stream=s),
        "prefill": lambda c, s: c.prefill(0, q[..., 0], k, v, cu, 1, stream=s),
        "prefill_attention": lambda c, s: c.prefill_attention(0, q, k, v, cu, 1, out, stream=s),
        "decode": lambda c, s: c.decode(0, q, k, v, out, stream=s),
        "decode_layers": lambda c, s: c.decode_layers(0, q[None], k[None], v[None], out, stream=s),
        "append": lambda c, s: c.append(0, q, k, v, stream=s),
        "attend": lambda c, s: c.attend(0, q, out, stream=s),
        "reorder": lambda c, s: c.reorder(parents, stream=s),
        "lengths": lambda c, s: c.lengths(0, stream=s),
        "export_heads": lambda c, s: c.export_heads(0, ids, 4, stream=s),
    }
    torch.cuda.synchronize()
    return calls


def made(stream=None):
    return DmcCache(1, 2, 2, 2, 128, BF16, 40, 16, 8, stream=stream)


@pytest.mark.parametrize("call", ["reset", "prefill", "prefill_attention", "decode", "decode_layers", "append", "attend",
                                  "reorder", "lengths", "export_heads"])
@pytest.mark.parametrize("where", ["named", "current", "created there"])
def test_a_cache_dropped_while_a_stream_works(inputs, call, where):
    """Its arena is not handed out again before the stream of its last call is done, whichever way the call got it."""
    side = torch.cuda.Stream()
    inputs[call](made(), None)  # (a kernel's first launch takes the host longer than the stream is busy)
    if where == "created there":
        cache = made(side)
    else:
        cache = made()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        if where == "current":
            inputs[call](cache, None)
    if where != "current":
        inputs[call](cache, side)
    place, size = cache.arena.data_ptr(), cache.nbytes
    assert not side.query()
    del cache
    again = torch.empty(size, dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(side):
        there = torch.empty(size, dtype=torch.uint8, device="cuda")
    places = [again.data_ptr()] + ([] if where == "created there" else [there.data_ptr()])
    side.synchronize()
    assert place not in places


def test_the_arena_is_memory_of_the_constructors_stream(cuda_dev):
    """Clearing it is in order with what the memory was used for before."""
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    here, there = made(), made(side)
    assert stream_of(here.arena) == [torch.cuda.current_stream().cuda_stream]
    assert stream_of(there.arena) == [side.cuda_stream]
    with torch.cuda.stream(side):
        assert stream_of(made(0).arena) == [0]
        assert stream_of(made().arena) == [side.cuda_stream]
    torch.cuda.synchronize()


def test_results_are_memory_of_the_calls_stream(cuda_dev):
    """A place that the current stream has just freed, and may still write, is not given to a call on another stream."""
    side, cache = torch.cuda.Stream(), made()
    q, k, v = (t.cuda() for t in tokens(torch.Generator().manual_seed(3), 2, 2, 2, 128, BF16, 1.0))
    cache.append(0, q, k, v)
    ids = torch.arange(4, dtype=torch.int32).cuda()
    torch.cuda.synchronize()
    for name in (side, side.cuda_stream):
        for call in (lambda **k: (cache.lengths(0, **k),), lambda **k: cache.export_heads(0, ids, 4, **k),
                     lambda **k: cache.export_heads(0, [0, 1, 2, 3], 4, **k)):
            want = [t.clone() for t in call()]
            torch.cuda.synchronize()
            freed = [torch.empty_like(t) for _ in range(4) for t in want]
            places = {t.data_ptr() for t in freed}
            del freed  # the current stream's to use again
            got = call(stream=name)
            side.synchronize()
            assert not places & {t.data_ptr() for t in got}
            assert all(stream_of(t) == [side.cuda_stream] for t in got)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_cache_used_in_a_captured_graph_alone(cuda_dev):
    """The capture's stream is noted like any other; the graph replays, and the cache can be dropped after it."""
    q, k, v = (t.cuda() for t in tokens(torch.Generator().manual_seed(2), 2, 2, 2, 64, F32, 1.0))
    cache, out = cache_of(2, 2, 2, 64, F32, 40), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cache.decode(0, q, k, v, out)
    for _ in range(5):
        graph.replay()
    assert cache.lengths(0).tolist() == [[5, 5], [5, 5]] and cache.status()[:2] == (0, 0)
    torch.cuda.synchronize()
    del graph, cache
    torch.empty(1 << 20, device="cuda").zero_()
    torch.cuda.synchronize()
