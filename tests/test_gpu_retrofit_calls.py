"""What the retrofitting calls refuse beside shapes and types: another device than the handle's, addresses that are
not aligned to their elements, outputs that lie in one place, tokens of no sequence; and whose memory a call on
another stream uses."""
import ctypes as C

import pytest
import torch

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300.retrofit import DmcRetrofit
from retrofit_harness import attention_inputs, cu_of, handle, on, states_inputs

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
LENS, HEADS = [40, 24], (4, 2, 64)


@pytest.fixture(scope="module")
def ready():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    dev = torch.device("cuda:0")
    x, s = on(attention_inputs(LENS, *HEADS, BF16), dev), on(states_inputs(LENS, *HEADS, BF16), dev)
    return x, s, cu_of(LENS, dev), dev


def both(dev):
    return DmcRetrofit(*HEADS, dtype=BF16, max_tokens=sum(LENS), max_seqs=2, hidden=64, vocab=50, device=dev)


def test_another_device_than_the_handles(ready):
    """A handle that says it belongs to another device than the current one (the number behind its config is
    changed for that): every call refuses before it launches anything."""
    x, s, cu, dev = ready
    h = both(dev)
    saved = h.states(s["q0"], s["k"], s["v"], cu, 40)[-1]
    o, lse = h.attention(x["q"], x["k"], x["v"], cu, 40)
    hid, w = torch.zeros(8, 64, dtype=BF16, device=dev), torch.zeros(50, 64, dtype=BF16, device=dev)
    t, f = torch.zeros(8, dtype=torch.int32, device=dev), torch.zeros(8, device=dev)
    device = C.c_int.from_address(h.handle + C.sizeof(P.dmc_retrofit_config))
    assert device.value == torch.cuda.current_device()
    calls = [lambda: h.states(s["q0"], s["k"], s["v"], cu, 40),
             lambda: h.states_backward(s["q0"], s["k"], s["v"], cu, 40, saved, s["dkt"], s["dvt"], s["dbias"]),
             lambda: h.attention(x["q"], x["k"], x["v"], cu, 40),
             lambda: h.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, cu, 40),
             lambda: h.loss(hid, w, t), lambda: h.loss_backward(f, hid, w, t, f)]
    for call in calls:
        call()
    device.value += 1
    try:
        for i, call in enumerate(calls):
            with pytest.raises(P.DmcError) as e:
                call()
            assert e.value.status == P.DMC_ERR_INVALID_ARG, i
        assert h.status()[0] == P.DMC_ERR_INVALID_ARG
    finally:
        device.value -= 1
    assert h.status() == (0, 0)


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_addresses_that_are_not_their_elements(ready, dtype):
    """q's and dq's first components may lie anywhere, but on whole elements; dbias too."""
    _, _, cu, dev = ready
    size = 4 if dtype == torch.float32 else 2
    h = handle(dev, *HEADS, dtype, LENS)
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device=dev)
    p, T = buf.data_ptr(), 64

    def states(q=p):
        return P.dmc_retrofit_states(h.handle, 2, q, 4, 1, p, p, None, 5.0, 0.1, cu.data_ptr(), T, 40, p, p, p, p, p, 0)

    def states_backward(q=p, dq=p, db=p, st=4, sh=1):
        return P.dmc_retrofit_states_backward(h.handle, 2, q, 4, 1, p, p, None, 5.0, 0.1, cu.data_ptr(), T, 40, p, p, p, db,
                                              None, dq, st, sh, p, p, 0)

    def attention_backward(db):
        return P.dmc_retrofit_attention_backward(h.handle, 2, p, p, p, p, p, p, p, cu.data_ptr(), T, 40, p, p, p, db, 0)

    bad = p + size // 2
    assert states(q=bad) == states_backward(q=bad) == states_backward(dq=bad) == P.DMC_ERR_INVALID_ARG
    assert states_backward(db=bad) == attention_backward(bad) == P.DMC_ERR_INVALID_ARG
    assert states_backward(st=0) == states_backward(sh=0) == P.DMC_ERR_INVALID_ARG  # tokens, heads in one place


def test_statuses_of_the_loss(ready):
    dev = ready[-1]
    h = both(dev)
    hid, w = torch.zeros(64, 64, dtype=BF16, device=dev), torch.zeros(50, 64, dtype=BF16, device=dev)
    f, t = torch.zeros(64, device=dev), torch.zeros(64, dtype=torch.int32, device=dev)
    dh, dw = torch.ones_like(hid), torch.ones_like(w)
    inv = P.DMC_ERR_INVALID_ARG

    def loss(n=64, hidden=hid.data_ptr(), weight=w.data_ptr(), targets=t.data_ptr(), out=f.data_ptr()):
        return P.dmc_retrofit_loss(h.handle, n, hidden, weight, targets, out, f.data_ptr(), 0)

    def backward(n=64, hidden=hid.data_ptr(), dloss=f.data_ptr(), dhidden=dh.data_ptr(), dweight=dw.data_ptr()):
        return P.dmc_retrofit_loss_backward(h.handle, n, hidden, w.data_ptr(), t.data_ptr(), f.data_ptr(), dloss, dhidden,
                                            dweight, 0)

    assert loss(n=-1) == loss(n=65) == loss(hidden=0) == loss(hidden=hid.data_ptr() + 8) == loss(weight=0) == inv
    assert loss(targets=0) == loss(targets=t.data_ptr() + 2) == loss(out=f.data_ptr() + 2) == inv
    assert backward(n=-1) == backward(n=65) == backward(hidden=0) == backward(dloss=0) == backward(dhidden=0) == inv
    assert backward(dweight=0) == backward(dweight=dw.data_ptr() + 4) == inv
    assert loss(n=0) == backward(n=0) == P.DMC_OK
    torch.cuda.synchronize()
    assert not bool(dw.any()) and bool(dh.all())  # no token: a gradient of zero
    assert h.status() == (0, 0)


def test_tokens_without_sequences(ready):
    x, s, _, dev = ready
    h = handle(dev, *HEADS, BF16, LENS)
    none = torch.zeros(1, dtype=torch.int32, device=dev)
    with pytest.raises(ValueError):
        h.attention(x["q"], x["k"], x["v"], none, 40)
    with pytest.raises(ValueError):
        h.states(s["q0"], s["k"], s["v"], none, 40)
    empty = h.attention(x["q"][:0], x["k"][:0], x["v"][:0], none, 0)
    assert empty[0].shape == (0, 4, 64)


def test_outputs_of_another_stream(ready):
    """They are that stream's: memory that work of the current stream may still use is not handed to a call that
    runs beside it."""
    x, s, cu, dev = ready
    h = both(dev)
    side = torch.cuda.Stream()
    hid, w = torch.zeros(64, 64, dtype=BF16, device=dev), torch.zeros(50, 64, dtype=BF16, device=dev)
    t, f = torch.zeros(64, dtype=torch.int32, device=dev), torch.zeros(64, device=dev)
    calls = [lambda **k: h.attention(x["q"], x["k"], x["v"], cu, 40, x["bias"], **k),
             lambda **k: h.states(s["q0"], s["k"], s["v"], cu, 40, s["noise"], **k),
             lambda **k: h.loss(hid, w, t, **k), lambda **k: h.loss_backward(f, hid, w, t, f, **k)]
    saved, (o, lse) = calls[1]()[-1], calls[0]()
    calls += [lambda **k: h.states_backward(s["q0"], s["k"], s["v"], cu, 40, saved, s["dkt"], s["dvt"], s["dbias"], **k),
              lambda **k: h.attention_backward(x["dout"], x["q"], x["k"], x["v"], o, lse, cu, 40, x["bias"], **k)]
    torch.cuda.synchronize()
    for call in calls:
        for stream in (side, side.cuda_stream):
            want = [t.clone() for t in call()]
            torch.cuda.synchronize()
            shapes = [(t.shape, t.dtype) for t in want]
            freed = [torch.empty(a, dtype=b, device=dev) for _ in range(4) for a, b in shapes]
            places = {t.data_ptr() for t in freed}
            del freed  # their places are the current stream's to use again
            got = call(stream=stream)
            side.synchronize()
            assert not places & {t.data_ptr() for t in got}
            for a, b in zip(got[:4], want):  # (states' fifth has rows that nobody writes or reads)
                assert torch.equal(a, b)
    assert h.status() == (0, 0)


def test_a_handle_dropped_while_another_stream_works(ready):
    """Its arena is not handed out again before that stream is done."""
    x, _, cu, dev = ready
    h = both(dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        h.attention(x["q"], x["k"], x["v"], cu, 40, x["bias"])
    place, size = h.arena.data_ptr(), h.nbytes
    del h
    again = torch.empty(size, dtype=torch.uint8, device=dev)
    assert again.data_ptr() != place
    side.synchronize()


def test_the_default_stream_named_from_another(ready):
    """Its number is 0: outputs and arena come from its memory, too."""
    x, _, cu, dev = ready

    def stream_of(t):
        at = t.data_ptr()
        return [s["stream"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        h = DmcRetrofit(*HEADS, dtype=BF16, max_tokens=sum(LENS), max_seqs=2, device=dev, stream=0)
        outs = h.attention(x["q"], x["k"], x["v"], cu, 40, x["bias"], stream=0)
        outs += h.attention(x["q"], x["k"], x["v"], cu, 40, x["bias"], stream=torch.cuda.default_stream())
        there = h.attention(x["q"], x["k"], x["v"], cu, 40, x["bias"])
    torch.cuda.synchronize()
    for t in (*outs, h.arena):
        assert stream_of(t) == [0]
    for t in there:
        assert stream_of(t) == [side.cuda_stream]
    assert h.status() == (0, 0)
