"""The retrofitting operators on the GPU against fp64 (oracle/retrofit_ref.py), within
bounds that follow from the roundings each of them makes."""
import math

import pytest
import torch

from oracle import retrofit_ref as R
from retrofit_harness import (OFFSET, TEMPERATURE, attention_inputs, check_attention, check_states, close, cu_of, gen,
                              handle, normal, on, states_inputs)
from paper_2403_09636_gb300 import (DMC_ERR_DEVICE_FAULT, DMC_FAULT_BAD_SEQLENS, DMC_FAULT_BAD_TARGET)
from paper_2403_09636_gb300.retrofit import DmcRetrofit

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

LENS = [[1], [2, 1, 3], [33, 0, 31, 64], [130, 127, 1, 257], [0, 700, 0]]
HEADS = [(4, 4, 64), (4, 4, 128), (8, 1, 128), (6, 2, 64), (5, 1, 128)]


def run_attention(dev, x, lens, heads, dtype):
    d = on(x, dev)
    h = handle(dev, *heads, dtype, lens)
    cu, longest = cu_of(lens, dev), max(lens)
    out, lse = h.attention(d["q"], d["k"], d["v"], cu, longest, d["bias"])
    grads = h.attention_backward(d["dout"], d["q"], d["k"], d["v"], out, lse, cu, longest, d["bias"])
    assert h.status() == (0, 0)
    return dict(zip(("out", "lse", "dq", "dk", "dv", "dbias"), (out, lse, *grads)))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", LENS)
def test_attention(cuda_dev, lens, heads, dtype):
    x = attention_inputs(lens, *heads, dtype)
    check_attention(x, lens, dtype, run_attention(cuda_dev, x, lens, heads, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bias", ["none", "hard"])
def test_attention_masks(cuda_dev, bias, dtype):
    """No bias at all, and one that hides rows entirely (the decisions of inference)."""
    lens, heads = [129, 300], (4, 2, 128)
    x = attention_inputs(lens, *heads, dtype, bias=bias)
    got = run_attention(cuda_dev, x, lens, heads, dtype)
    if bias == "none":
        assert got.pop("dbias") is None
    check_attention(x, lens, dtype, got)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_lowest_bias(cuda_dev, dtype):
    """A bias of the type's lowest value hides a row as -inf does."""
    lens, heads = [150, 70], (4, 2, 64)
    x = attention_inputs(lens, *heads, dtype, bias="hard")
    a = run_attention(cuda_dev, x, lens, heads, dtype)
    x["bias"] = x["bias"].clamp(min=torch.finfo(F32).min)
    b = run_attention(cuda_dev, x, lens, heads, dtype)
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_sequences_are_apart(cuda_dev, dtype):
    """NaN and infinities in one sequence reach no other one."""
    lens, heads = [100, 61, 90], (4, 2, 128)
    x = attention_inputs(lens, *heads, dtype)
    clean = run_attention(cuda_dev, x, lens, heads, dtype)
    for n in ("q", "k", "v", "dout"):
        x[n][100:161:3] = math.nan
        x[n][101:161:3] = math.inf
    x["bias"][:, 100:161] = math.nan
    got = run_attention(cuda_dev, x, lens, heads, dtype)
    for name, t in got.items():
        for a, b in ((0, 100), (161, 251)):
            part = (slice(None), slice(a, b)) if name in ("lse", "dbias") else slice(a, b)
            assert torch.equal(t[part], clean[name][part]), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [128, 129, 300])
def test_attention_many_sequences(cuda_dev, n, dtype):
    """Short and empty sequences in great number, a long one among them."""
    lens = [(7 * i) % 41 for i in range(n)]
    lens[n // 2] = 270
    x = attention_inputs(lens, 2, 1, 64, dtype)
    check_attention(x, lens, dtype, run_attention(cuda_dev, x, lens, (2, 1, 64), dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_twice_the_same(cuda_dev, dtype):
    lens, heads = [513, 260], (8, 2, 128)
    x = attention_inputs(lens, *heads, dtype)
    a, b = (run_attention(cuda_dev, x, lens, heads, dtype) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name


def run_states(dev, x, lens, heads, dtype, noise=True, dalpha=True, strided=False):
    d = on(x, dev)
    h = handle(dev, *heads, dtype, lens)
    cu, longest = cu_of(lens, dev), max(lens)
    q0 = d["q0"]
    if strided:  # as the first components of whole queries
        q = torch.full((*q0.shape, heads[2]), math.nan, dtype=dtype, device=dev)
        q[..., 0] = q0
        q0 = q[..., 0]
    gates = {"noise": d["noise"] if noise else None, "offset": OFFSET, "temperature": TEMPERATURE}
    kt, vt, alpha, bias, saved = h.states(q0, d["k"], d["v"], cu, longest, **gates)
    out = None
    if strided:
        full = torch.zeros_like(q)
        out = (full[..., 0], torch.empty_like(d["k"]), torch.empty_like(d["v"]))
    dq0, dk, dv = h.states_backward(q0, d["k"], d["v"], cu, longest, saved, d["dkt"], d["dvt"], d["dbias"],
                                    d["dalpha"] if dalpha else None, out=out, **gates)
    assert h.status() == (0, 0)
    if strided:
        assert not bool(full[..., 1:].any())
    return {"kt": kt, "vt": vt, "alpha": alpha, "bias": bias, "dq0": dq0, "dk": dk, "dv": dv}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("lens", LENS)
def test_states(cuda_dev, lens, heads, dtype):
    x = states_inputs(lens, *heads, dtype)
    check_states(x, lens, dtype, run_states(cuda_dev, x, lens, heads, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_states_options(cuda_dev, dtype):
    """No noise, no gradient of the decisions, first components inside whole queries."""
    lens, heads = [70, 33], (6, 3, 64)
    x = states_inputs(lens, *heads, dtype)
    check_states(x, lens, dtype, run_states(cuda_dev, x, lens, heads, dtype, False, False, True), False, False)


def test_states_long_segments(cuda_dev):
    """Decisions that nearly all merge: a state that remembers hundreds of tokens."""
    lens, heads = [900], (2, 2, 64)
    x = states_inputs(lens, *heads, F32, spread=0.0)
    x["k"][..., 0] += 0.4  # alpha around 0.98
    x["noise"].mul_(0.1)
    check_states(x, lens, F32, run_states(cuda_dev, x, lens, heads, F32))


LOSSES = [(1, 64, 5), (3, 8, 1), (65, 72, 130), (130, 264, 1009), (257, 128, 4099), (64, 1024, 700)]


def run_loss(dev, n, hidden, vocab, dtype, ignored, max_tokens=None, seed=3):
    g = gen(seed)
    x = {"hidden": normal(g, n, hidden, dtype=dtype),
         "weight": normal(g, vocab, hidden, scale=2.0 / math.sqrt(hidden), dtype=dtype),
         "targets": torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32),
         "dloss": torch.rand(n, generator=g) + 0.5}
    if ignored:
        x["targets"][::ignored] = -100
    d = on(x, dev)
    h = DmcRetrofit(dtype=dtype, max_tokens=max_tokens or n, hidden=hidden, vocab=vocab, device=dev)
    loss, lse = h.loss(d["hidden"], d["weight"], d["targets"])
    dh, dw = h.loss_backward(d["dloss"], d["hidden"], d["weight"], d["targets"], lse)
    assert h.status() == (0, 0)
    return x, {"loss": loss, "lse": lse, "dhidden": dh, "dweight": dw}


@pytest.mark.parametrize("ignored", [0, 3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", LOSSES)
def test_loss(cuda_dev, size, dtype, ignored):
    x, got = run_loss(cuda_dev, *size, dtype, ignored)
    for name, (want, bound) in R.loss_all(**x, dtype=dtype).items():
        close(name, got[name], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_loss_in_pieces(cuda_dev, dtype):
    """A handle for so many tokens that the vocabulary is taken in several pieces."""
    x, got = run_loss(cuda_dev, 70, 64, 2500, dtype, 5, max_tokens=300000)
    for name, (want, bound) in R.loss_all(**x, dtype=dtype).items():
        close(name, got[name], want, bound)


def test_loss_all_ignored(cuda_dev):
    _, got = run_loss(cuda_dev, 40, 64, 300, BF16, 1)
    for name in ("loss", "dhidden", "dweight"):
        assert not bool(got[name].any()), name


def test_loss_ignores_the_gradient_of_ignored_positions(cuda_dev):
    g = gen(4)
    hid, w = normal(g, 9, 64, dtype=BF16).to(cuda_dev), normal(g, 50, 64, dtype=BF16).to(cuda_dev)
    t = torch.tensor([3, -1, 7, -100, 0, 49, -5, 1, 2], dtype=torch.int32, device=cuda_dev)
    d = torch.where(t < 0, math.nan, 1.0).float()
    h = DmcRetrofit(dtype=BF16, max_tokens=9, hidden=64, vocab=50, device=cuda_dev)
    _, lse = h.loss(hid, w, t)
    dh, dw = h.loss_backward(d, hid, w, t, lse)
    assert bool(torch.isfinite(dh).all()) and bool(torch.isfinite(dw).all())
    assert not bool(dh[t < 0].any())


def test_loss_without_tokens(cuda_dev):
    h = DmcRetrofit(dtype=BF16, max_tokens=4, hidden=64, vocab=50, device=cuda_dev)
    e = torch.empty(0, 64, dtype=BF16, device=cuda_dev)
    w = torch.ones(50, 64, dtype=BF16, device=cuda_dev)
    t, f = torch.empty(0, dtype=torch.int32, device=cuda_dev), torch.empty(0, device=cuda_dev)
    loss, lse = h.loss(e, w, t)
    dh, dw = h.loss_backward(f, e, w, t, lse, out=(torch.empty_like(e), torch.ones_like(w)))
    assert loss.numel() == 0 and not bool(dw.any())


def test_bad_target_sets_its_bit(cuda_dev):
    h = DmcRetrofit(dtype=F32, max_tokens=4, hidden=64, vocab=50, device=cuda_dev)
    t = torch.tensor([1, 50, 2, 3], dtype=torch.int32, device=cuda_dev)
    loss, _ = h.loss(torch.randn(4, 64, device=cuda_dev), torch.randn(50, 64, device=cuda_dev), t)
    assert h.status() == (DMC_ERR_DEVICE_FAULT, DMC_FAULT_BAD_TARGET)
    assert float(loss[1]) == 0.0


@pytest.mark.parametrize("cu", [[0, 40, 30, 60], [0, 20, 40, 59], [1, 20, 40, 60], [0, 50, 55, 60], [0, -5, 40, 60],
                                [0, 20, 400, 60]])
def test_bad_seqlens_set_their_bit(cuda_dev, cu):
    lens, heads = [20, 20, 20], (4, 2, 64)
    x, s = (on(f(lens, *heads, BF16), cuda_dev) for f in (attention_inputs, states_inputs))
    c = torch.tensor(cu, dtype=torch.int32, device=cuda_dev)
    for call in ("attention", "attention_backward", "states", "states_backward"):
        h = handle(cuda_dev, *heads, BF16, lens)
        a = (x["q"], x["k"], x["v"])
        if call == "attention":
            h.attention(*a, c, 45, x["bias"])
        elif call == "attention_backward":
            h.attention_backward(x["dout"], *a, x["q"], torch.zeros(4, 60, device=cuda_dev), c, 45, x["bias"])
        elif call == "states":
            h.states(s["q0"], s["k"], s["v"], c, 45, s["noise"])
        else:
            saved = h.states(s["q0"], s["k"], s["v"], cu_of(lens, cuda_dev), 20, s["noise"])[-1]
            h.states_backward(s["q0"], s["k"], s["v"], c, 45, saved, s["dkt"], s["dvt"], s["dbias"], s["dalpha"],
                              s["noise"])
        assert h.status() == (DMC_ERR_DEVICE_FAULT, DMC_FAULT_BAD_SEQLENS), call


def test_empty_calls(cuda_dev):
    h = handle(cuda_dev, 4, 2, 64, BF16, [8])
    q, k = (torch.empty(0, n, 64, dtype=BF16, device=cuda_dev) for n in (4, 2))
    cu = torch.zeros(2, dtype=torch.int32, device=cuda_dev)
    out, lse = h.attention(q, k, k, cu, 0)
    assert out.shape == (0, 4, 64)
    h.attention_backward(q, q, k, k, out, lse, cu, 0)
    assert h.states(q[..., 0], k, k, cu, 0)[0].shape == (0, 2, 64)
    assert h.status() == (0, 0)
