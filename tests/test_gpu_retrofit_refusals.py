"""What the retrofitting calls refuse, and their use on another stream and in a graph."""
import pytest
import torch

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300.retrofit import DmcRetrofit, attention, cross_entropy
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
    return handle(dev, *HEADS, BF16, LENS), x, s, cu_of(LENS, dev), dev


def test_shapes_types_devices_and_layouts(ready):
    h, x, s, cu, dev = ready
    a = (x["q"], x["k"], x["v"])
    bad = [((x["q"].float(), *a[1:]), cu, x["bias"]),                       # type
           ((x["q"][:, :3], *a[1:]), cu, x["bias"]),                        # shape
           ((x["q"].transpose(0, 1).contiguous().transpose(0, 1), *a[1:]), cu, x["bias"]),  # layout
           ((x["q"].cpu(), *a[1:]), cu, x["bias"]),                         # device
           (a, cu.long(), x["bias"]), (a, cu, x["bias"].bfloat16()), (a, cu, x["bias"].t())]
    for args, c, bias in bad:
        with pytest.raises(ValueError):
            h.attention(*args, c, 40, bias)
    with pytest.raises(ValueError):
        h.attention(*a, cu, 40, out=(x["q"],))
    with pytest.raises(ValueError):
        h.states(s["q0"][:, :2], s["k"], s["v"], cu, 40)
    with pytest.raises(ValueError):
        h.loss(x["q"][:, 0], x["q"][:, 0], cu)  # made without a vocabulary
    with pytest.raises(ValueError):
        DmcRetrofit(4, 2, 64, dtype=torch.float16, max_tokens=8)
    with pytest.raises(P.DmcError):
        DmcRetrofit(4, 2, 80, dtype=BF16, max_tokens=8)
    words = DmcRetrofit(dtype=BF16, max_tokens=8, hidden=64, vocab=10, device=dev)
    with pytest.raises(ValueError):
        words.attention(*a, cu, 40)
    with pytest.raises(ValueError):
        words.loss(torch.empty(4, 64, dtype=BF16, device=dev), torch.empty(11, 64, dtype=BF16, device=dev),
                   torch.empty(4, dtype=torch.int32, device=dev))


def test_statuses_of_the_c_functions(ready):
    h, x, s, cu, dev = ready
    inv = P.DMC_ERR_INVALID_ARG
    out, lse = torch.empty_like(x["q"]), torch.empty(4, 64, device=dev)
    p = [t.data_ptr() for t in (x["q"], x["k"], x["v"], x["bias"], cu, out, lse)]

    def call(n=2, q=p[0], total=64, longest=40, cu=p[4], lse=p[6]):
        return P.dmc_retrofit_attention(h.handle, n, q, p[1], p[2], p[3], cu, total, longest, p[5], lse, 0)

    assert call(n=3) == call(n=-1) == call(total=65) == call(total=-1) == call(longest=65) == call(longest=-1) == inv
    assert call(q=p[0] + 2) == call(q=0) == call(cu=0) == call(lse=0) == call(lse=p[6] + 1) == inv
    assert call(n=0) == call(total=0, longest=0) == P.DMC_OK

    def states(temperature=0.1, offset=5.0, stride=4):
        d = [t.data_ptr() for t in (s["q0"], s["k"], s["v"], s["noise"])]
        return P.dmc_retrofit_states(h.handle, 2, d[0], stride, 1, *d[1:], offset, temperature, p[4], 64, 40, p[5],
                                     p[5], p[6], p[6], p[5], 0)

    assert states(temperature=0.0) == states(temperature=-1.0) == states(temperature=float("nan")) == inv
    assert states(offset=float("inf")) == states(stride=-1) == inv


def test_more_tokens_than_the_handle_was_made_for(ready):
    h, x, _, _, dev = ready
    big = {n: torch.cat([t, t]) for n, t in x.items() if n in ("q", "k", "v")}
    with pytest.raises(P.DmcError):
        h.attention(big["q"], big["k"], big["v"], cu_of([128], dev), 128)


def test_another_stream_and_a_graph(ready):
    h, x, _, cu, dev = ready
    a = (x["q"], x["k"], x["v"], cu, 40, x["bias"])
    out, lse = h.attention(*a)
    grads = h.attention_backward(x["dout"], *a[:3], out, lse, *a[3:])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2, l2 = h.attention(*a)
    side.synchronize()
    assert torch.equal(out, o2) and torch.equal(lse, l2)
    o3, l3 = torch.zeros_like(out), torch.zeros_like(lse)
    g3 = tuple(torch.zeros_like(t) for t in grads)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.attention(*a, out=(o3, l3))
        h.attention_backward(x["dout"], *a[:3], o3, l3, *a[3:], out=g3)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, o3) and all(torch.equal(s, t) for s, t in zip(grads, g3))
    assert h.status() == (0, 0)


def test_autograd(ready):
    """The autograd functions give what the calls give, the gates' gradients in the first components."""
    h, x, s, cu, dev = ready
    leaf = [t.clone().requires_grad_() for t in (x["q"], s["k"], s["v"])]
    out, alpha = attention(h, *leaf, cu, 40, noise=s["noise"])
    (out.float() * x["dout"].float()).sum().add((alpha * s["dalpha"]).sum()).backward()
    q, k, v = (t.detach() for t in leaf)
    gates = {"noise": s["noise"]}
    kt, vt, al, bias, saved = h.states(q[..., 0], k, v, cu, 40, **gates)
    o, lse = h.attention(q, kt, vt, cu, 40, bias)
    dq, dkt, dvt, db = h.attention_backward(x["dout"], q, kt, vt, o, lse, cu, 40, bias)
    assert not bool(dq[..., 0].any())  # the states' first components are zero
    dq0, dk, dv = h.states_backward(q[..., 0], k, v, cu, 40, saved, dkt, dvt, db, s["dalpha"], **gates)
    assert torch.equal(out, o) and torch.equal(alpha, al)
    assert torch.equal(leaf[0].grad[..., 1:], dq[..., 1:]) and torch.equal(leaf[0].grad[..., 0], dq0)
    assert torch.equal(leaf[1].grad, dk) and torch.equal(leaf[2].grad, dv)
    words = DmcRetrofit(dtype=BF16, max_tokens=64, hidden=64, vocab=99, device=dev)
    hid, w = x["q"][:, 0].clone().requires_grad_(), torch.randn(99, 64, device=dev).to(BF16).requires_grad_()
    t = torch.arange(64, dtype=torch.int32, device=dev)
    loss = cross_entropy(words, hid, w, t)
    loss.mean().backward()
    want = torch.nn.functional.cross_entropy(hid.detach().double() @ w.detach().double().t(), t.long())
    assert abs(float(loss.detach().mean()) - float(want)) < 1e-4
    assert hid.grad.shape == hid.shape and w.grad.shape == w.shape
