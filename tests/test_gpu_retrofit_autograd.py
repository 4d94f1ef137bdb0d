"""What the autograd functions of the retrofitting operators promise beside first gradients."""
import pytest
import torch

from retrofit_harness import OFFSET, TEMPERATURE, check_states, cu_of, handle, on, states_inputs
from paper_2403_09636_gb300.retrofit import DmcRetrofit, attention, cross_entropy

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
LENS, HEADS = [40, 24], (4, 2, 64)


def inputs(dev, dtype, **leaf):
    s = on(states_inputs(LENS, *HEADS, dtype), dev)
    g = torch.Generator(device=dev).manual_seed(9)
    q = torch.randn(sum(LENS), HEADS[0], HEADS[2], generator=g, device=dev).to(dtype)
    return handle(dev, *HEADS, dtype, LENS), q, s, cu_of(LENS, dev)


def test_second_derivatives_are_refused(cuda_dev):
    h, q, s, cu = inputs(cuda_dev, F32)
    q.requires_grad_()
    out, _ = attention(h, q, s["k"], s["v"], cu, 40, noise=s["noise"])
    (dq,) = torch.autograd.grad(out.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError):
        (dq.square().sum() + q.sum()).backward()
    words = DmcRetrofit(dtype=F32, max_tokens=64, hidden=64, vocab=99, device=cuda_dev)
    hid = q[:, 0].detach().contiguous().requires_grad_()
    w = torch.randn(99, 64, device=cuda_dev, requires_grad=True)
    loss = cross_entropy(words, hid, w, torch.arange(64, dtype=torch.int32, device=cuda_dev))
    (dh,) = torch.autograd.grad(loss.square().sum(), hid, create_graph=True)
    with pytest.raises(RuntimeError):
        (dh.square().sum() + hid.sum()).backward()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_noise_has_a_gradient(cuda_dev, dtype):
    """The noise is added to k's first component: it has its gradient."""
    h, q, s, cu = inputs(cuda_dev, dtype)
    k, noise = s["k"].clone().requires_grad_(), s["noise"].clone().requires_grad_()
    out, alpha = attention(h, q, k, s["v"], cu, 40, noise=noise)
    (out.float().square().sum() + alpha.sum()).backward()
    assert noise.grad.shape == noise.shape and noise.grad.dtype == F32
    assert bool(noise.grad.any())
    assert torch.equal(noise.grad, k.grad[..., 0].t().float())


def test_noise_changed_in_between_is_noticed(cuda_dev):
    h, q, s, cu = inputs(cuda_dev, F32)
    q.requires_grad_()
    noise = s["noise"].clone()
    out, _ = attention(h, q, s["k"], s["v"], cu, 40, noise=noise)
    noise.mul_(2.0)
    with pytest.raises(RuntimeError):
        out.sum().backward()
