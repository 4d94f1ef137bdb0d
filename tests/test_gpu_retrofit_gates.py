"""The states where the importance omega is far below the smallest fp32 number: only its ratios count."""
import pytest
import torch

from retrofit_harness import check_states, states_inputs
from test_gpu_retrofit import run_states

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,heads", [([1], (2, 2, 64)), ([1, 40, 90, 33], (4, 4, 64)), ([300], (6, 2, 128))])
@pytest.mark.parametrize("lo,hi", [(-87.0, -80.0), (-95.0, -85.0), (-110.0, -100.0), (-89.0, -88.0)])
def test_small_importance(cuda_dev, lo, hi, lens, heads, dtype):
    x = states_inputs(lens, *heads, dtype)
    g = torch.Generator().manual_seed(7)
    x["q0"] = (lo + (hi - lo) * torch.rand(x["q0"].shape, generator=g)).to(dtype)
    check_states(x, lens, dtype, run_states(cuda_dev, x, lens, heads, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_small_importance_before_and_after_large(cuda_dev, dtype):
    """Sequences whose importance rises or falls by a factor of 2^80 in the middle."""
    lens, heads = [70, 70], (2, 2, 64)
    x = states_inputs(lens, *heads, dtype, spread=0.1)
    x["k"][..., 0] += 0.3
    x["noise"].mul_(0.3)
    for t0 in (0, 105):
        x["q0"][t0:t0 + 35] -= 95.0
    check_states(x, lens, dtype, run_states(cuda_dev, x, lens, heads, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_no_importance_at_all(cuda_dev, dtype):
    """Below a mean of -110.9 it counts as that: the states are means of numbers, the first one the token itself."""
    lens, heads = [40], (2, 2, 64)
    x = states_inputs(lens, *heads, dtype)
    x["q0"][:] = -3.0e38
    got = run_states(cuda_dev, x, lens, heads, dtype)
    for name, t in got.items():
        assert bool(torch.isfinite(t).all()), name
    assert torch.equal(got["kt"][0, :, 1:].cpu(), x["k"][0, :, 1:]) and torch.equal(got["vt"][0].cpu(), x["v"][0])
    assert not bool(got["dq0"].any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128)])
def test_importance_near_one(cuda_dev, heads, dtype):
    """1 - omega is far smaller than what rounding leaves of a difference: q[0]'s gradient keeps its precision."""
    lens = [1, 2, 70, 200]
    x = states_inputs(lens, *heads, dtype)
    g = torch.Generator().manual_seed(8)
    # exact sums of a group; up to 17, where the 64-bit reference still has 1 - omega to 3e-9
    x["q0"] = (5.0 + 12.0 * torch.rand(x["q0"].shape, generator=g)).mul(8).round().div(8).to(dtype)
    check_states(x, lens, dtype, run_states(cuda_dev, x, lens, heads, dtype))
