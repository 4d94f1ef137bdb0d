"""fp32 attention of calls that fill the GPU (their kernels multiply operands split into three bf16 parts),
within the bounds of fp32 arithmetic, and nothing of a larger error's kind: values of very different sizes."""
import pytest
import torch

from retrofit_harness import attention_inputs, check_attention
from test_gpu_retrofit import run_attention

pytestmark = pytest.mark.gpu
F32 = torch.float32

CASES = [
    ([64] * 40, (8, 8, 128)),
    ([1, 63, 65, 127, 128, 129, 200, 0, 31] * 3, (16, 16, 64)),
    ([100, 33] * 20, (24, 8, 64)),       # grouped heads
    ([1300], (16, 16, 128)),             # one long sequence
    ([257, 300, 2, 190], (40, 40, 128)),
    ([5] * 310, (1, 1, 64)),
]


@pytest.mark.parametrize("bias", ["soft", "hard", "none"])
@pytest.mark.parametrize("lens,heads", CASES)
def test_attention_parts(cuda_dev, lens, heads, bias):
    x = attention_inputs(lens, *heads, F32, bias=bias)
    got = run_attention(cuda_dev, x, lens, heads, F32)
    if bias == "none":
        assert got.pop("dbias") is None
    check_attention(x, lens, F32, got)


def test_attention_parts_of_different_sizes(cuda_dev):
    """v and dout with factors from 2^-40 to 2^40 per channel: each channel keeps its own precision."""
    lens, heads = [300, 129], (40, 40, 64)
    x = attention_inputs(lens, *heads, F32)
    a = run_attention(cuda_dev, x, lens, heads, F32)
    factor = 2.0 ** torch.linspace(-40, 40, 64).round()
    x["v"], x["dout"] = x["v"] * factor, x["dout"] / factor
    b = run_attention(cuda_dev, x, lens, heads, F32)
    f = factor.to(cuda_dev)
    assert torch.equal(a["out"] * f, b["out"])
    assert torch.equal(a["dv"] / f, b["dv"])
    assert torch.equal(a["lse"], b["lse"])


def test_attention_parts_twice_the_same(cuda_dev):
    lens, heads = [333, 5, 128], (64, 64, 64)
    x = attention_inputs(lens, *heads, F32)
    a, b = (run_attention(cuda_dev, x, lens, heads, F32) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name
