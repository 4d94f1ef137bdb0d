"""Attention's backward pass where its work on K and V is split over a group's queries, and where it is not.

Tiles of 128 tokens times KV heads decide: few of them are split into shares of whole
heads, added up afterwards; from 304 on they are not, nor, in bf16, are sequences of up to 384 tokens.
"""
import pytest
import torch

from retrofit_harness import attention_inputs, check_attention
from test_gpu_retrofit import run_attention

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

CASES = [
    ([131], (64, 2, 128)),            # shares of a single head each
    ([600], (40, 8, 128)),
    ([1, 260, 127], (30, 6, 64)),     # shares of unequal sizes
    ([700, 90], (20, 20, 64)),        # nothing to split
    ([129] * 11, (36, 12, 64)),       # 263 of 3 heads: shares of 1 and 2
    ([40] * 18, (32, 16, 64)),        # just below the limit
    ([100, 33] * 20, (24, 8, 64)),    # above it: whole groups
    ([64] * 150, (10, 5, 128)),
    ([431], (64, 2, 128)),               # longer than three tiles: shares in bf16 too
    ([1, 390, 127], (30, 6, 64)),
    ([410, 129, 129, 1], (36, 12, 64)),
    ([385, 384], (7, 1, 128)),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,heads", CASES)
def test_attention_shares(cuda_dev, lens, heads, dtype):
    x = attention_inputs(lens, *heads, dtype)
    check_attention(x, lens, dtype, run_attention(cuda_dev, x, lens, heads, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_shares_twice_the_same(cuda_dev, dtype):
    lens, heads = [333, 5, 128], (24, 3, 128)
    x = attention_inputs(lens, *heads, dtype)
    a, b = (run_attention(cuda_dev, x, lens, heads, dtype) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name
