"""Attention's bias where it hides whole tiles of a sequence: values near the type's lowest hide as -inf does."""
import math

import pytest
import torch

from retrofit_harness import attention_inputs, check_attention
from test_gpu_retrofit import run_attention

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads", [(4, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("lens,hidden", [([700], (0, 128)), ([131, 500], (0, 400)), ([900], (256, 640)), ([260], (0, 260))])
def test_whole_tiles_hidden(cuda_dev, lens, hidden, heads, dtype):
    x = attention_inputs(lens, *heads, dtype)
    rows = slice(hidden[0] + lens[0] * (len(lens) - 1), hidden[1] + lens[0] * (len(lens) - 1))  # of the last sequence
    x["bias"][:, rows] = -math.inf
    want = run_attention(cuda_dev, x, lens, heads, dtype)
    check_attention(x, lens, dtype, want)
    for low in (torch.finfo(F32).min, -3e38, -2.4e38, -1e38, -1e30, -1e10, -1e9):
        x["bias"][:, rows] = low
        got = run_attention(cuda_dev, x, lens, heads, dtype)
        for name in want:
            assert torch.equal(got[name], want[name]), (low, name)
