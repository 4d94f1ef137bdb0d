"""The loss's gradients where the sums over words, or over tokens, are split into shares that are added up afterwards:
few tiles of 256 rows and columns, long sums."""
import pytest
import torch

from oracle import retrofit_ref as R
from retrofit_harness import close
from test_gpu_retrofit import run_loss

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("size", [(3, 64, 9001), (200, 136, 5000), (1500, 72, 97), (300, 520, 1100)])
def test_loss_shares(cuda_dev, size, dtype):
    x, got = run_loss(cuda_dev, *size, dtype, 4)
    for name, (want, bound) in R.loss_all(**x, dtype=dtype).items():
        close(name, got[name], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_loss_shares_of_pieces(cuda_dev, dtype):
    """Every piece of the vocabulary in shares, and dhidden of the pieces before added to them."""
    x, got = run_loss(cuda_dev, 33, 128, 2600, dtype, 0, max_tokens=300000)
    for name, (want, bound) in R.loss_all(**x, dtype=dtype).items():
        close(name, got[name], want, bound)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_loss_shares_twice_the_same(cuda_dev, dtype):
    a, b = (run_loss(cuda_dev, 90, 64, 4000, dtype, 0)[1] for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name
