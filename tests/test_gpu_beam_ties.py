"""Ties of beam search's selection (GPU): against the definition in 64 bits, tokens, parents and done equal."""
import pytest
import torch

from paper_2403_09636_gb300.beam import BeamSelect
from test_gpu_beam import check

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,V,keep", [(2, 8193, 4), (4, 20000, 4), (3, 40000, 16), (8, 130003, 32)])
def test_beams_that_are_alike_in_rows_of_several_pieces(cuda_dev, dt, B, V, keep):
    """The log-sum of a row that is cut into pieces is one number, whichever of its words it scores: equal logits have
    equal scores, so words of beams that are alike (the same logits and score) go by beam, then by word. The rows' best
    words are many equal ones among others, and sums of random numbers, which every order of adding rounds elsewhere."""
    select = BeamSelect(1, B, V, keep=keep, dtype=dt)
    for seed in range(24):
        g = torch.Generator().manual_seed(seed)
        row = (torch.randn(V, generator=g) * 2.5).to(torch.bfloat16)
        row[torch.randperm(V, generator=g)[:40]] = row.max()
        row[torch.randperm(V, generator=g)[:5]] = row.max() * 1.0625
        logits = row.to(dt).expand(B, V).contiguous().cuda()
        check(select, logits, torch.full((1, B), -3.0 - 0.37 * seed))
