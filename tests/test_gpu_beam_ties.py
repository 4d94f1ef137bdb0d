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


def test_logits_whose_scores_round_to_a_step_apart(cuda_dev):
    """A beam at minus its log-sum and two logits next to each other around -2^-22, half a step of its sum with them:
    rounded to 48 bits, some 4 % of the rows gave the lower one the higher score. With two such beams each, alike: every
    continuation is there once, in an order of scores, and a beam's in the order of its logits."""
    G, V = 4000, 64
    g = torch.Generator().manual_seed(0)
    row = -1e-3 - 0.1 * torch.rand(G, V, generator=g)
    low = torch.tensor(-2.0 ** -22)
    row[:, 9], row[:, 40] = low, torch.nextafter(low, torch.tensor(1.0))
    base = -torch.logsumexp(row.double(), 1).float()
    logits = row.repeat_interleave(2, 0).cuda()
    scores, tokens, parents, done = (t.cpu() for t in BeamSelect(G, 2, V, keep=4, dtype=F32).select(
        logits, base[:, None].expand(G, 2).contiguous().cuda()))
    where = (parents - 2 * torch.arange(G)[:, None]) * 2 + (tokens == 9)
    assert bool(((tokens == 9) | (tokens == 40)).all()) and not bool(done.any())
    assert torch.equal(where.sort(1)[0], torch.arange(4).expand(G, 4).to(where.dtype))
    assert bool((scores[:, 1:] <= scores[:, :-1]).all())
    place = where.argsort(1)  # of (beam 0, 40), (beam 0, 9), (beam 1, 40), (beam 1, 9)
    assert bool((place[:, 0] < place[:, 1]).all()) and bool((place[:, 2] < place[:, 3]).all())


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,V,keep", [(1, 40, 8), (2, 5001, 5), (3, 40000, 32)])
def test_zeros_of_both_signs_are_equal(cuda_dev, dt, B, V, keep):
    """Logits multiplied by a mask hold zeros of both signs, and so do scores: the lower word goes first, then the lower
    beam."""
    select = BeamSelect(2, B, V, keep=keep, dtype=dt)
    for seed in range(6):
        g = torch.Generator().manual_seed(seed)
        logits = -torch.randn(2 * B, V, generator=g).abs() * (torch.rand(2 * B, V, generator=g) < 0.7)
        logits[torch.rand(2 * B, V, generator=g) < 0.1] = 0.0  # beside those of -0.0
        assert bool((torch.signbit(logits) & (logits == 0)).any()) and bool((~torch.signbit(logits) & (logits == 0)).any())
        check(select, logits.to(dt).cuda(), torch.full((2, B), -1.0))


def test_finished_beams_whose_scores_are_zeros_of_both_signs(cuda_dev):
    for order in ([-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, -0.0]):
        select = BeamSelect(1, 4, 50, dtype=F32)
        check(select, torch.zeros(4, 50).cuda(), torch.tensor([order]), torch.ones(1, 4, dtype=torch.bool), 7)
