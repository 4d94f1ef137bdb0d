"""Beam search's selection against its definition in 64 bits (GPU).

Tokens, parents and done are equal. Scores: the log-sum is off by some 2^-20 relative to the sum (its terms by 3 steps of
2^-24 each, their sums by up to 9 more of what a lane adds), then the one rounding to fp32."""
import math

import pytest
import torch

import paper_2403_09636_gb300 as P
from generate_harness import near, picked
from paper_2403_09636_gb300.beam import BeamSelect

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def check(select, logits, scores, finished=None, eos=-1, x=None):
    got = select.select(logits if x is None else x, scores.cuda(), None if finished is None else finished.cuda(), eos)
    want = picked(logits.float().cpu(), scores, finished, eos, select.keep)
    assert torch.equal(got[1].cpu().long(), want[1])
    assert torch.equal(got[2].cpu().long(), want[2])
    assert torch.equal(got[3].cpu(), want[3])
    s, w = got[0].cpu().double(), want[0]
    assert torch.equal(torch.isinf(s), torch.isinf(w))
    f = torch.isfinite(w)
    near(s[f], w[f], 2.0 ** -20 + 2.0 ** -23 * w[f].abs())
    return got


def made(G, B, V, dt, seed=0, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(G * B, V, generator=g) * spread).to(dt).cuda(), -40 * torch.rand(G, B, generator=g), g


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("G,B,V,keep", [(1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 21), (1, 4, 32000, 4), (3, 5, 1009, 10),
                                        (2, 32, 4097, 32), (40, 8, 515, 16), (700, 1, 33, 3), (1, 2, 130003, 32),
                                        (5, 4, 2048, 1), (2, 2, 256, 32)])
def test_against_the_definition(cuda_dev, dt, G, B, V, keep):
    """(Logits of type bf16 have many equals among a row's best: those go to the lower word.)"""
    logits, scores, _ = made(G, B, V, dt)
    select = BeamSelect(G, B, V, keep=keep, dtype=dt)
    first = check(select, logits, scores)
    again = select.select(logits, scores.cuda())
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_rows_that_begin_anywhere(cuda_dev, dt):
    """Odd strides and starts, rows up to the buffer's last element; what lies between the rows is not read into
    anything. The result is the packed rows', bit for bit."""
    G, B, V = 2, 4, 3001
    logits, scores, _ = made(G, B, V, dt)
    select = BeamSelect(G, B, V, keep=8, dtype=dt)
    want = check(select, logits, scores)
    for stride, start in ((V, 1), (V + 1, 0), (V + 7, 3), (V + 8, 5)):
        buf = torch.full((start + stride * (G * B - 1) + V,), math.nan, dtype=dt).cuda()
        view = buf.as_strided((G * B, V), (stride, 1), start)
        view.copy_(logits)
        got = select.select(view, scores.cuda())
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (stride, start)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_equal_beams_and_equal_logits(cuda_dev, dt):
    """Nothing but ties: lower words first, then lower beams, wherever rows lie."""
    for V in (64, 5001, 40000):
        logits = torch.zeros(6, V, dtype=dt).cuda()
        select = BeamSelect(2, 3, V, keep=9, dtype=dt)
        check(select, logits, torch.zeros(2, 3))
        logits[:, V // 2] = 1.0  # the same best word in each
        check(select, logits, torch.zeros(2, 3))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_rising_logits(cuda_dev, dt):
    """Every element is a new best: the longest way through the lists."""
    V = 40000
    logits = torch.linspace(-5, 5, V).expand(2, V).contiguous().to(dt).cuda()
    check(BeamSelect(1, 2, V, keep=32, dtype=dt), logits, torch.tensor([[-1.0, -2.0]]))


@pytest.mark.parametrize("dt", [F32, BF16])
def test_the_first_step(cuda_dev, dt):
    """Scores 0, -inf, -inf, ...: all continuations are the first beam's."""
    logits, _, _ = made(2, 4, 1000, dt)
    scores = torch.full((2, 4), -math.inf)
    scores[:, 0] = 0.0
    got = check(BeamSelect(2, 4, 1000, dtype=dt), logits, scores)
    assert got[2].cpu().tolist() == [[0] * 4, [4] * 4]


@pytest.mark.parametrize("dt", [F32, BF16])
def test_finished_beams(cuda_dev, dt):
    G, B, V, eos = 6, 4, 777, 13
    logits, scores, g = made(G, B, V, dt, 1)
    finished = torch.rand(G, B, generator=g) < 0.5
    finished[0], finished[1] = True, False
    scores[2, 0], finished[2, 0] = -math.inf, True
    scores[3, 1], finished[3, 1] = math.nan, True
    logits[~finished.view(-1).cuda(), eos] += 9.0  # some end now
    logits[finished.view(-1).cuda()] = math.nan  # not read
    for keep in (4, 9, 32):
        check(BeamSelect(G, B, V, keep=keep, dtype=dt), logits, scores, finished, eos)
    check(BeamSelect(G, B, V, keep=5, dtype=dt), logits.nan_to_num(0.0), scores.nan_to_num(0.0, 0.0, -1.0), None, eos)
    for end in (0, V - 1):
        check(BeamSelect(G, B, V, keep=6, dtype=dt), logits, scores, torch.ones(G, B, dtype=torch.bool), end)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_masked_words_and_rows_that_offer_nothing(cuda_dev, dt):
    """Logits of -infinity, rows of nothing else, the type's lowest value, +infinity, values that are not numbers."""
    G, B, V = 3, 4, 3000
    logits, scores, _ = made(G, B, V, dt, 2)
    logits[0, 5:] = -math.inf            # five words
    logits[1] = -math.inf                # none
    logits[2, :] = torch.finfo(dt).min   # all alike, at the type's lowest
    logits[2, 70] = 3.0
    logits[4, 17] = math.nan             # the row's log-sum is none: it offers nothing
    logits[5, 2999] = math.inf
    logits[8:12] = -math.inf             # a group that has nothing at all
    for keep in (3, 16, 32):
        check(BeamSelect(G, B, V, keep=keep, dtype=dt), logits, scores)


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("B,V,keep", [(1, 5, 5), (1, 700, 4), (2, 9000, 32), (4, 33000, 4)])
def test_rows_of_values_that_are_not_numbers(cuda_dev, dt, B, V, keep):
    """Every place of the results is written, also where no logit is a number: words in their order, at -infinity."""
    logits, scores, _ = made(3, B, V, dt, 6)
    logits[:B] = math.nan          # a group of nothing else
    logits[B, V // 2 + 1:] = math.nan
    logits[2 * B, 2:] = math.nan   # fewer numbers than continuations
    check(BeamSelect(3, B, V, keep=keep, dtype=dt), logits, scores)


def test_scores_that_are_not_finite(cuda_dev):
    logits, scores, _ = made(2, 3, 100, F32, 3)
    scores[0, 0], scores[0, 1], scores[1, 2] = math.nan, math.inf, -math.inf
    check(BeamSelect(2, 3, 100, keep=7, dtype=F32), logits, scores)


def test_sharp_and_flat_logits(cuda_dev):
    """Logits that spread by hundreds: most exponentials are zero; and hardly at all."""
    for spread in (300.0, 1e-3):
        logits, scores, _ = made(2, 4, 9001, F32, 4, spread)
        check(BeamSelect(2, 4, 9001, keep=8, dtype=F32), logits, scores)


def test_in_place_graph_and_stream(cuda_dev):
    G, B, V, eos = 3, 4, 2000, 7
    logits, scores, g = made(G, B, V, BF16, 5)
    select = BeamSelect(G, B, V, dtype=BF16)
    finished = (torch.rand(G, B, generator=g) < 0.3).cuda()
    s = scores.cuda()
    want = select.select(logits, s, finished, eos)
    keep = [s.clone(), finished.clone()]
    tokens, parents = torch.zeros_like(want[1]), torch.zeros_like(want[2])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        select.select(logits, s, finished, eos, out=(s, tokens, parents, finished))
    for _ in range(2):
        s.copy_(keep[0])
        finished.copy_(keep[1])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((s, tokens, parents, finished), want))
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = select.select(logits, keep[0], keep[1], eos, stream=other)
    other.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(cuda_dev):
    select = BeamSelect(2, 3, 50, keep=4, dtype=BF16)
    logits, scores, _ = made(2, 3, 50, BF16)
    s, f = scores.cuda(), torch.zeros(2, 3, dtype=torch.bool).cuda()
    ok = dict(logits=logits, scores=s, finished=f, eos=0)
    for bad in (dict(logits=logits.float()), dict(logits=logits[:5]), dict(logits=logits[:, :49]), dict(logits=logits.cpu()),
                dict(logits=logits.t().contiguous().t()), dict(logits=logits[:1].expand(6, 50)), dict(scores=s.double()),
                dict(scores=s.view(-1)), dict(finished=f.int()), dict(finished=f.cpu()), dict(out=(s, s)),
                dict(out=(s, s, s, f))):
        with pytest.raises(ValueError):
            select.select(**{**ok, **bad})
    for bad in (dict(eos=50), dict(eos=-1)):  # no word; finished beams without an end word
        with pytest.raises(P.DmcError):
            select.select(**{**ok, **bad})
    # in place with another number of continuations than beams
    p = s.data_ptr()
    o = [torch.zeros(2, 4, dtype=t).cuda().data_ptr() for t in (F32, torch.int32, torch.int32, torch.bool)]
    call = lambda *a: P.dmc_beam_select(select.handle, logits.data_ptr(), 50, p, f.data_ptr(), 0, *a, 0)  # noqa: E731
    assert call(p, *o[1:]) == P.DMC_ERR_INVALID_ARG
    assert call(*o[:3], f.data_ptr()) == P.DMC_ERR_INVALID_ARG
    assert call(o[0] + 2, *o[1:]) == P.DMC_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        BeamSelect(1, 1, 10, dtype=torch.float16)
    with pytest.raises(P.DmcError):
        BeamSelect(1, 33, 10)
