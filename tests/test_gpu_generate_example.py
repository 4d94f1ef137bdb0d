"""The generation example: it runs, and the gradients that reach the model through the rotation are those of the rotation
written out in plain torch."""
import os
import sys

import torch
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def plain_turn(rotary, q, k, places):
    D = q.shape[-1]
    freq = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=q.device) / D)
    angle = places.double()[:, None] * freq
    angle[:, 0] = 0.0
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1).to(x.dtype)
    return turned(q), turned(k)


def test_taught_and_continued(cuda_dev):
    import generate as example

    model, rotary, loss = example.train(4, 3.0, cuda_dev, quiet=True)
    assert loss == loss
    said, want, slots, pages, apart = example.search(model, rotary, cuda_dev, beams=3, steps=40)
    assert said.shape == want.shape == (3, 40) and bool(((said >= 0) & (said < example.VOCAB)).all())
    assert 0.0 < slots <= 1.0 and 0 < pages <= apart


def test_gradients(cuda_dev):
    """Both rotations round the same fp32 values to bf16; where one is off by a step the rest of the pass differs by as
    much: gradients within 2^-5 of their norm, 8 roundings of 2^-8 in a row."""
    import generate as example

    torch.manual_seed(1)
    model = example.Model().to(cuda_dev)
    rotary = example.R.Rotary(example.HEAD_DIM, device=cuda_dev)
    dmc = example.DmcRetrofit(example.HEADS, example.KV_HEADS, example.HEAD_DIM, torch.bfloat16, max_tokens=400, max_seqs=4,
                              hidden=example.HIDDEN, vocab=example.VOCAB, device=cuda_dev)
    grads = []
    for turn in (example.R.apply, plain_turn):
        model.zero_grad()
        loss, kept = example.loss_of(model, dmc, rotary, [40, 71, 9], torch.Generator().manual_seed(2), noisy=False, turn=turn)
        (loss + kept).backward()
        grads.append([p.grad.double().clone() for p in model.parameters()])
    for a, b in zip(*grads):
        assert bool(b.any())
        assert float((a - b).norm()) <= 2.0 ** -5 * float(b.norm())
