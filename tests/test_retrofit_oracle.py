"""oracle/retrofit_ref.py against the inference-time oracle, known cases and
differences; what the C functions refuse before any CUDA call."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2403_09636_gb300 as P
from oracle import dmc_ref
from oracle import retrofit_ref as R
from paper_2403_09636_gb300 import build as B

D64 = torch.float64


def rnd(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=D64)


def test_binary_decisions_are_the_training_formulation():
    """Cold temperature and no noise: the states, mask and outputs of formulation B."""
    n, G, d = 23, 3, 6
    k, v, q = rnd(1, n, 1, d), rnd(2, n, 1, d), rnd(3, n, G, d)
    k[:, :, 0] = torch.where(k[:, :, 0] < 0, k[:, :, 0] - 0.1, k[:, :, 0] + 0.1)
    kt, vt, alpha, bias, z = R.states(q[:, :, 0], k, v, None, 0.0, 1e-5)
    ks, vs, zs, al = dmc_ref.unrolled_states(k[:, 0].numpy(), v[:, 0].numpy(), q[:, :, 0].numpy())
    assert np.allclose(kt[1:, 0], ks[1:]) and np.allclose(vt[:, 0], vs) and np.allclose(z[:, 0], zs)
    assert np.allclose(alpha[0, 1:], al[1:])
    out, _, _ = R.attention(q, kt, vt, bias)  # the states' first components are zero: q[0] adds nothing
    want = dmc_ref.masked_attention(k[:, 0].numpy(), v[:, 0].numpy(), q.numpy())
    assert np.allclose(out.numpy(), want, atol=1e-9)


def test_attention_without_bias_is_sdpa():
    q, k, v = rnd(4, 9, 4, 8), rnd(5, 9, 2, 8), rnd(6, 9, 2, 8)
    out, _, _ = R.attention(q, k, v, None)
    t = lambda x, r: x.permute(1, 0, 2).repeat_interleave(r, 0)  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(t(q, 1), t(k, 2), t(v, 2), is_causal=True)
    assert torch.allclose(out, want.permute(1, 0, 2))


def test_states_gradient_against_differences():
    n, H, d = 7, 2, 4
    x = {"q0": rnd(1, n, 4), "k": rnd(2, n, H, d), "v": rnd(3, n, H, d)}
    noise, w = rnd(4, H, n), [rnd(5 + i, *s) for i, s in enumerate([(n, H, d), (n, H, d), (H, n), (H, n)])]

    def f(q0, k, v):
        kt, vt, alpha, bias, _ = R.states(q0, k, v, noise, 0.2, 0.7)
        return (kt * w[0]).sum() + (vt * w[1]).sum() + (bias * w[2]).sum() + (alpha * w[3]).sum()

    assert torch.autograd.gradcheck(f, tuple(t.clone().requires_grad_() for t in x.values()))


def test_attention_and_loss_gradients_against_differences():
    q, k, v, b = rnd(1, 5, 4, 3), rnd(2, 5, 2, 3), rnd(3, 5, 2, 3), rnd(4, 2, 5)
    assert torch.autograd.gradcheck(lambda *a: R.attention(*a)[0], tuple(t.clone().requires_grad_() for t in (q, k, v, b)))
    h, w, t = rnd(5, 4, 6), rnd(6, 7, 6), torch.tensor([1, -100, 6, 0])
    got = R.loss_all(h, w, t, torch.ones(4, dtype=D64), torch.float32)
    hh, ww = h.clone().requires_grad_(), w.clone().requires_grad_()
    want = torch.nn.functional.cross_entropy(hh @ ww.t(), t, reduction="sum", ignore_index=-100)
    dh, dw = torch.autograd.grad(want, (hh, ww))
    want = want.detach()
    assert torch.allclose(got["loss"][0].sum(), want)
    assert torch.allclose(got["dhidden"][0], dh) and torch.allclose(got["dweight"][0], dw)


def test_bounds_hold_for_plain_fp32():
    """The bounds are wide enough for the same formulas in fp32 and too narrow for a wrong scale."""
    n, H, d = 40, 2, 8
    k = rnd(1, n, H, d).float()
    k[:, :, 0] = k[:, :, 0] * 0.5 + 5.0
    a = [rnd(3, n, 4).float(), k, rnd(2, n, H, d).float()]
    noise, g = rnd(4, H, n).float(), [rnd(5 + i, *s).float() for i, s in enumerate([(n, H, d), (n, H, d), (H, n), (H, n)])]
    res = R.states_all(*a, noise, 5.0, 0.1, *g, torch.float32)
    got = R.states(*a, noise, 5.0, 0.1)
    for name, x in zip(("kt", "vt", "alpha", "bias"), got):
        want, bound = res[name]
        assert bool(((x - want).abs() <= bound).all()), name
        assert not bool(((x * 1.001 - want).abs() <= bound).all()), name


# ---------------------------------------------------------------- the C functions' refusals

@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.lib()


def cfg(**kw):
    base = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, dtype=P.DMC_BF16, max_tokens=1000, max_seqs=4, hidden=256,
                vocab=1000)
    base.update(kw)
    return P.dmc_retrofit_config(*[base[f] for f, _ in P.dmc_retrofit_config._fields_])


def test_parts_of_a_config_can_be_left_out(lib):
    both = P.dmc_retrofit_required_bytes(cfg())
    heads = P.dmc_retrofit_required_bytes(cfg(hidden=0, vocab=0))
    words = P.dmc_retrofit_required_bytes(cfg(num_q_heads=0, num_kv_heads=0, head_dim=0))
    assert 0 < heads < both and 0 < words < both


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(num_q_heads=7), dict(num_q_heads=66), dict(dtype=2),
                                 dict(max_tokens=0), dict(max_seqs=0), dict(hidden=0), dict(vocab=0), dict(hidden=100),
                                 dict(num_kv_heads=0), dict(hidden=-8), dict(vocab=-1),
                                 dict(num_q_heads=0, num_kv_heads=0, head_dim=0, hidden=0, vocab=0)])
def test_invalid_configs_need_zero_bytes(lib, bad):
    c = cfg(**bad)
    assert P.dmc_retrofit_required_bytes(c) == 0
    assert P.dmc_retrofit_create(c, 4096, 1 << 40, 0) == (P.DMC_ERR_INVALID_ARG, None)


def test_create_rejects_a_bad_arena(lib):
    c = cfg()
    assert P.dmc_retrofit_create(c, 0, 1 << 40, 0)[0] == P.DMC_ERR_INVALID_ARG
    assert P.dmc_retrofit_create(c, 4097, 1 << 40, 0)[0] == P.DMC_ERR_INVALID_ARG
    assert P.dmc_retrofit_create(c, 4096, P.dmc_retrofit_required_bytes(c) - 1, 0)[0] == P.DMC_ERR_ARENA_TOO_SMALL


def test_calls_refuse_a_null_handle(lib):
    for name in P.EXPORTED:
        f = getattr(lib, name)
        if not name.startswith("dmc_retrofit_") or name in ("dmc_retrofit_required_bytes", "dmc_retrofit_create"):
            continue
        args = [a() if a in (C.c_int32, C.c_int64, C.c_float) else None for a in f.argtypes]
        want = {"dmc_retrofit_destroy": P.DMC_OK, "dmc_retrofit_saved_bytes": 0}.get(name, P.DMC_ERR_INVALID_ARG)
        assert f(*args) == want, name


def test_fp32_rows_are_multiples_of_16_bytes(lib):
    assert P.dmc_retrofit_required_bytes(cfg(dtype=P.DMC_F32, hidden=100)) > 0
    assert P.dmc_retrofit_required_bytes(cfg(dtype=P.DMC_F32, hidden=98)) == 0
    assert math.isfinite(P.dmc_retrofit_required_bytes(cfg(hidden=104)))
