"""Frequencies of the rotation as whole numbers, and what the rotation refuses (CPU)."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300 import build as B
from paper_2403_09636_gb300 import rotary as R


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()


def test_turns_are_the_frequencies_to_the_last_bit():
    """position * turns modulo 2^64 is the angle modulo a turn: against the same product of exact fractions."""
    r = R.Rotary(128, base=10000.0, device="cpu")
    pi = 2 * Fraction(0xC90FDAA22168C234C4C6628B80DC1CD129024E088A67CC74, 1 << 191)  # pi's bits
    assert abs(float(pi) - math.pi) < 1e-15
    for i in (1, 5, 33, 63):
        f = Fraction(10000.0 ** (-2.0 * i / 128))
        for at in (1, 7, 1 << 20, (1 << 31) - 1, -5):
            want = f * at / (2 * pi) % 1
            got = Fraction(int(r.turns[i]) * at % (1 << 64), 1 << 64)
            off = abs(got - want)
            assert min(off, 1 - off) <= Fraction(abs(at), 1 << 64), (i, at)


def test_given_frequencies_and_base_are_alike():
    a = R.Rotary(64, base=500.0, device="cpu")
    b = R.Rotary(64, inv_freq=[500.0 ** (-2.0 * i / 64) for i in range(32)], interleaved=True, device="cpu")
    assert torch.equal(a.turns, b.turns) and b.interleaved and not a.interleaved


@pytest.mark.parametrize("bad", [dict(head_dim=96), dict(head_dim=64, base=0.0), dict(head_dim=64, base=math.nan),
                                 dict(head_dim=64, inv_freq=[1.0] * 31), dict(head_dim=64, inv_freq=[math.inf] * 32)])
def test_rotary_refuses(bad):
    with pytest.raises(ValueError):
        R.Rotary(**bad, device="cpu")


def test_rotate_refuses_addresses_and_sizes_on_the_host():
    def call(dtype=P.DMC_BF16, D=64, T=2, at=64, turns=64, hq=2, q=64, qs=128, to=64, ts=128, hk=0, k=None, ks=0, kt=None, kts=0):
        return P.dmc_rotate(dtype, D, T, at, turns, 0, 0, hq, q, qs, to, ts, hk, k, ks, kt, kts, 0)

    assert call(T=0) == P.DMC_OK and call(hq=0) == P.DMC_OK
    for bad in (dict(dtype=2), dict(D=96), dict(T=-1), dict(at=None), dict(turns=None), dict(at=66), dict(turns=68),
                dict(hq=-1), dict(q=None), dict(to=None), dict(q=72), dict(to=72), dict(qs=127), dict(qs=132), dict(ts=100),
                dict(qs=136), dict(hk=1, k=64, ks=64, kt=None, kts=64), dict(hk=1, k=64, ks=32, kt=64, kts=64)):
        assert call(**bad) == P.DMC_ERR_INVALID_ARG, bad
