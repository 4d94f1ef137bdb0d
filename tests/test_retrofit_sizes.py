"""The bytes that a retrofitting handle asks for (CPU): never fewer than its largest parts take, however large the
numbers of a config are."""
import random

import pytest

import paper_2403_09636_gb300 as P
from paper_2403_09636_gb300 import build as B


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


def parts(c):
    """Bytes of some of a handle's parts, in numbers without an end."""
    f32 = c["dtype"] == P.DMC_F32
    sums = (c["max_tokens"] // 32 + c["max_seqs"]) * c["num_kv_heads"] * 2 * (c["head_dim"] + 2) * 8
    words = c["max_tokens"] * -(-c["vocab"] // 64) * 4 if c["hidden"] else 0
    three = 6 * c["max_tokens"] * c["hidden"] if f32 else 0
    return [2 * sums, 2 * words, three]


def need(**c):
    return P.dmc_retrofit_required_bytes(P.dmc_retrofit_config(*[c[f] for f, _ in P.dmc_retrofit_config._fields_]))


BASE = dict(num_q_heads=0, num_kv_heads=0, head_dim=0, dtype=P.DMC_BF16, max_tokens=8, max_seqs=1, hidden=0, vocab=0)


@pytest.mark.parametrize("c", [dict(max_tokens=2 ** 31 - 1, hidden=2 ** 31 - 8, vocab=2),
                               dict(max_tokens=2 ** 31 - 1, hidden=2 ** 31 - 8, vocab=2 ** 30),
                               dict(max_tokens=1750000000, hidden=1756800000, vocab=1, dtype=P.DMC_F32)])
def test_sizes_that_pass_64_bits_are_refused(c):
    assert need(**{**BASE, **c}) == 0


def test_large_configs():
    rng = random.Random(5)

    def number(hi):
        return max(1, min(hi, int(2 ** rng.uniform(0, hi.bit_length()))))

    counted = 0
    for _ in range(3000):
        c = dict(BASE, dtype=rng.choice([P.DMC_F32, P.DMC_BF16]), max_tokens=number(2 ** 31 - 1), max_seqs=number(2 ** 31 - 1))
        if rng.random() < 0.7:
            c["num_kv_heads"] = number(65535)
            c["num_q_heads"] = c["num_kv_heads"] * rng.randrange(1, 33)
            c["head_dim"] = rng.choice([64, 128])
        if rng.random() < 0.7 or not c["num_q_heads"]:
            c["hidden"], c["vocab"] = number((2 ** 31 - 8) // 8) * 8, number(2 ** 30)
        got = need(**c)
        if got:
            counted += 1
            assert got >= sum(parts(c)), c
    assert counted > 500
