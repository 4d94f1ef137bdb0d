"""How the chunks of the states' kernels wait for one another. On the CPU: the kernels' source is read, and the rule that
says how far a chunk looks back (csrc/dmc_chain.h, compiled here for the host) is run over chains of products
of alphas. On the GPU: gates that are not numbers."""
import ctypes as C
import math
import os
import random
import re
import subprocess

import pytest
import torch

from retrofit_harness import OFFSET, TEMPERATURE, cu_of, handle, on, states_inputs
from paper_2403_09636_gb300 import DMC_FAULT_BAD_SEQLENS, DMC_FAULT_BAD_TARGET
from paper_2403_09636_gb300 import build as B
from paper_2403_09636_gb300.retrofit import DmcRetrofit


def source():
    with open(os.path.join(B.CSRC, "dmc_retrofit_states.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_a_warp_leaves_a_wait_as_a_whole():
    """Between two tries a warp votes with all its lanes, so none may have gone on alone."""
    loops = re.findall(r"for \(int tries = 0;.*?give_up\(", source(), re.S)
    assert len(loops) >= 3
    for loop in loops:
        assert re.search(r"__all_sync\(0xffffffffu, (there|look)", loop), loop


# ---------------------------------------------------------------- which chunks are waited for

@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("chain") / "libchain.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", "chain_rule.cpp")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-I", B.CSRC, src, "-o", out])
    lib = C.CDLL(out)

    def run(prod):
        n = len(prod)
        walks, waits, publishes = ((C.c_int * n)() for _ in range(3))
        lib.dmc_chain_rule(n, (C.c_float * n)(*prod), walks, waits, publishes)
        return list(walks), list(waits), list(publishes)

    return run


def check_chain(rule, prod):
    walks, waits, publishes = rule(prod)
    for c in range(1, len(prod)):
        assert 1 <= walks[c] <= min(c, 16)
        if waits[c] >= 0:
            assert waits[c] < c and waits[c] == c - walks[c] and publishes[waits[c]], (c, waits[c], prod[waits[c]])


def test_every_anchor_that_is_waited_for_publishes(rule):
    values = [math.nan, 0.0, 1e-45, 1e-39, 1.17549435e-38, 1e-30, 1e-3, 0.5, 1.0]
    rng = random.Random(1)
    for _ in range(3000):
        few = rng.sample(values, rng.randrange(1, 5))
        check_chain(rule, [0.0] + [rng.choice(few) for _ in range(rng.randrange(1, 90))])


def test_a_gate_that_is_not_a_number_behind_a_closed_anchor(rule):
    """Nearly binary decisions, one NaN at chunk 20: chunk 21 may not wait for the anchor 16, which does not publish."""
    prod = [0.0] * 40
    prod[20] = math.nan
    check_chain(rule, prod)


def test_walks_reach_what_carries(rule):
    """Where all products are numbers: nothing that carries more than 2^-126 is left out."""
    rng = random.Random(2)
    for _ in range(300):
        prod = [0.0] + [rng.choice([1e-20, 1e-10, 0.5, 1.0, 1.0]) for _ in range(80)]
        walks, waits, _ = rule(prod)
        for c in range(1, len(prod)):
            upto = math.prod(prod[c - walks[c]:c])
            assert waits[c] >= 0 or walks[c] == c or upto < 2.0 ** -126


def long_inputs(lens, heads, dtype, merge):
    """Nearly binary decisions, or (merge) alphas near 1 that carry over hundreds of tokens."""
    x = states_inputs(lens, *heads, dtype, spread=0.5)
    if merge:
        x["k"][..., 0] = OFFSET + 0.7
        x["noise"].mul_(0.1)
    return x


def run_states(h, d, cu, longest):
    gates = {"noise": d["noise"], "offset": OFFSET, "temperature": TEMPERATURE}
    kt, vt, alpha, bias, saved = h.states(d["q0"], d["k"], d["v"], cu, longest, **gates)
    grads = h.states_backward(d["q0"], d["k"], d["v"], cu, longest, saved, d["dkt"], d["dvt"], d["dbias"], d["dalpha"],
                              **gates)
    return dict(zip(("kt", "vt", "dq0", "dk", "dv", "alpha", "bias"), (kt, vt, *grads, alpha, bias)))


@pytest.mark.gpu
@pytest.mark.parametrize("merge", [False, True])
@pytest.mark.parametrize("where", ["k", "noise"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_gate_that_is_not_a_number(cuda_dev, dtype, where, merge):
    """It stays in its head and sequence: no fault, and everything else as without it."""
    lens, heads, tok, head = [700, 1500, 900], (4, 4, 64), 700 + 641, 2
    x = long_inputs(lens, heads, dtype, merge)
    cu = cu_of(lens, cuda_dev)
    h = handle(cuda_dev, *heads, dtype, lens)
    want = run_states(h, on(x, cuda_dev), cu, max(lens))
    if where == "k":
        x["k"][tok, head, 0] = math.nan
    else:
        x["noise"][head, tok] = math.nan
    got = run_states(h, on(x, cuda_dev), cu, max(lens))
    assert h.status() == (0, 0)
    for name in got:
        a, b = ((t.transpose(0, 1) if name in ("alpha", "bias") else t) for t in (got[name], want[name]))
        touched = a[700:2200, head].isnan()
        assert bool(touched.any()), name
        for t in (a, b):
            t[700:2200, head] = 0.0
        assert torch.equal(a, b), name


# ---------------------------------------------------------------- faults of earlier calls

@pytest.mark.gpu
@pytest.mark.parametrize("fault", ["target", "seqlens"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_fault_of_an_earlier_call_changes_nothing(cuda_dev, dtype, fault):
    """A sticky bit (a target beyond the vocabulary, faulty cu_seqlens) says what happened; later calls give what a fresh
    handle's give, long waits along the chain among them."""
    lens, heads = [16384], (2, 2, 64)
    d = on(long_inputs(lens, heads, dtype, True), cuda_dev)
    cu = cu_of(lens, cuda_dev)

    def both():
        return DmcRetrofit(*heads, dtype=dtype, max_tokens=sum(lens), max_seqs=2, hidden=64, vocab=50, device=cuda_dev)

    want = run_states(both(), d, cu, max(lens))
    h = both()
    if fault == "target":
        h.loss(torch.zeros(3, 64, dtype=dtype, device=cuda_dev), torch.zeros(50, 64, dtype=dtype, device=cuda_dev),
               torch.tensor([1, 50, 2], dtype=torch.int32, device=cuda_dev))
    else:
        run_states(h, d, torch.tensor([0, 9000, 8000], dtype=torch.int32, device=cuda_dev), max(lens))
    bits = h.status()[1]
    assert bits == (DMC_FAULT_BAD_TARGET if fault == "target" else DMC_FAULT_BAD_SEQLENS)
    for _ in range(5):
        got = run_states(h, d, cu, max(lens))
        for name in got:
            assert torch.equal(got[name], want[name]), name
    assert h.status()[1] == bits
