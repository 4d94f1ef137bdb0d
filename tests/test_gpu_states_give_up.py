"""Waits between chunks of the states' kernels that run out (GPU).

A test-only kernel (tests/csrc/states_wait_probe.cu), built here with the limit at 2 ms, has warps wait for neighbours that
publish late or not at all. A wait that runs out sets DMC_FAULT_WAIT_TIMEOUT and leaves the launch's number, at which that
launch's other waits end, too; a later launch waits as if nothing had happened, although the fault bit stays."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2403_09636_gb300 import DMC_FAULT_BAD_TARGET, DMC_FAULT_WAIT_TIMEOUT
from paper_2403_09636_gb300 import build as B

pytestmark = pytest.mark.gpu

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "csrc", "states_wait_probe.cu")
LIMIT_NS = 2_000_000
STOP = 96  # the word beside the turns


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("wait") / "libwait.so")
    subprocess.check_call([B.nvcc()] + B.ARCH + B.FLAGS +
                          [f"-DDMC_WAIT_LIMIT_NS={LIMIT_NS}ull", "-shared", SRC, "-o", out])
    lib = C.CDLL(out)
    lib.dmc_states_wait_probe.argtypes = [C.c_int, C.c_uint, C.c_int, C.c_ulonglong] + [C.c_void_p] * 6
    return lib


def run(probe, dev, state, pairs, tag, published, delay):
    got = torch.full((pairs, 32, 3), -1.0, device=dev)
    ns = torch.zeros((pairs, 32), dtype=torch.int64, device=dev)
    assert probe.dmc_states_wait_probe(pairs, tag, published, delay, *[t.data_ptr() for t in (*state, got, ns)],
                                       torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return got, ns


def test_waits_that_run_out(cuda_dev, probe):
    pairs = 16
    state = [torch.zeros(n, dtype=torch.int64 if i == 0 else torch.int32, device=cuda_dev)
             for i, n in enumerate((pairs * 2 * 66, 128, 1))]
    rows, turns, err = state
    err.fill_(DMC_FAULT_BAD_TARGET)  # of an earlier call
    lane = torch.arange(32.0, device=cuda_dev)
    want = torch.stack([lane + 0.25, lane + 0.5, torch.full_like(lane, 3.0)], 1)

    got, _ = run(probe, cuda_dev, state, pairs, 5, pairs, LIMIT_NS // 4)  # late, far beyond the first tries
    assert bool((got == want).all()) and int(turns[STOP]) == 0 and int(err) == DMC_FAULT_BAD_TARGET

    _, ns = run(probe, cuda_dev, state, pairs, 6, pairs // 2, 0)  # half of them never
    assert int(err) == DMC_FAULT_BAD_TARGET | DMC_FAULT_WAIT_TIMEOUT and int(turns[STOP]) == 6
    assert int(ns[pairs // 2:].min()) >= LIMIT_NS // 2 and int(ns.max()) < 100 * LIMIT_NS

    for tag in (7, 8):  # the launches after it
        got, _ = run(probe, cuda_dev, state, pairs, tag, pairs, LIMIT_NS // 4)
        assert bool((got == want).all()) and int(turns[STOP]) == 6
    assert int(err) == DMC_FAULT_BAD_TARGET | DMC_FAULT_WAIT_TIMEOUT
