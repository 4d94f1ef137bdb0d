"""The states' backward kernel hands v's shares of the dots from one warp to the other through rows of
shared memory (CPU: its source is read). Between two barriers of the block no row may be both written and
read, since the warps run apart there."""
import os
import re

import pytest
import torch

from retrofit_harness import OFFSET, TEMPERATURE, cu_of, handle, on, states_inputs
from paper_2403_09636_gb300 import build as B


def backward_kernel():
    with open(os.path.join(B.CSRC, "dmc_retrofit_states.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    return text[text.index("states_backward_kernel("):text.index("cudaError_t forward(")]


def test_rows_are_not_written_and_read_between_two_barriers():
    written, read, seen = set(), set(), 0
    for m in re.finditer(r"__syncthreads\(\)|sh\.other\[(\w+)\]\[\w+\](\s*=(?!=))?", backward_kernel()):
        row = m.group(1)
        if row is None:
            written, read = set(), set()
            continue
        seen += 1
        (written if m.group(2) else read).add(row)
        assert row not in written & read, f"row {row} is written and read without a barrier between"
    assert seen >= 6


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradients_are_the_same_every_time(cuda_dev, dtype):
    """A grid that fills the GPU many times over, beside another one on a second stream: the bits stay."""
    lens, heads = [900, 33, 1400, 64], (32, 32, 128)
    d = on(states_inputs(lens, *heads, dtype), cuda_dev)
    cu, gates = cu_of(lens, cuda_dev), {"noise": d["noise"], "offset": OFFSET, "temperature": TEMPERATURE}
    one, two = (handle(cuda_dev, *heads, dtype, lens) for _ in range(2))

    def grads(h):
        saved = h.states(d["q0"], d["k"], d["v"], cu, max(lens), **gates)[-1]
        return h.states_backward(d["q0"], d["k"], d["v"], cu, max(lens), saved, d["dkt"], d["dvt"], d["dbias"],
                                 d["dalpha"], **gates)

    want = grads(one)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        beside = [grads(two) for _ in range(8)]
    got = [grads(one) for _ in range(8)]
    torch.cuda.synchronize()
    assert one.status() == two.status() == (0, 0)
    for g in got + beside:
        for name, a, b in zip(("dq0", "dk", "dv"), g, want):
            assert torch.equal(a, b), name
