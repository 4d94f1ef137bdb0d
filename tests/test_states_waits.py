"""How a chunk of the states' kernels waits for others (CPU: the kernels' source is read)."""
import os
import re

from paper_2403_09636_gb300 import build as B


def source():
    with open(os.path.join(B.CSRC, "dmc_retrofit_states.cu")) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_a_warp_leaves_a_wait_as_a_whole():
    """Between two tries a warp votes with all its lanes, so none may have gone on alone."""
    loops = re.findall(r"for \(int tries = 0;.*?give_up\(", source(), re.S)
    assert len(loops) >= 3
    for loop in loops:
        assert re.search(r"__all_sync\(0xffffffffu, (there|look)", loop), loop
