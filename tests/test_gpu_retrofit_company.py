"""bf16 calls with max_seqlen up to 384: a sequence's results are the same to the bit alone and in any company."""
import pytest
import torch

from retrofit_harness import attention_inputs, cu_of, handle, on

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def run(dev, d, lens, heads, longest):
    h = handle(dev, *heads, BF16, lens)
    a, cu = (d["q"], d["k"], d["v"]), cu_of(lens, dev)
    o, lse = h.attention(*a, cu, longest, d["bias"])
    grads = h.attention_backward(d["dout"], *a, o, lse, cu, longest, d["bias"])
    assert h.status() == (0, 0)
    return {n: t.transpose(0, 1) if n in ("lse", "dbias") else t
            for n, t in zip(("out", "lse", "dq", "dk", "dv", "dbias"), (o, lse, *grads))}


@pytest.mark.parametrize("heads", [(64, 8, 128), (30, 6, 64), (32, 1, 128), (4, 4, 128)])
@pytest.mark.parametrize("lens", [[300, 300], [1, 384, 127, 200], [40, 383] * 30])
def test_alone_and_in_company(cuda_dev, lens, heads):
    d = on(attention_inputs(lens, *heads, BF16), cuda_dev)
    got = run(cuda_dev, d, lens, heads, 384 if sum(lens) >= 384 else max(lens))
    a = 0
    for n in lens[:4]:
        part = {i: t[:, a:a + n].contiguous() if i == "bias" else t[a:a + n] for i, t in d.items()}
        for name, want in run(cuda_dev, part, [n], heads, n).items():
            assert torch.equal(got[name][a:a + n], want), (n, name)
        a += n
