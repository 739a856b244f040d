"""Prompts of linear attention that are divided among several CTAs per unit, for both head dimensions and types, against the
recurrence in 64 bits (inputs, bounds and checks of the prompt tests)."""
import pytest
import torch

import paper_2402_06262_b200 as R
from test_gpu_linear import check_prompt, inputs, make_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("lens", [[4500, 2111], [1, 129], [0, 1200], [128, 512], [3000, 33]])
def test_divided_prompt(dtype, d, lens):
    """Also prompts of fewer chunks than there are segments: empty segments, which pass the first state on."""
    q, k, v, state = inputs(5 + d, 2, 2, 4500, d, dtype)
    st, _ = check_prompt(q, k, v, state, [-2.0 ** -12, -0.02], lens, dtype)
    assert R.roco_linear_prefill_workspace_bytes(st, 4500) > 0      # it was divided


@pytest.mark.parametrize("d", [64, 128])
def test_divided_prompts_one_behind_the_other(d):
    """Many divided calls in a row on two streams: the two launches of a call overlap, and calls meet on the same SMs.  Bit for
    bit as one after the other."""
    data = [[t.to("cuda") for t in inputs(70 + i, 1, 9 + i, 2100, d, "bf16")] for i in range(2)]
    lens = torch.tensor([2099], dtype=torch.int32, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for at_once in (False, True):
        st = [make_state(x[3], [-0.01] * x[0].shape[1], "bf16") for x in data]
        out = [torch.zeros_like(x[0]) for x in data]
        torch.cuda.synchronize()
        for _ in range(8):
            for i in range(2):
                with torch.cuda.stream(streams[i if at_once else 0]):
                    R.roco_linear_prefill(st[i], *data[i][:3], lens, out[i])
        torch.cuda.synchronize()
        assert all(R.roco_linear_device_status(s) == 0 for s in st)
        got.append([s.state for s in st] + out)
    assert all(torch.equal(a, b) for a, b in zip(*got))
