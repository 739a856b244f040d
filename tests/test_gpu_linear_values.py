"""Linear attention over a prompt: a token's row does not depend on later tokens, however large they are."""
import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R
from test_gpu_linear import close, inputs, make_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L", [40, 300])
@pytest.mark.parametrize("log_decay", [0.0, -0.3])
def test_later_tokens_do_not_reach_a_row(dtype, d, L, log_decay):
    """Queries of size 2^70 and, behind the last of them, keys of size 2^60: their product leaves fp32's range, but no row
    contains it.  Every row of the definition is finite."""
    q, k, v, state = inputs(80 + d, 1, 2, L, d, dtype)
    large = list(range(5, L - 1, 64))
    q[:, :, large] *= 2.0 ** 70
    k[:, :, large[-1] + 1:] *= 2.0 ** 60
    v[:, :, large[-1] + 1:] *= 2.0 ** -60
    decay = [log_decay, -0.01]
    st = make_state(state, decay, dtype)
    out = torch.zeros_like(q).to("cuda")
    R.roco_linear_prefill(st, q.to("cuda"), k.to("cuda"), v.to("cuda"), torch.tensor([L], dtype=torch.int32, device="cuda"), out)
    assert bool(out.isfinite().all()) and bool(st.state.isfinite().all())
    for g in range(2):
        o, s, ob, sb = ref.linear(state[0, g].double(), float(torch.tensor(decay[g])), q[0, g].double(), k[0, g].double(),
                                  v[0, g].double(), d ** -0.5, low=dtype == "bf16")
        close(out[0, g], o, ob, f"out {g}")
        close(st.state[0, g], s, sb, f"state {g}")
