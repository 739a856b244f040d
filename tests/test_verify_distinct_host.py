"""The definition for siblings drawn without replacement gives the target's distribution, exactly enumerated, in bf16 rows too."""
import numpy as np
import pytest
import torch

import distinct_reference as ref


def rows(seed, V, lead, dtype):
    g = torch.Generator()
    g.manual_seed(seed)
    z = torch.randn(V, generator=g, dtype=torch.float64)
    x = z + torch.randn(V, generator=g, dtype=torch.float64)
    z[0] += lead
    return (torch.softmax(r, 0).to(dtype).double().numpy() for r in (x, z))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,n", [(4, 1), (5, 2), (6, 3), (3, 3)])
@pytest.mark.parametrize("lead", [0, 2, 3, 4, 5, 7, 9])
def test_what_comes_out_is_distributed_as_the_target(dtype, V, n, lead):
    """Flat drafts to one token of 0.9995.  The first test is off by as much as the two rows' sums are off one (e), a later one by that
    relative to M, which is at least 3/16 where it is not a sum: e (1 + 16/3) in all, and 10^-12 for the arithmetic."""
    for seed in range(25):
        p, q = rows(seed, V, lead, dtype)
        e = abs(p.sum() - 1) + abs(q.sum() - 1)
        off = np.abs(ref.first_token(p, q, n) - p / p.sum()).sum() / 2
        assert off <= e * (1 + 16 / 3) + 1e-12
