"""Verification of drafts without probabilities where next to nothing of a row is left after its rejections."""
import pytest
import torch

from test_gpu_verify import DT, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", [0.75, 1.25])
@pytest.mark.parametrize("dtype,e,n", [("f32", 20, 4), ("f32", 12, 6), ("bf16", 7, 10)])
@pytest.mark.parametrize("V,step", [(64, 1), (4096, 1), (4096, 311), (150001, 1), (150001, 9973)])
def test_rows_of_which_next_to_nothing_is_left(rest, dtype, e, n, V, step):
    """The k-th sibling takes all but about 2^-e of what its elders have left, so that after n rejections rest * 2^-(e n) is left of the
    row, below the last bit of its sum; half of that is the last sibling's.  All numbers are exact in their type."""
    S, T = 4, n + 2
    c = make(1, S, T, V, "fixed", True, dtype, "flat")
    row = torch.zeros(V, dtype=torch.float64)
    at = [3 + step * k for k in range(n + 3)]
    for k in range(n):
        row[at[k]] = 2.0 ** (-e * k) * (1 - 2.0 ** -e)
    row[at[n]], row[at[n + 1]] = rest / 2 * 2.0 ** (-e * n), rest / 2 * 2.0 ** (-e * n)
    assert torch.equal(row.to(DT[dtype]).double(), row)
    c["target_prefix"][:] = row.to(DT[dtype])
    c["tokens"][:, :n] = torch.tensor(at[:n], dtype=torch.int32)
    c["accept_u"][:, :n] = 1 - 2.0 ** -24          # rejected: what is left is larger than the sibling's by 2^-e of itself, or nearly so
    # the last two: one that the target cannot say, and then half of what is left
    c["tokens"][:, n], c["tokens"][:, n + 1] = at[n + 2], at[n]
    c["accept_u"][:, n] = 2.0 ** -20
    c["accept_u"][:, n + 1] = torch.tensor([0.45, 0.55, 0.501, 0.499])
    path, took, nxt = check(c, 1)
    assert path[:, 0].tolist() == [n + 1, -1, -1, n + 1]
    assert [int(nxt[1]), int(nxt[2])] == [at[n + 1]] * 2
