"""Probabilities of the target and of the draft at offsets beyond 32 bits, in both types: rows that decide and rows that are summed."""
import pytest
import torch

import paper_2402_06262_b200 as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("distinct", [False, True])
@pytest.mark.parametrize("dtype,S", [(torch.float32, 70), (torch.bfloat16, 150)])
def test_rows_beyond_two_to_the_32_bytes(dtype, S, distinct):
    T, V, A = 64, 250001, 16
    torch.manual_seed(S)
    way = [0] + list(range(50, 61))                    # what is accepted; node 63 hangs on its end and is rejected
    tokens = torch.randint(1, V // 4, (S, T), dtype=torch.int32, device="cuda")
    target, draft = (torch.zeros(S, T, V, dtype=dtype, device="cuda") for _ in range(2))
    for t in (target, draft):
        assert t.numel() * t.element_size() > 2 ** 32 and (dtype == torch.float32 or t.numel() > 2 ** 31)
    parent = torch.full((S, T), -1, dtype=torch.int32, device="cuda")
    each = torch.arange(S, device="cuda")
    for up, node in zip(way, way[1:]):
        parent[:, node] = up
        for t in (target, draft):
            t[each, up, tokens[:, node].long()] = 1
    parent[:, 63] = 60
    lo, hi = torch.randint(V // 4, V // 2, (S,), device="cuda"), torch.randint(V // 2, V, (S,), device="cuda")
    target[each, 60, lo], target[each, 60, hi] = 0.25, 0.75
    draft[each, 60, tokens[:, 63].long()], draft[each, 60, hi] = 0.5, 0.5
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    path, n, nxt, status = ints(S, A), ints(S), ints(S), ints(1)
    u = torch.full((S, T), 0.999, device="cuda")
    # without the draft a quarter and three, with it a quarter and a quarter of what is left
    for q, border in ((None, 0.25), (draft, 0.5)):
        for s, want in ((border - 1e-4, lo), (border + 1e-4, hi)):
            R.roco_tree_verify(target, tokens, parent, u, torch.full((S,), s, device="cuda"), path, n, nxt, status, draft=q,
                               distinct=distinct)
            assert n.tolist() == [len(way)] * S and torch.equal(nxt.long(), want) and int(status) == 0
            assert path.tolist() == [way + [-1] * (A - len(way))] * S
