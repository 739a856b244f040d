"""Siblings drawn without replacement from drafts that one token dominates: what is left of such a draft is little, and in bf16 as much
as the row's sum is off one."""
import numpy as np
import pytest
import torch

import distinct_reference as ref
import paper_2402_06262_b200 as R
from test_gpu_verify import DT, call

pytestmark = pytest.mark.gpu


def make(seed, S, T, V, prefix, dtype, shape, lead, kept=1.0):
    """Rows whose draft has a token of up to 1 - 1e-3, or several; kept: the share of each draft's tokens that have any probability."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = 1.5 * torch.randn(S, T + 1, V, generator=g, dtype=torch.float64)
    z = x + torch.randn(S, T + 1, V, generator=g, dtype=torch.float64)
    at = torch.randint(0, V, (S, T + 1, 2), generator=g)
    top = z.logsumexp(-1, keepdim=True) + lead * torch.rand(S, T + 1, 2, generator=g, dtype=torch.float64)
    z.scatter_(-1, at, top)
    if kept < 1:
        z = z.masked_fill(torch.rand(z.shape, generator=g) > kept, -torch.inf).scatter(-1, at, top)
    p, q = torch.softmax(x, -1).to(DT[dtype]), torch.softmax(z, -1).to(DT[dtype])
    par = torch.full((S, T), -1, dtype=torch.int32)
    for b in range(S):
        for i in range(T):
            if shape == "flat":
                par[b, i] = -1 if prefix else min(i, 1) - 1
            elif i and (not prefix or torch.rand((), generator=g) > 0.3):
                par[b, i] = int(torch.randint(0, min(i, 3), (), generator=g))
    tok = torch.zeros(S, T, dtype=torch.int32)
    for b in range(S):
        for up in set(par[b].tolist()):
            kids = [i for i in range(T) if par[b, i] == up]
            row = q[b, up + 1].float()
            n = min(len(kids), int((row > 0).sum()))
            tok[b, kids[:n]] = torch.multinomial(row, n, generator=g).int()
            for i in kids[n:]:                 # (more siblings than the draft can say: the first again)
                tok[b, i] = tok[b, kids[0]]
    return dict(target=p[:, 1:], draft=q[:, 1:], target_prefix=p[:, 0] if prefix else None, draft_prefix=q[:, 0] if prefix else None,
                tokens=tok, parent=par, accept_u=torch.rand(S, T, generator=g), sample_u=torch.rand(S, generator=g), nodes=None,
                distinct=True)


def check(c, A, near=0, views=False):
    """Every sequence against the definition; those whose decision hangs on less than 64 bits can tell (near) are left out."""
    path, n, nxt = call(c, A, views)
    f = lambda x, b: None if x is None else x[b].cpu().double().numpy()  # noqa: E731
    left_out = 0
    for b in range(path.shape[0]):
        want, token, margin = ref.verify(f(c["target"], b), f(c["draft"], b), f(c["target_prefix"], b), f(c["draft_prefix"], b),
                                         c["tokens"][b].tolist(), c["parent"][b].tolist(), c["accept_u"][b].double().numpy(),
                                         float(c["sample_u"][b]), A)
        if margin < 1e-12:
            left_out += 1
            continue
        assert path[b].tolist() == want + [-1] * (A - len(want)) and int(n[b]) == len(want), f"sequence {b}"
        assert int(nxt[b]) == token, f"sequence {b}: {int(nxt[b])}, {token}"
    assert left_out <= near


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("shape", ["flat", "random"])
@pytest.mark.parametrize("S,T,V,A", [(6, 4, 9, 2), (40, 5, 60, 3), (200, 4, 1001, 2), (20, 16, 4099, 5), (9, 6, 33001, 3), (3, 8, 150003, 4)])
def test_peaked_drafts(dtype, prefix, shape, S, T, V, A):
    for lead in (1.0, 4.0, 8.0):
        check(make(S + V, S, T, V, prefix, dtype, shape, lead), A)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5003, 70001])
def test_drafts_of_few_tokens(dtype, V):
    """Most of the draft's probabilities are zero, and siblings may use up all that it can say."""
    for kept in (0.0, 0.02, 0.3):
        check(make(V, 30, 5, V, True, dtype, "flat", 5.0, kept), 2)


@pytest.mark.parametrize("skip", [1, 3])
def test_rows_of_a_wider_matrix(skip):
    S, T, V = 12, 5, 2345
    for dtype in ("f32", "bf16"):
        c = make(7, S, T, V, True, dtype, "flat", 6.0)
        for name, lead in (("target", skip), ("draft", 2 * skip)):
            wide = torch.full((S, T + 1, V + 11), np.nan, dtype=DT[dtype], device="cuda")
            wide[:, 0, lead:lead + V], wide[:, 1:, lead:lead + V] = c[name + "_prefix"].cuda(), c[name].cuda()
            c[name + "_prefix"], c[name] = wide[:, 0, lead:lead + V], wide[:, 1:, lead:lead + V]
        check(c, 2, views=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0.9966, 0.993, 0.971, 0.908])
def test_what_comes_out_is_distributed_as_the_target(dtype, top):
    """The first token that a round gives: 200000 sequences with the same rows, two siblings and numbers at random, against the exact
    distribution (within five standard deviations of each of five counts: one in 200000 such tests would fail by chance)."""
    S, T, V = 200000, 2, 5
    q = torch.tensor([top, *((1 - top) * torch.tensor([0.45, 0.3, 0.2, 0.05])).tolist()]).to(DT[dtype])
    p = torch.tensor([0.55, 0.2, 0.1, 0.05, 0.1]).to(DT[dtype])
    g = torch.Generator()
    g.manual_seed(int(top * 1e4))
    tok = torch.multinomial(q.float().expand(S, V), T, generator=g).int()
    c = dict(target=p.expand(S, T, V).contiguous(), draft=q.expand(S, T, V).contiguous(), target_prefix=p.expand(S, V).contiguous(),
             draft_prefix=q.expand(S, V).contiguous(), tokens=tok, parent=torch.full((S, T), -1, dtype=torch.int32),
             accept_u=torch.rand(S, T, generator=g), sample_u=torch.rand(S, generator=g), nodes=None, distinct=True)
    path, n, nxt = call(c, 1)
    first = torch.where(n > 0, tok.gather(1, path.long().clamp_min(0))[:, 0], nxt).numpy()
    freq = np.bincount(first, minlength=V) / S
    p, q = p.double().numpy(), q.double().numpy()
    want = ref.first_token(p, q, T)
    sd = np.sqrt(want * (1 - want) / S)
    assert (np.abs(freq - want) < 5 * sd).all()
    e = abs(p.sum() - 1) + abs(q.sum() - 1)
    assert np.abs(freq - p / p.sum()).sum() / 2 < 2.5 * sd.sum() + e * (1 + 16 / 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_drafts_that_are_no_probabilities(dtype):
    """Nearly all of the draft is rejected and its row holds a NaN (nothing to draw from) or an infinity (which takes all of its token,
    and M stays what one less the rejected leaves)."""
    S, T, V = 3, 2, 3000
    c = make(11, S, T, V, True, dtype, "flat", 3.0)
    c["target_prefix"][:], c["draft_prefix"][:] = 2.0 ** -12, 2.0 ** -16
    c["tokens"][:] = torch.tensor([7, 8], dtype=torch.int32)
    c["draft_prefix"][:, 7], c["draft_prefix"][:, 8] = 0.875, 2.0 ** -4
    c["target_prefix"][:, 7], c["target_prefix"][:, 8] = 0, 0
    c["draft_prefix"][1, 1234], c["draft_prefix"][2, 1234] = np.nan, np.inf
    path, n, nxt = call(c, 1, status=32)
    assert n.tolist() == [0, 0, 0] and int(nxt[1]) == -1
    assert int(nxt[0]) >= 0 and int(nxt[2]) not in (-1, 7, 8, 1234)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_two_at_once(dtype):
    c = make(12, 40, 8, 20001, True, dtype, "flat", 7.0)
    d = {k: v.contiguous().cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def launch(out):
        R.roco_tree_verify(d["target"], d["tokens"], d["parent"], d["accept_u"], d["sample_u"], *out, status, draft=d["draft"],
                           target_prefix=d["target_prefix"], draft_prefix=d["draft_prefix"], distinct=True)

    new = lambda: (torch.zeros(40, 4, dtype=torch.int32, device="cuda"), *(torch.zeros(40, dtype=torch.int32, device="cuda") for _ in range(2)))  # noqa: E731
    first, one, two, held = new(), new(), new(), new()
    launch(first)
    torch.cuda.synchronize()
    for s, out in zip((torch.cuda.Stream(), torch.cuda.Stream()), (one, two)):
        with torch.cuda.stream(s):
            launch(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        launch(held)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for out in (one, two, held):
            assert all(torch.equal(x, y) for x, y in zip(first, out))
    assert int(status) == 0
