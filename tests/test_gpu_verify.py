"""Verification of drafted trees against the 64-bit reference: whole numbers, so equal."""
import math

import numpy as np
import pytest
import torch

import paper_2402_06262_b200 as R
import decoding_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BAD_TREE, BAD_PROBS = 8, 32


def softmax_rows(g, *shape, sharp=2.0):
    return torch.softmax(sharp * torch.randn(*shape, generator=g, dtype=torch.float64), -1)


def make(seed, S=3, T=6, V=50, drafts="drawn", prefix=True, dtype="f32", shape="random", near=0.7):
    """CPU inputs.  near: how far the draft's logits are from the target's."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = 2 * torch.randn(S, T + 1, V, generator=g, dtype=torch.float64)
    p = torch.softmax(x, -1).to(DT[dtype])
    q = torch.softmax(x + near * torch.randn(S, T + 1, V, generator=g, dtype=torch.float64), -1).to(DT[dtype])
    par = torch.full((S, T), -1, dtype=torch.int32)
    tok = torch.zeros(S, T, dtype=torch.int32)
    for b in range(S):
        for i in range(T):
            if shape == "chain":
                par[b, i] = i - 1
            elif shape == "flat":
                par[b, i] = -1 if prefix else min(i, 1) - 1
            elif i and (not prefix or torch.rand((), generator=g) > 0.25):
                par[b, i] = int(torch.randint(0, i, (), generator=g))
        kids = {}
        for i in range(T):
            kids.setdefault(int(par[b, i]), []).append(i)
        for up, nodes in kids.items():
            row = q[b, up + 1].float()
            if drafts == "fixed":
                tok[b, nodes] = row.topk(len(nodes)).indices.int() if len(nodes) <= V else torch.zeros(len(nodes), dtype=torch.int32)
            else:
                tok[b, nodes] = torch.multinomial(row, len(nodes), replacement=drafts == "drawn" or len(nodes) > V, generator=g).int()
    return dict(target=p[:, 1:], draft=None if drafts == "fixed" else q[:, 1:], target_prefix=p[:, 0] if prefix else None,
                draft_prefix=q[:, 0] if prefix and drafts != "fixed" else None, tokens=tok, parent=par,
                accept_u=torch.rand(S, T, generator=g), sample_u=torch.rand(S, generator=g), nodes=None, distinct=drafts == "distinct")


def call(c, A, views=False, status=0):
    S, T = c["tokens"].shape
    path = torch.full((S, A), 99, dtype=torch.int32, device="cuda")
    n, nxt = (torch.full((S,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    # (views of one tensor with the prefix's rows, or tensors of their own)
    dev = {k: v.cuda() if views and isinstance(v, torch.Tensor) else v.contiguous().cuda() if isinstance(v, torch.Tensor) else v
           for k, v in c.items()}
    nodes = None if c["nodes"] is None else torch.tensor(c["nodes"], dtype=torch.int32, device="cuda")
    R.roco_tree_verify(dev["target"], dev["tokens"], dev["parent"], dev["accept_u"], dev["sample_u"], path, n, nxt, flags, nodes=nodes,
                       draft=dev["draft"], target_prefix=dev["target_prefix"], draft_prefix=dev["draft_prefix"],
                       distinct=dev["distinct"])
    assert int(flags) == status
    return path.cpu(), n.cpu(), nxt.cpu()


def want(c, A):
    S, T = c["tokens"].shape
    f = lambda x, b: None if x is None else x[b].double().numpy()  # noqa: E731
    return [ref.verify(f(c["target"], b), f(c["draft"], b), f(c["target_prefix"], b), f(c["draft_prefix"], b), c["tokens"][b].tolist(),
                       c["parent"][b].tolist(), T if c["nodes"] is None else c["nodes"][b], c["accept_u"][b].double().numpy(),
                       float(c["sample_u"][b]), A, c["distinct"]) for b in range(S)]


def check(c, A, views=False, status=0, near=0):
    """Every sequence; those whose decision hangs on less than 64 bits can tell (near: how many there may be) are left out."""
    path, n, nxt = call(c, A, views, status)
    left_out = 0
    for b, w in enumerate(want(c, A)):
        if w.margin < 1e-12:
            left_out += 1
            continue
        assert path[b].tolist() == w.path + [-1] * (A - len(w.path)), f"sequence {b}"
        assert int(n[b]) == len(w.path) and int(nxt[b]) == w.next, f"sequence {b}: {int(nxt[b])}, {w.next}"
    assert left_out <= near
    return path, n, nxt


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("S,T,V,A", [(1, 1, 5, 1), (4, 6, 50, 4), (3, 16, 1000, 6), (2, 64, 777, 16), (5, 9, 32001, 3), (150, 4, 4099, 4)])
def test_trees(dtype, drafts, prefix, S, T, V, A):
    for shape in ("random", "chain", "flat"):
        check(make(S + T + V, S, T, V, drafts, prefix, dtype, shape), A)


@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
@pytest.mark.parametrize("V", [1, 2, 3, 31, 127, 128, 129, 511, 2047, 2049, 4095, 8193, 16385, 65537, 131073, 262147])
def test_vocabularies(drafts, V):
    """Every number of CTAs, warps and chunks that a row is cut into, odd ones and rows that start inside a chunk among them."""
    for dtype in ("f32", "bf16"):
        for S in (1, 40) if V < 70000 else (1, 20):
            check(make(V, S, 2, V, drafts, True, dtype, "flat", near=2.0), 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("skip", [0, 1, 3, 4])
def test_rows_of_a_wider_matrix(dtype, skip):
    """The prefix's rows and the nodes' in one tensor, a few elements into wider rows; the draft's aligned otherwise."""
    S, T, V = 4, 5, 1234
    c = make(5, S, T, V, "drawn", True, dtype)
    for name, lead in (("target", skip), ("draft", 2 * skip)):
        wide = torch.full((S, T + 1, V + 11), math.nan, dtype=DT[dtype], device="cuda")
        wide[:, 0, lead:lead + V], wide[:, 1:, lead:lead + V] = c[name + "_prefix"].cuda(), c[name].cuda()
        c[name + "_prefix"], c[name] = wide[:, 0, lead:lead + V], wide[:, 1:, lead:lead + V]
    path, n, nxt = call(c, 4, views=True)
    c = {k: v.cpu() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    for b, w in enumerate(want(c, 4)):
        assert w.margin > 1e-12 and path[b, :len(w.path)].tolist() == w.path and int(n[b]) == len(w.path) and int(nxt[b]) == w.next


@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
def test_node_counts(drafts):
    c = make(8, 6, 8, 60, drafts, True)
    c["nodes"] = [8, 0, 1, 5, 7, 2]
    check(c, 8)
    c = make(9, 6, 8, 60, drafts, False)
    c["nodes"] = [8, 0, 1, 5, 7, 2]
    path, n, nxt = check(c, 8)
    assert int(n[1]) == 0 and int(nxt[1]) == -1 and path[1].tolist() == [-1] * 8
    c["nodes"] = [8, -1, 9, 5, 2 ** 31 - 1, 2]
    path, n, nxt = call(c, 8, status=BAD_TREE)
    assert [int(n[b]) for b in (1, 2, 4)] == [0, 0, 0] and [int(nxt[b]) for b in (1, 2, 4)] == [-1, -1, -1]
    assert int(n[0]) >= 1 and int(n[3]) >= 1


def test_numbers_at_the_ends():
    """u = 0 accepts whatever the target can say; u' = 0 is the first token with any probability, u' just below 1 the last."""
    S, T, V = 6, 3, 40
    for drafts in ("drawn", "fixed"):
        c = make(3, S, T, V, drafts, True, shape="chain")
        c["target_prefix"][:, :4], c["target"][:, :, :4] = 0, 0
        c["target_prefix"][:, -5:], c["target"][:, :, -5:] = 0, 0
        c["accept_u"][:] = 0
        c["sample_u"][:] = 0
        path, n, nxt = check(c, 3)
        able = [all(4 <= int(t) < V - 5 for t in c["tokens"][b]) for b in range(S)]
        assert any(able) and all(int(n[b]) == 3 and int(nxt[b]) == 4 for b in range(S) if able[b])
        c["sample_u"][:] = 1 - 2.0 ** -24
        c["target"][:, :, V - 6] = 0.01
        path, n, nxt = call(c, 3)
        assert all(int(nxt[b]) == V - 6 for b in range(S) if able[b])


def test_equal_distributions_accept_everything():
    c = make(4, 30, 8, 100, "drawn", True, shape="chain", near=0.0)
    path, n, nxt = check(c, 8)
    assert n.tolist() == [8] * 30


def test_impossible_tokens_are_rejected():
    """A drafted token that the target cannot say is rejected even by u = 0, one that the draft cannot have said is taken where the
    target can say it."""
    S, T, V = 2, 1, 20
    for drafts in ("drawn", "distinct", "fixed"):
        c = make(6, S, T, V, drafts, True)
        c["accept_u"][:] = 0
        x = c["tokens"][:, 0].long()
        c["target_prefix"][torch.arange(S), x] = 0
        path, n, nxt = check(c, 1)
        assert n.tolist() == [0, 0] and all(int(nxt[b]) != int(x[b]) for b in range(S))
    c = make(6, S, T, V, "drawn", True)
    c["accept_u"][:] = 1 - 2.0 ** -24
    c["draft_prefix"][torch.arange(S), c["tokens"][:, 0].long()] = 0
    path, n, nxt = check(c, 1)
    assert n.tolist() == [1, 1]


@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
def test_the_same_token_twice_among_siblings(drafts):
    S, T, V = 64, 5, 6
    c = make(14, S, T, V, drafts, True, shape="flat", near=3.0)
    c["tokens"][:] = torch.tensor([2, 2, 4, 2, 4], dtype=torch.int32)
    check(c, 3)


def test_all_of_the_draft_rejected():
    """Siblings without replacement that cover every token the draft can say."""
    S, T, V = 16, 3, 7
    c = make(15, S, T, V, "distinct", True, shape="flat")
    c["draft_prefix"][:] = 0
    c["draft_prefix"][:, :3] = torch.tensor([0.5, 0.25, 0.25])
    c["tokens"][:] = torch.tensor([0, 1, 2], dtype=torch.int32)
    c["target_prefix"][:] = 0
    c["target_prefix"][:, 0], c["target_prefix"][:, 5] = 2.0 ** -10, 1 - 2.0 ** -10
    c["accept_u"][:] = 0.9
    path, n, nxt = check(c, 2)
    assert n.tolist() == [0] * S and nxt.tolist() == [5] * S


def test_nothing_left_falls_back_to_the_target():
    """Roundings can reject a token though no probability is left elsewhere: the target itself is then drawn from."""
    S, T, V = 3, 2, 4
    c = make(16, S, T, V, "drawn", True, shape="flat")
    c["target_prefix"][:] = torch.tensor([0.0, 0.5, 0.25, 0.0])
    c["draft_prefix"][:] = torch.tensor([0.0, 1.0, 0.5, 0.0])
    c["tokens"][:] = torch.tensor([1, 2], dtype=torch.int32)
    c["accept_u"][:] = 0.75
    c["sample_u"][:] = torch.tensor([0.0, 0.5, 0.9])
    path, n, nxt = check(c, 2)
    assert n.tolist() == [0, 0, 0] and nxt.tolist() == [1, 1, 2]
    c = make(16, S, T, V, "fixed", True, shape="flat")
    c["target_prefix"][:] = torch.tensor([0.0, 0.75, 0.125, 0.0])
    c["tokens"][:] = torch.tensor([1, 2], dtype=torch.int32)
    c["accept_u"][:, 0], c["accept_u"][:, 1] = 0.8, 1.0
    c["sample_u"][:] = torch.tensor([0.0, 0.5, 0.9])
    path, n, nxt = call(c, 2)
    assert n.tolist() == [0, 0, 0] and nxt.tolist() == [1, 1, 2]


def test_nodes_that_are_none():
    c = make(17, 4, 5, 30, "drawn", True, shape="chain")
    c["accept_u"][:] = 0
    c["tokens"][0, 2], c["tokens"][1, 0], c["parent"][2, 3], c["parent"][3, 1] = 30, -1, 3, -2
    path, n, nxt = check(c, 5, status=BAD_TREE)
    assert n.tolist() == [2, 0, 3, 1]
    c = make(17, 3, 3, 30, "drawn", False, shape="chain")
    c["tokens"][0, 0] = 1000                     # the token sampled last is not looked up
    c["parent"][1, 0] = 0                        # no root: nothing to verify
    c["parent"][2, 1] = -1                       # a second root is never accepted
    c["accept_u"][:] = 0
    path, n, nxt = check(c, 3, status=BAD_TREE)
    assert n.tolist() == [3, 0, 1] and int(nxt[1]) == -1


@pytest.mark.parametrize("bad", ["nan", "inf", "zero", "negative"])
def test_rows_that_are_no_probabilities(bad):
    S, T, V = 3, 2, 5000
    for drafts in ("drawn", "fixed"):
        c = make(18, S, T, V, drafts, True, shape="chain")
        c["accept_u"][:] = 0
        row = c["target"][1, 1]                  # where the second sequence's walk ends
        if bad == "nan":
            row[4321] = math.nan
        elif bad == "inf":
            row[17] = math.inf
        elif bad == "zero":
            row[:] = 0
        else:
            row[:] = -1
        path, n, nxt = call(c, 2, status=BAD_PROBS)
        assert n.tolist() == [2, 2, 2] and int(nxt[1]) == -1 and int(nxt[0]) >= 0 and int(nxt[2]) >= 0
        good = make(18, S, T, V, drafts, True, shape="chain")
        good["accept_u"][:] = 0
        p2, n2, x2 = call(good, 2)
        assert int(nxt[0]) == int(x2[0]) and int(nxt[2]) == int(x2[2])


def test_rows_that_no_walk_needs_may_hold_anything():
    c = make(19, 4, 4, 300, "drawn", True, shape="flat")
    a = check(c, 2)
    ends = [w.path[-1] if w.path else -1 for w in want(c, 2)]
    for b in range(4):
        for i in range(4):
            if i != ends[b]:
                c["target"][b, i], c["draft"][b, i] = math.nan, math.inf
    assert all(torch.equal(x, y) for x, y in zip(a, call(c, 2)))


@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
def test_what_comes_out_is_distributed_as_the_target(drafts):
    """The first token that a round gives: 40000 sequences with the same distributions, drafts and numbers at random.  A count is
    within five standard deviations (of 9 counts and 3 cases, one in 60000 such tests would fail by chance)."""
    S, T, V = 40000, 3, 9
    g = torch.Generator()
    g.manual_seed(77)
    p, q = softmax_rows(g, V, sharp=1.0).float(), softmax_rows(g, V, sharp=1.0).float()
    if drafts == "fixed":
        tok = q.topk(T).indices.expand(S, T)
    else:
        tok = torch.multinomial(q.expand(S, V), T, replacement=drafts == "drawn", generator=g)
    c = dict(target=p.expand(S, T, V).contiguous(), draft=None if drafts == "fixed" else q.expand(S, T, V).contiguous(),
             target_prefix=p.expand(S, V).contiguous(), draft_prefix=None if drafts == "fixed" else q.expand(S, V).contiguous(),
             tokens=tok.int(), parent=torch.full((S, T), -1, dtype=torch.int32), accept_u=torch.rand(S, T, generator=g),
             sample_u=torch.rand(S, generator=g), nodes=None, distinct=drafts == "distinct")
    path, n, nxt = call(c, 1)
    first = torch.where(n > 0, c["tokens"].gather(1, path.long().clamp_min(0))[:, 0], nxt).numpy()
    # the first sibling alone is accepted with probability p(x), or sum min(p, q) where x was drawn from q; sd <= sqrt(S) / 2
    alone = float(p[tok[0, 0]]) if drafts == "fixed" else float(torch.minimum(p, q).sum())
    assert alone * S - 2.5 * S ** 0.5 < int((n > 0).sum()) < S
    freq = np.bincount(first, minlength=V) / S
    sd = np.sqrt(p.double().numpy() * (1 - p.double().numpy()) / S)
    assert (np.abs(freq - p.double().numpy()) < 5 * sd + 1e-7).all()


def test_broadcast_rows():
    """Strides of zero: every sequence and node reads the same row."""
    S, T, V = 3, 4, 100
    c = make(20, S, T, V, "drawn", True)
    full = {k: c[k][:1, :1].expand(S, T, V) for k in ("target", "draft")}
    full.update({k: c[k][:1].expand(S, V) for k in ("target_prefix", "draft_prefix")})
    a = call({**c, **{k: v.contiguous() for k, v in full.items()}}, 3)
    dev = {k: (c[k][:1, :1] if k in ("target", "draft") else c[k][:1]).contiguous().cuda().expand(full[k].shape) for k in full}
    b = call({**c, **dev}, 3, views=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_another_stream_a_captured_call_and_two_at_once():
    c = make(21, 5, 6, 9000, "drawn", True)
    d = {k: v.contiguous().cuda() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def launch(out):
        R.roco_tree_verify(d["target"], d["tokens"], d["parent"], d["accept_u"], d["sample_u"], *out, status, draft=d["draft"],
                           target_prefix=d["target_prefix"], draft_prefix=d["draft_prefix"])

    new = lambda: (torch.zeros(5, 4, dtype=torch.int32, device="cuda"), *(torch.zeros(5, dtype=torch.int32, device="cuda") for _ in range(2)))  # noqa: E731
    first, one, two, held = new(), new(), new(), new()
    launch(first)
    torch.cuda.synchronize()
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    for s, out in zip(sides, (one, two)):
        with torch.cuda.stream(s):
            launch(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        launch(held)
    graph.replay()
    torch.cuda.synchronize()
    for out in (one, two, held):
        assert all(torch.equal(x, y) for x, y in zip(first, out))
    d["accept_u"].fill_(0.999)
    graph.replay()
    launch(first)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, held)) and int(status) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("drafts", ["drawn", "distinct", "fixed"])
def test_rows_cut_to_their_likeliest_tokens(dtype, drafts):
    """Most probabilities are exactly zero, as after a cut to the likeliest tokens, in the target and (elsewhere) in the draft."""
    for V in (40, 5003, 40000):
        c = make(23 + V, 20, 6, V, drafts, True, dtype, near=1.5)
        for name, keep in (("target", 0.02), ("target_prefix", 0.02), ("draft", 0.05), ("draft_prefix", 0.05)):
            if c[name] is None:
                continue
            x = c[name].double()
            border = x.quantile(1 - keep, dim=-1, keepdim=True) if V < 10000 else x.topk(int(keep * V), -1).values[..., -1:]
            x = torch.where(x >= border, x, 0)
            c[name] = (x / x.sum(-1, keepdim=True)).to(DT[dtype])
        check(c, 6)


@pytest.mark.parametrize("drafts", ["drawn", "fixed"])
def test_probabilities_below_the_normal_numbers(drafts):
    """A token of probability 2^-140 is one that can be drawn: by u' = 0 it is the first, and it is accepted by u = 0."""
    c = make(24, 4, 1, 5000, drafts, True)
    tiny = 2.0 ** -140
    c["target_prefix"][:, :7], c["target"][:, :, :7] = 0, 0
    c["target_prefix"][:, 3], c["target"][:, :, 3] = tiny, tiny
    c["tokens"][:2], c["tokens"][2:] = 3, 5
    c["accept_u"][:], c["sample_u"][:] = 0, 0
    path, n, nxt = check(c, 1)
    assert n.tolist() == [1, 1, 0, 0] and (nxt[:2] == 3).all()
    if drafts == "fixed":
        assert (nxt[2:] == 3).all()
    else:
        c["draft_prefix"][:, 3] = 0
        path, n, nxt = check(c, 1)
        assert n.tolist() == [1, 1, 0, 0] and (nxt[2:] == 3).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_drafts_that_are_no_probabilities(bad):
    """A draft's row with a NaN leaves nothing to draw from where a child was rejected against it; an infinity there takes all of its
    token; where the child was accepted the row is not looked at."""
    c = make(25, 2, 1, 3000, "drawn", True)
    c["draft_prefix"][:, 1234] = bad
    c["tokens"][:] = 77
    c["target_prefix"][0, 77], c["target_prefix"][1, 77] = 0.5, 0
    c["draft_prefix"][:, 77] = 0.25
    path, n, nxt = call(c, 1, status=BAD_PROBS if math.isnan(bad) else 0)
    assert n.tolist() == [1, 0] and int(nxt[0]) >= 0
    assert int(nxt[1]) == -1 if math.isnan(bad) else int(nxt[1]) not in (-1, 77, 1234)
