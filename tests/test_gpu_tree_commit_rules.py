"""Commit of an accepted path: the eviction rule on exact ties at different counts, paths through padding, and what a commit of
one token has in common with a decode step."""
import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R
from test_gpu_tree_commit import check
from tree_cases import CACHE_FIELDS, make

pytestmark = pytest.mark.gpu


def commit_without_mass(c, a, r, mode=R.ROCO_SCOPE_EXCLUDE_TOP_R):
    """Commits nodes 0 .. a - 1 of a chain with a log-sum-exp at which every probability is exactly zero: Acc and Acc^square stay
    as they are and Count grows by a."""
    cache = c.cache()
    q = c.dev("Q")
    lse = torch.full(c.t["Q"].shape[:4], 1000.0, device="cuda")
    ev, ep = (torch.zeros(c.S, c.G, a, dtype=torch.int32, device="cuda") for _ in range(2))
    R.roco_tree_commit(cache, q, c.dev("K_new"), c.dev("V_new"), lse, c.dev("parent"),
                       torch.arange(a, dtype=torch.int32, device="cuda").expand(c.S, a).contiguous(),
                       torch.full((c.S,), a, dtype=torch.int32, device="cuda"), r, ev, evicted_pos=ep, scope_mode=mode)
    assert R.roco_device_status(cache) == 0
    return ep.sort(-1)[0].cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,B", [(2, 400), (2, 1500), (1200, 160)])
@pytest.mark.parametrize("a", [1, 3, 16])
@pytest.mark.parametrize("den", [1, 3, 10, 49])
def test_equal_means_at_different_counts_fall_to_the_lowest_position(dtype, G, B, a, den):
    """Count = den m and Acc = m 2^-10, so every mean is 2^-10 / den, whatever the count, in fp32 or (3, 10, 49) not."""
    c = make(21, S=1, G=G, B=B, d=64, T=16, dtype=dtype, shape="chain")
    m = c.t["n"] + a                        # all different within a unit
    c.t["n"] = den * m - a                  # Count becomes den m
    c.t["s"] = m.float() * 2.0 ** -10
    c.t["q"] = m.float() * 2.0 ** -19
    got = commit_without_mass(c, a, 0)
    assert torch.equal(got, c.t["pos"].sort(-1)[0][..., :a])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,B", [(2, 400), (2, 1500), (1200, 160)])
@pytest.mark.parametrize("a", [1, 3, 16])
@pytest.mark.parametrize("r", [2, 60])
@pytest.mark.parametrize("mode", [R.ROCO_SCOPE_EXCLUDE_TOP_R, R.ROCO_SCOPE_LOWEST_R])
def test_equal_variances_at_different_counts_fall_to_the_lowest_position(dtype, G, B, a, r, mode):
    """Acc^square = Count (c^2 + 2^-20) with the mean c = 2^-10 at the low positions and 2^-11 at the others: every variance is 2^-20
    exactly, the scope is the lowest positions, and in it the lower mean leaves first, the lowest position of those."""
    c = make(22, S=1, G=G, B=B, d=64, T=16, dtype=dtype, shape="chain")
    n = (c.t["n"] + a).float()
    order = c.t["pos"].argsort(-1).argsort(-1)          # 0: the lowest position
    half = order >= B // 2
    c.t["s"] = n * torch.where(half, 2.0 ** -11, 2.0 ** -10)
    c.t["q"] = n * torch.where(half, 5 * 2.0 ** -22, 2.0 ** -19)
    got = commit_without_mass(c, a, r, mode)
    pos = c.t["pos"].sort(-1)[0]
    left, want = list(range(B)), []
    for _ in range(a):                                  # by rank of position
        m = max(1, min(len(left), r if mode == R.ROCO_SCOPE_LOWEST_R else len(left) - r))
        v = min(left[:m], key=lambda j: (j < B // 2, j))
        want.append(v)
        left.remove(v)
    assert torch.equal(got, pos[..., sorted(want)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_path_through_padding_is_refused(dtype):
    """Sequences of 6, 3 and 0 drafted nodes whose padding continues the chain, and whose log-sum-exps behind the last node are
    what happened to be there."""
    c = make(23, S=3, G=2, B=60, T=6, dtype=dtype, shape="chain", nodes=[6, 3, 0])
    cache, before = c.cache(), c.cache()
    q = c.dev("Q")
    nodes = torch.tensor(c.nodes, dtype=torch.int32, device="cuda")
    lse = torch.zeros(q.shape[:4], device="cuda")
    args = (q, c.dev("K_new"), c.dev("V_new"), c.dev("parent"))
    R.roco_tree_attend(cache, *args, torch.zeros_like(q), nodes=nodes, lse_out=lse)
    ev = torch.zeros(3, 2, 4, dtype=torch.int32, device="cuda")
    path = torch.arange(4, dtype=torch.int32, device="cuda").expand(3, 4).contiguous()
    R.roco_tree_commit(cache, *args[:3], lse, args[3], path, torch.tensor([4, 4, 1], dtype=torch.int32, device="cuda"), 5, ev,
                       nodes=nodes)
    assert R.roco_device_status(cache) == 8
    for f in CACHE_FIELDS:
        x, y = getattr(cache, f), getattr(before, f)
        assert torch.equal(x[1:].view(torch.uint8), y[1:].view(torch.uint8)), f
    assert bool((ev[0] >= 0).all()) and bool((ev[1:] == -1).all())
    # the nodes that there are, and a node count that is none
    for n, good in (([6, 3, 0], True), ([7, 3, 0], False), ([-1, 3, 0], False)):
        cache = c.cache()
        R.roco_tree_commit(cache, *args[:3], lse, args[3], path, torch.tensor([4, 3, 0], dtype=torch.int32, device="cuda"), 5, ev,
                           nodes=torch.tensor(n, dtype=torch.int32, device="cuda"))
        assert R.roco_device_status(cache) == (0 if good else 8)
        assert (cache.t_next - before.t_next)[:, 0].tolist() == [4 if good else 0, 3, 0]
        assert bool((ev[0] >= 0).all()) == good


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_with_room_a_commit_of_one_token_is_a_decode_step(dtype, d):
    """Where nothing is evicted, a tree of one node that is attended and committed leaves what roco_decode_step leaves (EVICT_FIRST:
    the query sees its own key): the same output, log-sum-exp and insertion, and statistics that differ by roundings."""
    S, G, B = 2, 3, 200
    c = make(24, S=S, G=G, B=B, T=1, d=d, dtype=dtype, live=[150, 199], junk=0.0)
    tree, step = c.cache(), c.cache()
    q, k, v = c.dev("Q"), c.dev("K_new"), c.dev("V_new")
    out, lse = torch.zeros_like(q), torch.zeros(S, G, 1, 1, device="cuda")
    R.roco_tree_attend(tree, q, k, v, c.dev("parent"), out, lse_out=lse)
    one, zero = (f((S, 1), dtype=torch.int32, device="cuda") for f in (torch.ones, torch.zeros))
    R.roco_tree_commit(tree, q, k, v, lse, c.dev("parent"), zero, one[:, 0].contiguous(), 20,
                       torch.zeros(S, G, 1, dtype=torch.int32, device="cuda"))
    out2 = torch.zeros(S, G, d, dtype=q.dtype, device="cuda")
    R.roco_decode_step(step, q.reshape(S, G, d), k.reshape(S, G, d), v.reshape(S, G, d), 20, out2,
                       torch.zeros(S, G, dtype=torch.int32, device="cuda"), step_order=R.ROCO_EVICT_FIRST)
    for f in ("K", "V", "n", "pos", "live", "t_next"):
        a, b = getattr(tree, f), getattr(step, f)
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f
    for b in range(S):
        n = c.live[b] + 1
        for g in range(G):
            st = {f: c.t[f][b, g].clone().double() if f in ("K", "V", "s", "q") else c.t[f][b, g].clone() for f in CACHE_FIELDS}
            st["live"], st["t_next"] = c.live[b], int(st["t_next"])
            x = {f: c.t[f][b, g].double() for f in ("K", "V", "Q", "K_new", "V_new")}
            o, l, ob, lb = ref.tree_attend(x["K"], x["V"], c.live[b], x["Q"], x["K_new"], x["V_new"], [-1], 1, d ** -0.5,
                                           low=dtype == "bf16")
            _, _, _, sb, qb = ref.tree_commit(st, x["Q"], x["K_new"], x["V_new"], l, [0], 20, False, d ** -0.5)
            # the log-sum-exp that each took carries its own error into the probabilities (at most 1 each)
            sb, qb = sb[:n] + 1.01 * float(lb), qb[:n] + 2.02 * float(lb)
            for cache in (tree, step):
                assert bool(((cache.s[b, g, :n].double().cpu() - st["s"][:n]).abs() <= sb).all())
                assert bool(((cache.q[b, g, :n].double().cpu() - st["q"][:n]).abs() <= qb).all())
            for y in (out[b, g, 0, 0], out2[b, g]):
                assert bool(((y.double().cpu() - o[0, 0]).abs() <= ob[0, 0]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [3, 200, 1300])
@pytest.mark.parametrize("mode,r", [(R.ROCO_SCOPE_EXCLUDE_TOP_R, 2), (R.ROCO_SCOPE_EXCLUDE_TOP_R, 70), (R.ROCO_SCOPE_EXCLUDE_TOP_R, 200),
                                    (R.ROCO_SCOPE_LOWEST_R, 30)])
def test_every_number_of_threads_for_a_unit(dtype, G, mode, r):
    """Few units, more than a B200 has SMs, more than eight to an SM; scopes that leave out two tokens, 70, most."""
    c = make(25 + r, S=1, G=G, B=230, d=64, T=4, dtype=dtype, shape="chain", live=[229])
    check(c, [[0, 1, 2, 3]], 4, r, mode)
