"""Attention of a tree of drafted tokens over the cache against its definition in 64 bits, at the sizes, masks and contents
where it can go wrong."""
import math

import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R
from tree_cases import make

pytestmark = pytest.mark.gpu
SENTINEL = 2.0 ** 100   # no result comes near it


def run(c, scale=None, cache=None, **kw):
    cache = cache or c.cache()
    out = torch.full_like(c.t["Q"], SENTINEL).to("cuda")
    lse = torch.full(c.t["Q"].shape[:4], SENTINEL, device="cuda")
    R.roco_tree_attend(cache, c.dev("Q"), c.dev("K_new"), c.dev("V_new"), c.dev("parent"), out,
                       nodes=torch.tensor(c.nodes, dtype=torch.int32, device="cuda"), lse_out=lse, scale=scale, **kw)
    torch.cuda.synchronize()
    return cache, out, lse


def check(c, scale=None, units=None):
    cache, out, lse = run(c, scale)
    scale = c.d ** -0.5 if scale is None else scale
    for b in range(c.S):
        N = c.nodes[b]
        assert bool((out[b, :, N:] == SENTINEL).all()) and bool((lse[b, :, N:] == SENTINEL).all())
        for g in range(c.G) if units is None else units:
            f = {k: c.t[k][b, g].double() for k in ("K", "V", "Q", "K_new", "V_new")}
            o, l, ob, lb = ref.tree_attend(f["K"], f["V"], c.live[b], f["Q"], f["K_new"], f["V_new"], c.t["parent"][b].tolist(),
                                           N, scale, low=c.dtype == "bf16")
            do = (out[b, g, :N].double().cpu() - o).abs()
            dl = (lse[b, g, :N].double().cpu() - l).abs()
            assert bool((do <= ob).all()), f"unit {b},{g}: out off by {float((do / ob).max())} of its bound"
            assert bool((dl <= lb).all()), f"unit {b},{g}: lse off by {float((dl / lb).max())} of its bound"
    assert R.roco_device_status(cache) == 0
    for k in ("K", "V", "s", "q", "n", "pos", "live", "t_next"):     # the cache stays as it was, bit for bit
        assert torch.equal(getattr(cache, k).view(torch.uint8), c.dev(k).view(torch.uint8)), k


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("B,T,group,live,nodes", [
    (1, 1, 1, [0, 1], [1, 1]),
    (5, 3, 2, [0, 5], [3, 0]),
    (63, 7, 1, [63, 17], [7, 5]),
    (127, 16, 1, [127, 1], [16, 9]),
    (128, 17, 1, [128, 128], [17, 1]),
    (129, 5, 3, [129, 128], [5, 5]),
    (300, 8, 4, [256, 299], [8, 7]),
    (515, 33, 1, [515, 385], [33, 20]),
    (700, 64, 1, [700, 640], [64, 63]),
    (640, 13, 5, [640, 511], [13, 12]),
    (400, 12, 16, [400, 399], [12, 3]),
    (1030, 40, 8, [1030, 1], [40, 39]),
])
def test_tree_attend(dtype, d, B, T, group, live, nodes):
    check(make(B * 31 + T, S=2, G=2, B=B, d=d, T=T, group=group, dtype=dtype, live=live, nodes=nodes))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", ["chain", "flat"])
def test_tree_shapes(dtype, shape):
    check(make(3, S=1, G=2, B=200, T=64, group=1, dtype=dtype, live=[133], shape=shape))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [(8, 1), (24, 4), (50, 8)])
def test_long_budget_few_units(dtype, rows):
    """The cached tokens of a unit divided among several CTAs."""
    T, group = rows
    check(make(11, S=2, G=1, B=8192, T=T, group=group, dtype=dtype, live=[8192, 4099], nodes=[T, T - 1]))


def test_many_units():
    c = make(12, S=3, G=300, B=260, T=6, live=[260, 259, 3], nodes=[6, 6, 2])
    check(c, units=[0, 1, 148, 299])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7])
def test_any_scale(dtype, scale):
    # (0.3 and 1.7 against keys a quarter as long keep the scores in the range that bf16 tests use elsewhere)
    check(make(5, S=1, G=2, B=150, T=9, dtype=dtype, live=[149], key_scale=0.25), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_maximum_moves_in_every_tile(dtype):
    """Keys that grow along the slots: every tile's scores are far above the ones before; then far below."""
    c = make(6, S=2, G=1, B=1024, T=16, dtype=dtype)
    grow = torch.linspace(0.1, 12.0, 1024)
    u = c.t["Q"].float().mean(dim=(2, 3), keepdim=False)
    u = u / u.norm(dim=-1, keepdim=True)
    ramp = torch.stack((grow, grow.flip(0)))[:, None, :, None]
    c.t["K"] = (c.t["K"].float() * 0.2 + ramp * 11.3 * u[:, :, None]).to(c.t["K"].dtype)
    c.t["Q"] = (c.t["Q"].float() * 0.1 + 2 * u[:, :, None, None]).to(c.t["Q"].dtype)
    check(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -3e38])
def test_other_branches_may_hold_anything(dtype, value):
    """Two branches from the prefix; the keys and values of one are NaN or infinite and must not reach the other."""
    T = 20
    c = make(7, S=1, G=2, B=140, T=T, dtype=dtype, live=[139])
    par = [-1 if i < 2 else i - 2 for i in range(T)]              # even and odd chains
    c.t["parent"][0] = torch.tensor(par, dtype=torch.int32)
    for f in ("K_new", "V_new"):
        c.t[f][:, :, 1::2] = value
    cache, out, lse = run(c)
    for g in range(c.G):
        f = {k: c.t[k][0, g].double() for k in ("K", "V", "Q", "K_new", "V_new")}
        o, l, ob, lb = ref.tree_attend(f["K"], f["V"], c.live[0], f["Q"], f["K_new"], f["V_new"], par, T, c.d ** -0.5,
                                       low=dtype == "bf16")
        assert bool(((out[0, g, ::2].double().cpu() - o[::2]).abs() <= ob[::2]).all())
        assert bool(((lse[0, g, ::2].double().cpu() - l[::2]).abs() <= lb[::2]).all())


def test_optional_arguments():
    c = make(8, S=2, G=2, B=90, T=6)
    _, out, lse = run(c)
    again = torch.zeros_like(out)
    R.roco_tree_attend(c.cache(), c.dev("Q"), c.dev("K_new"), c.dev("V_new"), c.dev("parent"), again)
    assert torch.equal(out, again)


def test_bad_node_counts_and_parents_are_reported():
    c = make(9, S=3, G=2, B=90, T=6, shape="chain")
    good = run(c)[1]
    c.nodes = [6, 7, -1]
    cache, out, _ = run(c)
    assert R.roco_device_status(cache) == 8
    assert torch.equal(out[0], good[0]) and bool((out[1:] == SENTINEL).all())
    c.nodes = [6, 6, 6]
    c.t["parent"][1] = torch.tensor([-1, 1, 1, 9, -2, 3], dtype=torch.int32)     # itself, later, below -1: the prefix
    cache, out, _ = run(c)
    assert R.roco_device_status(cache) == 8
    c.t["parent"][1] = torch.tensor([-1, -1, 1, -1, -1, 3], dtype=torch.int32)
    assert torch.equal(out, run(c)[1]) and torch.equal(out[0], good[0])
    c.t["live"][2] = 91
    cache, out, _ = run(c)
    assert R.roco_device_status(cache) == 2


def test_same_bits_every_time_and_on_another_stream():
    c = make(10, S=2, G=3, B=2100, T=10, group=2, live=[2100, 77])
    _, a, la = run(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _, b, lb = run(c)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_in_a_graph():
    """Captured with a workspace of its own and replayed on new queries and a new number of nodes."""
    c, c2 = (make(s, S=1, G=2, B=4100, T=8, group=2, live=[4100]) for s in (20, 21))
    cache = c.cache()
    ws = torch.empty(max(256, R.roco_tree_attend_workspace_bytes(cache, 8, 2)), dtype=torch.uint8, device="cuda")
    t = {k: c.dev(k) for k in ("Q", "K_new", "V_new", "parent")}
    nodes = torch.tensor([8], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(t["Q"]), torch.zeros(t["Q"].shape[:4], device="cuda")
    call = lambda: R.roco_tree_attend(cache, t["Q"], t["K_new"], t["V_new"], t["parent"], out, nodes=nodes, lse_out=lse,  # noqa: E731
                                      workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in t:
        t[k].copy_(c2.t[k])
    nodes.fill_(5)
    out.fill_(SENTINEL)
    g.replay()
    got = out.clone()
    out.fill_(SENTINEL)
    call()
    assert torch.equal(got, out) and bool((out[:, :, 5:] == SENTINEL).all()) and not bool((out[:, :, :5] == SENTINEL).any())
    assert math.isfinite(float(lse[:, :, :5].sum()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [2, 4, 8])
@pytest.mark.parametrize("live", [0, 1, 300])
@pytest.mark.parametrize("value", [float("nan"), -3e38])
def test_other_branches_may_hold_anything_however_many_rows(dtype, group, live, value):
    """40 to 64 and more rows, whose groups of columns share the drafted tokens; with and without cached tokens in front."""
    T = 20
    c = make(30 + group, S=1, G=2, B=300, T=T, group=group, dtype=dtype, live=[live])
    par = [-1 if i < 2 else i - 2 for i in range(T)]
    c.t["parent"][0] = torch.tensor(par, dtype=torch.int32)
    for f in ("K_new", "V_new"):
        c.t[f][:, :, 1::2] = value
    _, out, lse = run(c)
    for g in range(c.G):
        f = {k: c.t[k][0, g].double() for k in ("K", "V", "Q", "K_new", "V_new")}
        o, l, ob, lb = ref.tree_attend(f["K"], f["V"], c.live[0], f["Q"], f["K_new"], f["V_new"], par, T, c.d ** -0.5,
                                       low=dtype == "bf16")
        assert bool(((out[0, g, ::2].double().cpu() - o[::2]).abs() <= ob[::2]).all())
        assert bool(((lse[0, g, ::2].double().cpu() - l[::2]).abs() <= lb[::2]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", [(5, 1), (7, 3), (20, 2), (25, 5)])
@pytest.mark.parametrize("ranks", [2, 3, 4, 5, 6, 7, 8])
def test_every_number_of_ctas_that_share_a_unit(dtype, T, group, ranks):
    """Two to eight ranges on either path, of a full cache, one that ends inside the first range (the others are empty) and
    none."""
    B = ranks * (256 if dtype == "bf16" else 128) - 3
    check(make(40 + ranks, S=3, G=2, B=B, T=T, group=group, dtype=dtype, live=[B, 70, 0], nodes=[T, T - 1, T]))
