"""Attention of a tree of drafted tokens on values that a row does see: NaN and infinities have to come out, large finite
values must not turn into them, and a log-sum-exp is good to single precision in every row."""
import math

import pytest
import torch

import operator_reference as ref
from test_gpu_tree import run
from tree_cases import make

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
ROWS = [(8, 1), (8, 4), (10, 4), (24, 4), (40, 5)]      # nodes and heads: 8, 32, 40, 96 and 200 query rows


def defined(c, b, g):
    """(out, lse) of a unit from the formula, in 64 bits, whatever the values; what a row does not see takes no part."""
    N, live = c.nodes[b], c.live[b]
    f = {k: c.t[k][b, g].double() for k in ("K", "V", "Q", "K_new", "V_new")}
    k, v = torch.cat((f["K"][:live], f["K_new"][:N])), torch.cat((f["V"][:live], f["V_new"][:N]))
    sees = torch.cat((torch.ones(N, live, dtype=torch.bool), ref.ancestors(c.t["parent"][b].tolist()[:N])), 1)
    x = torch.where(sees[:, None], torch.einsum("thd,jd->thj", f["Q"][:N], k) * c.d ** -0.5, -INF)
    e = torch.exp(x - x.amax(-1, keepdim=True))
    out = torch.einsum("thj,jd->thd", e, torch.where(v.isnan(), 0, v)) / e.sum(-1, keepdim=True)
    return out, x.amax(-1) + torch.log(e.sum(-1))


def check_finiteness(c, low_bound=True):
    """Rows that come out NaN or infinite in the definition do so here, and the others are right."""
    _, out, lse = run(c)
    for g in range(c.G):
        o, l = defined(c, 0, g)
        got, gl = out[0, g, :c.nodes[0]].double().cpu(), lse[0, g, :c.nodes[0]].double().cpu()
        bad = ~o.isfinite().all(-1)
        assert bool((~got[bad].isfinite()).all()) and bool((~gl[bad].isfinite()).all()), (
            f"{int(got[bad].isfinite().all(-1).sum())} of {int(bad.sum())} rows lost what they see")
        assert bool(got[~bad].isfinite().all()) and bool(gl[~bad].isfinite().all())
        f = {k: c.t[k][0, g].double().nan_to_num(0, 0, 0) for k in ("K", "V", "Q", "K_new", "V_new")}
        ro, rl, ob, lb = ref.tree_attend(f["K"], f["V"], c.live[0], f["Q"], f["K_new"], f["V_new"], c.t["parent"][0].tolist(),
                                         c.nodes[0], c.d ** -0.5, low=c.dtype == "bf16")
        ok = ~bad
        assert bool(((got - ro).abs() <= ob)[ok].all()) and bool(((gl - rl).abs() <= lb)[ok].all())
    return bad


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("live", [0, 300])
def test_nan_in_a_query_stays_in_its_row(dtype, T, group, live):
    c = make(3 + T, S=1, G=1, B=300, T=T, group=group, dtype=dtype, live=[live])
    flat = c.t["Q"].reshape(1, 1, T * group, c.d)
    rows = [0, 2, 5, T * group - 1]
    flat[0, 0, rows, 7] = NAN
    bad = check_finiteness(c)
    assert bad.flatten().nonzero().flatten().tolist() == rows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("value", [NAN, INF])
@pytest.mark.parametrize("slot", [0, 130, 299])
def test_a_cached_key_that_is_not_finite_reaches_every_row(dtype, T, group, value, slot):
    """NaN in one component of a key, and an infinite score (all queries positive there)."""
    c = make(5 + T, S=1, G=1, B=300, T=T, group=group, dtype=dtype)
    c.t["K"][0, 0, slot, 3] = value
    c.t["Q"][..., 3] = c.t["Q"][..., 3].abs() + 0.5
    bad = check_finiteness(c)
    assert bool(bad.all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("live", [0, 200])
@pytest.mark.parametrize("value", [NAN, INF])
def test_a_drafted_key_that_is_not_finite_reaches_the_rows_that_see_it(dtype, T, group, live, value):
    c = make(7 + T, S=1, G=1, B=300, T=T, group=group, dtype=dtype, live=[live])
    c.t["K_new"][0, 0, 2, 3] = value
    c.t["Q"][..., 3] = c.t["Q"][..., 3].abs() + 0.5
    _, out, lse = run(c)
    sees = ref.ancestors(c.t["parent"][0].tolist())[:, 2]
    assert bool(out[0, 0][sees].isnan().all()) and bool((~lse[0, 0][sees].isfinite()).all())
    assert bool(out[0, 0][~sees].isfinite().all()) and bool(lse[0, 0][~sees].isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("live", [1, 2, 300])
def test_keys_of_score_minus_infinity_take_no_part(dtype, T, group, live):
    """The first cached key and others at minus infinity for every row: as if they were not there."""
    c = make(9 + T, S=1, G=1, B=300, T=T, group=group, dtype=dtype, live=[live])
    c.t["Q"][..., 3] = c.t["Q"][..., 3].abs() + 0.5
    gone = torch.arange(0, live, 2)
    c.t["K"][0, 0, gone, 3] = -INF
    _, out, lse = run(c)
    keep = torch.arange(1, live, 2)
    k, v = c.t["K"][0, 0, keep].double(), c.t["V"][0, 0, keep].double()
    f = {n: c.t[n][0, 0].double() for n in ("Q", "K_new", "V_new")}
    o, l, ob, lb = ref.tree_attend(k, v, len(keep), f["Q"], f["K_new"], f["V_new"], c.t["parent"][0].tolist(), T, c.d ** -0.5,
                                   low=dtype == "bf16")
    assert bool(((out[0, 0].double().cpu() - o).abs() <= ob).all()) and bool(((lse[0, 0].double().cpu() - l).abs() <= lb).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("live", [40, 300, 2000])
@pytest.mark.parametrize("bits", [10, 31, 50, 90])
def test_large_values(dtype, T, group, live, bits):
    """Values up to 2^80 behind a first cached key whose score lies 10 to 90 binary orders below the others': the definition is
    a mean of the values and stays finite.  (The second product's terms are far from the end of fp32 in the bound's
    arithmetic too: it scales with the values.)"""
    c = make(11 + T, S=1, G=1, B=2000, T=T, group=group, dtype=dtype, live=[live])
    big = 2.0 ** 76
    c.t["V"], c.t["V_new"] = c.t["V"] * big, c.t["V_new"] * big
    assert float(c.t["V"][0, 0, :live].abs().max()) < 2.0 ** 80 and float(c.t["V_new"].abs().max()) < 2.0 ** 80
    c.t["Q"][..., 5] = 4.0
    c.t["K"][..., 5] = 0.0
    c.t["K"][0, 0, 0, 5] = -bits * math.log(2) * math.sqrt(c.d) / 4
    _, out, lse = run(c)
    f = {n: c.t[n][0, 0].double() for n in ("K", "V", "Q", "K_new", "V_new")}
    o, l, ob, lb = ref.tree_attend(f["K"], f["V"], live, f["Q"], f["K_new"], f["V_new"], c.t["parent"][0].tolist(), T, c.d ** -0.5,
                                   low=dtype == "bf16")
    assert bool(out[0, 0].isfinite().all())
    assert bool(((out[0, 0].double().cpu() - o).abs() <= ob).all()) and bool(((lse[0, 0].double().cpu() - l).abs() <= lb).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
def test_the_log_sum_exp_is_good_to_single_precision(dtype, T, group):
    """Two cached keys of scores 0 and x (many x, one to a unit), the same for every row, and a drafted token far below both:
    lse = log(1 + e^x), x exact in the inputs' type.  Where an error can come from, u = 2^-24: the score times its factor (the
    factor is rounded, the product is: 2 u |x|), its distance to the reference (u |x|), both exponentials (2^-22 of each), the
    sum of two (u), and of the final formula the reference times log 2 and the sum's logarithm (2^-22 of it, rounded constants
    and products: 4 u |lse|).  The sum's error counts as it is in the logarithm."""
    G = 64
    c = make(13, S=1, G=G, B=4, T=T, group=group, dtype=dtype, live=[2], d=64, shape="flat")
    for n in ("K", "Q", "K_new"):
        c.t[n][:] = 0
    c.t["Q"][..., 0] = 1.0
    x = (1.0 + torch.arange(G) / 128.0)
    c.t["K"][0, :, 1, 0] = 8 * x.to(c.t["K"].dtype)       # (scale 1/8)
    assert torch.equal(c.t["K"][0, :, 1, 0].double(), 8 * x.double())
    c.t["K_new"][..., 0] = -8 * 64.0                      # e^-64: nothing
    _, _, lse = run(c)
    x = x.double()
    want = torch.log1p(torch.exp(x))
    u = 2.0 ** -24
    bound = 3 * u * x + 2.0 ** -22 + u + 4 * u * want + 2.0 ** -22 * want
    off = (lse[0].double().cpu() - want[:, None, None]).abs()
    assert bool((off <= bound[:, None, None]).all()), f"off by {float((off / bound[:, None, None]).max())} of its bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,group", ROWS)
@pytest.mark.parametrize("B,live,far", [(300, 1, 1), (300, 200, 200), (700, 700, 300), (700, 700, 690), (8192, 8000, 5000)])
def test_a_range_of_cached_keys_without_a_finite_score(dtype, T, group, B, live, far):
    """The first `far` cached keys at scores below fp32's range (finite keys and queries), all others and the drafted ones 200
    binary orders below zero: what is left is an ordinary softmax."""
    c = make(15 + T, S=1, G=1, B=B, T=T, group=group, dtype=dtype, live=[live])
    c.t["Q"][..., 3] = 200.0
    for f in ("K", "K_new"):
        c.t[f][..., 3] = -200 * math.log(2) * math.sqrt(c.d) / 200
    c.t["K"][0, 0, :far, 3] = -3e38
    _, out, lse = run(c)
    k, v = c.t["K"][0, 0, far:live].double(), c.t["V"][0, 0, far:live].double()
    f = {n: c.t[n][0, 0].double() for n in ("Q", "K_new", "V_new")}
    o, l, ob, lb = ref.tree_attend(k, v, live - far, f["Q"], f["K_new"], f["V_new"], c.t["parent"][0].tolist(), T, c.d ** -0.5,
                                   low=dtype == "bf16")
    assert bool(((out[0, 0].double().cpu() - o).abs() <= ob).all()) and bool(((lse[0, 0].double().cpu() - l).abs() <= lb).all())
