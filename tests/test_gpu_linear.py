"""Linear attention with a decay for each head, prompts and single tokens, against the recurrence in 64 bits."""
import math

import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
SENTINEL = 2.0 ** 100   # no result comes near it
DECAYS = [0.0, -1e-4, -0.01, -0.7, -20.0, -math.inf]


def inputs(seed, S, G, L, d, dtype, zero_state=False):
    g = torch.Generator()
    g.manual_seed(seed)
    q, k, v = (torch.randn(S, G, L, d, generator=g).to(DT[dtype]) for _ in range(3))
    state = torch.zeros(S, G, d, d) if zero_state else torch.randn(S, G, d, d, generator=g)
    return q, k, v, state


def make_state(state, log_decay, dtype):
    return R.LinearState.wrap(state.to("cuda").clone(), torch.tensor(log_decay, dtype=torch.float32, device="cuda"), DT[dtype],
                              torch.zeros(1, dtype=torch.int32, device="cuda"))


def close(got, want, bound, what, rel=None):
    d = (got.double().cpu() - want).abs()
    assert bool((d <= bound).all()), f"{what} off by {float((d / bound).max())} of its bound"
    if rel is not None and want.shape[0] >= 16:
        off = float((got.double().cpu() - want).norm()) / max(1e-30, float(want.norm()))
        assert off <= rel, f"{what}: relative error {off}"


# In the 2-norm: three independent roundings to bf16 (scores, state, result) of at most 2^-8 each; in fp32 the rounding of
# the state at each of the tokens it lasts, which a random sign keeps below sqrt(L) 2^-24 times a small factor.  Both are
# relative to the terms of the sums, so they hold for the norm over many rows only: a lone row is scale (q.k) v, and with
# 128 products of size one in q.k the error of up to 128 * 128 * 2^-24 = 1e-3 stands against a sum that may be anywhere near
# zero.  The bound of every single element, above, counts that and holds for all.
REL = {"bf16": 3 * 2.0 ** -8, "f32": 4e-6}


def check_prompt(q, k, v, state, log_decay, lens, dtype, scale=None, pieces=None):
    S, G, L, d = q.shape
    st = make_state(state, log_decay, dtype)
    out = torch.full_like(q, SENTINEL).to("cuda")
    qd, kd, vd = q.clone(), k.clone(), v.clone()
    for b in range(S):     # what lies behind the last token must not matter
        for t in (qd, kd, vd):
            t[b, :, lens[b]:] = float("nan")
    R.roco_linear_prefill(st, qd.to("cuda"), kd.to("cuda"), vd.to("cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                          out, scale=scale)
    torch.cuda.synchronize()
    scale = d ** -0.5 if scale is None else scale
    for b in range(S):
        assert bool((out[b, :, lens[b]:] == SENTINEL).all())
        for g in range(G):
            n = lens[b]
            o, s, ob, sb = ref.linear(state[b, g].double(), float(torch.tensor(log_decay[g])), q[b, g, :n].double(),
                                      k[b, g, :n].double(), v[b, g, :n].double(), scale, low=dtype == "bf16")
            close(out[b, g, :n], o, ob, f"out {b},{g} (decay {log_decay[g]})", REL[dtype])
            close(st.state[b, g], s, sb, f"state {b},{g} (decay {log_decay[g]})", 1e-5)
    assert R.roco_linear_device_status(st) == 0
    return st, out


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("L,lens", [(1, [1, 0]), (2, [2, 1]), (63, [63, 17]), (64, [64, 33]), (127, [127, 64]), (128, [128, 127]),
                                    (129, [129, 128]), (255, [255, 130]), (300, [300, 257]), (513, [513, 1])])
def test_prompt(dtype, d, L, lens):
    q, k, v, state = inputs(L * 3 + d, 2, len(DECAYS), L, d, dtype)
    check_prompt(q, k, v, state, DECAYS, lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_prompt_few_units(dtype):
    """The prompt of a unit divided among several CTAs."""
    q, k, v, state = inputs(5, 2, 2, 4500, 128, dtype)
    check_prompt(q, k, v, state, [-2.0 ** -12, -0.02], [4500, 2111], dtype)


def test_many_units():
    q, k, v, state = inputs(6, 3, 110, 140, 128, "bf16")
    check_prompt(q, k, v, state, [-0.001 * (g + 1) for g in range(110)], [140, 139, 9], "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.5, 1.0])
def test_any_scale(dtype, scale):
    q, k, v, state = inputs(7, 1, 2, 150, 128, dtype)
    check_prompt(q, k, v, state, [-0.1, -0.003], [150], dtype, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_and_small_values(dtype):
    """Keys and values over many binary orders: products are formed at full range, and small tokens stay beside large ones
    as far as the result's type goes."""
    q, k, v, state = inputs(8, 1, 2, 200, 128, dtype)
    k[:, :, ::3] *= 2.0 ** 20
    v[:, :, 1::5] *= 2.0 ** -20
    check_prompt(q, k, v, state, [-0.05, 0.0], [200], dtype)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
def test_step(dtype, d):
    S, G = 3, len(DECAYS)
    q, k, v, state = inputs(20 + d, S, G, 1, d, dtype)
    for active in (None, [1, 0, 5]):
        st = make_state(state, DECAYS, dtype)
        out = torch.full((S, G, d), SENTINEL, dtype=DT[dtype], device="cuda")
        R.roco_linear_step(st, *(t[:, :, 0].contiguous().to("cuda") for t in (q, k, v)), out,
                           active=None if active is None else torch.tensor(active, dtype=torch.int32, device="cuda"))
        for b in range(S):
            for g in range(G):
                if active and not active[b]:
                    assert torch.equal(st.state[b, g].cpu(), state[b, g]) and bool((out[b, g] == SENTINEL).all())
                    continue
                o, s, ob, sb = ref.linear(state[b, g].double(), float(torch.tensor(DECAYS[g])), q[b, g].double(), k[b, g].double(),
                                          v[b, g].double(), d ** -0.5)
                if dtype == "bf16":
                    ob = ob + ref.U16 * o.abs()
                close(out[b, g], o[0], ob[0], f"out {b},{g}")
                close(st.state[b, g], s, sb, f"state {b},{g}")
        assert R.roco_linear_device_status(st) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_in_pieces_then_tokens(dtype):
    """As a program uses them: a prompt in three pieces of different lengths per sequence, then single tokens while one
    sequence has already ended; the whole against one recurrence."""
    S, G, d, L, steps = 2, 3, 128, 400, 5
    log_decay = [-0.004, -0.1, 0.0]
    q, k, v, state = inputs(30, S, G, L + steps, d, dtype, zero_state=True)
    st = make_state(state, log_decay, dtype)
    total = [L, 277]
    cuts = [[0, 130, 131, L], [0, 77, 200, 277]]
    outs = [[[] for _ in range(G)] for _ in range(S)]
    for piece in range(3):
        n = [cuts[b][piece + 1] - cuts[b][piece] for b in range(S)]
        Lm = max(n)
        part = []
        for t in (q, k, v):
            x = torch.full((S, G, Lm, d), float("nan"), dtype=t.dtype)
            for b in range(S):
                x[b, :, :n[b]] = t[b, :, cuts[b][piece]:cuts[b][piece + 1]]
            part.append(x.to("cuda"))
        out = torch.zeros_like(part[0])
        R.roco_linear_prefill(st, *part, torch.tensor(n, dtype=torch.int32, device="cuda"), out)
        for b in range(S):
            for g in range(G):
                outs[b][g].append(out[b, g, :n[b]].cpu())
    for i in range(steps):
        active = [1, int(i < 2)]
        tok = [torch.stack([t[b, :, total[b] + i] for b in range(S)]).to("cuda") for t in (q, k, v)]
        out = torch.zeros_like(tok[0])
        R.roco_linear_step(st, *tok, out, active=torch.tensor(active, dtype=torch.int32, device="cuda"))
        for b in range(S):
            if active[b]:
                for g in range(G):
                    outs[b][g].append(out[b, g][None].cpu())
    for b in range(S):
        n = total[b] + (steps if b == 0 else 2)
        for g in range(G):
            o, s, ob, sb = ref.linear(state[b, g].double(), log_decay[g], q[b, g, :n].double(), k[b, g, :n].double(),
                                      v[b, g, :n].double(), d ** -0.5, low=dtype == "bf16")
            close(torch.cat(outs[b][g]), o, ob, f"out {b},{g}", REL[dtype])
            close(st.state[b, g], s, sb, f"state {b},{g}", 1e-5)


def test_bad_lengths_are_reported_and_change_nothing():
    q, k, v, state = inputs(40, 3, 2, 70, 128, "bf16")
    st = make_state(state, [-0.1, -0.2], "bf16")
    out = torch.full_like(q, SENTINEL).to("cuda")
    R.roco_linear_prefill(st, q.to("cuda"), k.to("cuda"), v.to("cuda"), torch.tensor([71, -1, 70], dtype=torch.int32, device="cuda"),
                          out)
    assert R.roco_linear_device_status(st) == 16
    assert torch.equal(st.state[:2].cpu(), state[:2]) and bool((out[:2] == SENTINEL).all())
    assert not torch.equal(st.state[2].cpu(), state[2]) and not bool((out[2] == SENTINEL).any())


@pytest.mark.parametrize("L", [260, 4000])
def test_same_bits_every_time_on_another_stream_and_in_a_graph(L):
    q, k, v, state = (t.to("cuda") for t in inputs(41, 1, 3, L, 128, "bf16"))
    lens = torch.tensor([L - 3], dtype=torch.int32, device="cuda")
    decay = [-0.01, -0.001, -0.3]

    def fresh():
        return make_state(state, decay, "bf16"), torch.zeros_like(q)
    a, oa = fresh()
    R.roco_linear_prefill(a, q, k, v, lens, oa)
    b, ob = fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        R.roco_linear_prefill(b, q, k, v, lens, ob)
    torch.cuda.synchronize()
    assert torch.equal(oa, ob) and torch.equal(a.state, b.state)
    c, oc = fresh()
    ws = torch.empty(max(256, R.roco_linear_prefill_workspace_bytes(c, L)), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.roco_linear_prefill(c, q, k, v, lens, oc, workspace=ws)
    assert torch.equal(c.state, state)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(oa, oc) and torch.equal(a.state, c.state)
    lens.fill_(100)
    c.state.copy_(state)
    oc.zero_()
    g.replay()
    torch.cuda.synchronize()
    d, od = fresh()
    R.roco_linear_prefill(d, q, k, v, lens, od)
    assert torch.equal(od, oc) and torch.equal(d.state, c.state) and not bool(oc[:, :, 100:].any())


def test_step_in_a_graph():
    q, k, v, state = (t.to("cuda") for t in inputs(42, 2, 2, 1, 64, "f32"))
    tok = [t[:, :, 0].contiguous() for t in (q, k, v)]
    a, b = (make_state(state, [-0.1, -0.2], "f32") for _ in range(2))
    out = torch.zeros_like(tok[0])
    for _ in range(3):
        R.roco_linear_step(a, *tok, out)
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.roco_linear_step(b, *tok, out)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(want, out) and torch.equal(a.state, b.state)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_at_once(dtype):
    """Divided prompts of two states on two streams, bit for bit as one after the other."""
    data = [[t.to("cuda") for t in inputs(50 + i, 1, 3, 2000 + 300 * i, 128, dtype)] for i in range(2)]
    lens = [torch.tensor([1990 + 300 * i], dtype=torch.int32, device="cuda") for i in range(2)]
    decay = [-0.01, -0.001, -0.3]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for at_once in (False, True):
        st, out = [make_state(d[3], decay, dtype) for d in data], [torch.zeros_like(d[0]) for d in data]
        torch.cuda.synchronize()
        for _ in range(3):
            for i in range(2):
                with torch.cuda.stream(streams[i if at_once else 0]):
                    R.roco_linear_prefill(st[i], *data[i][:3], lens[i], out[i])
        torch.cuda.synchronize()
        got.append([s.state for s in st] + out)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_many_steps_do_not_drift():
    """A decay near one, keys with one component: component 0 of the state is the sum of g^j, whose relative error stays below
    that of its roundings (each at most 2^-24 of the state, decaying with it), n 2^-24 at most; a decay rounded to fp32 alone
    could use that up.  A third of the bound is asserted, which random signs keep by far: the root of n terms."""
    n, d = 2000, 64
    tok = [torch.zeros(1, 4, d, device="cuda") for _ in range(3)]
    for t in tok:
        t[..., 0] = 1
    decay = [-1e-5, -3e-5, -1.7e-4, -9.1e-4]
    st = make_state(torch.zeros(1, 4, d, d), decay, "f32")
    out = torch.zeros_like(tok[0])
    for _ in range(n):
        R.roco_linear_step(st, *tok, out, scale=1.0)
    for g in range(4):
        x = float(torch.tensor(decay[g]))
        want = math.expm1(n * x) / math.expm1(x)
        assert abs(float(st.state[0, g, 0, 0]) - want) <= n / 3 * 2.0 ** -24 * want
        assert abs(float(out[0, g, 0]) - want) <= n / 3 * 2.0 ** -24 * want
