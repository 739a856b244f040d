"""Norm and rotation of a layer's heads against the 64-bit reference."""
import math

import pytest
import torch

import paper_2402_06262_b200 as R
import decoding_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def run(seed, S=2, N=3, G=2, group=2, d=128, rot=None, adjacent=False, axes=1, norm="qk", dtype="bf16", lens=None, start=None,
        positions=None, axis=None, rows="fused", scale=1.0, theta=1e4, skip=(), freq=None, x=None):
    """One call and its check: every row against the reference, everything behind lens as it was, the status."""
    g, dt = gen(seed), DT[dtype]
    rot = d if rot is None else rot
    H = G * (group + 2)
    if x is None:
        x = (torch.randn(S, N, H, d, generator=g) * scale).to(dt)
    ls = [N] * S if lens is None else lens
    for b in range(S):
        x[b, ls[b]:] = math.nan
    cut = [G * group, G, G]
    if rows == "fused":            # rows of one product
        dev = x.cuda().reshape(S, N, H * d).split([c * d for c in cut], dim=2)
        dev = [t.reshape(S, N, -1, d) if t.is_contiguous() else t.unflatten(2, (-1, d)) for t in dev]
    elif rows == "apart":
        dev = [t.contiguous().cuda() for t in x.split(cut, dim=2)]
    elif rows == "padded":         # wider rows, sequences behind one another with a gap
        wide = torch.full((S, N + 2, H + 3, d), math.nan, dtype=dt, device="cuda")
        wide[:, :N, :H] = x.cuda()
        dev = wide[:, :N, :H].split(cut, dim=2)
    else:                          # tokens first
        dev = x.transpose(0, 1).contiguous().cuda().transpose(0, 1).split(cut, dim=2)
    if freq is None:
        freq = torch.tensor([theta ** (-2 * i / max(1, rot)) for i in range(rot // 2)], dtype=torch.float32)
    w = {n: (1 + 0.3 * torch.randn(d, generator=g)) if n in norm else None for n in "qk"}
    rotary = R.Rotary(d, freq, pairing=R.ROCO_PAIR_ADJACENT if adjacent else R.ROCO_PAIR_HALVES, axes=axes, axis=axis, q_weight=w["q"],
                      k_weight=w["k"], eps=1e-5)
    junk = -7.0
    Q = torch.full((S, G, N, group, d), junk, dtype=dt, device="cuda")
    K, V = (torch.full((S, G, N, d), junk, dtype=dt, device="cuda") for _ in range(2))
    opt = lambda t: None if t is None else torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    st = None
    if start is not None:          # a column of a wider table, as t_next of a cache is
        st = torch.tensor(start, dtype=torch.int32, device="cuda")[:, None].expand(S, G + 1).contiguous()[:, 0]
    R.roco_norm_rotate(rotary, dev[0], None if "k" in skip else dev[1], None if "v" in skip else dev[2], Q, None if "k" in skip else K,
                       None if "v" in skip else V, lens=opt(lens), start=st, positions=None if positions is None else positions.cuda())
    assert R.roco_rotary_device_status(rotary) == 0
    at = torch.arange(N)[None, :, None].expand(S, N, axes) if positions is None else positions.reshape(S, N, axes)
    eps = float(torch.tensor(1e-5, dtype=torch.float32))
    xq, xk, xv = x.split(cut, dim=2)
    for name, out, src, per, weight in (("Q", Q, xq, group, w["q"]), ("K", K, xk, 1, w["k"])):
        got = out.cpu().reshape(S, G, N, per, d)
        if name == "K" and "k" in skip:
            assert bool((got == junk).all())
            continue
        y, bound = ref.norm_rotate(src, per, None if weight is None else weight.double(), eps, rot, adjacent, freq.double(),
                                   [0] * (rot // 2) if axis is None else axis, [0] * S if start is None else start, at, ls)
        for b in range(S):
            assert bool((got[b, :, ls[b]:] == junk).all()), name
            err = (got[b, :, :ls[b]].double() - y[b, :, :ls[b]]).abs()
            allowed = bound[b, :, :ls[b]] + (y[b, :, :ls[b]].abs() + bound[b, :, :ls[b]]) * (ref.U16 if dtype == "bf16" else ref.U32)
            assert bool((err <= allowed).all()), f"{name}[{b}]: {float((err / allowed).max())} of the bound"
    got = V.cpu()
    for b in range(S):
        if "v" not in skip:
            assert torch.equal(got[b, :, :ls[b]], xv[b, :ls[b]].transpose(0, 1))
        assert bool((got[b, :, 0 if "v" in skip else ls[b]:] == junk).all())
    return Q, K, V


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("norm", ["qk", "", "q"])
def test_pairs_and_norms(dtype, d, adjacent, rot, norm):
    if rot <= d:
        run(rot + d, d=d, rot=rot, adjacent=adjacent, norm=norm, dtype=dtype, S=2, N=5, G=2, group=2, lens=[5, 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,N,G,group,lens", [(1, 1, 1, 1, None), (5, 1, 3, 1, None), (1, 33, 1, 5, None), (3, 17, 4, 4, [17, 0, 9]),
                                              (2, 40, 3, 16, [1, 40]), (40, 1, 2, 8, None), (1, 130, 2, 1, [129])])
@pytest.mark.parametrize("rows", ["fused", "apart", "padded", "tokens"])
def test_sizes_and_strides(dtype, S, N, G, group, lens, rows):
    run(7, S=S, N=N, G=G, group=group, d=64, dtype=dtype, lens=lens, rows=rows)


def test_more_heads_than_one_cta_takes_and_more_tokens_than_a_tile():
    run(11, S=3, N=70, G=10, group=3, d=128, lens=[70, 5, 64])
    run(12, S=1, N=2, G=40, group=8, d=128, adjacent=True, dtype="f32")


def test_heads_per_cta_change_no_bit():
    """The number of heads that a thread goes through depends on the number of tokens and changes no bit: a call that fills the GPU
    gives what calls of a few sequences each give."""
    S, N, G, group, d = 16, 513, 10, 2, 128
    x = torch.randn(S, N, G * 4, d, generator=gen(3)).bfloat16().cuda()
    rotary = R.Rotary(d, [1e4 ** (-i / 64) for i in range(64)], q_weight=torch.ones(d), k_weight=torch.ones(d))
    outs = []
    for step in (S, 1):
        Q = torch.zeros(S, G, N, group, d, dtype=torch.bfloat16, device="cuda")
        K, V = (torch.zeros(S, G, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for b in range(0, S, step):
            s = slice(b, b + step)
            R.roco_norm_rotate(rotary, x[s, :, :20], x[s, :, 20:30], x[s, :, 30:], Q[s], K[s], V[s])
        outs.append((Q, K, V))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_axes(dtype, adjacent, axes):
    S, N, d = 2, 7, 64
    pos = torch.randint(-50, 5000, (S, N, axes), generator=gen(axes), dtype=torch.int32)
    axis = torch.randint(0, axes, (d // 2,), generator=gen(axes + 9)).tolist()
    run(5, S=S, N=N, d=d, dtype=dtype, adjacent=adjacent, axes=axes, positions=pos, axis=axis, start=[100, -3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 131072, 10 ** 7, 2 ** 31 - 1, -2 ** 31])
def test_far_positions(dtype, at):
    """Angles of far positions, a sum of start and position beyond 32 bits among them."""
    pos = torch.tensor([[0, 1, 2 ** 31 - 1, -2 ** 31 + 1]], dtype=torch.int32)
    run(9, S=1, N=4, d=64, dtype=dtype, start=[at], positions=pos[..., None])
    run(9, S=1, N=4, d=64, dtype=dtype, start=[at], freq=torch.full((32,), 3.1415927, dtype=torch.float32))


@pytest.mark.parametrize("dtype,scale", [("bf16", 0.0), ("bf16", 1e-15), ("f32", 1e15), ("f32", 0.0)])
def test_small_and_large_rows(dtype, scale):
    run(13, scale=scale, dtype=dtype, d=64)


def test_only_queries_only_keys_left_out():
    run(15, skip=("v",))
    run(15, skip=("k", "v"))
    run(15, skip=("k",))


def test_a_row_that_is_not_finite_stays_alone():
    g = gen(4)
    x = torch.randn(1, 6, 8, 64, generator=g)
    clean = run(4, S=1, N=6, G=2, group=2, d=64, dtype="f32", x=x.clone())
    bad = x.clone()
    bad[0, 2, 1, 5], bad[0, 3, 4, 63], bad[0, 4, 6, 0] = math.nan, math.inf, -math.inf
    rotary = R.Rotary(64, [1e4 ** (-i / 32) for i in range(32)], q_weight=torch.ones(64), k_weight=torch.ones(64))
    same = []
    for y in (x, bad):
        Q, K, V = torch.zeros(1, 2, 6, 2, 64).cuda(), torch.zeros(1, 2, 6, 64).cuda(), torch.zeros(1, 2, 6, 64).cuda()
        z = y.cuda()
        R.roco_norm_rotate(rotary, z[:, :, :4], z[:, :, 4:6], z[:, :, 6:], Q, K, V)
        same.append((Q, K, V))
    differ = [(a != b).nonzero() for a, b in zip(*same)]
    assert {tuple(r[1:4].tolist()) for r in differ[0]} == {(0, 2, 1)}       # head 1 is the first unit's second
    assert {tuple(r[1:3].tolist()) for r in differ[1]} == {(0, 3)}
    assert [tuple(r.tolist()) for r in differ[2]] == [(0, 0, 4, 0)]
    assert clean is not None


def test_unrotated_elements_do_not_meet_what_turns():
    """An infinity behind the rotated elements stays where it is, and without a norm nothing else sees it."""
    for adjacent in (False, True):
        for dtype in (torch.bfloat16, torch.float32):
            x = torch.ones(1, 1, 3, 128, dtype=dtype, device="cuda")
            x[..., 100] = math.inf
            rotary = R.Rotary(128, [1.0] * 16, pairing=int(adjacent))
            Q, K, V = (torch.zeros(1, 1, 1, 1, 128, dtype=dtype, device="cuda") for _ in range(3))
            R.roco_norm_rotate(rotary, x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], Q, K[:, :, :, 0], V[:, :, :, 0], start=torch.tensor(
                [2], dtype=torch.int32, device="cuda"))
            for out in (Q, K):
                assert torch.isinf(out).nonzero()[:, -1].tolist() == [100] and not torch.isnan(out).any()


def test_bad_lengths_and_axes_are_flagged():
    S, N, d = 4, 3, 64
    x = torch.randn(S, N, 3, d).cuda()
    Q, K, V = torch.zeros(S, 1, N, 1, d).cuda(), torch.zeros(S, 1, N, d).cuda(), torch.zeros(S, 1, N, d).cuda()
    rotary = R.Rotary(d, [0.5] * 32)
    R.roco_norm_rotate(rotary, x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], Q, K, V, lens=torch.tensor([3, 4, -1, 2 ** 31 - 1],
                       dtype=torch.int32).cuda())
    assert R.roco_rotary_device_status(rotary) == 16
    assert bool((V[0] != 0).all()) and not V[1:].any() and not Q[1:].any()
    axis = [0] * 32
    axis[3], axis[4] = 2, -1
    rotary = R.Rotary(d, [0.5] * 32, axes=2, axis=axis)
    plain = R.Rotary(d, [0.5] * 32, axes=2)
    pos = torch.randint(0, 9, (S, N, 2), dtype=torch.int32).cuda()
    R.roco_norm_rotate(rotary, x[:, :, :1], x[:, :, 1:2], x[:, :, 2:], Q, K, V, positions=pos)
    assert R.roco_rotary_device_status(rotary) == 64
    Q2 = torch.zeros_like(Q)
    R.roco_norm_rotate(plain, x[:, :, :1], None, None, Q2, None, None, positions=pos)
    assert torch.equal(Q, Q2)


def test_another_stream_and_a_captured_call():
    S, N, G, group, d = 2, 9, 3, 2, 128
    x = torch.randn(S, N, G * 4, d).bfloat16().cuda()
    rotary = R.Rotary(d, [1e4 ** (-i / 64) for i in range(64)], q_weight=torch.ones(d), k_weight=torch.ones(d))
    t_next = torch.full((S, G), 77, dtype=torch.int32, device="cuda")

    def call():
        out = (torch.zeros(S, G, N, group, d, dtype=torch.bfloat16, device="cuda"),
               *(torch.zeros(S, G, N, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        R.roco_norm_rotate(rotary, x[:, :, :6], x[:, :, 6:9], x[:, :, 9:], *out, start=t_next[:, 0])
        return out

    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    t_next += 5                      # what the call reads at replay
    want = call()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
