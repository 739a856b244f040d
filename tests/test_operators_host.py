"""Host-side checks of the operators beside the budgeted cache that need no GPU: refusals of the C entry points and of the
binding, and the 64-bit references against independent forms."""
import ctypes as C
import math

import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R
from paper_2402_06262_b200 import binding
from test_abi_cpu import fake_cache

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def attend(c, Q=0x10000, parent=0x13000, T=4, group=1, out=0x20000, ws=0x100000, wsb=1 << 40, scale=0.1):
    return R.lib().roco_tree_attend(C.byref(c), Q, 0x11000, 0x12000, parent, None, T, group, scale, out, None, ws, wsb, None)


def test_tree_attend_refuses_on_the_host():
    assert R.lib().roco_tree_attend(None, 1, 1, 1, 1, None, 1, 1, 0.1, 1, None, None, 0, None) == INVALID
    assert attend(fake_cache(K=None)) == INVALID
    assert attend(fake_cache(d=96)) == UNSUPPORTED
    assert attend(fake_cache(kv_dtype=5)) == UNSUPPORTED
    assert attend(fake_cache(B=8193)) == UNSUPPORTED
    assert attend(fake_cache(), T=0) == INVALID and attend(fake_cache(), group=0) == INVALID
    assert attend(fake_cache(), T=65) == UNSUPPORTED and attend(fake_cache(), group=17) == UNSUPPORTED
    assert attend(fake_cache(), Q=None) == INVALID and attend(fake_cache(), parent=None) == INVALID
    assert attend(fake_cache(), Q=0x10008) == INVALID and attend(fake_cache(), out=0x20004) == INVALID
    big = fake_cache(B=8192)
    need = R.lib().roco_tree_attend_workspace_bytes(C.byref(big), 4, 1)
    assert need > 0 and need % 256 == 0
    assert attend(big, ws=None) == WORKSPACE and attend(big, wsb=need - 1) == WORKSPACE and attend(big, ws=0x100080) == WORKSPACE
    assert R.lib().roco_tree_attend_workspace_bytes(None, 4, 1) == 0
    assert R.lib().roco_tree_attend_workspace_bytes(C.byref(big), 65, 1) == 0


def commit(c, Q=0x10000, lse=0x13000, path=0x15000, T=4, group=1, A=2, r=3, mode=R.ROCO_SCOPE_EXCLUDE_TOP_R, ev=0x30000):
    return R.lib().roco_tree_commit(C.byref(c), Q, 0x11000, 0x12000, lse, 0x14000, path, 0x16000, T, group, A, r, mode, 0.1, ev,
                                    None, None)


def test_tree_commit_refuses_on_the_host():
    assert commit(fake_cache(V=0x1008)) == INVALID
    assert commit(fake_cache(d=32)) == UNSUPPORTED
    assert commit(fake_cache(), Q=None) == INVALID and commit(fake_cache(), lse=None) == INVALID
    assert commit(fake_cache(), path=None) == INVALID and commit(fake_cache(), ev=None) == INVALID
    assert commit(fake_cache(), Q=0x10004) == INVALID
    assert commit(fake_cache(), A=0) == INVALID and commit(fake_cache(), A=5) == INVALID          # A <= T
    assert commit(fake_cache(B=64), T=20, A=17) == UNSUPPORTED
    assert commit(fake_cache(), r=15) == INVALID                                                  # r + A <= B = 16
    assert commit(fake_cache(), r=-1) == INVALID and commit(fake_cache(), mode=4) == INVALID
    assert commit(fake_cache(), r=0, mode=R.ROCO_SCOPE_LOWEST_R) == INVALID


def linear_state(**kw):
    v = dict(dtype=R.ROCO_BF16, S=1, G=2, d=128, state=0x1000, log_decay=0x2000, status=0x3000)
    v.update(kw)
    return R.roco_linear_state(*v.values())


def prefill(s, Q=0x10000, lens=0x14000, L=8, out=0x20000, ws=0x100000, wsb=1 << 40):
    return R.lib().roco_linear_prefill(C.byref(s), Q, 0x11000, 0x12000, lens, L, 0.1, out, ws, wsb, None)


def step(s, q=0x10000, out=0x20000):
    return R.lib().roco_linear_step(C.byref(s), q, 0x11000, 0x12000, None, 0.1, out, None)


@pytest.mark.parametrize("call", [prefill, step])
def test_linear_refuses_on_the_host(call):
    assert call(linear_state(state=None)) == INVALID and call(linear_state(log_decay=None)) == INVALID
    assert call(linear_state(status=None)) == INVALID and call(linear_state(state=0x1008)) == INVALID
    assert call(linear_state(S=0)) == INVALID
    assert call(linear_state(d=96)) == UNSUPPORTED and call(linear_state(dtype=3)) == UNSUPPORTED
    assert call(linear_state(), 0) == INVALID and call(linear_state(), 0x10008) == INVALID
    assert call(linear_state(), out=None) == INVALID


def test_linear_prefill_refuses_lengths_and_workspaces():
    assert prefill(linear_state(), L=0) == INVALID and prefill(linear_state(), lens=None) == INVALID
    one = linear_state(G=1)
    need = R.lib().roco_linear_prefill_workspace_bytes(C.byref(one), 8192)
    if need:
        assert prefill(one, L=8192, ws=None) == WORKSPACE and prefill(one, L=8192, wsb=need - 1) == WORKSPACE
        assert prefill(one, L=8192, ws=0x100010) == WORKSPACE
    assert R.lib().roco_linear_prefill_workspace_bytes(None, 8) == 0
    assert R.lib().roco_linear_prefill_workspace_bytes(C.byref(one), 0) == 0


def test_binding_refuses_wrong_tensors():
    """Tensors of the wrong type, shape or place are refused before the library sees a pointer."""
    x = torch.zeros(1, 2, 3, 1, 128, dtype=torch.bfloat16)
    c = binding.Cache.__new__(binding.Cache)
    c.S, c.G, c.B, c.d, c.dtype, c.c, c.K = 1, 2, 16, 128, torch.bfloat16, fake_cache(), torch.zeros(1)
    par = torch.full((1, 3), -1, dtype=torch.int32)
    for bad in (x, x.float(), x[:, :, :, :, ::2], x[0], None):       # (the first: right, but not on a GPU)
        with pytest.raises(R.RocoError) as e:
            R.roco_tree_attend(c, bad, x[:, :, :, 0], x[:, :, :, 0], par, x)
        assert e.value.code == INVALID
        with pytest.raises(R.RocoError):
            R.roco_tree_commit(c, bad, x[:, :, :, 0], x[:, :, :, 0], torch.zeros(1, 2, 3, 1), par, par, par[:, 0], 1,
                               torch.zeros(1, 2, 3, dtype=torch.int32))
    with pytest.raises(R.RocoError):
        R.LinearState(1, 2, 128, torch.bfloat16, [-0.1, -0.2], device="cpu")
    with pytest.raises(R.RocoError):
        R.LinearState.wrap(torch.zeros(2, 2), torch.zeros(2), torch.float16, torch.zeros(1))
    with pytest.raises(R.RocoError):
        R.Cache.wrap(*([torch.zeros(1, 2, 16, 128)] * 9))
    s = binding.LinearState.__new__(binding.LinearState)
    s.S, s.G, s.d, s.dtype, s.c, s.state = 1, 2, 128, torch.bfloat16, linear_state(), torch.zeros(1)
    y = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(R.RocoError):
        R.roco_linear_prefill(s, y, y, y, torch.ones(1, dtype=torch.int32), y)
    with pytest.raises(R.RocoError):
        R.roco_linear_step(s, y[:, :, 0], y[:, :, 0], y[:, :, 0], y[:, :, 0])


def randn(seed, *shape):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def test_reference_tree_of_one_chain_is_causal_attention():
    B, live, T, d = 12, 9, 5, 64
    K, V, Q, kn, vn = randn(1, B, d), randn(2, B, d), randn(3, T, 1, d), randn(4, T, d), randn(5, T, d)
    out, lse, ob, lb = ref.tree_attend(K, V, live, Q, kn, vn, [-1, 0, 1, 2, 3], T, 0.3)
    k, v = torch.cat((K[:live], kn)), torch.cat((V[:live], vn))
    mask = torch.cat((torch.zeros(T, live), torch.full((T, T), -math.inf).triu(1)), 1).double()
    z = Q[:, 0] @ k.T * 0.3 + mask
    assert torch.allclose(out[:, 0], torch.softmax(z, -1) @ v) and torch.allclose(lse[:, 0], torch.logsumexp(z, -1))
    assert bool((ob > 0).all()) and bool((ob < 1e-3).all()) and bool((lb < 1e-3).all())


def test_reference_ancestors():
    m = ref.ancestors([-1, 0, 0, 1, -1, 3])
    assert [r.nonzero().flatten().tolist() for r in m] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [0, 1, 3, 5]]


def test_reference_commit_keeps_the_mass():
    """Every accepted query hands out a probability of one over what it sees; Count grows by the queries that saw a token."""
    B, live, T, d, a = 10, 8, 4, 64, 4
    st = dict(K=randn(1, B, d), V=randn(2, B, d), s=randn(3, B).abs(), q=randn(4, B).abs() + 1, n=torch.full((B,), 20, dtype=torch.int32),
              pos=torch.arange(B, dtype=torch.int32), live=live, t_next=30)
    s0 = st["s"].clone()
    Q, kn, vn = randn(5, T, 2, d), randn(6, T, d), randn(7, T, d)
    par = [-1, 0, 1, 2]
    lse = ref.tree_attend(st["K"], st["V"], live, Q, kn, vn, par, T, 0.2)[1]
    gone, gone_pos, margin, _, _ = ref.tree_commit(st, Q, kn, vn, lse, [0, 1, 2, 3], 2, False, 0.2)
    assert len(gone) == 2 and st["live"] == B and st["t_next"] == 34
    kept = [j for j in range(live) if j not in gone]
    assert sorted(st["pos"].tolist()) == sorted([j for j in kept] + [30, 31, 32, 33])
    new = [int((st["pos"] == 30 + m).nonzero()) for m in range(a)]
    assert [int(st["n"][j]) for j in new] == [4, 3, 2, 1]
    assert float(st["s"][kept].sum() - s0[kept].sum() + st["s"][new].sum()) <= a + 1e-9


@pytest.mark.parametrize("log_decay", [0.0, -0.05, -math.inf])
def test_reference_linear_is_the_sum_over_pairs(log_decay):
    L, d = 9, 64
    q, k, v, s0 = randn(1, L, d), randn(2, L, d), randn(3, L, d), randn(4, d, d)
    out, s, _, _ = ref.linear(s0, log_decay, q, k, v, 0.5)
    gap = (torch.arange(L)[:, None] - torch.arange(L)).double()
    g = math.exp(log_decay) if log_decay > -math.inf else 0.0
    w = torch.where(gap >= 0, g ** gap.clamp_min(0), 0)
    want = ((q @ k.T) * w) @ v + (g ** torch.arange(1, L + 1).double())[:, None] * (q @ s0)
    assert torch.allclose(out, 0.5 * want)
    assert torch.allclose(s, g ** L * s0 + (k * (g ** (L - 1 - torch.arange(L)).double())[:, None]).T @ v)
