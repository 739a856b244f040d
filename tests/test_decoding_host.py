"""Host-side checks of norm and rotation, verification and reordering that need no GPU: refusals of the C entry points and of the
binding, and the 64-bit references against independent forms."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2402_06262_b200 as R
import decoding_reference as ref
from paper_2402_06262_b200 import binding
from test_abi_cpu import fake_cache
from test_operators_host import linear_state

INVALID, UNSUPPORTED = 1, 2


def rotary(**kw):
    v = dict(d=128, rot=128, pairing=0, axes=1, freq=0x1000, axis=None, q_weight=None, k_weight=None, eps=1e-6, status=0x2000)
    v.update(kw)
    return R.roco_rotary(*v.values())


def rotate(r, **kw):
    v = dict(dtype=R.ROCO_BF16, S=2, N=3, G=4, group=1, start_stride=0, q=0x10000, k=0x20000, v=0x30000, q_seq=512, q_row=512, k_seq=512,
             k_row=512, v_seq=512, v_row=512, lens=None, start=None, positions=None, Q=0x40000, K=0x50000, V=0x60000)
    v.update(kw)
    return R.lib().roco_norm_rotate(r if r is None else C.byref(r), bytes(R.roco_heads(*v.values())), None)


def test_norm_rotate_refuses_on_the_host():
    assert rotate(None) == INVALID and rotate(rotary(status=None)) == INVALID
    assert R.lib().roco_norm_rotate(C.byref(rotary()), None, None) == INVALID
    for kw in (dict(q=None), dict(Q=None), dict(k=None), dict(K=None), dict(v=None), dict(V=None), dict(S=0), dict(N=0), dict(G=0),
               dict(group=0), dict(q=0x10008), dict(Q=0x40008), dict(V=0x60004), dict(q_row=4), dict(k_seq=4), dict(v_row=1)):
        assert rotate(rotary(), **kw) == INVALID, kw
    for kw in (dict(freq=None), dict(axes=0), dict(pairing=2), dict(rot=-16), dict(rot=144)):
        assert rotate(rotary(**kw)) == INVALID, kw
    for kw in (dict(d=96), dict(rot=24), dict(axes=5)):
        assert rotate(rotary(**kw)) == UNSUPPORTED, kw
    for kw in (dict(dtype=4), dict(group=17), dict(S=1 << 20, N=1 << 12, G=1), dict(S=1 << 20, G=1 << 10)):
        assert rotate(rotary(), **kw) == UNSUPPORTED, kw


def verify(**kw):
    v = dict(dtype=R.ROCO_F32, S=2, T=4, V=100, A=3, distinct=0, target=0x1000, draft=0x2000, target_prefix=0x3000, draft_prefix=0x4000,
             target_seq=400, target_row=100, draft_seq=400, draft_row=100, target_prefix_seq=100, draft_prefix_seq=100, tokens=0x5000,
             parent=0x6000, nodes=None, accept_u=0x7000, sample_u=0x8000, path=0x9000, path_len=0xa000, next_token=0xb000, status=0xc000)
    v.update(kw)
    return R.lib().roco_tree_verify(bytes(R.roco_verify(*v.values())), None)


def test_tree_verify_refuses_on_the_host():
    assert R.lib().roco_tree_verify(None, None) == INVALID
    for name in ("target", "tokens", "parent", "accept_u", "sample_u", "path", "path_len", "next_token", "status", "draft_prefix"):
        assert verify(**{name: None}) == INVALID, name
    for kw in (dict(S=0), dict(T=0), dict(V=0), dict(A=0), dict(A=5), dict(distinct=2), dict(target=0x1002), dict(draft=0x2001),
               dict(target_prefix=0x3002), dict(dtype=R.ROCO_BF16, draft_prefix=0x4001)):
        assert verify(**kw) == INVALID, kw
    for kw in (dict(dtype=7), dict(T=65), dict(T=20, A=17), dict(V=(1 << 30) + 1), dict(S=(1 << 24) + 1)):
        assert verify(**kw) == UNSUPPORTED, kw


def two_caches(**kw):
    v = dict(S=2, G=2, d=64, B=16, K=0x100000, V=0x200000, s=0x300000, q=0x400000, n=0x500000, pos=0x600000, live=0x700000, t_next=0x800000)
    v.update(kw)
    return fake_cache(**v)


def test_cache_reorder_refuses_on_the_host():
    call = lambda a, b, m=0x10000: R.lib().roco_cache_reorder(a and C.byref(a), b and C.byref(b), m, None)  # noqa: E731
    far = dict(K=0x1100000, V=0x1200000)
    a = two_caches()
    assert call(None, a) == INVALID and call(a, None) == INVALID and call(a, a, None) == INVALID
    assert call(two_caches(live=None), a) == INVALID and call(a, two_caches(d=96, **far)) == UNSUPPORTED
    for kw in (dict(kv_dtype=R.ROCO_F32), dict(G=3), dict(d=128), dict(B=15)):
        assert call(a, two_caches(**far, **kw)) == INVALID, kw
    for kw in (dict(V=0x1200000), dict(s=0x1300000), dict(live=0x1700000), dict(S=3), dict(B=17)):    # the same K: not in place
        assert call(a, two_caches(**kw)) == INVALID, kw
    assert call(a, two_caches(K=0x100010, V=0x1200000)) == INVALID                                    # overlaps
    assert call(a, two_caches(K=0x1100000, V=0x200000)) == INVALID
    big = two_caches(S=257)
    assert call(big, big) == UNSUPPORTED


def test_linear_reorder_refuses_on_the_host():
    call = lambda a, b, m=0x10000: R.lib().roco_linear_reorder(a and C.byref(a), b and C.byref(b), m, None)  # noqa: E731
    a, far = linear_state(state=0x100000), dict(state=0x9000000)
    assert call(None, a) == INVALID and call(a, None) == INVALID and call(a, a, None) == INVALID
    assert call(a, linear_state(G=3, **far)) == INVALID and call(a, linear_state(d=64, **far)) == INVALID
    assert call(a, linear_state(S=2, state=0x100000)) == INVALID and call(a, linear_state(state=0x100100)) == INVALID
    assert call(linear_state(dtype=9), a) == UNSUPPORTED
    big = linear_state(S=257, state=0x100000)
    assert call(big, big) == UNSUPPORTED


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(2, 3, 4, 64)
    for bad in (None, x, x.double()):
        with pytest.raises(R.RocoError) as e:
            R.roco_norm_rotate(binding.Rotary.__new__(binding.Rotary), x, x, x, bad, x, x)
        assert e.value.code == INVALID
    with pytest.raises(R.RocoError):
        R.Rotary(64, [1.0] * 32, device="cpu")
    for kw in (dict(d=96), dict(freq=[1.0] * 40), dict(freq=[1.0] * 4), dict(axes=5), dict(axes=0), dict(pairing=2)):
        with pytest.raises(R.RocoError):
            R.Rotary(**{"d": 64, "freq": [1.0] * 32, "device": "cpu", **kw})
    p, i, u = torch.zeros(2, 4, 10), torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, 4)
    for bad in (p, None, p.half(), p[0]):                        # (the first: right, but not on a GPU)
        with pytest.raises(R.RocoError) as e:
            R.roco_tree_verify(bad, i, i, u, u[:, 0], i, i[:, 0], i[:, 0], i[0, :1])
        assert e.value.code == INVALID


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("adjacent", [False, True])
def test_reference_rotation(adjacent):
    """Lengths stay, positions add up, and the product of two rotated rows depends on their distance alone."""
    x, y = (torch.randn(64, generator=gen(s), dtype=torch.float64) for s in (1, 2))
    w = torch.tensor([1e4 ** (-i / 24) for i in range(24)], dtype=torch.float64)
    turn = lambda v, t: ref.rotate_row(v, None, 0.0, 48, adjacent, t * w)[0]  # noqa: E731
    assert torch.allclose(turn(x, 5).norm(), x.norm()) and torch.equal(turn(x, 7)[48:], x[48:])
    assert torch.allclose(turn(turn(x, 5), 9), turn(x, 14))
    assert torch.allclose(turn(x, 11) @ turn(y, 4), turn(x, 107) @ turn(y, 100))
    a, b = (0, 1) if adjacent else (0, 24)
    e = torch.zeros(64, dtype=torch.float64)
    e[a] = 1
    z = turn(e, 0.5)
    assert math.isclose(z[a], math.cos(0.5)) and math.isclose(z[b], math.sin(0.5))
    n, bound = ref.rotate_row(x, torch.full((64,), 2.0, dtype=torch.float64), 0.0, 0, adjacent, w[:0])
    assert torch.allclose(n, 2 * torch.nn.functional.rms_norm(x, (64,), eps=0.0)) and bool((bound > 0).all())


@pytest.mark.parametrize("kind", ["drawn", "distinct", "fixed"])
def test_reference_verification_gives_the_target(kind):
    """Summed over all drafts of two siblings and integrated over all random numbers, the first token is distributed as the target
    says: the accepted share of every draft is exact, the rest is what is drawn from."""
    V = 4
    p, q = (torch.softmax(torch.randn(V, generator=gen(s), dtype=torch.float64), 0).numpy() for s in (3, 4))
    out = np.zeros(V)
    for x in range(V):
        for y in range(V):
            if kind == "distinct" and x == y or kind == "fixed" and (x, y) != (2, 0):
                continue
            chance = 1.0 if kind == "fixed" else q[x] * (q[y] if kind == "drawn" else q[y] / (1 - q[x]))
            steps = 400                                     # a grid of the two acceptances' numbers
            for u in ((np.arange(steps) + 0.5) / steps):
                draft = None if kind == "fixed" else np.stack([q, q])
                # the second sibling's share of acceptance, found from its border
                lo, hi = 0.0, 1.0
                walk = lambda v, s=0.5: ref.verify(np.stack([p, p]), draft, p, q, [x, y], [-1, -1], 2, [u, v], s, 1, kind == "distinct")  # noqa: E731,B023
                if walk(0.0).path == [0]:
                    out[x] += chance / steps
                    continue
                if walk(1 - 1e-12).path == [1]:
                    share = 1.0
                elif walk(0.0).path != [1]:
                    share = 0.0
                else:
                    for _ in range(20):
                        mid = (lo + hi) / 2
                        lo, hi = (mid, hi) if walk(mid).path == [1] else (lo, mid)
                    share = lo
                out[y] += chance / steps * share
                if share < 1:
                    rest = np.zeros(V)                      # what is drawn from, read off the borders of the last number
                    for s in ((np.arange(25) + 0.5) / 25):
                        rest[walk(1 - 1e-12, s).next] += 1 / 25
                    out += chance / steps * (1 - share) * rest
        if kind != "fixed":
            continue
    assert np.abs(out - p).max() < 0.03


def test_reference_reorder():
    t = {f: torch.arange(3)[:, None, None].expand(3, 1, 4).clone() for f in ref.CACHE[2:6]}
    t.update({f: torch.arange(3.)[:, None, None, None].expand(3, 1, 4, 2).clone() for f in ("K", "V")},
             live=torch.tensor([[2], [4], [1]]), t_next=torch.tensor([[7], [8], [9]]))
    new = ref.reorder_cache(t, t, [1, 0, -2])
    assert new["live"].flatten().tolist() == [4, 2, 0] and new["t_next"].flatten().tolist() == [8, 7, 0]
    assert new["pos"][1, 0].tolist() == [0, 0, -1, -1] and new["s"][1, 0].tolist() == [0, 0, 1, 1] and new["pos"][2, 0].tolist() == [-1] * 4
