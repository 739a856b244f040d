"""What the binding refuses of norm and rotation, verification and reordering: whole calls with one wrong argument."""
import re

import pytest
import torch

import paper_2402_06262_b200 as R
from test_operators_arguments import INVALID, ints, wrong, zeros

pytestmark = pytest.mark.gpu
S, N, G, H, d, T, V, A, B = 2, 5, 3, 2, 64, 4, 30, 3, 20
F32 = torch.float32


def rotate_call():
    rotary = R.Rotary(d, [0.1] * 32, axes=2, axis=[0, 1] * 16, q_weight=torch.ones(d), k_weight=torch.ones(d))
    args = dict(q=zeros(S, N, G * H, d), k=zeros(S, N, G, d), v=zeros(S, N, G, d), Q=zeros(S, G, N, H, d), K=zeros(S, G, N, d),
                V=zeros(S, G, N, d), lens=ints(S) + N, positions=ints(S, N, 2))
    return lambda **kw: R.roco_norm_rotate(rotary, start=ints(S), **{**args, **kw}), args


def rotary_call():
    args = dict(freq=zeros(32, dtype=F32), axis=ints(32), q_weight=zeros(d, dtype=F32), k_weight=zeros(d, dtype=F32), status=ints(1))
    return lambda **kw: R.Rotary(d, **{**args, **kw}), args


def verify_call():
    args = dict(target=zeros(S, T, V) + 0.1, draft=zeros(S, T, V) + 0.1, target_prefix=zeros(S, V) + 0.1, draft_prefix=zeros(S, V) + 0.1,
                tokens=ints(S, T), parent=ints(S, T) - 1, accept_u=zeros(S, T, dtype=F32), sample_u=zeros(S, dtype=F32),
                path=ints(S, A), path_len=ints(S), next_token=ints(S), status=ints(1), nodes=ints(S) + T)
    return lambda **kw: R.roco_tree_verify(**{**args, **kw}), args


def reorder_call():
    cache = R.Cache(S, G, B, d, torch.bfloat16)
    args = dict(source=ints(S))
    return lambda **kw: R.roco_cache_reorder(cache, **{**args, **kw}), args


def linear_call():
    state = R.LinearState(S, G, d, torch.bfloat16, [-0.1] * G)
    args = dict(source=ints(S))
    return lambda **kw: R.roco_linear_reorder(state, **{**args, **kw}), args


CALLS = dict(rotate=rotate_call, rotary=rotary_call, verify=verify_call, reorder=reorder_call, linear=linear_call)


@pytest.mark.parametrize("how", ["type", "shape", "rank", "strides", "device"])
@pytest.mark.parametrize("what", list(CALLS))
def test_one_wrong_argument(what, how):
    call, args = CALLS[what]()
    for name, t in args.items():
        if t.numel() == 1 and how == "strides":
            continue
        if what == "rotary" and how in ("type", "device") and name != "status":
            continue                      # the constructor converts these
        before = [x.clone() for x in args.values()]
        with pytest.raises(R.RocoError) as e:
            call(**{name: wrong(t, how)})
        if what == "rotary" and name == "freq":
            assert e.value.code in (INVALID, 2)
        elif how == "shape" and name in ("Q", "target"):
            assert e.value.code == INVALID        # sizes are taken from this one, and the next is refused
        else:
            assert e.value.code == INVALID and re.search(rf"\b{name}\b(:| is)", str(e.value)), f"{name} ({how}): {e.value}"
        assert all(torch.equal(x, y) for x, y in zip(before, args.values()))
    call()                                # and the right ones are taken


def test_projections_may_be_views_of_rows_but_not_of_columns():
    call, args = rotate_call()
    wide = zeros(S, N + 1, G * H + 7, d)
    call(q=wide[:, 1:, 7:])
    heads_first = zeros(S, G * H, N, d).transpose(1, 2)
    with pytest.raises(R.RocoError, match="q: a token's heads lie"):
        call(q=heads_first)
    off = zeros(S * N * (G * H * d + 4)).as_strided((S, N, G * H, d), (N * (G * H * d + 4), G * H * d + 4, d, 1))
    with pytest.raises(R.RocoError):      # tokens eight bytes off the boundary
        call(q=off)
    shifted = zeros(S * N * G * H * d + 4)[4:].view(S, N, G * H, d)
    with pytest.raises(R.RocoError):
        call(q=shifted)


def test_optional_arguments_and_pairs():
    call, args = rotate_call()
    call(lens=None, positions=None, k=None, K=None, v=None, V=None)
    for kw in (dict(k=None), dict(K=None), dict(v=None), dict(V=None)):
        with pytest.raises(R.RocoError) as e:
            call(**kw)
        assert e.value.code == INVALID
    rotary = R.Rotary(128, None)
    with pytest.raises(R.RocoError, match="heads of 64"):
        R.roco_norm_rotate(rotary, args["q"], None, None, args["Q"], None, None)
    for start in (ints(S + 1), ints(S).long(), ints(S).cpu(), [0, 0]):
        with pytest.raises(R.RocoError, match="start"):
            R.roco_norm_rotate(R.Rotary(d, [0.1] * 32), args["q"], None, None, args["Q"], None, None, start=start)
    call, args = verify_call()
    call(nodes=None, draft=None, target_prefix=None, draft_prefix=None)
    call(target_prefix=None)
    with pytest.raises(R.RocoError) as e:
        call(draft_prefix=None)
    assert e.value.code == INVALID


def test_caches_that_do_not_match():
    a = R.Cache(S, G, B, d, torch.bfloat16)
    for other in (R.Cache(S, G + 1, B, d, torch.bfloat16), R.Cache(S, G, B, 128, torch.bfloat16), R.Cache(S, G, B, d, F32),
                  R.Cache(S, G, B - 1, d, torch.bfloat16)):
        with pytest.raises(R.RocoError) as e:
            R.roco_cache_reorder(a, ints(S), other)
        assert e.value.code == INVALID
    R.roco_cache_reorder(a, ints(S), R.Cache(S, G, B + 1, d, torch.bfloat16))
    big = R.Cache(257, 1, 2, 64, torch.bfloat16)
    with pytest.raises(R.RocoError) as e:
        R.roco_cache_reorder(big, ints(257))
    assert e.value.code == 2
    x = R.LinearState(2, 1, 64, torch.bfloat16, [-0.1])
    for other in (R.LinearState(2, 2, 64, torch.bfloat16, [-0.1] * 2), R.LinearState(2, 1, 128, torch.bfloat16, [-0.1])):
        with pytest.raises(R.RocoError) as e:
            R.roco_linear_reorder(x, ints(2), other)
        assert e.value.code == INVALID
