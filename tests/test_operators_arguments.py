"""What the binding refuses of the operators beside the budgeted cache, each argument and each reason on its own: on the CPU the
check itself, on a GPU whole calls with one wrong argument."""
import re

import pytest
import torch

import paper_2402_06262_b200 as R
from paper_2402_06262_b200 import binding

INVALID, WORKSPACE = 1, 3


def test_the_check_takes_the_right_tensor_only():
    ok = torch.zeros(2, 3, 4)
    binding._need("call", "x", ok, (2, 3, 4), torch.float32, -1)       # (-1: where CPU tensors say they are)
    binding._need("call", "x", ok, ok.shape, torch.float32, -1)
    for bad, shape, dtype, dev in ((ok.double(), (2, 3, 4), torch.float32, -1), (ok.int(), (2, 3, 4), torch.float32, -1),
                                   (ok, (2, 3, 5), torch.float32, -1), (ok, (2, 12), torch.float32, -1),
                                   (ok[:, :, 0], (2, 3), torch.float32, -1), (ok.transpose(0, 1), (3, 2, 4), torch.float32, -1),
                                   (ok, (2, 3, 4), torch.float32, 0), (ok, (2, 3, 4), torch.float32, -2),
                                   (None, (2, 3, 4), torch.float32, -1), ([0.0], (1,), torch.float32, -1)):
        with pytest.raises(R.RocoError, match="call: x: ") as e:
            binding._need("call", "x", bad, shape, dtype, dev)
        assert e.value.code == INVALID


S, G, B, d, T, H, A, L = 2, 3, 40, 64, 5, 2, 3, 20


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def ints(*shape):
    return zeros(*shape, dtype=torch.int32)


def attend_call():
    cache = R.Cache(S, G, B, d, torch.bfloat16)
    args = dict(Q=zeros(S, G, T, H, d), K_new=zeros(S, G, T, d), V_new=zeros(S, G, T, d), parent=ints(S, T) - 1,
                attn_out=zeros(S, G, T, H, d), nodes=ints(S) + T, lse_out=zeros(S, G, T, H, dtype=torch.float32))
    return lambda **kw: R.roco_tree_attend(cache, **{**args, **kw}), args


def commit_call():
    cache = R.Cache(S, G, B, d, torch.bfloat16)
    args = dict(Q=zeros(S, G, T, H, d), K_new=zeros(S, G, T, d), V_new=zeros(S, G, T, d), lse=zeros(S, G, T, H, dtype=torch.float32),
                parent=ints(S, T) - 1, path=ints(S, A), path_len=ints(S), evicted_slot=ints(S, G, A), evicted_pos=ints(S, G, A),
                nodes=ints(S) + T)
    return lambda **kw: R.roco_tree_commit(cache, r=4, **{**args, **kw}), args


def prefill_call():
    state = R.LinearState(S, G, d, torch.bfloat16, [-0.1] * G)
    args = dict(Q=zeros(S, G, L, d), K=zeros(S, G, L, d), V=zeros(S, G, L, d), lens=ints(S) + L, out=zeros(S, G, L, d))
    return lambda **kw: R.roco_linear_prefill(state, **{**args, **kw}), args


def step_call():
    state = R.LinearState(S, G, d, torch.bfloat16, [-0.1] * G)
    args = dict(q=zeros(S, G, d), k=zeros(S, G, d), v=zeros(S, G, d), out=zeros(S, G, d), active=ints(S))
    return lambda **kw: R.roco_linear_step(state, **{**args, **kw}), args


def wrap_cache_call():
    args = dict(K=zeros(S, G, B, d), V=zeros(S, G, B, d), s=zeros(S, G, B, dtype=torch.float32), q=zeros(S, G, B, dtype=torch.float32),
                n=ints(S, G, B), pos=ints(S, G, B), live=ints(S, G), t_next=ints(S, G), status=ints(1))
    return lambda **kw: R.Cache.wrap(**{**args, **kw}), args


def wrap_state_call():
    args = dict(state=zeros(S, G, d, d, dtype=torch.float32), log_decay=zeros(G, dtype=torch.float32), status=ints(1))
    return lambda **kw: R.LinearState.wrap(**{**args, "dtype": torch.bfloat16, **kw}), args


CALLS = dict(attend=attend_call, commit=commit_call, prefill=prefill_call, step=step_call, cache=wrap_cache_call, state=wrap_state_call)


def wrong(t, how):
    if how == "type":
        return t.to(torch.int64 if t.dtype is torch.int32 else torch.float64)
    if how == "shape":       # one more sequence
        return torch.zeros(t.shape[0] + 1, *t.shape[1:], dtype=t.dtype, device=t.device)
    if how == "rank":
        return t[None]
    if how == "strides":
        return torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype, device=t.device)[..., ::2]
    return t.cpu()


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["type", "shape", "rank", "strides", "device"])
@pytest.mark.parametrize("what", list(CALLS))
def test_one_wrong_argument(what, how):
    call, args = CALLS[what]()
    for name, t in args.items():
        if (t.numel() == 1 and how == "strides") or (what in ("cache", "state") and name in ("K", "state") and how == "shape"):
            continue           # one element has no strides; a wrap takes its sizes from this one, and the next is refused
        before = [x.clone() for x in args.values()]
        with pytest.raises(R.RocoError) as e:
            call(**{name: wrong(t, how)})
        assert e.value.code == INVALID and re.search(rf"\b{name}\b(:| is)", str(e.value)), f"{name} ({how}): {e.value}"
        assert all(torch.equal(x, y) for x, y in zip(before, args.values()))
    call()                     # and the right ones are taken


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["attend", "prefill"])
def test_wrong_workspaces(what):
    if what == "attend":
        big = R.Cache(1, 1, 8192, d, torch.bfloat16)
        x, kv = zeros(1, 1, T, H, d), zeros(1, 1, T, d)
        need = R.roco_tree_attend_workspace_bytes(big, T, H)
        call = lambda ws: R.roco_tree_attend(big, x, kv, kv, ints(1, T) - 1, torch.zeros_like(x), workspace=ws)  # noqa: E731
    else:
        state = R.LinearState(1, 1, d, torch.bfloat16, [-0.1])
        x = zeros(1, 1, 8192, d)
        need = R.roco_linear_prefill_workspace_bytes(state, 8192)
        call = lambda ws: R.roco_linear_prefill(state, x, x, x, ints(1), torch.zeros_like(x), workspace=ws)  # noqa: E731
    assert need > 0
    room = torch.zeros(2 * need + 512, dtype=torch.uint8, device="cuda")
    assert room.data_ptr() % 256 == 0
    for ws in (room[:need - 1], room[128:128 + need], room[:2 * need:2], torch.zeros(need, dtype=torch.uint8)):
        with pytest.raises(R.RocoError) as e:
            call(ws)
        assert e.value.code == WORKSPACE
    call(room[:need])
    call(room[:need].view(torch.float32))
