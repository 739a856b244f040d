"""A program with both kinds of memory-bounded attention, as a model that interleaves them runs: a prompt through a layer with a
budgeted cache and one with linear attention, then tokens through both in one captured graph, then drafted tokens."""
import pytest
import torch

import operator_reference as ref
import paper_2402_06262_b200 as R
from test_gpu_linear import close
from tree_cases import CACHE_FIELDS

pytestmark = pytest.mark.gpu


def test_prompt_and_tokens_through_both():
    S, G, L, B, r, d, steps = 2, 3, 300, 200, 16, 128, 6
    g = torch.Generator()
    g.manual_seed(3)
    log_decay = [-0.002, -0.05, -0.4]
    # [layer: queries, keys, values]; the prompt and the tokens behind it
    x = [[torch.randn(S, G, L + steps, d, generator=g).bfloat16() for _ in range(3)] for _ in range(2)]
    prompt = [[t[:, :, :L].contiguous().to("cuda") for t in layer] for layer in x]
    token = [[torch.zeros(S, G, d, dtype=torch.bfloat16, device="cuda") for _ in range(3)] for _ in range(2)]
    lens = torch.full((S,), L, dtype=torch.int32, device="cuda")

    def after_prompt():
        cache, state = R.Cache(S, G, B, d, torch.bfloat16), R.LinearState(S, G, d, torch.bfloat16, log_decay)
        outs = [torch.zeros_like(prompt[0][0]) for _ in range(2)]
        R.roco_prefill(*prompt[0], [L] * S, B, r, cache, attn_out=outs[0])
        R.roco_linear_prefill(state, *prompt[1], lens, outs[1])
        return cache, state, outs

    def step(cache, state, outs, evicted):
        R.roco_decode_step(cache, *token[0], r, outs[0], evicted)
        R.roco_linear_step(state, *token[1], outs[1])

    def set_token(i):
        for layer in range(2):
            for t, src in zip(token[layer], x[layer]):
                t.copy_(src[:, :, L + i])

    def buffers():
        return [torch.zeros(S, G, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)], torch.zeros(S, G, dtype=torch.int32, device="cuda")

    eager, graphed, warm = after_prompt(), after_prompt(), after_prompt()
    (o1, e1), (o2, e2) = buffers(), buffers()
    step(warm[0], warm[1], *buffers())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed[0], graphed[1], o2, e2)
    linear_rows = []
    for i in range(steps):
        set_token(i)
        step(eager[0], eager[1], o1, e1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(o1 + [e1], o2 + [e2])) and bool((e1 >= 0).all())
        linear_rows.append(o1[1].cpu())
    assert torch.equal(eager[1].state, graphed[1].state)
    assert all(torch.equal(getattr(eager[0], f), getattr(graphed[0], f)) for f in CACHE_FIELDS)
    # the linear layer against one recurrence over prompt and tokens
    for b in range(S):
        for h in range(G):
            o, s, ob, sb = ref.linear(torch.zeros(d, d, dtype=torch.float64), float(torch.tensor(log_decay[h])),
                                      *(t[b, h].double() for t in x[1]), d ** -0.5, low=True)
            close(torch.cat([eager[2][1][b, h].cpu()] + [row[b, h][None] for row in linear_rows]), o, ob, f"out {b},{h}")
            close(eager[1].state[b, h], s, sb, f"state {b},{h}")
    # drafted tokens through the cache as the steps left it
    cache, T = eager[0], 5
    c64 = {f: getattr(cache, f).cpu().double() for f in ("K", "V")}
    q, k, v = (torch.randn(S, G, T, d, generator=g).bfloat16() for _ in range(3))
    parent = torch.tensor([[-1, 0, 0, 1, -1]] * S, dtype=torch.int32)
    out, lse = torch.zeros(S, G, T, 1, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(S, G, T, 1, device="cuda")
    draft = q[:, :, :, None].to("cuda"), k.to("cuda"), v.to("cuda")
    R.roco_tree_attend(cache, *draft, parent.to("cuda"), out, lse_out=lse)
    for b in range(S):
        for h in range(G):
            o, l, ob, lb = ref.tree_attend(c64["K"][b, h], c64["V"][b, h], B, q[b, h, :, None].double(), k[b, h].double(), v[b, h].double(),
                                           parent[b].tolist(), T, d ** -0.5, low=True)
            close(out[b, h], o, ob, f"drafted {b},{h}")
            close(lse[b, h], l, lb, f"log-sum-exp {b},{h}")
    before = cache.t_next.clone()
    path = torch.tensor([[0, 1, 3], [4, 0, 0]], dtype=torch.int32, device="cuda")
    gone = torch.zeros(S, G, 3, dtype=torch.int32, device="cuda")
    R.roco_tree_commit(cache, *draft, lse, parent.to("cuda"), path, torch.tensor([3, 1], dtype=torch.int32, device="cuda"), r, gone)
    assert (cache.t_next - before).tolist() == [[3] * G, [1] * G] and bool((cache.live == B).all())
    assert bool((gone[0] >= 0).all()) and bool((gone[1, :, 0] >= 0).all()) and bool((gone[1, :, 1:] == -1).all())
    assert R.roco_device_status(cache) == 0 and R.roco_linear_device_status(eager[1]) == 0
