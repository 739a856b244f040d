"""Rounds of speculative decoding with sampling over a budgeted cache, as a program runs them: projections, norm and rotation behind
what the cache has seen, attention of the drafted tree, verification, commit, and the batch forked and compacted in between."""
import pytest
import torch

import operator_reference as ops
import paper_2402_06262_b200 as R
import decoding_reference as ref
from tree_cases import CACHE_FIELDS

pytestmark = pytest.mark.gpu


class Model:
    """One layer with random weights; tokens in, probabilities out.  All in torch except what is under test."""

    def __init__(self, G, group, d, V, dtype):
        g = torch.Generator()
        g.manual_seed(5)
        self.G, self.group, self.d, self.V, self.dtype = G, group, d, V, dtype
        H = G * (group + 2)
        rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.embed = rand(V, 48).cuda()
        self.proj = (rand(48, H * d) / 48 ** 0.5).cuda()
        self.head = (2 * rand(G * group * d, V) / (G * group * d) ** 0.5).cuda()
        self.rotary = R.Rotary(d, [1e4 ** (-2 * i / d) for i in range(d // 2)], q_weight=1 + 0.1 * rand(d), k_weight=1 + 0.1 * rand(d))

    def heads(self, tokens, start, positions=None, lens=None):
        S, N = tokens.shape
        rows = (self.embed[tokens.long()] @ self.proj).to(self.dtype)
        q, k, v = (x.unflatten(2, (-1, self.d)) for x in rows.split([self.G * self.group * self.d, self.G * self.d, self.G * self.d], 2))
        Q = torch.zeros(S, self.G, N, self.group, self.d, dtype=self.dtype, device="cuda")
        K, V = (torch.zeros(S, self.G, N, self.d, dtype=self.dtype, device="cuda") for _ in range(2))
        R.roco_norm_rotate(self.rotary, q, k, v, Q, K, V, lens=lens, start=start, positions=positions)
        return Q, K, V

    def probs(self, att):          # [S][G][T][group][d] -> [S][T][V]
        x = att.permute(0, 2, 1, 3, 4).flatten(2).float()
        return torch.softmax(x @ self.head, -1)


class Round:
    """The buffers of a round, made once."""

    def __init__(self, model, cache, T, A):
        S, G, group, d, V = cache.S, model.G, model.group, model.d, model.V
        ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.m, self.cache, self.T, self.A, self.r = model, cache, T, A, 3
        self.att = torch.zeros(S, G, T, group, d, dtype=model.dtype, device="cuda")
        self.lse = torch.zeros(S, G, T, group, device="cuda")
        self.tokens, self.parent, self.depth, self.nodes = ints(S, T), ints(S, T), ints(S, T), ints(S)
        self.draft = torch.zeros(S, T, V, device="cuda")
        self.accept_u, self.sample_u = torch.zeros(S, T, device="cuda"), torch.zeros(S, device="cuda")
        self.path, self.n, self.next, self.status, self.gone = ints(S, A), ints(S), ints(S), ints(1), ints(S, G, A)
        self.ws = torch.zeros(max(1, R.roco_tree_attend_workspace_bytes(cache, T, group)), dtype=torch.uint8, device="cuda")
        self.target = None

    def run(self):
        c = self.cache
        self.q, self.k, self.v = self.m.heads(self.tokens, c.t_next[:, 0], self.depth[..., None], lens=self.nodes)
        R.roco_tree_attend(c, self.q, self.k, self.v, self.parent, self.att, nodes=self.nodes, lse_out=self.lse, workspace=self.ws)
        self.target = self.m.probs(self.att)
        R.roco_tree_verify(self.target, self.tokens, self.parent, self.accept_u, self.sample_u, self.path, self.n, self.next, self.status,
                           nodes=self.nodes, draft=self.draft)
        R.roco_tree_commit(c, self.q, self.k, self.v, self.lse, self.parent, self.path, self.n, self.r, self.gone, nodes=self.nodes)

    def fill(self, seed, last):
        """A new tree per sequence: its root is the token sampled last, children drawn from the draft's probabilities."""
        g = torch.Generator()
        g.manual_seed(seed)
        S, T, V = self.tokens.shape[0], self.T, self.m.V
        q = torch.softmax(0.7 * torch.randn(S, T, V, generator=g), -1)
        par, tok, depth = torch.full((S, T), -1), torch.zeros(S, T, dtype=torch.long), torch.zeros(S, T, dtype=torch.long)
        nodes = torch.randint(1, T + 1, (S,), generator=g)
        nodes[0] = T
        for b in range(S):
            tok[b, 0] = int(last[b])
            for i in range(1, T):
                par[b, i] = int(torch.randint(0, i, (), generator=g)) if i > 2 else i - 1
                depth[b, i] = depth[b, par[b, i]] + 1
                tok[b, i] = int(torch.multinomial(q[b, par[b, i]], 1, generator=g))
        self.parent.copy_(par), self.tokens.copy_(tok), self.depth.copy_(depth), self.nodes.copy_(nodes), self.draft.copy_(q)
        self.accept_u.copy_(torch.rand(S, T, generator=g)), self.sample_u.copy_(torch.rand(S, generator=g))


def prompted(model, S, B, L, seed):
    g = torch.Generator()
    g.manual_seed(seed)
    cache = R.Cache(S, model.G, B, model.d, model.dtype)
    lens = [L - b for b in range(S)]
    tokens = torch.randint(0, model.V, (S, L), generator=g).cuda()
    Q, K, V = model.heads(tokens, None, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert not Q[1, :, lens[1]:].any()
    R.roco_prefill(Q[:, :, :, 0].contiguous(), K, V, lens, B, 3, cache)
    return cache


def state(cache):
    return {f: getattr(cache, f).cpu().clone() for f in CACHE_FIELDS}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_stage_of_the_rounds(dtype):
    """Each stage against its definition on what it was given."""
    S, B, T, A = 3, 40, 6, 4
    m = Model(2, 1, 64, 50, dtype)
    cache = prompted(m, S, B, 45, 1)
    rd = Round(m, cache, T, A)
    last, accepted = [1, 2, 3], 0
    w = {n: getattr(m.rotary, n + "_weight").cpu().double() for n in "qk"}
    eps = float(torch.tensor(1e-6, dtype=torch.float32))
    for step in range(4):
        rd.fill(step, last)
        before = state(cache)
        rd.run()
        torch.cuda.synchronize()
        assert int(rd.status) == 0 and R.roco_device_status(cache) == 0 and R.roco_rotary_device_status(m.rotary) == 0
        nodes, par, tok = rd.nodes.tolist(), rd.parent.tolist(), rd.tokens.tolist()
        # norm and rotation
        rows = (m.embed[rd.tokens.long()] @ m.proj).to(dtype).cpu()
        q, k, _ = (x.unflatten(2, (-1, 64)) for x in rows.split([128, 128, 128], 2))
        for x, got, name in ((q, rd.q.cpu(), "q"), (k, rd.k.cpu()[:, :, :, None], "k")):
            y, bound = ref.norm_rotate(x, 1, w[name], eps, 64, False, m.rotary.freq.cpu().double(), [0] * 32,
                                       before["t_next"][:, 0].tolist(), rd.depth.cpu()[..., None], nodes)
            u = ref.U16 if dtype == torch.bfloat16 else ref.U32
            assert bool(((got.double() - y).abs() <= bound + (y.abs() + bound) * u).all())
        for b in range(S):
            # attention of the tree
            for g in range(2):
                out, lse, ob, lb = ops.tree_attend(before["K"][b, g].double(), before["V"][b, g].double(), int(before["live"][b, g]),
                                                   rd.q[b, g].cpu().double(), rd.k[b, g].cpu().double(), rd.v[b, g].cpu().double(),
                                                   par[b], nodes[b], 64 ** -0.5, low=dtype == torch.bfloat16)
                assert bool(((rd.att[b, g, :nodes[b]].cpu().double() - out).abs() <= ob).all())
                assert bool(((rd.lse[b, g, :nodes[b]].cpu().double() - lse).abs() <= lb).all())
            # verification
            walk = ref.verify(rd.target[b].cpu().double().numpy(), rd.draft[b].cpu().double().numpy(), None, None, tok[b], par[b], nodes[b],
                              rd.accept_u[b].cpu().double().numpy(), float(rd.sample_u[b]), A, False)
            assert walk.margin > 1e-12
            assert rd.path[b, :len(walk.path)].tolist() == walk.path and int(rd.n[b]) == len(walk.path) and int(rd.next[b]) == walk.next
            # commit: what was accepted is in the cache, at the positions that follow
            a = len(walk.path)
            accepted += a
            for g in range(2):
                assert int(cache.t_next[b, g]) == int(before["t_next"][b, g]) + a
                pos = cache.pos[b, g].cpu()
                for i, node in enumerate(walk.path):
                    slot = (pos == int(before["t_next"][b, g]) + i).nonzero()
                    assert len(slot) == 1 and torch.equal(cache.K[b, g, int(slot)], rd.k[b, g, node])
                    assert torch.equal(cache.V[b, g, int(slot)], rd.v[b, g, node])
        last = rd.next.tolist()
        # the batch: the first sequence goes on twice, the others move up
        source = torch.tensor([0, 0, 1] if step % 2 else [2, 0, 1], dtype=torch.int32, device="cuda")
        was = state(cache)
        R.roco_cache_reorder(cache, source)
        want = ref.reorder_cache(was, was, source.tolist())
        assert all(torch.equal(getattr(cache, f).cpu(), want[f]) for f in CACHE_FIELDS)
        last = [last[a] for a in source.tolist()]
    assert accepted > 12


def test_captured_rounds_give_what_eager_ones_give():
    """A whole round as one CUDA graph, replayed over new trees, beside the same calls one by one."""
    m = Model(2, 1, 64, 50, torch.bfloat16)
    caches = [prompted(m, 3, 40, 45, 7) for _ in range(2)]
    rounds = [Round(m, c, 6, 4) for c in caches]
    source = torch.tensor([1, 1, 2], dtype=torch.int32, device="cuda")
    start = state(caches[0])

    def both(rd):
        rd.run()
        R.roco_cache_reorder(rd.cache, source)

    rounds[0].fill(0, [0, 0, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):          # (a first run outside, as libraries want it before a capture)
        both(rounds[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(rounds[0])
    for f in CACHE_FIELDS:
        getattr(caches[0], f).copy_(start[f])
    last = [[1, 2, 3], [1, 2, 3]]
    for step in range(6):
        for i, rd in enumerate(rounds):
            rd.fill(50 + step, last[i])
            graph.replay() if i == 0 else both(rd)
            torch.cuda.synchronize()
            last[i] = [rd.next.tolist()[a] for a in source.tolist()]
        assert last[0] == last[1] and rounds[0].path.tolist() == rounds[1].path.tolist()
        x, y = state(caches[0]), state(caches[1])
        for f in CACHE_FIELDS:             # (what lies in empty slots is of no meaning)
            held = torch.arange(40) < x["live"][..., None]
            if x[f].dim() >= 3:
                held = held.reshape(held.shape + (1,) * (x[f].dim() - 3)).expand(x[f].shape)
                assert torch.equal(x[f][held], y[f][held]), f
            else:
                assert torch.equal(x[f], y[f]), f
    assert all(R.roco_device_status(c) == 0 for c in caches)
