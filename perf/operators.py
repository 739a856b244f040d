"""The operators beside the budgeted cache, in plain form and as the library's calls, on cases of real use.

Four operators, in two groups:

  tree_attend, tree_commit    speculative decoding over the budgeted cache: every node of a tree of drafted tokens
                              attends over the cached tokens and its own ancestors; the accepted root-to-leaf path then
                              enters the cache (statistics of its queries added, evictions to the budget, insertion)
  linear_prefill, linear_step attention whose memory is bounded by construction: a d x d state per head that decays by a
                              factor of the head's own at every token; a prompt in pieces, and single tokens

A unit is one (sequence, head of one layer); G counts the heads of all layers of a call, S the sequences.
"""
import math

import torch

own = False
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one layer of one sequence, a handful of drafts: the smallest call, where latency counts
        dict(name="tree one layer", op="tree_attend", S=1, G=32, B=1024, d=128, T=8, group=1, dtype="bf16"),
        # all layers of a batch of eight at once, a tree of 16 nodes
        dict(name="tree batch", op="tree_attend", S=8, G=1024, B=1024, d=128, T=16, group=1, dtype="bf16"),
        # one layer with shared key-value heads over a long budget: 96 query rows on few units
        dict(name="tree grouped long", op="tree_attend", S=3, G=8, B=8192, d=128, T=24, group=4, dtype="bf16"),
        # single precision and the small head dimension, odd sizes
        dict(name="tree fp32 odd", op="tree_attend", S=2, G=8, B=1001, d=64, T=5, group=1, dtype="f32"),
        # the commits that follow those trees
        dict(name="commit one layer", op="tree_commit", S=1, G=32, B=1024, d=128, T=8, group=1, A=4, r=64, dtype="bf16"),
        dict(name="commit batch", op="tree_commit", S=8, G=1024, B=1024, d=128, T=16, group=1, A=5, r=64, dtype="bf16"),
        dict(name="commit grouped long", op="tree_commit", S=3, G=8, B=4093, d=128, T=24, group=4, A=6, r=64, dtype="bf16"),
        # one layer's heads over a long prompt: few units, so the length has to be split
        dict(name="linear prompt layer", op="linear_prefill", S=1, G=32, L=8192, d=128, decay="mild", dtype="bf16"),
        # every layer of that prompt at once
        dict(name="linear prompt all", op="linear_prefill", S=1, G=1024, L=8192, d=128, decay="steep", dtype="bf16"),
        # ragged short prompts in single precision
        dict(name="linear prompt fp32", op="linear_prefill", S=3, G=8, L=777, d=64, decay="mild", dtype="f32"),
        # single tokens: one layer of one sequence, and all layers of a batch
        dict(name="linear step layer", op="linear_step", S=1, G=32, d=128, decay="mild", dtype="bf16"),
        dict(name="linear step batch", op="linear_step", S=8, G=1024, d=128, decay="steep", dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tree_attend", "tree_commit", "linear_prefill", "linear_step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 64])
    S = _log(rng, 1, 16)
    G = rng.choice([4, 8, 10, 32, 40, 64, 256])
    if op in ("tree_attend", "tree_commit"):
        group = rng.choice([1, 1, 2, 4, 5, 8])
        T = _log(rng, 1, 64)
        B = _log(rng, 48, 8192)
        while S * G * B > 8192 * 1024 // (2 if dtype == "f32" else 1) or S * G * T * group > 131072:
            G = max(4, G // 2)
            S = max(1, S // 2)
            T = max(1, T // 2)
        c = dict(op=op, S=S, G=G, B=B, d=d, T=T, group=group, dtype=dtype)
        if op == "tree_commit":
            A = min(_log(rng, 1, 16), T)
            c.update(A=A, r=_log(rng, 1, max(1, (B - A) // 4)))
        return c
    c = dict(op=op, S=S, G=G, d=d, decay=rng.choice(["mild", "steep"]), dtype=dtype)
    if op == "linear_prefill":
        L = _log(rng, 1, 16384)
        while S * G * L > 2 ** 21:
            S, G, L = max(1, S // 2), max(4, G // 2), max(1, (L * 3) // 4)
        c.update(S=S, G=G, L=L)
    return c


def _tree_shape(c):
    """Sizes of a tree case and the number of sequences' cached tokens, nodes and accepted tokens, from the case alone
    (the same for every seed): sequences differ in all three."""
    S, B, T = c["S"], c["B"], c["T"]
    live = [B if b % 4 != 3 else max(1, B - 1 - (7 * b) % max(1, B // 3)) for b in range(S)]
    nodes = [T if b % 3 != 2 else max(1, T - 1 - b % max(1, T // 2)) for b in range(S)]
    return live, nodes


def _lens(c):
    S, L = c["S"], c["L"]
    return [L if b % 3 == 0 else max(1, L - (b * 997) % max(1, (2 * L) // 3)) for b in range(S)]


def _active(c):
    return [1 if b % 8 != 5 else 0 for b in range(c["S"])]


def _accepted(c, b):
    """The tokens of sequence b that were accepted (none at all for one sequence in seven)."""
    return 0 if b % 7 == 5 else 1 + (c["A"] - 1) * (3 + b) // (3 + b + b % 3)


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    d, G = c["d"], c["G"]
    if c["op"] in ("tree_attend", "tree_commit"):
        live, nodes = _tree_shape(c)
        by = fl = 0
        for b in range(c["S"]):
            if c["op"] == "tree_attend":
                rows = nodes[b] * c["group"]
                by += G * (2 * (live[b] + nodes[b]) * d * e + 2 * rows * d * e + 4 * rows)
                fl += G * 4 * rows * (live[b] + nodes[b] / 2) * d
            else:
                a = min(_accepted(c, b), nodes[b])
                if a:
                    # the keys once, the three statistics read and written, the accepted tokens in and their slots out
                    by += G * (live[b] * d * e + 24 * live[b] + a * (c["group"] + 4) * d * e + 16 * c["A"])
                    fl += G * 2 * a * c["group"] * live[b] * d
        return {"bytes": by, "flops": fl}
    if c["op"] == "linear_prefill":
        tok = G * sum(_lens(c))
        return {"bytes": 4 * tok * d * e + 8 * c["S"] * G * d * d, "flops": 4 * tok * d * d}
    units = G * sum(_active(c))
    return {"bytes": units * (8 * d * d + 4 * d * e), "flops": units * 5 * d * d}


# ------------------------------------------------------------------------------------------------ the inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    return g


def _parents(c, seed):
    """A random tree per sequence: node 0 hangs on the cached prefix, a later one on an earlier node or (rarely) on the
    prefix; every parent comes before its children.  A long chain through the first nodes, so that there is a path to
    accept."""
    g = torch.Generator()
    g.manual_seed(seed * 31 + 5)
    S, T = c["S"], c["T"]
    chain = c.get("A", (T + 1) // 2)
    par = torch.empty(S, T, dtype=torch.int32)
    for b in range(S):
        for i in range(T):
            x = torch.rand((), generator=g).item()
            par[b, i] = i - 1 if i < chain else (-1 if x < 0.1 else int(x * i))
    return par


def prepare(c, seed):
    g = _gen(seed)
    dt, d, S, G = DT[c["dtype"]], c["d"], c["S"], c["G"]
    randn = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    if c["op"] in ("tree_attend", "tree_commit"):
        return _prepare_tree(c, seed, g, randn, dt)
    heads = min(G, 32)
    h = torch.arange(G, dtype=torch.float64) % heads
    if c["decay"] == "mild":  # memory of 32 to 4096 tokens
        logd = torch.log1p(-torch.exp2(-5 - 7 * h / max(1, heads - 1)))
    else:                     # memory of about one token to 256
        logd = -torch.exp2(-8 * (h + 1) / heads)
    st = dict(case=dict(c), state=0.5 * randn(S, G, d, d), log_decay=logd.float().to(DEV),
              status=torch.zeros(1, dtype=torch.int32, device=DEV), scale=d ** -0.5)
    if c["op"] == "linear_prefill":
        L = c["L"]
        for n in ("q", "k", "v"):
            st[n] = randn(S, G, L, d).to(dt)
        st["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device=DEV)
        st["out"] = torch.zeros(S, G, L, d, dtype=dt, device=DEV)
    else:
        for n in ("q", "k", "v"):
            st[n] = randn(S, G, d).to(dt)
        st["active"] = torch.tensor(_active(c), dtype=torch.int32, device=DEV)
        st["out"] = torch.zeros(S, G, d, dtype=dt, device=DEV)
    return st


def _prepare_tree(c, seed, g, randn, dt):
    S, G, B, d, T, group = (c[k] for k in ("S", "G", "B", "d", "T", "group"))
    live_b, nodes_b = _tree_shape(c)
    unit = randn(S, G, 1, d)
    unit /= unit.norm(dim=-1, keepdim=True)              # the head's mean query direction
    rank = torch.rand(S, G, B, device=DEV, generator=g).argsort(dim=-1, stable=True)   # a slot's place in the order of mean attention
    slot = torch.arange(B, device=DEV)
    live = torch.tensor(live_b, dtype=torch.int32, device=DEV)[:, None].expand(S, G).contiguous()
    K = randn(S, G, B, d)
    # queries share a direction; a few keys lie along it (sinks, which hold much of the mass) and the tokens that have
    # received least so far lie against it
    low = min(64, B // 2)
    K += math.sqrt(d) * unit * (3.0 * (rank >= B - 4) - 2.0 * (rank < low))[..., None]
    st = dict(case=dict(c), K=K.to(dt), V=randn(S, G, B, d).to(dt), live=live, scale=d ** -0.5,
              Q=(randn(S, G, T, group, d) + 2 * unit[:, :, :, None]).to(dt),
              K_new=(randn(S, G, T, d) + math.sqrt(d) * unit).to(dt), V_new=randn(S, G, T, d).to(dt),
              parent=_parents(c, seed).to(DEV), nodes=torch.tensor(nodes_b, dtype=torch.int32, device=DEV),
              status=torch.zeros(1, dtype=torch.int32, device=DEV))
    del K
    # positions: the slots of a full budget in an order of their own, twice as many tokens seen as kept; Count is the age
    # (the least attended are older than most)
    t_next = torch.full((S, G), 2 * B + 100, device=DEV)
    age = torch.rand(S, G, B, device=DEV, generator=g) + 0.5 * (rank >= low)
    pos = 2 * age.argsort(dim=-1, stable=True).argsort(dim=-1, stable=True).to(torch.int32)
    n = (t_next[..., None] - pos).to(torch.int32)
    # mean attention: a ladder of 4 % steps below the uniform share for the least attended, spread widely above it
    up = torch.rand(S, G, B, device=DEV, generator=g)
    mean = torch.where(rank < low, 0.05 / B * 1.04 ** rank, 1.0 / B * torch.exp(3 * up)).double()
    s = mean * n
    std = mean * (0.3 + 0.4 * torch.rand(S, G, B, device=DEV, generator=g).double())
    q = n * (std * std + mean * mean)
    empty = slot >= live[..., None]
    st["s"] = s.masked_fill(empty, 0).float()
    st["q"] = q.masked_fill(empty, 0).float()
    st["n"] = n.masked_fill(empty, 0)
    st["pos"] = pos.masked_fill(empty, -1)
    st["t_next"] = t_next.to(torch.int32)
    if c["op"] == "tree_attend":
        st["out"] = torch.zeros(S, G, T, group, d, dtype=dt, device=DEV)
        st["lse"] = torch.zeros(S, G, T, group, device=DEV)
        return st
    A = c["A"]
    st["path"] = torch.arange(A, dtype=torch.int32, device=DEV).expand(S, A).contiguous()
    st["path_len"] = torch.tensor([min(_accepted(c, b), nodes_b[b]) for b in range(S)], dtype=torch.int32, device=DEV)
    st["lse"] = torch.zeros(S, G, T, group, device=DEV)
    for b in range(S):   # what the attention over the tree returned
        st["lse"][b] = _tree_scores(st, slice(b, b + 1))[0][0]
    st["evicted_slot"] = torch.zeros(S, G, A, dtype=torch.int32, device=DEV)
    st["evicted_pos"] = torch.zeros(S, G, A, dtype=torch.int32, device=DEV)
    return st


# ------------------------------------------------------------------------------------------------ plain forms

def _ancestors(parent):
    """[S][T][T]: node i sees node j (its ancestors and itself).  With P the matrix of the parents, (I + P)^T is positive
    exactly there."""
    T = parent.shape[1]
    P = torch.zeros(parent.shape[0], T, T + 1, device=parent.device)
    P.scatter_(2, torch.where(parent >= 0, parent, T).long()[..., None], 1.0)
    return torch.linalg.matrix_power(P[..., :T] + torch.eye(T, device=parent.device), T) > 0


def _tree_scores(st, b=slice(None)):
    """Row log-sum-exp and the scores' exponentials (against the row's maximum) over [cached | drafted], in 32 bits."""
    K, Q, Kn = st["K"][b].float(), st["Q"][b].float(), st["K_new"][b].float()
    S, G, T, group, d = Q.shape
    B = K.shape[2]
    z = (Q.reshape(S, G, T * group, d) @ torch.cat((K, Kn), 2).transpose(2, 3)) * st["scale"]
    z = z.reshape(S, G, T, group, B + T)
    sees = torch.cat(((torch.arange(B, device=K.device) < st["live"][b][..., None])[:, :, None].expand(S, G, T, B),
                      _ancestors(st["parent"][b])[:, None].expand(S, G, T, T)), -1)[:, :, :, None]
    z = torch.where(sees, z, -math.inf)
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    return (top + torch.log(total)).squeeze(-1), e, total


def _plain_tree_attend(st):
    lse, e, total = _tree_scores(st)
    S, G, T, group, _ = e.shape
    held = torch.arange(st["K"].shape[2], device=e.device) < st["live"][..., None]
    V = torch.cat((torch.where(held[..., None], st["V"], 0).float(), st["V_new"].float()), 2)
    o = (e.reshape(S, G, T * group, -1) @ V).reshape(S, G, T, group, -1) / total
    used = (torch.arange(T, device=e.device) < st["nodes"][:, None])[:, None, :, None]
    st["out"].copy_(torch.where(used[..., None], o.to(st["out"].dtype), st["out"]))
    st["lse"].copy_(torch.where(used, lse, st["lse"]))
    return {"out": st["out"], "lse": st["lse"]}


def _first(order, second, count):
    """A truth value for each slot: whether it is among the first `count` in (order, second) order."""
    by2 = second.argsort(dim=-1, stable=True)
    by = by2.gather(-1, order.gather(-1, by2).argsort(dim=-1, stable=True))
    at = torch.empty_like(by).scatter_(-1, by, torch.arange(by.shape[-1], device=by.device).expand_as(by))
    return at < count[..., None]


def _plain_tree_commit(st):
    c = st["case"]
    S, G, B, d, A, r = (c[k] for k in ("S", "G", "B", "d", "A", "r"))
    a = st["path_len"][:, None]                                     # accepted tokens, [S][1]
    steps = torch.arange(A, device=DEV)
    node = torch.where(steps < a, st["path"], 0).long()             # [S][A]
    at = node[:, None, :].expand(S, G, A)
    pick = lambda x: x.gather(2, at.reshape(S, G, A, *([1] * (x.dim() - 3))).expand(S, G, A, *x.shape[3:]))  # noqa: E731
    Q, Kn, Vn, lse = pick(st["Q"]), pick(st["K_new"]), pick(st["V_new"]), pick(st["lse"])
    taken = (steps < a)[:, None, :]                                 # [S][1][A]
    # probabilities of the accepted queries over the cached and over the accepted tokens, averaged over a token's heads
    rows = Q.float().reshape(S, G, -1, d)
    p = torch.exp((rows @ st["K"].float().transpose(2, 3)).reshape(S, G, A, -1, B) * st["scale"] - lse[..., None]).mean(3)
    pn = torch.exp((rows @ Kn.float().transpose(2, 3)).reshape(S, G, A, -1, A) * st["scale"] - lse[..., None]).mean(3)
    slot = torch.arange(B, device=DEV)
    held = slot < st["live"][..., None]
    p = torch.where(taken[..., None] & held[:, :, None], p, 0)
    pn = torch.where(taken[..., None] & (steps[:, None] >= steps), pn, 0)
    st["s"] += p.sum(2)
    st["q"] += (p * p).sum(2)
    st["n"] += torch.where(held, a[..., None], 0).to(torch.int32)
    # the slots that leave, decided next to a border in 64 bits
    need = (st["live"] + a - B).clamp_min(0) * (a > 0)
    n64 = st["n"].double().clamp_min(1)
    mean = st["s"].double() / n64
    var = (st["q"].double() / n64 - mean * mean).clamp_min(0)
    scope = _first(torch.where(held, var, math.inf), st["pos"], torch.minimum((st["live"] - r).clamp_min(1), st["live"]))
    leave = _first(torch.where(held & scope, mean, math.inf), st["pos"], need) & held
    freed = torch.where(leave, slot, B).sort(-1).values
    freed = torch.cat((freed, freed.new_full((S, G, A), B)), -1)[..., :A]
    gone = steps < need[..., None]
    st["evicted_slot"].copy_(torch.where(gone, freed, -1))
    st["evicted_pos"].copy_(torch.where(gone, st["pos"].gather(-1, freed.clamp_max(B - 1)).long(), -1))
    to = torch.where(gone, freed, st["live"][..., None] + steps - need[..., None])
    x, y, z = torch.nonzero(taken.expand(S, G, A), as_tuple=True)
    w = to[x, y, z]
    st["K"][x, y, w] = Kn[x, y, z]
    st["V"][x, y, w] = Vn[x, y, z]
    st["s"][x, y, w] = pn.sum(2)[x, y, z]
    st["q"][x, y, w] = (pn * pn).sum(2)[x, y, z]
    st["n"][x, y, w] = (a[x, 0] - z).to(torch.int32)
    st["pos"][x, y, w] = (st["t_next"][x, y] + z).to(torch.int32)
    st["live"] += (a - need).to(torch.int32)
    st["t_next"] += a
    return {k: st[k] for k in ("K", "V", "s", "q", "n", "pos", "live", "t_next", "evicted_slot", "evicted_pos")}


def _plain_linear_prefill(st):
    """In pieces of C tokens: products inside a piece, the state before it for the rest; the states before all pieces by
    one product with the matrix of the decays between pieces."""
    S, G, L, d = st["q"].shape
    C = 256
    P = -(-L // C)
    pad = lambda x: torch.nn.functional.pad(x.float(), (0, 0, 0, P * C - L)).reshape(S, G, P, C, d)  # noqa: E731
    lens, logd = st["lens"].long(), st["log_decay"].double()
    held = (torch.arange(P * C, device=DEV) < lens[:, None]).reshape(S, 1, P, C, 1)
    q, k, v = pad(st["q"]), torch.where(held, pad(st["k"]), 0), torch.where(held, pad(st["v"]), 0)
    i = torch.arange(C, device=DEV)
    gap = (i[:, None] - i).double()
    inside = torch.where(gap >= 0, torch.exp(logd[:, None, None] * gap.clamp_min(0)), 0).float()      # [G][C][C]
    to_end = torch.exp(logd[:, None] * (C - 1 - i).double()).float()                                  # [G][C]
    from_start = torch.exp(logd[:, None] * (i + 1).double()).float()
    o = ((q @ k.transpose(3, 4)) * inside[:, None]) @ v
    added = (k * to_end[:, None, :, None]).transpose(3, 4) @ v                                        # [S][G][P][d][d]
    t = torch.arange(P, device=DEV)
    gap = (t[:, None] - 1 - t).double()
    between = torch.where(gap >= 0, torch.exp(logd[:, None, None] * C * gap.clamp_min(0)), 0).float()  # [G][P][P]
    before = (between @ added.reshape(S, G, P, d * d)).reshape(S, G, P, d, d)
    before += torch.exp(logd[:, None] * C * t.double()).float()[:, :, None, None] * st["state"][:, :, None]
    o += (q @ before) * from_start[:, None, :, None]
    o = (o * st["scale"]).reshape(S, G, P * C, d)[:, :, :L].to(st["out"].dtype)
    rows = (torch.arange(L, device=DEV) < lens[:, None])[:, None, :, None]
    st["out"].copy_(torch.where(rows, o, st["out"]))
    left = (lens[:, None] - 1 - torch.arange(P * C, device=DEV)).double().clamp_min(0)                # [S][P C]
    w = torch.exp(logd[:, None] * left[:, None]).float()[..., None]
    end = (k.reshape(S, G, -1, d) * w).transpose(2, 3) @ v.reshape(S, G, -1, d)
    st["state"].copy_(torch.exp(logd * lens[:, None].double()).float()[..., None, None] * st["state"] + end)
    return {"out": st["out"], "state": st["state"]}


def _plain_linear_step(st):
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    on = (st["active"] != 0)[:, None, None]
    decay = torch.exp(st["log_decay"].double()).float()[:, None, None]
    new = decay * st["state"] + k[..., None] * v[..., None, :]
    st["state"].copy_(torch.where(on[..., None], new, st["state"]))
    o = ((q[..., None] * st["state"]).sum(2) * st["scale"]).to(st["out"].dtype)
    st["out"].copy_(torch.where(on, o, st["out"]))
    return {"out": st["out"], "state": st["state"]}


# ------------------------------------------------------------------------------------------------ one pass

def _own(st):
    import paper_2402_06262_b200 as R
    c = st["case"]
    h = st.get("handle")
    if h is None:  # what a program makes once and keeps: the C struct over its tensors, the workspace
        if c["op"] in ("tree_attend", "tree_commit"):
            h = R.Cache.wrap(st["K"], st["V"], st["s"], st["q"], st["n"], st["pos"], st["live"], st["t_next"], st["status"])
            if c["op"] == "tree_attend":
                st["ws"] = torch.empty(R.roco_tree_attend_workspace_bytes(h, c["T"], c["group"]), dtype=torch.uint8, device=DEV)
        else:
            h = R.LinearState.wrap(st["state"], st["log_decay"], DT[c["dtype"]], st["status"])
            if c["op"] == "linear_prefill":
                st["ws"] = torch.empty(R.roco_linear_prefill_workspace_bytes(h, c["L"]), dtype=torch.uint8, device=DEV)
        st["handle"] = h
    if c["op"] == "tree_attend":
        R.roco_tree_attend(h, st["Q"], st["K_new"], st["V_new"], st["parent"], st["out"], nodes=st["nodes"], lse_out=st["lse"],
                           scale=st["scale"], workspace=st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    if c["op"] == "tree_commit":
        R.roco_tree_commit(h, st["Q"], st["K_new"], st["V_new"], st["lse"], st["parent"], st["path"], st["path_len"], c["r"],
                           st["evicted_slot"], evicted_pos=st["evicted_pos"], scale=st["scale"])
        return {k: st[k] for k in ("K", "V", "s", "q", "n", "pos", "live", "t_next", "evicted_slot", "evicted_pos")}
    if c["op"] == "linear_prefill":
        R.roco_linear_prefill(h, st["q"], st["k"], st["v"], st["lens"], st["out"], scale=st["scale"], workspace=st["ws"])
    else:
        R.roco_linear_step(h, st["q"], st["k"], st["v"], st["out"], active=st["active"], scale=st["scale"])
    return {"out": st["out"], "state": st["state"]}


def run(st):
    if own:
        return _own(st)
    return {"tree_attend": _plain_tree_attend, "tree_commit": _plain_tree_commit, "linear_prefill": _plain_linear_prefill,
            "linear_step": _plain_linear_step}[st["case"]["op"]](st)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits

def _sees(parent, T):
    m = torch.zeros(T, T, dtype=torch.bool)
    for i in range(T):
        j = i
        while j >= 0:
            m[i, j] = True
            j = int(parent[j])
    return m.to(DEV)


def _exact_tree_attend(st, c):
    out, lse = st["out"].double(), st["lse"].double()
    for b in range(c["S"]):
        live, N = int(st["live"][b, 0]), int(st["nodes"][b])
        see = _sees(st["parent"][b].tolist(), N)
        for g0 in range(0, c["G"], 64):
            g = slice(g0, g0 + 64)
            k = torch.cat((st["K"][b, g, :live], st["K_new"][b, g, :N]), 1).double()
            v = torch.cat((st["V"][b, g, :live], st["V_new"][b, g, :N]), 1).double()
            z = torch.einsum("gthd,gjd->gthj", st["Q"][b, g, :N].double(), k) * st["scale"]
            z[..., live:].masked_fill_(~see[None, :, None], -math.inf)
            lse[b, g, :N] = torch.logsumexp(z, -1)
            out[b, g, :N] = torch.einsum("gthj,gjd->gthd", torch.softmax(z, -1), v)
    return {"out": out, "lse": lse}


def _exact_tree_commit(st, c):
    s_all, q_all = st["s"].double(), st["q"].double()
    B, r = c["B"], c["r"]
    for b in range(c["S"]):
        a, live = int(st["path_len"][b]), int(st["live"][b, 0])
        if not a:
            continue
        path = st["path"][b, :a].long()
        for g0 in range(0, c["G"], 64):
            g = slice(g0, g0 + 64)
            qa, l = st["Q"][b, g][:, path].double(), st["lse"][b, g][:, path].double()
            prob = lambda k: torch.exp(torch.einsum("gahd,gjd->gahj", qa, k.double()) * st["scale"] - l[..., None]).mean(2)  # noqa: E731,B023
            p = prob(st["K"][b, g, :live])
            pn = prob(st["K_new"][b, g][:, path]) * (torch.arange(a, device=DEV)[:, None] >= torch.arange(a, device=DEV))
            s, q = s_all[b, g, :live] + p.sum(1), q_all[b, g, :live] + p.pow(2).sum(1)
            n, pos = st["n"][b, g, :live].double() + a, st["pos"][b, g, :live].double()
            s_all[b, g, :live], q_all[b, g, :live] = s, q
            need = max(0, live + a - B)
            var = q / n - (s / n) ** 2
            m = min(max(1, live - r), live)
            # one slot after the other: the lowest (mean, position) of those whose (variance, position) is among the m lowest
            keys = torch.stack((var, pos), -1)
            kth = keys[..., 0].sort(-1).values[:, m - 1:m]
            mean = torch.where(var <= kth, s / n, math.inf)
            chosen = mean.topk(need, -1, largest=False).indices.sort(-1).values if need else torch.zeros(len(s), 0, dtype=torch.long, device=DEV)
            fill = torch.arange(live, live + a - need, device=DEV).expand(len(s), -1)
            to = torch.cat((chosen, fill), -1)
            s_all[b, g] = s_all[b, g].scatter(-1, to, pn.sum(1))
            q_all[b, g] = q_all[b, g].scatter(-1, to, pn.pow(2).sum(1))
    return {"K": None, "V": None, "s": s_all, "q": q_all, "n": None, "pos": None, "live": None, "t_next": None, "evicted_slot": None,
            "evicted_pos": None}


def _exact_linear_prefill(st, c):
    """out_i = sum over j <= i of decay^(i - j) (q_i . k_j) v_j + decay^(i + 1) q_i state, every pair of tokens."""
    out, state = st["out"].double(), st["state"].double()
    logd = st["log_decay"].double()
    for b in range(c["S"]):
        L = int(st["lens"][b])
        i = torch.arange(L, device=DEV, dtype=torch.float64)
        for g in range(c["G"]):
            q, k, v = (st[n][b, g, :L].double() for n in ("q", "k", "v"))
            s0 = state[b, g].clone()
            for lo in range(0, L, 2048):
                hi = min(L, lo + 2048)
                gap = i[lo:hi, None] - i[None, :hi]
                w = torch.exp(logd[g] * gap).masked_fill_(gap < 0, 0)
                o = ((q[lo:hi] @ k[:hi].T) * w) @ v[:hi] + torch.exp(logd[g] * (i[lo:hi, None] + 1)) * (q[lo:hi] @ s0)
                out[b, g, lo:hi] = o * st["scale"]
            state[b, g] = torch.exp(logd[g] * L) * s0 + (k * torch.exp(logd[g] * (L - 1 - i))[:, None]).T @ v
    return {"out": out, "state": state}


def _exact_linear_step(st, c):
    out, state = st["out"].double(), st["state"].double()
    for b in range(c["S"]):
        if int(st["active"][b]):
            state[b] = torch.exp(st["log_decay"].double())[:, None, None] * state[b] + torch.einsum(
                "gi,gj->gij", st["k"][b].double(), st["v"][b].double())
            out[b] = torch.einsum("gi,gij->gj", st["q"][b].double(), state[b]) * st["scale"]
    return {"out": out, "state": state}


def exact(c, seed):
    st = prepare(c, seed)
    return {"tree_attend": _exact_tree_attend, "tree_commit": _exact_tree_commit, "linear_prefill": _exact_linear_prefill,
            "linear_step": _exact_linear_step}[c["op"]](st, c)
