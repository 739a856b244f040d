"""What one round of speculative decoding or parallel sampling needs around the attention over the budgeted cache, in plain form
and as the library's calls, on cases of real use.

Four operators:

  norm_rotate     queries, keys and values of a layer out of its projections: norm of each head's query and key, rotation by the
                  token's position (one number, or several axes), layout by unit
  tree_verify     which path of a tree of drafted tokens the target's probabilities accept, from given random numbers, and the
                  token behind it
  cache_reorder   sequences of the budgeted cache forked, reordered, compacted, freed
  linear_reorder  the same for the states of linear attention

A unit is one (sequence, key-value head of one layer); G counts the heads of a call, S the sequences.
"""
import math

import torch

own = False
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
KEEP, FREE = -1, -2


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the next token of a batch in one layer: the smallest call, where latency counts
        dict(name="rotate step", op="norm_rotate", S=8, N=1, G=32, group=1, d=128, rot=128, pairing="halves", axes=1,
             norm="qk", at="start", dtype="bf16"),
        # the drafted trees of a batch, positions from the cache and the nodes' depths, shared key-value heads
        dict(name="rotate tree", op="norm_rotate", S=8, N=16, G=8, group=4, d=128, rot=64, pairing="adjacent", axes=1,
             norm="qk", at="tree", dtype="bf16"),
        # ragged long prompts in one layer
        dict(name="rotate prompts", op="norm_rotate", S=4, N=8192, G=32, group=1, d=128, rot=128, pairing="halves", axes=1,
             norm="qk", at="prompt", dtype="bf16"),
        # frames of a video: time, height and width turn a third of the pairs each; single precision, odd length
        dict(name="rotate video", op="norm_rotate", S=2, N=3001, G=10, group=2, d=64, rot=64, pairing="halves", axes=3,
             norm="qk", at="grid", dtype="f32"),
        # one sequence, a few drafts
        dict(name="verify one", op="tree_verify", S=1, T=8, V=32000, A=4, drafts="drawn", prefix=False, dtype="f32"),
        # a batch with trees of 16 nodes over a large vocabulary
        dict(name="verify batch", op="tree_verify", S=64, T=16, V=128000, A=6, drafts="distinct", prefix=False, dtype="f32"),
        # drafts without probabilities (the likeliest tokens of each node), an odd vocabulary, verified from the prefix on
        dict(name="verify odd", op="tree_verify", S=32, T=63, V=50257, A=8, drafts="fixed", prefix=True, dtype="bf16"),
        # one layer: a prompt forked into eight samples
        dict(name="fork one layer", op="cache_reorder", S=8, G=32, B=1024, d=128, how="fork", dtype="bf16"),
        # every layer of a batch: two groups of four beams follow their best continuations
        dict(name="beams all layers", op="cache_reorder", S=8, G=1024, B=1024, d=128, how="beams", dtype="bf16"),
        # a running batch without the sequences that ended, into a cache of another size; odd budget, single precision
        dict(name="compact odd", op="cache_reorder", S=13, G=24, B=1001, d=64, how="compact", dtype="f32"),
        # the linear-attention layers beside them
        dict(name="linear fork", op="linear_reorder", S=8, G=32, d=128, how="fork"),
        dict(name="linear beams", op="linear_reorder", S=16, G=512, d=64, how="beams"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rotate", "norm_rotate", "tree_verify", "tree_verify", "cache_reorder", "cache_reorder", "linear_reorder"])
    d = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    S = _log(rng, 1, 64)
    if op == "norm_rotate":
        at = rng.choice(["start", "tree", "prompt", "prompt", "grid"])
        N = 1 if at == "start" else _log(rng, 1, 64) if at == "tree" else _log(rng, 1, 16384)
        G, group = rng.choice([4, 8, 10, 32, 40]), rng.choice([1, 1, 2, 4, 5, 8])
        while S * N * G * (group + 2) > 4 * 8192 * 96 // (2 if dtype == "f32" else 1):
            S, N, G = max(1, S // 2), max(1, (2 * N) // 3), max(4, (3 * G) // 4)
        return dict(op=op, S=S, N=N, G=G, group=group, d=d, rot=rng.choice([d, d, d // 2, 3 * d // 4]),
                    pairing=rng.choice(["halves", "adjacent"]), axes=rng.choice([2, 3]) if at == "grid" else 1,
                    norm=rng.choice(["qk", "qk", "none"]), at=at, dtype=dtype)
    if op == "tree_verify":
        T, V = _log(rng, 1, 64), _log(rng, 500, 150000)
        while S * V > 64 * 128000 or S * T * V > 64 * 16 * 128000:
            S, T, V = max(1, (2 * S) // 3), max(1, (2 * T) // 3), (4 * V) // 5
        return dict(op=op, S=S, T=T, V=V, A=min(T, _log(rng, 1, 16)), drafts=rng.choice(["drawn", "distinct", "fixed"]),
                    prefix=rng.random() < 0.5, dtype=dtype)
    how = rng.choice(["fork", "beams", "compact"])
    S, G = max(2, S), rng.choice([4, 8, 10, 32, 40, 64, 256])
    if op == "linear_reorder":
        while S * G * d * d > 16 * 512 * 64 * 64:
            S, G = max(2, S // 2), max(4, G // 2)
        return dict(op=op, S=S, G=G, d=d, how=how)
    B = _log(rng, 48, 8192)
    while S * G * B > 8192 * 1024 // (2 if dtype == "f32" else 1):
        S, G, B = max(2, S // 2), max(4, G // 2), max(48, (3 * B) // 4)
    return dict(op=op, S=S, G=G, B=B, d=d, how=how, dtype=dtype)


def _lens(c):
    """Tokens of each sequence, from the case alone: ragged for prompts and frames, drafted nodes for trees."""
    S, N = c["S"], c["N"]
    if c["at"] == "start":
        return [N] * S
    return [N if b % 3 == 0 else max(1, N - (b * 997) % max(1, N // 2)) for b in range(S)]


def _nodes(c):
    S, T = c["S"], c["T"]
    return [T if b % 4 != 3 else T - 1 - b % max(1, T // 2) for b in range(S)]


def _live(c):
    S, B = c["S"], c["B"]
    return [B if b % 4 != 3 else max(1, B - 1 - (7 * b) % max(1, B // 3)) for b in range(S)]


def _map(c, seed=0):
    """source[b] of every destination.  fork: all from sequence 0.  beams: groups of four follow members of the group.  compact:
    the sequences that go on (two in three), in order; the room behind them is freed or stays as it is."""
    S = c["S"]
    if c["how"] == "fork":
        return [0] * S
    g = torch.Generator()
    g.manual_seed(seed * 13 + 3)
    if c["how"] == "beams":
        step = torch.randint(0, 4, (S,), generator=g).tolist()
        # (the first of a group follows its second, so that the group always moves)
        return [min(S - 1, b + 1) if b % 4 == 0 else min(S - 1, 4 * (b // 4) + step[b]) for b in range(S)]
    on = [b for b in range(S) if b % 3 != 1]
    return on + [FREE if b % 2 else KEEP for b in range(len(on), S)]


def work(c):
    if c["op"] == "norm_rotate":
        e = 2 if c["dtype"] == "bf16" else 4
        tok, heads = sum(_lens(c)), c["G"] * (c["group"] + 2)
        turned = tok * c["G"] * (c["group"] + 1)
        return {"bytes": 2 * tok * heads * c["d"] * e, "flops": turned * (3 * c["rot"] + (4 * c["d"] if c["norm"] == "qk" else 0))}
    if c["op"] == "tree_verify":
        e = 2 if c["dtype"] == "bf16" else 4
        rows = 1 if c["drafts"] == "fixed" else 2
        # the row at which each walk ends, and the nodes' own numbers
        return {"bytes": c["S"] * (rows * c["V"] * e + c["T"] * (12 + rows * e)), "flops": c["S"] * c["V"] * (rows + 1)}
    S, G, d = c["S"], c["G"], c["d"]
    src = _map(c)
    moved = [b for b in range(S) if src[b] >= 0 and (c["how"] == "compact" or src[b] != b)]
    read = {src[b] for b in moved}
    if c["op"] == "linear_reorder":
        return {"bytes": (len(moved) + len(read)) * G * d * d * 4, "flops": 0}
    e = 2 if c["dtype"] == "bf16" else 4
    live = _live(c)
    slots = sum(live[src[b]] for b in moved) + sum(live[b] for b in read)
    return {"bytes": slots * G * (2 * d * e + 16), "flops": 0}


# ------------------------------------------------------------------------------------------------ the inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    return g


def prepare(c, seed):
    return {"norm_rotate": _prepare_rotate, "tree_verify": _prepare_verify, "cache_reorder": _prepare_cache,
            "linear_reorder": _prepare_linear}[c["op"]](c, seed, _gen(seed))


def _tree(c, seed):
    """A random tree per sequence, every parent before its children: node 0 hangs on the prefix, half the others continue the
    node before them, the rest branch off anywhere."""
    g = torch.Generator()
    g.manual_seed(seed * 31 + 7)
    S, T = c["S"], c.get("T", c.get("N"))
    x, y = torch.rand(S, T, generator=g), torch.rand(S, T, generator=g)
    i = torch.arange(T)
    back = (y * i).long().clamp_max(i - 1)
    return torch.where(x < 0.5, i - 1, back).to(torch.int32)


def _prepare_rotate(c, seed, g):
    S, N, G, group, d, rot = (c[k] for k in ("S", "N", "G", "group", "d", "rot"))
    dt = DT[c["dtype"]]
    H = G * (group + 2)
    # the projections of a token lie side by side in one row, as one matrix product leaves them
    rows = torch.empty(S, N, H * d, dtype=dt, device=DEV)
    for b in range(S):
        rows[b] = torch.randn(N, H * d, device=DEV, generator=g).to(dt)
    q, k, v = (x.reshape(S, N, -1, d) for x in rows.split([G * group * d, G * d, G * d], dim=2))
    lens = _lens(c)
    st = dict(case=dict(c), q=q, k=k, v=v, eps=1e-6,
              freq=torch.tensor([1e4 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float32, device=DEV),
              lens=torch.tensor(lens, dtype=torch.int32, device=DEV), axis=None, start=None, positions=None,
              status=torch.zeros(1, dtype=torch.int32, device=DEV), q_weight=None, k_weight=None,
              Q=torch.zeros(S, G, N, group, d, dtype=dt, device=DEV), K=torch.zeros(S, G, N, d, dtype=dt, device=DEV),
              V=torch.zeros(S, G, N, d, dtype=dt, device=DEV))
    if c["norm"] == "qk":
        st["q_weight"], st["k_weight"] = (1 + 0.2 * torch.randn(d, device=DEV, generator=g) for _ in range(2))
    if c["at"] in ("start", "tree"):    # behind what the cache has seen (t_next, one number per unit)
        t_next = torch.randint(1000, 100000, (S, 1), device=DEV, generator=g, dtype=torch.int32).expand(S, G).contiguous()
        st["start"] = t_next[:, 0]
    if c["at"] == "tree":
        par = _tree(c, seed)
        depth = torch.zeros(S, N, dtype=torch.int32)
        for i in range(1, N):
            depth[:, i] = depth.gather(1, par[:, i:i + 1].long())[:, 0] + 1
        st["positions"] = depth[..., None].to(DEV)
    if c["at"] == "grid":               # tokens in raster order over frames
        w = max(1, int(N ** 0.4))
        n = torch.arange(N, device=DEV)
        pos = torch.stack((n // (w * w), n // w % w, n % w)[3 - c["axes"]:], -1).to(torch.int32)
        st["positions"] = (pos + torch.randint(0, 50, (S, 1, c["axes"]), device=DEV, generator=g, dtype=torch.int32)).contiguous()
        st["axis"] = (torch.arange(rot // 2, device=DEV) * c["axes"] // (rot // 2)).to(torch.int32)
    return st


def _prepare_verify(c, seed, g):
    S, T, V = c["S"], c["T"], c["V"]
    dt = DT[c["dtype"]]
    par = _tree(c, seed)
    if c["prefix"] and T > 2:
        par[:, T // 2] = -1                       # a second candidate for the first token
    R = T + 1 if c["prefix"] else T               # rows: behind the prefix (where it is asked for), then behind every node
    st = dict(case=dict(c), parent=par.to(DEV), nodes=torch.tensor(_nodes(c), dtype=torch.int32, device=DEV),
              status=torch.zeros(1, dtype=torch.int32, device=DEV))
    target = torch.empty(S, T, V, dtype=dt, device=DEV)
    draft = None if c["drafts"] == "fixed" else torch.empty(S, T, V, dtype=dt, device=DEV)
    first = [torch.empty(S, V, dtype=dt, device=DEV) if c["prefix"] else None for _ in range(2)]
    tokens = torch.zeros(S, T, dtype=torch.int32, device=DEV)
    for b in range(S):
        # a few likely tokens and a long tail; the draft model is near the target
        x = 2.2 * torch.randn(R, V, device=DEV, generator=g)
        x += 7 * (torch.rand(R, V, device=DEV, generator=g) < 12.0 / V)
        p = torch.softmax(x, -1).to(dt)
        q = torch.softmax(x + 0.7 * torch.randn(R, V, device=DEV, generator=g), -1).to(dt)
        target[b] = p[R - T:]
        if draft is not None:
            draft[b] = q[R - T:]
        if c["prefix"]:
            first[0][b], first[1][b] = p[0], q[0]
        # children of a row: its likeliest tokens in order, or drawn from it one by one (with their like or all different)
        kids = {}
        for i in range(T):
            kids.setdefault(int(par[b, i]), []).append(i)
        for up, nodes in kids.items():
            row = up + R - T
            if row < 0:                            # the token that was sampled last time
                tokens[b, nodes] = torch.randint(0, V, (len(nodes),), device=DEV, generator=g, dtype=torch.int32)
            elif c["drafts"] == "fixed":
                tokens[b, nodes] = q[row].float().topk(len(nodes)).indices.to(torch.int32)
            else:
                tokens[b, nodes] = torch.multinomial(q[row].float(), len(nodes), replacement=c["drafts"] == "drawn",
                                                     generator=g).to(torch.int32)
    st.update(target=target, draft=draft, target_prefix=first[0], draft_prefix=None if draft is None else first[1], tokens=tokens,
              accept_u=torch.rand(S, T, device=DEV, generator=g), sample_u=torch.rand(S, device=DEV, generator=g),
              path=torch.zeros(S, c["A"], dtype=torch.int32, device=DEV), path_len=torch.zeros(S, dtype=torch.int32, device=DEV),
              next_token=torch.zeros(S, dtype=torch.int32, device=DEV))
    return st


FIELDS = ("K", "V", "s", "q", "n", "pos", "live", "t_next")


def _random_cache(c, g, S, live):
    G, B, d, dt = c["G"], c["B"], c["d"], DT[c["dtype"]]
    st = {}
    for name in ("K", "V"):
        st[name] = torch.empty(S, G, B, d, dtype=dt, device=DEV)
        for b in range(S):
            st[name][b] = torch.randn(G, B, d, device=DEV, generator=g).to(dt)
    live = torch.tensor(live, dtype=torch.int32, device=DEV)[:, None].expand(S, G).contiguous()
    empty = torch.arange(B, device=DEV) >= live[..., None]
    pos = torch.rand(S, G, B, device=DEV, generator=g).argsort(-1).to(torch.int32) * 2
    n = (2 * B + 100 - pos).to(torch.int32)
    s = torch.rand(S, G, B, device=DEV, generator=g) * n / B
    st.update(s=s.masked_fill(empty, 0), q=(s * s).masked_fill(empty, 0), n=n.masked_fill(empty, 0), pos=pos.masked_fill(empty, -1),
              live=live, t_next=torch.randint(2 * B, 3 * B, (S, 1), device=DEV, generator=g, dtype=torch.int32).expand(S, G).contiguous(),
              status=torch.zeros(1, dtype=torch.int32, device=DEV))
    return st


def _prepare_cache(c, seed, g):
    S = c["S"]
    st = dict(case=dict(c), source=torch.tensor(_map(c, seed), dtype=torch.int32, device=DEV), src=_random_cache(c, g, S, _live(c)))
    st["dst"] = _random_cache(c, g, S, [1 + b % c["B"] for b in range(S)]) if c["how"] == "compact" else st["src"]
    return st


def _prepare_linear(c, seed, g):
    S, G, d = c["S"], c["G"], c["d"]
    st = dict(case=dict(c), source=torch.tensor(_map(c, seed), dtype=torch.int32, device=DEV),
              log_decay=torch.full((G,), -0.05, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV),
              src=torch.randn(S, G, d, d, device=DEV, generator=g))
    st["dst"] = torch.randn(S, G, d, d, device=DEV, generator=g) if c["how"] == "compact" else st["src"]
    return st


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_norm_rotate(st):
    c = st["case"]
    S, N, G, group, d, rot = (c[k] for k in ("S", "N", "G", "group", "d", "rot"))
    n = torch.arange(N, device=DEV)
    at = (n[:, None] if st["positions"] is None else st["positions"]).double().expand(S, N, c["axes"])
    if st["start"] is not None:
        at = at + st["start"][:, None, None]
    axis = torch.zeros(rot // 2, dtype=torch.long, device=DEV) if st["axis"] is None else st["axis"].long()
    turn = at[..., axis] * st["freq"].double()                                    # [S][N][rot / 2]
    cos, sin = torch.cos(turn).float()[:, :, None], torch.sin(turn).float()[:, :, None]
    held = (n < st["lens"][:, None])[:, None, :, None]
    for x, w, out, heads in ((st["q"], st["q_weight"], st["Q"], group), (st["k"], st["k_weight"], st["K"], 1), (st["v"], None, st["V"], 0)):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + st["eps"]) * w
        if heads:
            z = y[..., :rot]
            a, b = (z[..., :rot // 2], z[..., rot // 2:]) if c["pairing"] == "halves" else (z[..., ::2], z[..., 1::2])
            a, b = a * cos - b * sin, b * cos + a * sin
            z = torch.cat((a, b), -1) if c["pairing"] == "halves" else torch.stack((a, b), -1).flatten(-2)
            y = torch.cat((z, y[..., rot:]), -1)
        y = y.to(out.dtype).reshape(S, N, G, -1).transpose(1, 2)                  # a group's heads stay together
        flat = out.view(S, G, N, -1)
        flat.copy_(torch.where(held, y, flat))
    return {"Q": st["Q"], "K": st["K"], "V": st["V"]}


def _plain_tree_verify(st):
    """Node after node in 64 bits: a node is tried where its parent is the end of the sequence's path so far.  With p the target's
    and q the draft's probabilities behind that end, what is left of p after rejections is max(p - C q, 0)."""
    c = st["case"]
    S, T, V, A = (c[k] for k in ("S", "T", "V", "A"))
    tokens, parent, nodes = st["tokens"].long(), st["parent"], st["nodes"]
    seq = torch.arange(S, device=DEV)

    def rows(after, first):
        at = after[seq, tip.clamp_min(0)].double()
        return at if first is None else torch.where((tip < 0)[:, None], first.double(), at)

    f64 = dict(dtype=torch.float64, device=DEV)
    tip = torch.full((S,), -1, dtype=torch.long, device=DEV)
    n = torch.zeros(S, dtype=torch.int32, device=DEV)
    path = torch.full((S, A), -1, dtype=torch.int32, device=DEV)
    begin = 0
    if not c["prefix"]:                   # node 0 is the token sampled last: accepted as it stands
        on = nodes > 0
        tip = torch.where(on, 0, tip)
        path[:, 0] = torch.where(on, 0, -1)
        n += on.to(torch.int32)
        begin = 1
    C, R, M = torch.zeros(S, **f64), torch.ones(S, **f64), torch.ones(S, **f64)
    gone = torch.zeros(S, V, dtype=torch.bool, device=DEV)      # drafted tokens rejected behind the path's end
    for i in range(begin, T):
        x, u = tokens[:, i], st["accept_u"][:, i].double()
        tried = (parent[:, i] == tip) & (i < nodes) & (n < A) & (c["prefix"] | (tip >= 0))
        p = rows(st["target"], st["target_prefix"])
        if st["draft"] is None:
            left = torch.where(gone, 0, p)
            yes = tried & (u * R < left[seq, x])
        else:
            q = rows(st["draft"], st["draft_prefix"])
            qx = torch.where(gone[seq, x], 0, q[seq, x]) if c["drafts"] == "distinct" else q[seq, x]
            yes = tried & (u * qx * R < (p[seq, x] - C * q[seq, x]).clamp_min(0) * M)
        no = tried & ~yes
        gone[seq, x] |= no
        if st["draft"] is None:
            rest = torch.where(gone, 0, p).sum(-1)
        else:
            C = torch.where(no & (M > 0), C + R / M, C)
            if c["drafts"] == "distinct":
                M = torch.where(no, M - qx, M)
            rest = (p - C[:, None] * q).clamp_min(0).sum(-1)
        R = torch.where(no, rest, R)
        # a step down the tree
        path[seq, n.long().clamp_max(A - 1)] = torch.where(yes, i, path[seq, n.long().clamp_max(A - 1)])
        n += yes.to(torch.int32)
        tip = torch.where(yes, i, tip)
        C, R, M = torch.where(yes, 0, C), torch.where(yes, 1, R), torch.where(yes, 1, M)
        gone &= ~yes[:, None]
    p = rows(st["target"], st["target_prefix"])
    left = torch.where(gone, 0, p) if st["draft"] is None else (p - C[:, None] * rows(st["draft"], st["draft_prefix"])).clamp_min(0)
    left = torch.where((left.sum(-1) > 0)[:, None], left, p)
    upto = left.cumsum(-1)
    pick = torch.searchsorted(upto, (st["sample_u"].double() * upto[:, -1])[:, None], right=True)[:, 0]
    last = V - 1 - (left.flip(-1) > 0).to(torch.int8).argmax(-1)
    pick = torch.minimum(pick, last)
    st["path"].copy_(path)
    st["path_len"].copy_(n)
    st["next_token"].copy_(torch.where((tip >= 0) | c["prefix"], pick, -1))
    return {"path": st["path"], "path_len": st["path_len"], "next_token": st["next_token"]}


def _plain_cache_reorder(st):
    src, dst, source = st["src"], st["dst"], st["source"]
    B = src["K"].shape[2]
    at = source.clamp_min(0).long()
    taken = source >= 0
    live = src["live"][at]
    held = (torch.arange(B, device=DEV) < live[..., None]) & taken[:, None, None]
    cleared = ~held & (source != KEEP)[:, None, None]
    new = {}
    for name in ("K", "V"):
        new[name] = torch.where(held[..., None], src[name][at], dst[name])
    for name in ("s", "q", "n", "pos"):
        new[name] = torch.where(held, src[name][at], dst[name])
    new["pos"] = torch.where(cleared, -1, new["pos"])
    for name in ("live", "t_next"):
        new[name] = torch.where(taken[:, None], src[name][at], torch.where((source == FREE)[:, None], 0, dst[name]))
    for name in FIELDS:
        dst[name].copy_(new[name])
    return {name: dst[name] for name in FIELDS}


def _plain_linear_reorder(st):
    source = st["source"][:, None, None, None]
    new = torch.where(source >= 0, st["src"][st["source"].clamp_min(0).long()], torch.where(source == FREE, 0, st["dst"]))
    st["dst"].copy_(new)
    return {"state": st["dst"]}


# ------------------------------------------------------------------------------------------------ one pass

def _own(st):
    import paper_2402_06262_b200 as R
    c = st["case"]
    if c["op"] == "norm_rotate":
        if "handle" not in st:   # what a program makes once and keeps
            st["handle"] = R.Rotary(c["d"], st["freq"], pairing=R.ROCO_PAIR_HALVES if c["pairing"] == "halves" else R.ROCO_PAIR_ADJACENT,
                                    axes=c["axes"], axis=st["axis"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=st["eps"],
                                    status=st["status"])
        R.roco_norm_rotate(st["handle"], st["q"], st["k"], st["v"], st["Q"], st["K"], st["V"], lens=st["lens"], start=st["start"],
                           positions=st["positions"])
        return {"Q": st["Q"], "K": st["K"], "V": st["V"]}
    if c["op"] == "tree_verify":
        R.roco_tree_verify(st["target"], st["tokens"], st["parent"], st["accept_u"], st["sample_u"], st["path"], st["path_len"],
                           st["next_token"], st["status"], nodes=st["nodes"], draft=st["draft"], target_prefix=st["target_prefix"],
                           draft_prefix=st["draft_prefix"], distinct=c["drafts"] == "distinct")
        return {"path": st["path"], "path_len": st["path_len"], "next_token": st["next_token"]}
    if c["op"] == "cache_reorder":
        if "handles" not in st:
            src = R.Cache.wrap(*(st["src"][f] for f in FIELDS), st["src"]["status"])
            st["handles"] = src, src if st["dst"] is st["src"] else R.Cache.wrap(*(st["dst"][f] for f in FIELDS), st["dst"]["status"])
        R.roco_cache_reorder(st["handles"][0], st["source"], st["handles"][1])
        return {name: st["dst"][name] for name in FIELDS}
    if "handles" not in st:
        src = R.LinearState.wrap(st["src"], st["log_decay"], torch.bfloat16, st["status"])
        st["handles"] = src, src if st["dst"] is st["src"] else R.LinearState.wrap(st["dst"], st["log_decay"], torch.bfloat16, st["status"])
    R.roco_linear_reorder(st["handles"][0], st["source"], st["handles"][1])
    return {"state": st["dst"]}


def run(st):
    if own:
        return _own(st)
    return {"norm_rotate": _plain_norm_rotate, "tree_verify": _plain_tree_verify, "cache_reorder": _plain_cache_reorder,
            "linear_reorder": _plain_linear_reorder}[st["case"]["op"]](st)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits

def _exact_norm_rotate(st, c):
    """Head after head, pairs as complex numbers."""
    S, G, group, d, rot = (c[k] for k in ("S", "G", "group", "d", "rot"))
    out = {}
    for name, x, w in (("Q", st["q"], st["q_weight"]), ("K", st["k"], st["k_weight"]), ("V", st["v"], None)):
        res = st[name].double()
        per = group if name == "Q" else 1
        for b in range(S):
            L = int(st["lens"][b])
            for h in range(x.shape[2]):
                y = x[b, :L, h].double()
                if w is not None:
                    y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / d + st["eps"]) * w.double()
                if name != "V":
                    base = 0 if st["start"] is None else int(st["start"][b])
                    cols = []
                    for a in range(c["axes"]):
                        cols.append(base + (torch.arange(L, device=DEV) if st["positions"] is None else st["positions"][b, :L, a]).double())
                    where = torch.stack(cols, -1)
                    pick = [0] * (rot // 2) if st["axis"] is None else st["axis"].tolist()
                    z = torch.complex(y[:, :rot // 2], y[:, rot // 2:rot]) if c["pairing"] == "halves" else torch.view_as_complex(
                        y[:, :rot].reshape(L, rot // 2, 2).contiguous())
                    t = where[:, pick] * st["freq"].double()
                    z = z * torch.polar(torch.ones_like(t), t)
                    y = y.clone()
                    y[:, :rot] = torch.cat((z.real, z.imag), -1) if c["pairing"] == "halves" else torch.view_as_real(z).reshape(L, rot)
                (res[b, h // per, :L, h % per] if name == "Q" else res[b, h, :L]).copy_(y)
        out[name] = res
    return out


def _exact_tree_verify(st, c):
    """The walk in its own words: normalised distributions, one sequence after the other."""
    S, T, V, A = (c[k] for k in ("S", "T", "V", "A"))
    path, length, nxt = torch.full((S, A), -1.0), torch.zeros(S), torch.full((S,), -1.0)
    parent, tokens, nodes = st["parent"].tolist(), st["tokens"].tolist(), st["nodes"].tolist()
    accept, sample = st["accept_u"].double().tolist(), st["sample_u"].double().tolist()
    for b in range(S):
        way, tip = [], -1
        if not c["prefix"]:
            if not nodes[b]:
                continue
            way, tip = [0], 0
        while True:
            p = (st["target_prefix"][b] if tip < 0 else st["target"][b, tip]).double()
            q = None if st["draft"] is None else (st["draft_prefix"][b] if tip < 0 else st["draft"][b, tip]).double().clone()
            whole, found = p.clone(), None
            kids = [i for i in range(tip + 1, nodes[b]) if parent[b][i] == tip] if len(way) < A else []
            for i in kids:
                x, u = tokens[b][i], accept[b][i]
                if q is None:
                    yes = u < float(p[x])
                    rest = p.clone()
                    rest[x] = 0
                else:
                    yes = u * float(q[x]) < float(p[x])
                    rest = (p - q).clamp_min(0)
                if yes:
                    found = i
                    break
                total = float(rest.sum())
                p = rest / total if total > 0 else rest
                if q is not None and c["drafts"] == "distinct":
                    keep = 1 - float(q[x])
                    q[x] = 0
                    q = q / keep if keep > 0 else q
            if found is None:
                break
            way.append(found)
            tip = found
        if float(p.sum()) <= 0:
            p = whole
        upto = torch.cumsum(p, 0)
        over = (upto > sample[b] * float(upto[-1])).nonzero()
        nxt[b] = int(over[0]) if len(over) else int((p > 0).nonzero()[-1])
        length[b] = len(way)
        path[b, :len(way)] = torch.tensor(way, dtype=torch.float32)
    return {"path": path.int().to(DEV), "path_len": length.int().to(DEV), "next_token": nxt.int().to(DEV)}


def _exact_cache_reorder(st, c):
    """Sequence after sequence, from a copy of what was there."""
    was = {name: st["src"][name] if st["dst"] is not st["src"] else st["src"][name].clone() for name in FIELDS}
    new = st["dst"]
    for b, a in enumerate(st["source"].tolist()):
        if a == KEEP:
            continue
        n = 0 if a == FREE else _live(c)[a]
        for name in FIELDS[:6]:
            if n:
                new[name][b, :, :n] = was[name][a, :, :n]
        new["pos"][b, :, n:] = -1
        for name in FIELDS[6:]:
            new[name][b] = 0 if a == FREE else was[name][a]
    return {name: new[name].double() if new[name].is_floating_point() else new[name] for name in FIELDS}


def _exact_linear_reorder(st, c):
    was = st["src"].clone()
    for b, a in enumerate(st["source"].tolist()):
        if a != KEEP:
            st["dst"][b] = 0 if a == FREE else was[a]
    return {"state": st["dst"].double()}


def exact(c, seed):
    return {"norm_rotate": _exact_norm_rotate, "tree_verify": _exact_tree_verify, "cache_reorder": _exact_cache_reorder,
            "linear_reorder": _exact_linear_reorder}[c["op"]](prepare(c, seed), c)
