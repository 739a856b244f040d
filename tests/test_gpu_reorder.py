"""Sequences of a cache and of linear states forked, reordered, compacted and freed: bit for bit."""
import pytest
import torch

import paper_2402_06262_b200 as R
import decoding_reference as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BAD_LIVE, BAD_MAP = 2, 64


def fields(seed, S, G, B, d, dtype, live=None):
    g = torch.Generator()
    g.manual_seed(seed)
    t = {f: torch.randn(S, G, B, d, generator=g).to(DT[dtype]) for f in ("K", "V")}
    t.update({f: torch.rand(S, G, B, generator=g) for f in ("s", "q")})
    t.update({f: torch.randint(0, 10 ** 6, (S, G, B), generator=g, dtype=torch.int32) for f in ("n", "pos")})
    t["live"] = torch.randint(0, B + 1, (S, G), generator=g, dtype=torch.int32) if live is None else torch.tensor(
        live, dtype=torch.int32)[:, None].expand(S, G).contiguous()
    t["t_next"] = torch.randint(B, 10 ** 6, (S, G), generator=g, dtype=torch.int32)
    return t


def wrap(t):
    dev = {f: t[f].cuda() for f in ref.CACHE}
    return R.Cache.wrap(*(dev[f] for f in ref.CACHE), torch.zeros(1, dtype=torch.int32, device="cuda"))


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(cache, want):
    for f in ref.CACHE:
        assert torch.equal(getattr(cache, f).cpu(), want[f]), f


def random_map(seed, S_src, S_dst):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.randint(-2, S_src, (S_dst,), generator=g).tolist()


MAPS = {"keep": [-1] * 6, "itself": [0, 1, 2, 3, 4, 5], "fork": [0] * 6, "rotate": [1, 2, 3, 4, 5, 0], "swap": [1, 0, 3, 2, 5, 4],
        "chain": [0, 0, 1, 2, 3, 4], "back": [1, 2, 3, 4, 5, 5], "free": [-2, -2, -2, -2, -2, -2], "free a source": [3, -1, 3, -2, 0, -2],
        "mixed": [5, -1, 0, -2, 2, 2]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(MAPS))
def test_in_place(dtype, d, name):
    for B in (1, 33, 200):
        t = fields(B + d, 6, 3, B, d, dtype)
        c = wrap(t)
        R.roco_cache_reorder(c, ints(MAPS[name]))
        assert R.roco_device_status(c) == 0
        same(c, ref.reorder_cache(t, t, MAPS[name]))


@pytest.mark.parametrize("S,G,B,d,dtype", [(1, 1, 7, 64, "bf16"), (8, 32, 128, 128, "bf16"), (13, 5, 1001, 64, "f32"), (17, 2, 300, 128, "f32"),
                                           (40, 3, 65, 128, "bf16"), (100, 2, 50, 64, "bf16"), (256, 2, 30, 64, "f32"), (2, 1, 8192, 128, "bf16"),
                                           (3, 700, 40, 64, "bf16")])
def test_in_place_any_map(S, G, B, d, dtype):
    for seed in range(3):
        t = fields(seed, S, G, B, d, dtype)
        m = random_map(seed + S, S, S)
        c = wrap(t)
        R.roco_cache_reorder(c, ints(m))
        assert R.roco_device_status(c) == 0
        same(c, ref.reorder_cache(t, t, m))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,S2,G,B,B2,d", [(6, 6, 2, 50, 50, 128), (3, 9, 4, 33, 70, 64), (9, 2, 3, 200, 201, 128), (5, 300, 2, 20, 20, 64),
                                           (600, 400, 1, 9, 11, 64), (1, 1, 1, 1, 8192, 64)])
def test_into_another_cache(dtype, S, S2, G, B, B2, d):
    for seed in range(2):
        a, b = fields(seed, S, G, B, d, dtype), fields(seed + 50, S2, G, B2, d, dtype)
        m = random_map(seed + S, S, S2)
        src, dst = wrap(a), wrap(b)
        R.roco_cache_reorder(src, ints(m), dst)
        assert R.roco_device_status(src) == 0 and R.roco_device_status(dst) == 0
        same(dst, ref.reorder_cache(a, b, m))
        same(src, a)


def test_bad_maps_and_occupancies_are_flagged():
    S, G, B, d = 5, 2, 20, 64
    t = fields(1, S, G, B, d, "bf16")
    c = wrap(t)
    m = [5, -3, 0, 2 ** 31 - 1, -2 ** 31]
    R.roco_cache_reorder(c, ints(m))
    assert R.roco_device_status(c) == BAD_MAP
    same(c, ref.reorder_cache(t, t, [-1, -1, 0, -1, -1]))
    for into in (False, True):
        t = fields(2, S, G, B, d, "bf16")
        t["live"][3, 1], t["live"][1, 0] = B + 1, -1
        u = fields(3, S, G, B, d, "bf16")
        src, m = wrap(t), [3, 0, 1, -1, 2]
        dst = wrap(u) if into else src
        R.roco_cache_reorder(src, ints(m), dst if into else None)
        assert R.roco_device_status(dst) == BAD_LIVE
        same(dst, ref.reorder_cache(t, u if into else t, m))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("S,S2,G", [(1, 1, 1), (6, 6, 3), (20, 20, 2), (256, 256, 1), (4, 300, 2), (7, 3, 40)])
def test_linear_states(d, S, S2, G):
    g = torch.Generator()
    g.manual_seed(S + d)
    for into in (False, True) if S == S2 else (True,):
        x, y = torch.randn(S, G, d, d, generator=g), torch.randn(S2, G, d, d, generator=g)
        decay = torch.zeros(G, device="cuda")
        make = lambda t: R.LinearState.wrap(t.cuda(), decay, torch.bfloat16, torch.zeros(1, dtype=torch.int32, device="cuda"))  # noqa: E731
        src = make(x)
        dst = make(y) if into else src
        m = random_map(S + d, S, S2)
        R.roco_linear_reorder(src, ints(m), dst if into else None)
        want = (y if into else x).clone()
        for b, a in enumerate(m):
            if a >= 0:
                want[b] = x[a]
            elif a == -2:
                want[b] = 0
        assert torch.equal(dst.state.cpu(), want) and R.roco_linear_device_status(dst) == 0
        if into:
            assert torch.equal(src.state.cpu(), x)
            R.roco_linear_reorder(src, ints([S] * S2), dst)
            assert R.roco_linear_device_status(dst) == BAD_MAP and torch.equal(dst.state.cpu(), want)


def test_another_stream_and_a_captured_call():
    t = fields(4, 6, 4, 100, 128, "bf16")
    m, seq = MAPS["mixed"], MAPS["rotate"]
    c = wrap(t)
    source = ints(m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        R.roco_cache_reorder(c, source)
    side.synchronize()
    t = ref.reorder_cache(t, t, m)
    same(c, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.roco_cache_reorder(c, source)
        R.roco_cache_reorder(c, source)
    source.copy_(ints(seq))             # the map is read at replay
    graph.replay()
    torch.cuda.synchronize()
    for _ in range(2):
        t = ref.reorder_cache(t, t, seq)
    same(c, t)


def test_two_calls_at_once():
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    ts = [fields(30 + i, 8, 16, 300, 128, "bf16") for i in range(2)]
    caches, maps = [wrap(t) for t in ts], [random_map(3 + i, 8, 8) for i in range(2)]
    sources = [ints(m) for m in maps]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, s, side in zip(caches, sources, sides):
            with torch.cuda.stream(side):
                R.roco_cache_reorder(c, s)
    torch.cuda.synchronize()
    for t, c, m in zip(ts, caches, maps):
        for _ in range(3):
            t = ref.reorder_cache(t, t, m)
        same(c, t)
