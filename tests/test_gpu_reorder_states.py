"""States of linear attention reordered in place: sequences that are freed and go on elsewhere, bit for bit."""
import pytest
import torch

import paper_2402_06262_b200 as R
from test_gpu_reorder import BAD_MAP, MAPS, ints, random_map

pytestmark = pytest.mark.gpu
FREE = R.ROCO_REORDER_FREE


def states(seed, S, G, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(S, G, d, d, device="cuda", generator=g)
    return R.LinearState.wrap(x, torch.zeros(G, device="cuda"), torch.bfloat16, ints([0]))


def reordered(x, source):
    """What the states x become."""
    new = x.clone()
    for b, a in enumerate(source):
        if 0 <= a < x.shape[0]:
            new[b] = x[a]
        elif a == FREE:
            new[b] = 0
    return new


def check(st, source, status=0):
    want = reordered(st.state, source)
    R.roco_linear_reorder(st, ints(source))
    assert torch.equal(st.state, want) and R.roco_linear_device_status(st) == status


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(MAPS))
def test_maps(d, name):
    for G in (1, 3, 40):
        check(states(G + d, 6, G, d), MAPS[name])


def compactions(S):
    """Sequences that end, at the front, at the back and in between, with the others moved up; forks of a sequence that is freed."""
    half = S // 2
    yield [S // 4] + [FREE] * (S - 1)
    yield list(range(half, S)) + [FREE] * half
    yield [b for b in range(S) if b % 3] + [FREE] * len([b for b in range(S) if b % 3 == 0])
    yield [FREE] * half + [0] * (S - half)
    yield [FREE if b % 2 == 0 else b - 1 for b in range(S)]
    yield [FREE] * S


# up to many more CTAs than reside at once, with one and several columns per thread, few and many distinct sources
@pytest.mark.parametrize("S,G,d", [(2, 2048, 64), (8, 512, 128), (16, 512, 64), (5, 37, 128), (20, 60, 128), (64, 40, 64), (256, 4, 64)])
def test_compactions_that_free_a_source(S, G, d):
    for i, source in enumerate(compactions(S)):
        st = states(i, S, G, d)
        for _ in range(3):
            check(st, source)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("S,G", [(8, 300), (16, 40), (33, 7), (100, 3)])
def test_any_map(d, S, G):
    for seed in range(6):
        check(states(seed, S, G, d), random_map(seed + S, S, S))


def test_bad_maps_are_flagged():
    check(states(1, 5, 8, 128), [5, -3, FREE, 2, 2 ** 31 - 1], BAD_MAP)


def test_another_stream_and_a_captured_call():
    st = states(2, 8, 64, 128)
    first, second = [4, 5, 6, 7] + [FREE] * 4, [1, FREE, 0, 0, FREE, 2, 3, 1]
    want = reordered(st.state, first)
    source = ints(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        R.roco_linear_reorder(st, source)
    side.synchronize()
    assert torch.equal(st.state, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.roco_linear_reorder(st, source)
        R.roco_linear_reorder(st, source)
    source.copy_(ints(second))          # the map is read at replay
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(st.state, reordered(reordered(want, second), second)) and R.roco_linear_device_status(st) == 0
