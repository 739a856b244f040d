"""The largest calls: offsets beyond 32 bits in the projections, in the probabilities and in a cache that is reordered."""
import pytest
import torch

import paper_2402_06262_b200 as R

pytestmark = pytest.mark.gpu


def test_projections_beyond_two_to_the_32_bytes():
    """33000 tokens of 520 heads, 4.4 GB in and out: the last rows are those of a call of their own."""
    S, N, G, group, d = 3, 11000, 104, 3, 128
    x = torch.empty(S, N, G * 5, d, dtype=torch.bfloat16, device="cuda")
    for b in range(S):
        x[b].normal_()
    assert x.numel() * 2 > 2 ** 32
    rotary = R.Rotary(d, [1e4 ** (-i / 64) for i in range(64)], q_weight=torch.ones(d), k_weight=torch.ones(d))
    cut = lambda t: (t[:, :, :G * group], t[:, :, G * group:G * (group + 1)], t[:, :, G * (group + 1):])  # noqa: E731
    out = lambda s, n: (torch.zeros(s, G, n, group, d, dtype=torch.bfloat16, device="cuda"),  # noqa: E731
                        *(torch.zeros(s, G, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    start = torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")
    whole, part = out(S, N), out(1, 50)
    R.roco_norm_rotate(rotary, *cut(x), *whole, start=start)
    R.roco_norm_rotate(rotary, *cut(x[2:, N - 50:]), *part, start=start[2:] + N - 50)
    assert all(torch.equal(a[2:, :, N - 50:], b) for a, b in zip(whole, part))
    assert R.roco_rotary_device_status(rotary) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_probabilities_beyond_two_to_the_32_bytes(dtype):
    S, T, V = 70, 64, 250001
    torch.manual_seed(3)
    target = torch.zeros(S, T, V, dtype=dtype, device="cuda")
    assert target.numel() * target.element_size() > 2 ** 31
    # a chain that is accepted to its 16th node, whose row holds two tokens
    tokens = torch.randint(0, V, (S, T), dtype=torch.int32, device="cuda")
    target.scatter_(2, tokens.roll(-1, 1).long()[..., None], 1.0)
    lo, hi = torch.randint(0, V // 2, (S,), device="cuda"), torch.randint(V // 2, V, (S,), device="cuda")
    target[:, 15] = 0
    target[torch.arange(S), 15, lo], target[torch.arange(S), 15, hi] = 0.25, 0.75
    parent = torch.arange(-1, T - 1, dtype=torch.int32, device="cuda").repeat(S, 1)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    path, n, nxt, status = ints(S, 16), ints(S), ints(S), ints(1)
    u = torch.full((S, T), 0.999, device="cuda")
    for s, want in ((0.2499, lo), (0.2501, hi)):
        R.roco_tree_verify(target, tokens, parent, u, torch.full((S,), s, device="cuda"), path, n, nxt, status)
        assert n.tolist() == [16] * S and torch.equal(nxt.long(), want) and int(status) == 0
        assert path.tolist() == [list(range(16))] * S


def test_a_cache_beyond_two_to_the_32_bytes():
    """Ten sequences x 512 units x 4000 slots, 5.2 GB of keys: the last units of a cycle, and of a copy into a larger cache."""
    S, G, B, d = 10, 512, 4000, 128
    cache = R.Cache(S, G, B, d, torch.bfloat16)
    for t in (cache.K, cache.V):
        for b in range(S):
            t[b].normal_()
    assert cache.K.numel() * 2 > 2 ** 32
    cache.live.fill_(B)
    cache.live[9, 511] = B - 7
    cache.pos.copy_(torch.arange(B, device="cuda").expand(S, G, B))
    cache.s.uniform_()
    was = [(f[9, 511].clone(), f[0, 511].clone(), f[8, 3].clone()) for f in (cache.K, cache.V, cache.s)]
    source = torch.tensor([9, 0, 1, 2, 3, 4, 5, 6, 7, 8], dtype=torch.int32, device="cuda")
    R.roco_cache_reorder(cache, source)
    for f, (a, b, c) in zip((cache.K, cache.V, cache.s), was):
        assert torch.equal(f[0, 511, :B - 7], a[:B - 7]) and torch.equal(f[1, 511], b) and torch.equal(f[9, 3], c)
    assert int(cache.live[0, 511]) == B - 7 and cache.pos[0, 511, B - 7:].tolist() == [-1] * 7
    larger = R.Cache(2, G, B + 9, d, torch.bfloat16)
    R.roco_cache_reorder(cache, torch.tensor([0, 9], dtype=torch.int32, device="cuda"), larger)
    assert torch.equal(larger.K[0, 511, :B - 7], was[0][0][:B - 7]) and torch.equal(larger.V[1, 3, :B], was[1][2])
    assert R.roco_device_status(cache) == 0 and R.roco_device_status(larger) == 0
