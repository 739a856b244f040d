"""Inputs of the draft-tree tests, made on the CPU from a seed, and the library's calls on them."""
import dataclasses
from typing import List

import torch

import paper_2402_06262_b200 as R

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CACHE_FIELDS = ("K", "V", "s", "q", "n", "pos", "live", "t_next")


@dataclasses.dataclass
class Case:
    S: int
    G: int
    B: int
    d: int
    T: int
    group: int
    dtype: str
    live: List[int]        # per sequence
    nodes: List[int]
    t: dict                # CPU tensors

    def dev(self, name):
        return self.t[name].to("cuda")

    def cache(self) -> R.Cache:
        return R.Cache.wrap(*(self.dev(f) for f in CACHE_FIELDS), torch.zeros(1, dtype=torch.int32, device="cuda"))


def trees(S, T, gen, shape):
    """Parents: "random" (a tenth of the nodes hang on the prefix), "chain", "flat" (every node on the prefix)."""
    par = torch.full((S, T), -1, dtype=torch.int32)
    for b in range(S):
        for i in range(T):
            if shape == "chain":
                par[b, i] = i - 1
            elif shape == "random" and i and torch.rand((), generator=gen) > 0.1:
                par[b, i] = int(torch.randint(0, i, (), generator=gen))
    return par


def make(seed, S=1, G=2, B=64, d=128, T=4, group=1, dtype="bf16", live=None, nodes=None, shape="random", junk=float("nan"),
         key_scale=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    dt = DT[dtype]
    live = [B] * S if live is None else live
    nodes = [T] * S if nodes is None else nodes
    randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    t = dict(K=(randn(S, G, B, d) * key_scale).to(dt), V=randn(S, G, B, d).to(dt), Q=randn(S, G, T, group, d).to(dt),
             K_new=(randn(S, G, T, d) * key_scale).to(dt), V_new=randn(S, G, T, d).to(dt), parent=trees(S, T, g, shape))
    age = torch.stack([torch.randperm(B, generator=g) for _ in range(S * G)]).reshape(S, G, B)
    t["pos"] = (2 * age).to(torch.int32)
    t["t_next"] = torch.full((S, G), 2 * B + 3, dtype=torch.int32)
    t["n"] = (t["t_next"][..., None] - t["pos"]).to(torch.int32)
    mean = torch.exp(2 * randn(S, G, B)) / B
    t["s"] = (mean * t["n"]).float()
    t["q"] = (t["n"] * mean * mean * (1 + torch.rand(S, G, B, generator=g))).float()
    t["live"] = torch.tensor(live, dtype=torch.int32)[:, None].expand(S, G).contiguous()
    for b in range(S):     # what lies behind the last token or node must not matter
        for f in ("K", "V", "s", "q"):
            t[f][b, :, live[b]:] = junk
        t["n"][b, :, live[b]:] = -7
        t["pos"][b, :, live[b]:] = -1
        for f in ("Q", "K_new", "V_new"):
            t[f][b, :, nodes[b]:] = junk
    return Case(S, G, B, d, T, group, dtype, live, nodes, t)
