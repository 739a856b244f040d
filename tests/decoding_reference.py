"""Norm and rotation of heads, verification of drafted trees and reordering of sequences in 64 bits on the CPU, straight from their
definitions, with bounds on what rounding may cost the library.  Test infrastructure: shares nothing with csrc/.

u32 = 2^-24 and u16 = 2^-8 are the largest relative errors of one rounding to fp32 and to bf16.
"""
from __future__ import annotations

import numpy as np
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
F64 = torch.float64


def rotate_row(x, weight, eps, rot, adjacent, angles):
    """One head of one token: x [d] (64 bits), angles [rot/2] (64 bits).  Returns (y, bound on the error before the last rounding).

    Norm: the sum of d squares in fp32 is off by (d + 1) u32 of itself, its root by half of that; mean and eps 2, rsqrt 4 (2 ulp),
    two products 2 u32.  Angles: in turns, three roundings to 64 bits (2^-51 of itself), then one to fp32 of a number up to 1 (times pi: under 4
    u32), sine and cosine 2 ulp (under 4 u32).  Each result is a sum of two products: 3 u32 of their magnitudes."""
    y = x.clone()
    d = x.shape[0]
    rel = 0.0
    if weight is not None:
        y = x / torch.sqrt((x * x).sum() / d + eps) * weight
        rel = (d / 2 + 10) * U32
    bound = y.abs() * rel
    if rot:
        h = rot // 2
        a = torch.arange(0, rot, 2) if adjacent else torch.arange(h)
        b = a + 1 if adjacent else a + h
        c, s = torch.cos(angles), torch.sin(angles)
        ya, yb = y[a], y[b]
        each = (ya.abs() + yb.abs()) * (rel + 11 * U32 + angles.abs() * 2.0 ** -50)
        y[a], y[b] = ya * c - yb * s, yb * c + ya * s
        bound[a], bound[b] = each, each
    return y, bound + 1e-38


def norm_rotate(x, heads_per_unit, weight, eps, rot, adjacent, freq, axis, start, positions, lens):
    """x [S][N][heads][d], positions [S][N][axes] -> (y, bound) [S][G][N][heads_per_unit][d], zero behind lens."""
    S, N, H, d = x.shape
    y, bound = (torch.zeros(S, H // heads_per_unit, N, heads_per_unit, d, dtype=F64) for _ in range(2))
    for b in range(S):
        for n in range(lens[b]):
            angles = torch.tensor([(start[b] + int(positions[b, n, axis[i]])) * float(freq[i]) for i in range(rot // 2)], dtype=F64)
            for h in range(H):
                at = b, h // heads_per_unit, n, h % heads_per_unit
                y[at], bound[at] = rotate_row(x[b, n, h].double(), weight, eps, rot, adjacent, angles)
    return y, bound


class Walk:
    """One sequence's walk with normalised distributions.  margin: how near (relative to the probabilities' own size) a decision was
    to going the other way."""

    def __init__(self):
        self.path, self.next, self.margin = [], -1, float("inf")


def verify(target, draft, target_prefix, draft_prefix, tokens, parent, nodes, accept_u, sample_u, A, distinct):
    """target, draft [T][V] numpy rows in 64 bits (draft None: no probabilities), target_prefix None: node 0 is taken as it stands."""
    w = Walk()
    V = target.shape[1]
    ok = [0 <= tokens[i] < V and -1 <= parent[i] < i for i in range(nodes)]
    tip = -1
    if target_prefix is None:
        if not nodes or parent[0] != -1:
            return w
        w.path, tip = [0], 0
    while True:
        p = np.array(target_prefix if tip < 0 else target[tip], dtype=np.float64)
        q = None if draft is None else np.array(draft_prefix if tip < 0 else draft[tip], dtype=np.float64)
        whole, taken, seen = p.copy(), None, set()
        for i in range(nodes) if len(w.path) < A else ():
            if not ok[i] or parent[i] != tip or (target_prefix is None and i == 0):
                continue
            x, u = tokens[i], float(accept_u[i])
            if q is None:
                left, chance = (0.0 if x in seen else p[x]), 1.0
            else:
                left, chance = max(p[x], 0.0), (0.0 if distinct and x in seen else q[x])
            if u * chance != left or u * chance != 0:
                w.margin = min(w.margin, abs(u * chance - left) / (u * chance + left))
            if u * chance < left:
                taken = i
                break
            seen.add(x)
            if q is None:
                p[x] = 0
            else:
                p = np.maximum(p - q, 0)
                if distinct:
                    keep = 1 - chance if q[x] else 1.0
                    q[x] = 0
                    q = q / keep if keep > 0 else q * 0
            total = p.sum()
            p = p / total if total > 0 else p * 0
        if taken is None:
            break
        w.path.append(taken)
        tip = taken
    if p.sum() == 0:
        p = np.maximum(whole, 0)
    p = np.where(p <= 0, 0, p)
    total = p.sum()
    if not (0 < total < np.inf):
        return w
    upto = np.cumsum(p)
    place = float(sample_u) * upto[-1]
    over = np.nonzero((upto > place) & (p > 0))[0]
    w.next = int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])
    # (a place of exactly zero is before every token with any probability, however the sums are rounded)
    w.margin = min(w.margin, float(np.abs(upto - place).min() / upto[-1]) if place > 0 else float("inf"))
    return w


CACHE = ("K", "V", "s", "q", "n", "pos", "live", "t_next")


def reorder_cache(src, dst, source):
    """src, dst: dicts of CPU tensors (the same dict: in place).  Returns dst's new tensors."""
    S_src, G, B = src["K"].shape[:3]
    new = {f: dst[f].clone() for f in CACHE}
    for b, a in enumerate(source):
        if a == -2:
            new["pos"][b], new["live"][b], new["t_next"][b] = -1, 0, 0
        if not 0 <= a < S_src or (a == b and src is dst):
            continue
        for g in range(G):
            live = int(src["live"][a, g])
            if not 0 <= live <= B:
                continue
            for f in CACHE[:6]:
                new[f][b, g, :live] = src[f][a, g, :live]
            new["pos"][b, g, live:] = -1
            new["live"][b, g], new["t_next"][b, g] = live, src["t_next"][a, g]
    return new
