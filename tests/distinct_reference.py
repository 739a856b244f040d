"""Verification of siblings drawn without replacement in 64 bits on the CPU, by the definition in C, R and M, and the exact distribution
of the first token over all draws and random numbers.  Shares nothing with csrc/."""
from __future__ import annotations

import numpy as np

LITTLE = 3.0 / 16     # below it M is the sum of what was not rejected


class Node:
    """The tests behind one node: p, q rows in 64 bits."""

    def __init__(self, p, q):
        self.p, self.q, self.C, self.R, self.M, self.gone = p, q, 0.0, 1.0, 1.0, []

    def left(self):
        return np.maximum(self.p - self.C * self.q, 0)

    def accepts(self, x, u):
        """Whether x is accepted, and how near that was to going the other way, relative to the numbers it is formed of."""
        q = 0.0 if x in self.gone else self.q[x]
        a, b = u * q * self.R, max(self.p[x] - self.C * self.q[x], 0) * self.M
        scale = a + (self.p[x] + self.C * self.q[x]) * self.M
        return a < b, abs(a - b) / scale if scale > 0 and a != b else np.inf

    def reject(self, x):
        if self.M > 0:
            self.C += self.R / self.M
        if x not in self.gone:
            self.gone.append(x)
            self.M -= self.q[x]
        self.R = self.left().sum()
        if self.M < LITTLE:
            rest = self.q.copy()
            rest[self.gone] = 0
            self.M = rest.sum()


def verify(target, draft, target_prefix, draft_prefix, tokens, parent, accept_u, sample_u, A):
    """(path, next token, margin) of one sequence; target, draft [T][V], the prefix's rows [V] (None: node 0 is taken as it stands)."""
    path, tip, margin = [], -1, np.inf
    if target_prefix is None:
        path, tip = [0], 0
    while True:
        node = Node(*((target_prefix, draft_prefix) if tip < 0 else (target[tip], draft[tip])))
        taken = None
        for i in range(len(tokens)) if len(path) < A else ():
            if parent[i] != tip or (target_prefix is None and i == 0):
                continue
            yes, near = node.accepts(tokens[i], float(accept_u[i]))
            margin = min(margin, near)
            if yes:
                taken = i
                break
            node.reject(tokens[i])
        if taken is None:
            break
        path.append(taken)
        tip = taken
    left = node.left()
    if left.sum() == 0:
        left = node.p
    upto = np.cumsum(left)
    place = float(sample_u) * upto[-1]
    over = np.nonzero((upto > place) & (left > 0))[0]
    if place > 0:
        margin = min(margin, float(np.abs(upto - place).min()) / (node.p.sum() + node.C * node.q.sum()))
    return path, int(over[0]) if len(over) else int(np.nonzero(left > 0)[0][-1]), margin


def first_token(p, q, n):
    """The distribution of the first token that comes out, n siblings drawn from q (as a distribution) without replacement: every draw,
    random numbers integrated."""
    out = np.zeros(len(p))

    def go(chance, node, k):
        left = node.left()
        if k == n:
            out[:] += chance * (left if left.sum() > 0 else p) / (left.sum() if left.sum() > 0 else p.sum())
            return
        rest = q.copy()
        rest[node.gone] = 0
        for x in np.nonzero(rest)[0]:
            need = q[x] * node.R
            yes = min(1.0, left[x] * node.M / need) if need > 0 else 0.0
            each = chance * rest[x] / rest.sum()
            out[x] += each * yes
            if yes < 1:
                then = Node(p, q)
                then.C, then.R, then.M, then.gone = node.C, node.R, node.M, list(node.gone)
                then.reject(x)
                go(each * (1 - yes), then, k + 1)

    go(1.0, Node(p, q), 0)
    return out
