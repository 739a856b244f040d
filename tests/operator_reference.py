"""The operators beside the budgeted cache in 64 bits on the CPU, straight from their definitions (one unit at a time),
with bounds on what rounding may cost the library.  Test infrastructure: shares nothing with csrc/.

Bounds.  u32 = 2^-24 and u16 = 2^-8 are the largest relative errors of one rounding to fp32 and to bf16.  A sum of n
products in fp32 is off by at most (n + 1) u32 times the sum of the products' magnitudes, whatever the order.
"""
from __future__ import annotations

import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
F64 = torch.float64


def ancestors(parent):
    """[T][T] truth values: row i marks node i's ancestors and itself."""
    T = len(parent)
    m = torch.zeros(T, T, dtype=torch.bool)
    for i in range(T):
        j = i
        while j >= 0:
            m[i, j] = True
            j = int(parent[j])
    return m


def score_error(q, k, scale):
    """Bound on the error of scale * q.k (natural units) formed in fp32, for rows q [R][d], keys k [J][d]: the sum, its
    scaling (by a factor that was itself rounded) and, in the exponential, one subtraction and the exponential's own error
    of at most 4 ulp."""
    d = q.shape[-1]
    return (abs(scale) * (q.abs() @ k.abs().T)) * (d + 4) * U32


def tree_attend(K, V, live, Q, K_new, V_new, parent, nodes, scale, low=False):
    """One unit.  K, V [B][d], Q [T][group][d], K_new, V_new [T][d] (64 bits).  Returns (out, lse, out_bound, lse_bound),
    the first two [nodes][group][d] and [nodes][group].  low: bf16 output and bf16 probabilities."""
    N, group, d = nodes, Q.shape[1], Q.shape[2]
    k = torch.cat((K[:live], K_new[:N]))
    v = torch.cat((V[:live], V_new[:N]))
    see = torch.cat((torch.ones(N, live, dtype=torch.bool), ancestors(parent[:N])), 1)
    see = see[:, None].expand(N, group, live + N).reshape(N * group, live + N)
    rows = Q[:N].reshape(N * group, d)
    # what a row does not see takes no part, whatever it holds
    kk, vv = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
    x = torch.where(see, rows @ kk.T * scale, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[:, None])
    out = p @ vv
    ex = torch.where(see, score_error(rows, kk, scale), 0).amax(-1)
    n = k.shape[0]
    # a probability: the error of its score and of the others' (through the sum), the exponential (2^-21), the sum
    ep = 2 * ex + 2.0 ** -21 + (n + 8) * U32
    mass = p @ vv.abs()
    ob = mass * (ep + (n + 8) * U32)[:, None] + out.abs() * 4 * U32 + 1e-30
    if low:
        ob = ob + U16 * mass + (U16 * (1 + U16)) * out.abs()
    lb = ex + 2.0 ** -21 + (n + 8) * U32 + 4 * U32 * lse.abs() + 4 * U32 * (x.masked_fill(~see, 0).abs().amax(-1))
    return (out.reshape(N, group, d), lse.reshape(N, group), ob.reshape(N, group, d), lb.reshape(N, group))


def scope_order(first, second):
    """Slots in (first, second) order."""
    return sorted(range(len(first)), key=lambda j: (float(first[j]), int(second[j])))


def victims(s, q, n, pos, need, r, lowest_r):
    """`need` slots by the rule of Sec. 4.3 on frozen statistics, one after the other, and the smallest relative margin of
    the decisions."""
    mean = s / n
    var = (q / n - mean * mean).clamp_min(0)
    left, gone, margin = list(range(len(s))), [], math.inf
    for _ in range(need):
        m = max(1, min(len(left), r if lowest_r else len(left) - r))
        by_var = sorted(left, key=lambda j: (float(var[j]), int(pos[j])))
        scope, out = by_var[:m], by_var[m:]
        by_mean = sorted(scope, key=lambda j: (float(mean[j]), int(pos[j])))
        v = by_mean[0]
        if len(by_mean) > 1:
            margin = min(margin, float((mean[by_mean[1]] - mean[v]) / (mean[by_mean[1]] + mean[v])))
        # a token outside with a lower mean, or the victim itself, must not be near the border of the scope
        if out:
            border = float(var[out[0]] + var[scope[-1]]) / 2
            for j in [v] + [j for j in out if float(mean[j]) <= float(mean[v])]:
                margin = min(margin, abs(float(var[j]) - border) / float(q[j] / n[j] + mean[j] ** 2 + 1e-300))
        gone.append(v)
        left.remove(v)
    return sorted(gone), margin


def tree_commit(st, Q, K_new, V_new, lse, path, r, lowest_r, scale):
    """One unit in place: st = dict of K, V [B][d], s, q [B] (64 bits), n, pos [B] and live, t_next.  Returns (evicted
    slots, their positions, margin, bound on s, bound on q)."""
    a, B, live = len(path), st["K"].shape[0], st["live"]
    sb, qb = torch.zeros(B, dtype=F64), torch.zeros(B, dtype=F64)
    if a == 0:
        return [], [], math.inf, sb, qb
    path = torch.as_tensor(path).long()

    def prob(keys):
        rows = Q[path]                                               # [a][group][d]
        x = torch.einsum("ahd,jd->ahj", rows, keys) * scale - lse[path][..., None]
        e = score_error(rows.reshape(-1, rows.shape[-1]), keys, scale).reshape(x.shape) + 4 * U32 * (
            x.abs() + lse[path][..., None].abs()) + 2.0 ** -21
        p = torch.exp(x)
        return p.mean(1), (p * e).mean(1) * 1.01

    p, ep = prob(st["K"][:live])
    pn, epn = prob(K_new[path])
    seen = torch.ones(a, a, dtype=torch.bool).tril()
    pn, epn = torch.where(seen, pn, 0), torch.where(seen, epn, 0)
    st["s"][:live] += p.sum(0)
    st["q"][:live] += p.pow(2).sum(0)
    st["n"][:live] += a
    sb[:live] = ep.sum(0) + (a + 20) * U32 * st["s"][:live]
    qb[:live] = (2 * p * ep).sum(0) * 1.01 + (a + 20) * U32 * st["q"][:live]
    need = max(0, live + a - B)
    gone, margin = victims(st["s"][:live], st["q"][:live], st["n"][:live].to(F64), st["pos"][:live], need, r, lowest_r)
    gone_pos = [int(st["pos"][j]) for j in gone]
    to = gone + list(range(live, live + a - need))
    for m, j in enumerate(to):
        st["K"][j], st["V"][j] = K_new[path[m]], V_new[path[m]]
        st["s"][j], st["q"][j] = pn[:, m].sum(), pn[:, m].pow(2).sum()
        sb[j] = epn[:, m].sum() + (a + 20) * U32 * st["s"][j]
        qb[j] = (2 * pn[:, m] * epn[:, m]).sum() * 1.01 + (a + 20) * U32 * st["q"][j]
        st["n"][j], st["pos"][j] = a - m, st["t_next"] + m
    st["live"] += a - need
    st["t_next"] += a
    return gone, gone_pos, margin, sb, qb


def linear(state, log_decay, q, k, v, scale, low=False):
    """One unit, token by token: state [d][d], q, k, v [L][d] (64 bits).  Returns (out, state, out_bound, state_bound).
    Bounds: every term decay^(i-j) (q_i.k_j) v_j (and the one of the first state) may have been rounded a few times to fp32
    in each of its factors and once more for every token that it stayed in the state; with low, in pieces on the tensor
    cores, the scores and the state enter one product as bf16; the keys of a state update are the sum of three bf16, which
    are all of an fp32."""
    g = math.exp(log_decay) if log_decay > -math.inf else 0.0
    S, A = state.clone(), state.abs()
    outs, mags = [], []
    for t in range(q.shape[0]):
        S = g * S + torch.outer(k[t], v[t])
        A = g * A + torch.outer(k[t].abs(), v[t].abs())
        outs.append(scale * (q[t] @ S))
        mags.append(abs(scale) * (q[t].abs() @ A))
    L, d = q.shape
    n = min(L, 1 / (1 - g) if g < 1 else L) + d + 150
    sb = A * (2 * n * U32) + 1e-30
    out = torch.stack(outs) if outs else q.new_zeros(0, d)
    mag = torch.stack(mags) if mags else q.new_zeros(0, d)
    ob = mag * (3 * n * U32 + (2 * U16 if low else 0)) + (2 * U32 + (U16 if low else 0)) * out.abs() + 1e-30
    return out, S, ob, sb
