"""A step of speculative decoding with a tree of drafted tokens, in fp64. Test
infrastructure: used by tests/ only.

Eq. (mla_compact) with an additive mask that lets node t see the context, the nodes above
it and itself; verification of the tree against the target's probabilities by rejection
sampling with several candidates a node (each refusal leaves the residual distribution);
and the cache rows of the accepted path moved together.
"""
from __future__ import annotations

import numpy as np


def line_of(parents, t: int) -> list[int] | None:
    """Node t and the nodes above it, or None where one of them has no valid parent."""
    line = []
    while t >= 0:
        line.append(t)
        p = int(parents[t])
        if not -1 <= p < t:
            return None
        t = p
    return line


def attend_tree(q_lat, q_pe, C, K, parents, n: int, tau: float, values=None):
    """All T nodes' rows (q_lat [T, H, 512], q_pe [T, H, 64]) over a sequence whose rows C [L, 512]
    and K [L, 64] end with those of its n nodes: (out [T, H, 512], lse [T, H], the same with
    |C| in C's place, for error bounds). values: what is summed in C's place."""
    q_lat, q_pe, C, K = (np.asarray(x, np.float64) for x in (q_lat, q_pe, C, K))
    V = C if values is None else np.asarray(values, np.float64)
    T, H = q_lat.shape[:2]
    out, mass, lse = np.zeros((T, H, C.shape[1])), np.zeros((T, H, C.shape[1])), np.full((T, H), -np.inf)
    ctx = C.shape[0] - n
    for t in range(n):
        line = line_of(parents, t)
        if line is None:
            continue
        at = np.concatenate([np.arange(ctx), ctx + np.array(line, int)])
        S = tau * (q_lat[t] @ C[at].T + q_pe[t] @ K[at].T)
        top = S.max(1, keepdims=True)
        e = np.exp(S - top)
        den = e.sum(1, keepdims=True)
        out[t], mass[t] = (e / den) @ V[at], (e / den) @ np.abs(V[at])
        lse[t] = (top + np.log(den))[:, 0]
    return out, lse, mass


def verify_tree(target, draft, tokens, parents, n: int, u):
    """The walk through one tree: (kept nodes, next token). target, draft [T, V] (draft None: the
    drafts are certain); -1 as the next token where nothing is left to draw from. The normalised
    residuals are computed step by step, as the method has them."""
    target = np.asarray(target, np.float64)
    V = target.shape[1]
    u = np.clip(np.nan_to_num(np.asarray(u, np.float64), nan=0.0), 0.0, 1.0 - 2.0 ** -24)
    if n == 0:
        return [], -1
    path, cur = [0], 0
    while True:
        p, out = np.maximum(target[cur], 0.0), []  # (out: certain drafts that were refused)
        took = None
        for t in range(cur + 1, n):
            if int(parents[t]) != cur or not 0 <= int(tokens[t]) < V:
                continue
            x = int(tokens[t])
            q = np.eye(1, V, x)[0] if draft is None else np.asarray(draft[cur], np.float64)
            if u[t] * q[x] < p[x]:
                took = t
                break
            if draft is None:
                out.append(x)
                p = np.maximum(target[cur], 0.0)
                rest = 1.0 - p[sorted(set(out))].sum()  # (the row sums to one)
                p[out] = 0.0
            else:
                p = np.maximum(p - q, 0.0)
                rest = p.sum()
            p = p / rest if rest > 0 else 0.0 * p
        if took is None:
            s = p.sum()
            if not (s > 0 and np.isfinite(s)):
                return path, -1
            over = np.nonzero(np.cumsum(p) > u[0] * s)[0]
            return path, int(over[0]) if len(over) else int(np.nonzero(p > 0)[0][-1])
        path.append(took)
        cur = took
