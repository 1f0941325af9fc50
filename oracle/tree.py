"""Float64 CPU oracle of decoding with a tree of drafted tokens: cache entries, attention,
verification, rows as 8-bit integers.

TEST INFRASTRUCTURE ONLY. The product path never imports this module; only ``tests/``
does. Each function is the definition, written out with loops over sequences, nodes and
heads.
"""

from __future__ import annotations

import numpy as np

from .decode import argmax, draw, filtered_probs


def way_up(parents, i):
    """Node ``i`` and its ancestors; None where the tree does not have the node."""
    way = [i]
    while parents[way[-1]] != -1:
        p = parents[way[-1]]
        if not 0 <= p < way[-1]:
            return None
        way.append(int(p))
    return way


def attention(q, k, v, lengths, parents, scale=None):
    """``out [B, n, H, D]`` for ``q [B, n, H, D]`` over entries ``k``, ``v [B][t, Hk, D]``:
    the context's ``lengths[b]``, then the nodes'. Entries that are None are not there."""
    B, n, H, D = q.shape
    out = np.zeros(q.shape)
    scale = D ** -0.5 if scale is None else scale
    for b in range(B):
        if lengths[b] < 0:
            continue
        for i in range(n):
            way = way_up(parents[b], i)
            if way is None:
                continue
            ts = list(range(lengths[b])) + [lengths[b] + j for j in sorted(way)]
            ts = [t for t in ts if t < len(k[b]) and k[b][t] is not None]
            if not ts:
                continue
            kk, vv = np.array([k[b][t] for t in ts]), np.array([v[b][t] for t in ts])
            for h in range(H):
                hk = h // (H // kk.shape[1])
                z = scale * (kk[:, hk] @ q[b, i, h])
                w = np.exp(z - z.max())
                with np.errstate(invalid="ignore"):
                    out[b, i, h] = (w[:, None] * vv[:, hk]).sum(0) / w.sum()
    return out


def verify(target, tokens, parents, u_accept, u_sample, temperature, top_p, draft=None, greedy=False):
    """``(n_accepted [B], path [B, n], next_token [B])``."""
    B, n, V = target.shape
    n_acc, path, nxt = np.zeros(B, int), np.full((B, n), -1), np.zeros(B, int)
    for b in range(B):
        way = [0]
        while True:
            c = way[-1]
            children = [i for i in range(c + 1, n) if parents[b][i] == c]
            if greedy:
                y = argmax(target[b, c])
                taken = next((i for i in children if tokens[b][i] == y), None)
            else:
                p = filtered_probs(target[b, c], temperature, top_p)
                q = filtered_probs(draft[b, c], temperature, top_p) if draft is not None and children else None
                taken = None
                for i in children:
                    x = int(tokens[b][i])
                    here = 0 <= x < V
                    px = p[x] if here else 0.0
                    qx = 1.0 if draft is None else q[x] if here else 0.0
                    if float(u_accept[b][i]) * qx < px:
                        taken = i
                        break
                    if draft is None:
                        left = p.copy()
                        if here:
                            left[x] = 0.0
                    else:
                        left = np.maximum(p - q, 0.0)
                    if left.sum() > 0:
                        p = left / left.sum()
                if taken is None:
                    y = draw(p, float(u_sample[b]))
            if taken is None:
                break
            way.append(taken)
        n_acc[b], nxt[b] = len(way) - 1, y
        path[b, :len(way)] = way
    return n_acc, path, nxt


def quantize(x):
    """``(q [T, d], scale [T])`` of float32 rows (as float64 arrays of float32 or bf16 values)."""
    scale = np.float32(np.abs(x).max(1) / 127.0).astype(np.float64)
    q = np.zeros(x.shape)
    rows = scale > 0
    q[rows] = np.clip(np.rint(x[rows] / scale[rows, None]), -127, 127)
    return q, scale
