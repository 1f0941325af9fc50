"""Float64 CPU oracle of the post-training operators: layer norm, token
log-probabilities, the clipped policy loss and gradient clipping.

TEST INFRASTRUCTURE ONLY. The product path never imports this module; only
``tests/`` does. Each function is the definition, written out; the gradients are
pinned by central differences in ``tests/test_post_oracle.py``.
"""

from __future__ import annotations

import math

import numpy as np


def layer_norm(x, w, b=None, eps=1e-5):
    mu = x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
    y = (x - mu) * r * w
    return y if b is None else y + b


def layer_norm_backward(x, w, g_y, eps=1e-5):
    """``(g_x, g_w, g_b)``."""
    mu = x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt(((x - mu) ** 2).mean(1, keepdims=True) + eps)
    xh = (x - mu) * r
    u = g_y * w
    g_x = r * (u - u.mean(1, keepdims=True) - xh * (u * xh).mean(1, keepdims=True))
    return g_x, (g_y * xh).sum(0), g_y.sum(0)


def _log_softmax(z):
    m = z.max(1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(1, keepdims=True))


def token_logp(h, W, tokens, temperature=1.0, ignore_index=-100):
    """``(logp [T], entropy [T])``; a token outside [0, V) counts as ignored."""
    V = W.shape[0]
    logp, entropy = np.zeros(len(h)), np.zeros(len(h))
    rows = np.flatnonzero((tokens != ignore_index) & (tokens >= 0) & (tokens < V))
    if rows.size:
        lp = _log_softmax(h[rows] @ W.T / temperature)
        logp[rows] = lp[np.arange(rows.size), tokens[rows]]
        entropy[rows] = -(np.exp(lp) * lp).sum(1)
    return logp, entropy


def token_logp_backward(h, W, tokens, g, temperature=1.0, ignore_index=-100):
    """``(grad_h, grad_W)`` for the gradient ``g`` of the log-probabilities."""
    V = W.shape[0]
    gh, gW = np.zeros_like(h), np.zeros_like(W)
    rows = np.flatnonzero((tokens != ignore_index) & (tokens >= 0) & (tokens < V))
    if rows.size:
        G = -np.exp(_log_softmax(h[rows] @ W.T / temperature))
        G[np.arange(rows.size), tokens[rows]] += 1.0
        G *= (g[rows] / temperature)[:, None]
        gh[rows] = G @ W
        gW = G.T @ h[rows]
    return gh, gW


def policy(logp, old, adv, ref=None, mask=None, cu=None, per_sequence=False, clip_low=0.2, clip_high=0.2,
           kl_coef=0.0, reduction="token"):
    """``(loss, kl, clipped, gradient of logp)``, token by token."""
    n = len(logp)
    owner = np.zeros(n, dtype=int) if cu is None else np.full(n, -1)
    if cu is not None:
        for s in range(len(cu) - 1):
            owner[cu[s]:cu[s + 1]] = s
    counted = [t for t in range(n) if owner[t] >= 0 and (mask is None or mask[t])]
    per = {}
    for t in counted:
        per[owner[t]] = per.get(owner[t], 0) + 1
    loss, kl, clipped, grad = [], [], [], np.zeros(n)
    for t in counted:
        w = 1.0 / len(counted) if reduction == "token" else 1.0 / (len(per) * per[owner[t]])
        a = adv[owner[t]] if per_sequence else adv[t]
        r = math.exp(logp[t] - old[t])
        free, bound = r * a, min(max(r, 1.0 - clip_low), 1.0 + clip_high) * a
        loss.append(-w * min(free, bound))
        clipped.append(w if free > bound else 0.0)
        grad[t] = 0.0 if free > bound else -w * free
        if ref is not None:
            d = ref[t] - logp[t]
            kl.append(w * (math.exp(d) - d - 1.0))
            loss.append(kl_coef * kl[-1])
            grad[t] += w * kl_coef * (1.0 - math.exp(d))
    return math.fsum(loss), math.fsum(kl), math.fsum(clipped), grad


def clip(grads, max_norm):
    """``(norm, scaled gradients)``."""
    norm = math.sqrt(math.fsum(float((g.astype(np.float64) ** 2).sum()) for g in grads))
    c = min(1.0, max_norm / norm) if norm > 0 and math.isfinite(norm) else 1.0
    return norm, [g * c for g in grads]
