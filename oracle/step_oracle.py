"""Plain CPU definitions of a step's operators around the tied weight, in 64 bits (log probabilities and their gradient,
root-mean-square norm and its gradient, gradient norm and clipping).  Test infrastructure: shares no code with the CUDA
library."""
from __future__ import annotations

import numpy as np


def log_probabilities(x, scale=1.0):
    """(log p [rows, vocab], lse, entropy, r) of softmax(scale x); r: the sum of exp(z) without the largest logit's 1."""
    x = np.asarray(x, np.float64)
    top = x.max(-1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        z = scale * (x - top)
        e = np.exp(z)
        first = np.argmax(x == top, axis=-1)
        others = e.copy()
        others[np.arange(len(x)), first] = np.where(np.isnan(top[:, 0]), np.nan, 0.0)
        r = others.sum(-1)
        log_p = z - np.log1p(r)[:, None]
        p = np.exp(log_p)
        entropy = -np.where(p > 0, p * log_p, np.where(np.isnan(p), np.nan, 0.0)).sum(-1)
        lse = scale * top[:, 0] + np.log1p(r)
    undefined = ~(top[:, 0] < np.inf)                                      # a NaN or +infinity in the row
    log_p[undefined], lse[undefined], entropy[undefined], r[undefined] = np.nan, np.nan, np.nan, np.nan
    empty = top[:, 0] == -np.inf
    log_p[empty], lse[empty], entropy[empty], r[empty] = -np.inf, -np.inf, 0.0, -1.0
    return log_p, lse, entropy, r


def top_tokens(x, n):
    """Indices of the n largest logits by value, then by index; -1 where nothing but -infinity and NaN is left."""
    out = np.full((len(x), n), -1)
    for i, row in enumerate(np.asarray(x, np.float64)):
        order = np.lexsort((np.arange(len(row)), -np.where(np.isnan(row), -np.inf, row)))[:n]
        order = order[row[order] > -np.inf]
        out[i, :len(order)] = order
    return out


def logits_gradient(x, targets, scale, dlogprob, dentropy):
    """The logits' gradient of sum(dlogprob * logprob + dentropy * entropy); rows whose derivatives are both zero are zero."""
    log_p, _, entropy, _ = log_probabilities(x, scale)
    p = np.exp(log_p)
    given = np.asarray(targets) >= 0
    weight = np.where(given, dlogprob, 0.0)
    with np.errstate(invalid="ignore"):
        g = -p * (weight[:, None] + np.asarray(dentropy)[:, None] * np.where(p > 0, log_p + entropy[:, None], 0.0))
    rows = np.flatnonzero(given)
    g[rows, np.asarray(targets)[rows]] += weight[rows]
    g *= scale
    g[(weight == 0) & (np.asarray(dentropy) == 0)] = 0.0
    g[np.max(np.asarray(x, np.float64), -1) == -np.inf] = 0.0
    return g


def rmsnorm(h, weight, eps):
    """(y, inv_rms)"""
    inv = 1.0 / np.sqrt((h * h).mean(-1) + eps)
    return h * inv[:, None] * weight, inv


def rmsnorm_gradient(dy, h, weight, inv, dsum):
    """(dx, dweight)"""
    u = h * inv[:, None]
    g = dy * weight
    return dsum + inv[:, None] * (g - u * (g * u).mean(-1, keepdims=True)), (dy * u).sum(0)


def clip(tensors, max_norm):
    """(norm, factor, scaled tensors)"""
    norm = float(np.sqrt(sum(float((np.asarray(t, np.float64) ** 2).sum()) for t in tensors)))
    factor = min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 0.0
    return norm, factor, [np.zeros_like(t) if factor == 0 else np.asarray(t, np.float64) * factor for t in tensors]
