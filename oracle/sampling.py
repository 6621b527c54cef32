"""Sampling under temperature, top-k, min-p and top-p, and the norm and clipping of gradients, in float64 numpy, straight
from their definitions: the oracle of the GPU kernels of the same names."""
from __future__ import annotations

import math

import numpy as np


def kept_tokens(x, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(indices kept, in the order of the logits; weights of all tokens, the largest 1) of one row."""
    x = np.asarray(x, np.float64)
    w = np.exp(scale * (x - x.max()))
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if top_k > 0:
        order = order[:top_k]
    order = [i for i in order if w[i] >= min_p]
    if top_p < 1:
        asked = top_p * math.fsum(w[i] for i in order)
        so_far, n = 0.0, 0
        while n < 1 or so_far < asked:
            so_far += w[order[n]]
            n += 1
        order = order[:n]
    return order, w


def sample(x, uniform, scale=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens, logp, log_kept) of the rows x [n, V]; every parameter is a number or a vector over the rows."""
    x = np.asarray(x, np.float64)
    n = len(x)
    scale, top_k, top_p, min_p = (np.broadcast_to(np.asarray(v, np.float64), n) for v in (scale, top_k, top_p, min_p))
    tokens, logp, log_kept = np.full(n, -1), np.full(n, np.nan), np.full(n, np.nan)
    for r in range(n):
        if np.isnan(x[r]).any() or np.isposinf(x[r]).any() or not 0 < scale[r] < np.inf:
            continue
        if np.isneginf(x[r]).all():
            logp[r], log_kept[r] = -np.inf, 0.0
            continue
        order, w = kept_tokens(x[r], scale[r], int(top_k[r]), top_p[r], min_p[r])
        total, chosen = math.fsum(w), np.sort(order)
        running = np.cumsum(w[chosen])  # its own end is the total that the random number is a share of
        tokens[r] = chosen[np.nonzero(running > uniform[r] * running[-1])[0][0]]
        logp[r] = scale[r] * (x[r, tokens[r]] - x[r].max()) - math.log(total)
        dropped = np.ones(len(w), bool)
        dropped[order] = False
        log_kept[r] = math.log1p(-math.fsum(w[dropped]) / total)
    return tokens, logp, log_kept


def grad_norm(tensors):
    return math.sqrt(math.fsum(float(v) ** 2 for t in tensors for v in np.asarray(t, np.float64).ravel()))


def grad_clip(tensors, norm, max_norm, eps=1e-6):
    factor = min(1.0, max_norm / (norm + eps))
    return [np.asarray(t, np.float64) * factor for t in tensors]
