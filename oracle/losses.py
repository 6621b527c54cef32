"""Token log-probabilities, preference and policy losses in float64 numpy, straight from their
definitions (no running maxima, no shared sums): the oracle of the GPU kernels of the same names."""
from __future__ import annotations

import numpy as np


def token_logp(x, targets, scale=1.0):
    """(logp, entropy, stats [n, 2]) of float64 logits x [n, V]; targets outside [0, V) do not count."""
    x = np.asarray(x, np.float64)
    n, V = x.shape
    logp, entropy, stats = np.zeros(n), np.zeros(n), np.zeros((n, 2))
    with np.errstate(invalid="ignore", over="ignore"):
        for i, t in enumerate(targets):
            if not 0 <= t < V:
                continue
            m = x[i].max()
            if m == -np.inf:
                logp[i], stats[i] = -np.inf, (-np.inf, 0.0)
                continue
            z = scale * (x[i] - m)
            log_sum = np.log(np.exp(z).sum())
            p = np.exp(z - log_sum)
            logp[i] = z[t] - log_sum
            entropy[i] = -sum_of(np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, z - log_sum)))
            stats[i] = m, log_sum
    return logp, entropy, stats


def sum_of(v):
    return np.sum(v, dtype=np.float64)


def token_logp_grad(x, targets, grad_logp, grad_entropy=None, scale=1.0):
    """d(sum grad_logp * logp + grad_entropy * entropy) / dx."""
    x = np.asarray(x, np.float64)
    out = np.zeros_like(x)
    for i, t in enumerate(targets):
        if not 0 <= t < x.shape[1] or x[i].max() == -np.inf:
            continue
        z = scale * (x[i] - x[i].max())
        p = np.exp(z) / np.exp(z).sum()
        log_p = np.where(p > 0, z - np.log(np.exp(z).sum()), 0.0)
        one = np.arange(x.shape[1]) == t
        out[i] = grad_logp[i] * (one - p)
        if grad_entropy is not None:
            out[i] -= grad_entropy[i] * p * (log_p - (p * log_p).sum())
    return scale * out


def _segments(offsets, n):
    """Clamped [a, b) of every segment."""
    off = np.asarray(offsets, np.int64)
    a = np.clip(off[:-1], 0, n)
    return list(zip(a, np.clip(off[1:], a, n)))


def margins(logp, seq_offsets, ref_logp=None, mask=None, beta=0.1, mean=False):
    """(h, dh/dlogp of a counted token) of each sequence."""
    lp = np.asarray(logp, np.float64)
    h, w = [], []
    for a, b in _segments(seq_offsets, len(lp)):
        use = np.ones(b - a, bool) if mask is None else np.asarray(mask[a:b]) != 0
        v = lp[a:b][use] - (0.0 if ref_logp is None else np.asarray(ref_logp[a:b], np.float64)[use])
        w.append(beta / max(int(use.sum()), 1) if mean else beta)
        h.append(w[-1] * sum_of(v))
    return np.array(h), np.array(w)


def preference_loss(logp, seq_offsets, scores, group_offsets, ref_logp=None, mask=None, beta=0.1, smoothing=0.0,
                    grad_scale=1.0, mean=False):
    """(loss [n_groups], margins [n_seqs], gradient [n_tokens])."""
    h, w = margins(logp, seq_offsets, ref_logp, mask, beta, mean)
    slope = np.zeros(len(h))
    groups = _segments(group_offsets, len(h))
    loss = np.zeros(len(groups))
    for g, (a, b) in enumerate(groups):
        s = np.asarray(scores[a:b], np.float64)
        i, j = np.nonzero(s[:, None] > s[None, :])
        if not len(i):
            continue
        d = h[a + i] - h[a + j]
        loss[g] = np.mean((1 - smoothing) * np.logaddexp(0, -d) + smoothing * np.logaddexp(0, d))
        dl = (-(1 - smoothing) / (1 + np.exp(d)) + smoothing / (1 + np.exp(-d))) / len(i)
        np.add.at(slope, a + i, dl)
        np.add.at(slope, a + j, -dl)
    grad = np.zeros(len(np.asarray(logp)))
    for s, (a, b) in enumerate(_segments(seq_offsets, len(grad))):
        use = np.ones(b - a) if mask is None else (np.asarray(mask[a:b]) != 0).astype(np.float64)
        grad[a:b] = grad_scale * slope[s] * w[s] * use
    return loss, h, grad


def group_advantage(scores, group_offsets, eps, center_only=False):
    s = np.asarray(scores, np.float64)
    out = np.zeros(len(s))
    with np.errstate(invalid="ignore"):
        for a, b in _segments(group_offsets, len(s)):
            if b > a:
                out[a:b] = s[a:b] - s[a:b].mean() if np.isfinite(s[a:b]).all() else np.nan
                if not center_only:
                    out[a:b] /= s[a:b].std() + eps
    return out


def policy_loss(logp, old_logp, advantages, seq_offsets, ref_logp=None, mask=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                grad_scale=1.0, mean=False):
    """(loss [n_seqs], kl [n_seqs], gradient [n_tokens])."""
    lp = np.asarray(logp, np.float64)
    spans = _segments(seq_offsets, len(lp))
    loss, kl, grad = np.zeros(len(spans)), np.zeros(len(spans)), np.zeros(len(lp))
    with np.errstate(over="ignore"):
        for s, (a, b) in enumerate(spans):
            at = np.arange(a, b) if mask is None else a + np.nonzero(np.asarray(mask[a:b]))[0]
            A = float(advantages[s])
            share = 1.0 / max(len(at), 1) if mean else 1.0
            ratio = np.ones(len(at)) if old_logp is None else np.exp(lp[at] - np.asarray(old_logp, np.float64)[at])
            q = np.zeros(len(at)) if ref_logp is None else np.asarray(ref_logp, np.float64)[at] - lp[at]
            k = np.where(np.isposinf(q), np.inf, np.expm1(q) - np.where(np.isposinf(q), 0.0, q))
            edge = 1 + clip_high if A >= 0 else 1 - clip_low
            out = ratio > edge if A >= 0 else ratio < edge
            gain = np.where(out, edge, ratio) * A
            loss[s] = share * sum_of((kl_coef * k if kl_coef else 0.0) - gain)
            kl[s] = share * sum_of(k)
            pull = kl_coef * np.expm1(q) if kl_coef else 0.0
            grad[at] = grad_scale * share * (-np.where(out, 0.0, A * np.where(out, 0.0, ratio)) - pull)
    return loss, kl, grad
