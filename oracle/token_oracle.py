"""CPU oracle for the losses on token logits and for clipping by the global gradient norm.

TEST INFRASTRUCTURE ONLY: plain float64 statements of what the CUDA library computes, sharing no code with it.

    lp_i = z_it - log sum_j exp z_ij,   z = logit_scale * y[:, :vocab]
    d lp_i / d y_ij = logit_scale * ([j = t] - p_ij)

Rows of weight 0 or with a target outside [0, vocab) are left out.
"""
from __future__ import annotations

import numpy as np


def live_rows(targets, weights, vocab):
    t = np.asarray(targets)
    return (t >= 0) & (t < vocab) & (np.asarray(weights) != 0)


def log_probs(y, targets, vocab, scale, live):
    """lp of the live rows (0 elsewhere) and the softmax of those rows."""
    M = y.shape[0]
    lp = np.zeros(M)
    p = np.zeros((M, vocab))
    for i in np.flatnonzero(live):
        z = scale * np.asarray(y[i, :vocab], dtype=np.float64)
        z = z - z.max()
        e = np.exp(z)
        p[i] = e / e.sum()
        lp[i] = z[targets[i]] - np.log(e.sum())
    return lp, p


def logit_grad(y, targets, vocab, scale, live, p, coef):
    g = np.zeros((y.shape[0], y.shape[1]))
    for i in np.flatnonzero(live):
        g[i, :vocab] = -coef[i] * scale * p[i]
        g[i, targets[i]] += coef[i] * scale
    return g


def policy(y, targets, weights, adv, old, ref, vocab, scale, lo, hi, beta):
    """(stats[4], lp, dY, c): the clipped policy loss with its KL term; old / ref may be None."""
    live = live_rows(targets, weights, vocab)
    lp, p = log_probs(y, targets, vocab, scale, live)
    w = np.where(live, weights, 0.0).astype(np.float64)
    r = np.where(live, np.exp(lp - (lp if old is None else old)), 1.0)
    rc = np.clip(r, 1 - lo, 1 + hi)
    first, second = r * adv, rc * adv
    clipped = (first > second) & live
    if ref is None:
        kl, dkl = np.zeros_like(lp), np.zeros_like(lp)
    else:
        d = np.where(live, ref - lp, 0.0)
        with np.errstate(over="ignore"):
            grown = np.exp(d)
        kl, dkl = np.where(d == np.inf, np.inf, grown - 1 - np.where(d == np.inf, 0.0, d)), 1 - grown
    slope = np.where(clipped, 0.0, -first)
    if beta:                                     # a divergence that is reported only may be infinite
        slope = slope + beta * dkl
    coef = w * slope
    part1, part2 = -(w * np.minimum(first, second)).sum(), np.where(w != 0, w * np.where(w != 0, kl, 0.0), 0.0).sum()
    stats = np.array([part1 + beta * part2 if beta else part1, part1, part2, (w * clipped).sum()])
    return stats, lp, logit_grad(y, targets, vocab, scale, live, p, coef), coef


def pair_loss(x, kind, beta, eps):
    """Loss of one pair and its slope in x."""
    if kind == 0:
        up, down = np.logaddexp(0, -x), np.logaddexp(0, x)       # -log sigmoid(x), -log sigmoid(-x)
        return (1 - eps) * up + (eps * down if eps else 0.0), -(1 - eps) * np.exp(-np.logaddexp(0, x)) + eps * np.exp(-np.logaddexp(0, -x))
    if kind == 1:
        h = x / beta - 1 / (2 * beta)
        return h * h, 2 * h / beta
    return max(0.0, 1 - x), (-1.0 if x < 1 else 0.0)


def preference(y, targets, weights, begin, ref, vocab, scale, kind, beta, eps):
    """(stats[4], S, dY, c)"""
    M = y.shape[0]
    P = (len(begin) - 1) // 2
    w = np.ones(M) if weights is None else np.asarray(weights, dtype=np.float64)
    inside = np.zeros(M, dtype=bool)
    b = [min(max(int(v), 0), M) for v in begin]
    for q in range(2 * P):
        inside[b[q]:max(b[q], b[q + 1])] = True
    live = live_rows(targets, np.where(inside, w, 0.0), vocab)
    lp, p = log_probs(y, targets, vocab, scale, live)
    S = np.zeros(2 * P)
    for q in range(2 * P):
        rows = np.arange(b[q], max(b[q], b[q + 1]))
        rows = rows[live[rows]]
        S[q] = (w[rows] * lp[rows]).sum()
    reward = beta * (S - (0.0 if ref is None else np.asarray(ref, dtype=np.float64)))
    coef = np.zeros(M)
    losses, wins = [], []
    for k in range(P):
        x = reward[2 * k] - reward[2 * k + 1]
        loss, dx = pair_loss(x, kind, beta, eps)
        losses.append(loss)
        wins.append(float(x > 0))
        for q, sign in ((2 * k, 1.0), (2 * k + 1, -1.0)):
            rows = np.arange(b[q], max(b[q], b[q + 1]))
            rows = rows[live[rows]]
            coef[rows] = sign * beta * dx / P * w[rows]
    stats = np.array([np.mean(losses), reward[0::2].mean(), reward[1::2].mean(), np.mean(wins)])
    return stats, S, logit_grad(y, targets, vocab, scale, live, p, coef), coef


def clip_factor(grads, max_norm):
    """(norm, factor) over a list of arrays."""
    norm = float(np.sqrt(sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads)))
    if not np.isfinite(norm):
        return norm, 0.0
    return norm, (max_norm / norm if norm > max_norm else 1.0)
