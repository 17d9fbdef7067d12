"""The preference loss over pairs of token sequences and its gradient, and gradient
clipping over many tensors, in float64."""
from __future__ import annotations

import numpy as np


def row_logps(logits, labels):
    """(log-probability of each row's label, log sum exp); 0 and 0 where the label is outside the vocabulary."""
    x = np.asarray(logits, dtype=np.float64)
    rows, vocab = x.shape
    lp, lse = np.zeros(rows), np.zeros(rows)
    with np.errstate(all="ignore"):
        for r in range(rows):
            if 0 <= labels[r] < vocab:
                top = np.max(x[r])
                ln = np.log(np.sum(np.exp(x[r] - top)))
                lse[r] = top + ln
                lp[r] = (x[r, labels[r]] - top) - ln     # apart from top, which may be far larger
    return lp, lse


def log_sigmoid(z):
    with np.errstate(all="ignore"):
        return np.minimum(z, 0.0) - np.log1p(np.exp(-np.abs(z)))


def preference(logits, labels, offsets, ref, beta, smoothing, scale):
    """losses [P], logps [2P], gradient of scale * sum(losses) by the logits."""
    x = np.asarray(logits, dtype=np.float64)
    rows, vocab = x.shape
    off = np.clip(np.asarray(offsets), 0, rows)
    seqs = len(off) - 1
    p = seqs // 2
    lp, lse = row_logps(x, labels)
    logps = np.array([np.sum(lp[off[s]:off[s + 1]]) for s in range(seqs)])
    with np.errstate(all="ignore"):
        ratio = logps - np.asarray(ref, dtype=np.float64)
        z = beta * (ratio[:p] - ratio[p:])
        losses = np.where(np.isnan(z), np.nan, 0.0)
        if smoothing < 1:
            losses = losses - (1 - smoothing) * log_sigmoid(z)
        if smoothing > 0:
            losses = losses - smoothing * log_sigmoid(-z)
        # sigma(z) - (1 - smoothing), without its cancellation where sigma(z) is close to 1
        w = scale * beta * (smoothing / (1 + np.exp(-z)) - (1 - smoothing) / (1 + np.exp(z)))
        w = np.concatenate([w, -w])
        grads = np.zeros((rows, vocab))
        for s in range(seqs):
            for r in range(off[s], off[s + 1]):
                if 0 <= labels[r] < vocab:
                    grads[r] = -w[s] * np.exp((x[r] - x[r, labels[r]]) + lp[r] if np.isfinite(lp[r]) else x[r] - lse[r])
                    grads[r, labels[r]] += w[s]
    return losses, logps, grads, w, lse


def clip(workers, max_norm):
    """Per worker: (norm over all its tensors, coefficient, clipped tensors)."""
    out = []
    with np.errstate(all="ignore"):
        for tensors in workers:
            norm = np.sqrt(sum(float(np.sum(np.asarray(t, dtype=np.float64) ** 2)) for t in tensors))
            c = max_norm / (norm + 1e-6) if max_norm else 1.0
            c = 1.0 if c > 1.0 else c
            out.append((norm, c, [np.asarray(t, dtype=np.float64) * c for t in tensors]))
    return out
