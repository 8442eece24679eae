"""Float64 numpy definitions of the operators at the vocabulary ends of a stack: scaled embedding and its gradient, top
logits of a row, distillation loss and its gradient.  Written from the formulas; shares no code with the GPU path."""
from __future__ import annotations

import numpy as np


def embed_fwd(tokens, table, scale=1.0):
    ids = np.clip(tokens, 0, table.shape[0] - 1)
    return scale * table[ids]


def embed_bwd(tokens, dx, vocab, scale=1.0):
    d = np.zeros((vocab, dx.shape[-1]))
    np.add.at(d, np.clip(tokens, 0, vocab - 1).reshape(-1), scale * dx.reshape(-1, dx.shape[-1]))
    return d


def top_logits(logits, k):
    """(values, ids): descending, equal ones by ascending id, NaN above everything."""
    x = np.where(np.isnan(logits), np.inf, logits)
    ids = np.stack([np.lexsort((np.arange(r.size), -r, ~np.isnan(l)))[:k] for r, l in zip(x, logits)])
    return np.take_along_axis(logits, ids, 1), ids


def _lse(x):
    m = x.max(-1)
    return m + np.log(np.exp(x - m[..., None]).sum(-1))


def teacher_probs(t, ids, vocab, temperature):
    """[rows, K] probabilities over the entries that count (0 for the others), and whether a row has any."""
    on = (ids >= 0) & (ids < vocab)
    s = np.where(on, t / temperature, -np.inf)
    m = s.max(1)
    has = m > -np.inf
    w = np.exp(s - np.where(has, m, 0.0)[:, None])
    w = np.where(on, w, 0.0)
    tot = w.sum(1)
    return np.where(has[:, None], w / np.where(has, tot, 1.0)[:, None], 0.0), has


def distill_loss(logits, targets, t, ids, temperature=1.0, soft=1.0, z_loss=0.0, want_grad=True):
    """(mean loss, row losses, gradient of the mean).  targets None: every row counts."""
    x = np.asarray(logits, np.float64)
    rows, vocab = x.shape
    counted = np.ones(rows, bool) if targets is None else (targets >= 0) & (targets < vocab)
    n = max(int(counted.sum()), 1)
    row = np.zeros(rows)
    grad = np.zeros_like(x)
    p, has = teacher_probs(np.asarray(t, np.float64), ids, vocab, temperature)
    for r in np.flatnonzero(counted):
        m = x[r].max()
        d = x[r] - m  # (relative to the largest: next to 1e38 the sum's logarithm would be lost)
        log_s, log_st = _lse(d), _lse(d / temperature)
        lse = m + log_s
        row[r] = z_loss * lse ** 2 if z_loss else 0.0
        if soft < 1:
            row[r] += (1 - soft) * (log_s - d[targets[r]])
        pos = p[r] > 0
        if soft > 0 and has[r]:
            at = ids[r][pos]
            row[r] += soft * temperature ** 2 * np.sum(p[r][pos] * (np.log(p[r][pos]) - (d[at] / temperature - log_st)))
        if want_grad:
            g = np.exp(d - log_s) * (1 - soft + 2 * z_loss * lse)
            if soft < 1:
                g[targets[r]] -= 1 - soft
            if has[r]:
                g += soft * temperature * np.exp(d / temperature - log_st)
                np.add.at(g, ids[r][pos], -soft * temperature * p[r][pos])
            grad[r] = g / n
    return row.sum() / n, row, grad
