"""Divergence of rows of logits from a teacher's top entries, and its gradient, fp64 (test infrastructure).

p over a list's entries is the softmax of their logits over T, q the softmax of the row's logits over T:

  kl_r = sum_j p_j (ln p_j - ln q[id_j]),  loss = sum_r w_r kl_r,  dz_v = w_r / T (q_v - sum_{j: id_j = v} p_j)

A row of weight 0, or with no entry of positive probability, has kl 0 and no gradient.  An id of -1 is no entry.
"""
from __future__ import annotations

import math

import numpy as np


def distill(logits, ids, teacher, weights, rows=None, temperature=1.0):
    """(loss, kl [rows], dlogits [rows, vocab]), row by row and entry by entry."""
    n, vocab = logits.shape
    loss, kl, grad = 0.0, np.zeros(n), np.zeros((n, vocab))
    for r in range(n):
        w, at = float(weights[r]), r if rows is None else int(rows[r])
        entries = [(int(i), float(t) / temperature) for i, t in zip(ids[at], teacher[at]) if i >= 0 and t > -math.inf]
        if w == 0.0 or not entries:
            continue
        top = max(t for _, t in entries)
        total = sum(math.exp(t - top) for _, t in entries)
        z = np.asarray(logits[r], np.float64) / temperature
        z = z - z.max()      # before the sum's logarithm, which a large maximum would absorb
        lse = math.log(np.exp(z).sum())
        grad[r] = np.exp(z - lse)
        for i, t in entries:
            p = math.exp(t - top) / total
            if p > 0:
                kl[r] += p * (math.log(p) - (z[i] - lse))
            grad[r, i] -= p
        grad[r] *= w / temperature
        loss += w * kl[r]
    return loss, kl, grad
