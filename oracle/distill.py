"""CPU oracle: distillation of one row of joint logits from a teacher's top logits (TEST INFRASTRUCTURE ONLY).

With q = softmax(l / T) over the row's columns and p = softmax(t / T) over the teacher's entries whose column the
row has: loss = T^2 sum_j p_j (log p_j - log q_{id_j}), its derivative for l_c is T (q_c - sum of p_j over
id_j = c).  A row without columns of finite logit, or without a teacher entry of finite logit, has loss 0 and
gradient 0.  fp64, column by column.

Pins: tests/test_oracle_operators.py (differences of the loss, automatic differentiation in fp64, loss 0 where the
student is the teacher, duplicates, empty rows).
"""
from __future__ import annotations

import numpy as np


def row(l: np.ndarray, ids, t, T: float):
    """(loss, lse, gradient for l) of one row: l are the row's columns, ids / t the teacher's entries."""
    l = np.asarray(l, dtype=np.float64)
    ids, t = np.asarray(ids, dtype=np.int64), np.asarray(t, dtype=np.float64)
    grad = np.zeros(l.shape[0])
    if l.size == 0 or l.max() == -np.inf:
        return 0.0, -np.inf, grad
    m = l.max()
    s = np.exp((l - m) / T).sum()
    lse = m / T + np.log(s)
    keep = (ids >= 0) & (ids < l.shape[0]) & (t > -np.inf)
    ids, t = ids[keep], t[keep]
    if ids.size == 0:
        return 0.0, lse, grad
    x = (t - t.max()) / T
    p = np.exp(x) / np.exp(x).sum()
    logp = x - np.log(np.exp(x).sum())
    loss = 0.0
    for j in range(ids.size):
        if p[j] > 0:
            loss += p[j] * (logp[j] - ((l[ids[j]] - m) / T - np.log(s)))
    grad = np.exp((l - m) / T) / s
    for j in range(ids.size):
        grad[ids[j]] -= p[j]
    return T * T * loss, lse, T * grad
