"""The loss against a teacher's top logits and its gradient in fp64, by their
definition (include/dgap.h): q = softmax(t / T) over a row's entries,
p = softmax(z / T) over the vocabulary, loss = T^2 sum q (log q - log p_i),
gradient = T (p - q at its places)."""
from __future__ import annotations

import numpy as np


def distill_row(z, teacher, index, T: float):
    """(loss, lse, gradient) of one row for grad_loss = 1."""
    z = np.asarray(z, dtype=np.float64)
    have = [(float(t), int(i)) for t, i in zip(teacher, index) if 0 <= i < len(z) and t != -np.inf]
    x = z / T
    top = x.max()
    e = np.where(np.isneginf(x), 0.0, np.exp(x - top))
    lse = top + np.log(e.sum())
    if not have:
        return 0.0, lse, np.zeros_like(z)
    t = np.array([v for v, _ in have]) / T
    w = np.exp(t - t.max())
    q = w / w.sum()
    logq = t - t.max() - np.log(w.sum())
    grad = T * e / e.sum()
    loss = 0.0
    for k, (_, i) in enumerate(have):
        loss += q[k] * (logq[k] - x[i] + lse) if q[k] > 0 else 0.0
        grad[i] -= T * q[k]
    return T * T * loss, lse, grad
