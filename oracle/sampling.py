"""Token selection from a row of logits in fp64, by its definition (include/dgap.h).

In the row's descending order (equal logits by lower index), with weights
e^((z - z_max) / T): top-k keeps the first k, top-p the shortest beginning
holding at least p of their mass, min-p the elements of weight >= m; the token
is the first kept one with which the mass is more than u times the kept total.
"""
from __future__ import annotations

import math
from typing import Tuple

import numpy as np


def sample_row(z, T: float = 1.0, k: int = 0, p: float = 1.0, m: float = 0.0, u: float = 0.0) -> Tuple[int, float]:
    """(token, log-probability); (-1, nan) for a row without a token."""
    z = np.asarray(z, dtype=np.float64)
    if not (math.isfinite(T) and T >= 0) or any(math.isnan(x) for x in (p, m, u)) or np.isnan(z).any() \
            or (z == np.inf).any() or not np.isfinite(z).any():
        return -1, math.nan
    order = np.argsort(-z, kind="stable")
    if T == 0:
        return int(order[0]), 0.0
    w = np.exp((z[order] - z[order[0]]) / T)
    n = len(w) if k < 1 or k >= len(w) else k
    if m > 1:
        n = 1
    if p < 1:
        upto = np.cumsum(w[:n])
        n = max(1, int(np.searchsorted(upto, p * upto[-1], side="left")) + 1)
    n = max(1, min(n, int((w >= m).sum())))
    upto = np.cumsum(w[:n])
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24)
    at = int(np.searchsorted(upto, u * upto[-1], side="right"))
    return int(order[at]), math.log(w[at] / upto[-1])
