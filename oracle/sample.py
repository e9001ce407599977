"""The draw of a token from a row of logits (pipo_op_sample), in 64 bits."""
from __future__ import annotations

from typing import Tuple

import numpy as np


def sample(x: np.ndarray, u: float, T: float = 1.0, top_k: int = 0, top_p: float = 1.0,
           min_p: float = 0.0) -> Tuple[int, float]:
    """(token, log of its share of the kept weights)"""
    x = np.asarray(x, np.float32).astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return 0, -np.inf
    if not T > 0:
        return int(np.argmax(x)), 0.0
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    z = np.zeros(len(order))
    other = x[order] != top
    z[other] = (x[order][other] - top) / T
    w = np.exp(z)
    n = int((w > 0).sum())
    if top_k > 0:
        n = min(n, top_k)
    if min_p > 0:
        # (of the logarithms: a weight just under 1 rounds to 1)
        n = min(n, int((z >= np.log(min(min_p, 1.0))).sum()))
    run = np.cumsum(w[:n])
    if top_p < 1:
        n = min(n, int((run < max(top_p, 0.0) * run[-1]).sum()) + 1)
    total = run[n - 1]
    at = min(int((run[:n] <= np.clip(u, 0.0, 1.0) * total).sum()), n - 1)
    return int(order[at]), float(z[at] - np.log(total))
