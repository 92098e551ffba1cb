"""What sdvg.h says of sdvg_sample_tokens, row by row in 64 bits on the host."""
import math

import numpy as np


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob) of one row of logits."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or x.max() == -np.inf:
        return -1, math.nan
    if not temperature > 0:
        return int(np.argmax(x)), 0.0
    top = x.max()
    there = np.flatnonzero(x > -np.inf)
    order = there[np.argsort(-x[there], kind="stable")]
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / temperature)) if top < np.inf else (x[order] == top).astype(np.float64)
    if 0 < top_k < len(x):
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        goal = top_p * math.fsum(w)
        n = int(np.argmax(np.cumsum(w) >= goal)) + 1 if np.cumsum(w)[-1] >= goal else len(w)
        order, w = order[:n], w[:n]
    if min_p > 0:
        n = max(1, int((w >= min(min_p, 1.0)).sum()))
        order, w = order[:n], w[:n]
    by_index = np.argsort(order)
    order, w = order[by_index], w[by_index]
    total = math.fsum(w)
    u = 0.0 if not u > 0 else min(float(u), 1 - 2.0**-24)
    over = np.cumsum(w) > u * total
    at = int(np.argmax(over)) if over.any() else int(np.flatnonzero(w)[-1])
    return int(order[at]), math.log(w[at] / total)
