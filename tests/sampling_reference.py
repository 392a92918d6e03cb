"""The next token of one row of logits by definition, in 64 bits: (token, log-probability)."""
import math

import numpy as np


def kept_mass(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Each token's weight, 0 where it is not kept; None where nothing can be drawn; an index where the likeliest is taken."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    if not (x > -np.inf).any():
        return None
    top = x.max()
    if not temperature > 0 or top_k == 1:
        return int(np.argmax(x))
    with np.errstate(invalid="ignore", over="ignore"):
        y = np.where(x == top, 0.0, np.where(np.isinf(x) | np.isinf(top), -np.inf, (x - top) / temperature))
    w = np.exp(y)
    order = np.argsort(-x, kind="stable")
    keep = np.ones(len(x), bool)
    if 0 < top_k < len(x):
        keep[order[top_k:]] = False
    if min_p > 0:
        keep &= (y >= math.log(min(min_p, 1.0)))
    w = np.where(keep, w, 0.0)
    if top_p < 1:
        s = w[order]
        c = np.cumsum(s)
        reached = int(np.searchsorted(c, max(top_p, 0.0) * c[-1], side="left"))     # first with cumulative >= top_p of all
        w[order[reached + 1:]] = 0.0
    return w


def pick(x, u, **kw):
    w = kept_mass(x, **kw)
    if w is None:
        return -1, -math.inf
    if isinstance(w, int):
        return w, 0.0
    c = np.cumsum(w)
    u = 0.0 if not u > 0 else u
    i = min(int(np.searchsorted(c, u * c[-1], side="right")), int(np.flatnonzero(w)[-1]))
    return i, math.log(w[i] / c[-1])
