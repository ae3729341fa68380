"""One token from a row of logits by a uniform number, float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

Tokens are ordered by falling logit, equal ones by rising index.  Kept are those
among the first top_k, in the shortest run from the front with at least top_p of
their weight exp((x - max) / T) (the first one always), and of a weight of at least
min_p.  The token is the first one by index up to which the kept ones' weights pass
u times their sum.
"""
from __future__ import annotations

import math

import numpy as np


def kept(x, T=1.0, k=0, p=1.0, minp=0.0):
    """Indices of the tokens that are kept, rising, and their weights."""
    x = np.asarray(x, np.float64)
    live = [i for i in range(len(x)) if x[i] > -np.inf]
    live.sort(key=lambda i: (-x[i], i))
    if T == 0.0:
        live = live[:1]
        return np.array(live), np.ones(1)
    with np.errstate(under="ignore"):
        w = {i: math.exp((x[i] - x[live[0]]) / T) for i in live}
    if 0 < k:
        live = live[:k]
    if p < 1.0:
        total, run, mass = math.fsum(w[i] for i in live), [], 0.0
        for i in live:
            if run and mass >= p * total:
                break
            run.append(i)
            mass += w[i]
        live = run
    if minp > 0.0:
        live = [i for i in live if w[i] >= min(minp, 1.0)]
    live.sort()
    return np.array(live), np.array([w[i] for i in live])


def draw(x, u, T=1.0, k=0, p=1.0, minp=0.0):
    """token, log-probability in softmax(x), log-probability among the kept, how
    many are kept."""
    x = np.asarray(x, np.float64)
    if np.isnan(x).any() or np.isposinf(x).any() or any(math.isnan(v) for v in (u, T, p, minp)) or T < 0.0:
        return -1, math.nan, math.nan, 0
    if not (x > -np.inf).any():
        return -1, -math.inf, -math.inf, 0
    at, w = kept(x, T, k, p, minp)
    c = np.cumsum(w)
    full = np.flatnonzero(w > 0.0)
    j = int(np.searchsorted(c, min(max(u, 0.0), 1.0) * c[-1], side="right"))
    j = min(j, int(full[-1]))
    with np.errstate(over="ignore", under="ignore"):
        lse = math.log(np.exp(x - x.max()).sum())
    return int(at[j]), float(x[at[j]] - x.max() - lse), math.log(w[j] / c[-1]), len(at)
