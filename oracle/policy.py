"""Clipped policy loss with KL and entropy terms, float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

With l the log-probability of the row's action, r = exp(l - old), u = ref - l:

    row  = -min(r adv, clip(r, 1 - lo, 1 + hi) adv) + beta (exp(u) - 1 - u) - eta H
    loss = sum w row / sum w

The KL term counts only where beta is not 0 (its mean is formed either way).
Rows of weight 0 or with a negative action do not count (l and H are formed for
weight 0 all the same); a row of nothing but
-inf has l = -inf, H = 0 and adds nothing; an action past the vocabulary, a NaN
or +inf in a row that counts gives NaN.
"""
from __future__ import annotations

import numpy as np


def rows(logits, actions, weights=None):
    """Log-probabilities, entropies, probabilities, and which rows count and
    which have nothing to choose from."""
    x = np.asarray(logits, np.float64)
    R, V = x.shape
    w = np.ones(R) if weights is None else np.asarray(weights, np.float64)
    counts = (np.asarray(actions) >= 0) & (w != 0.0)
    l, H, P, dead = np.zeros(R), np.zeros(R), np.zeros((R, V)), np.zeros(R, bool)
    for r in range(R):
        a = int(actions[r])
        if a < 0:
            continue
        if a >= V or np.isnan(x[r]).any() or np.isposinf(x[r]).any():
            l[r] = H[r] = np.nan
            P[r] = np.nan
            continue
        m = x[r].max()
        if np.isneginf(m):
            l[r], dead[r] = -np.inf, True
            continue
        e = np.exp(x[r] - m)
        S = e.sum()
        P[r] = e / S
        l[r] = x[r, a] - m - np.log(S)
        on = e > 0.0
        H[r] = np.log(S) - (e[on] * (x[r][on] - m)).sum() / S
    return l, H, P, counts, dead, w


def loss(logits, actions, old, adv, ref=None, weights=None, lo=0.2, hi=0.2, beta=0.0, eta=0.0):
    """Returns dict(stats [6], logp, entropy, dlogits)."""
    l, H, P, counts, dead, w = rows(logits, actions, weights)
    R, V = P.shape
    W = w[counts].sum()
    sums, d = np.zeros(4), np.zeros((R, V))
    for r in range(R):
        if not counts[r] or dead[r]:
            continue
        ratio = np.exp(l[r] - old[r])
        free, cut = ratio * adv[r], np.clip(ratio, 1.0 - lo, 1.0 + hi) * adv[r]
        off = free > cut
        c, kl = (0.0 if off else -free), 0.0
        if ref is not None:
            u = ref[r] - l[r]
            kl = np.expm1(u) - u if u < np.inf else u
            if beta:
                c -= beta * np.expm1(u)
        sums += w[r] * np.array([-(cut if off else free), kl, H[r], float(off)])
        lp = np.where(P[r] > 0.0, np.log(np.where(P[r] > 0.0, P[r], 1.0)), 0.0) if not np.isnan(l[r]) else P[r]
        g = -c * P[r] + eta * P[r] * (lp + H[r])
        if actions[r] < V:
            g[actions[r]] += c
        d[r] = g * w[r] / W
    s = sums / W if W > 0.0 else sums
    total = s[0] + (beta * s[1] if ref is not None and beta else 0.0) - (eta * s[2] if eta else 0.0)
    return dict(stats=np.array([total, *s, W]), logp=l, entropy=H, dlogits=d)
