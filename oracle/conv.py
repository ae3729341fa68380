"""Short causal convolution over variable-length sequences, float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

    p_t[d] = bias[d] + sum_k w[d, k] x_{t-K+1+k}[d],   y = p or p s(p)

for t < len_b, with the carried state (the K - 1 inputs before t = 0, oldest
first) in front of the sequence; y is 0 from len_b on.  The loop runs over
sequences and time steps as the imperative program would; the backward is
derived by hand from the same sums.
"""
from __future__ import annotations

import numpy as np


def _sig(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def _seq(x, s0, b, n, K):
    """[K - 1 + n, D] inputs of sequence b with its state in front."""
    D = x.shape[2]
    front = np.zeros((K - 1, D)) if s0 is None else np.asarray(s0[b], np.float64)
    return np.concatenate([front, np.asarray(x[:n, b], np.float64)])


def forward(x, lengths, w, bias, s0, silu):
    """x [T, B, D], w [D, K], bias [D] or None, s0 [B, K-1, D] or None.
    Returns y [T, B, D], sT [B, K-1, D]."""
    T, B, D = x.shape
    K = w.shape[1]
    w = np.asarray(w, np.float64)
    y, sT = np.zeros((T, B, D)), np.zeros((B, K - 1, D))
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        v = _seq(x, s0, b, n, K)
        for t in range(n):
            p = (w.T * v[t:t + K]).sum(0) + (0.0 if bias is None else bias)
            y[t, b] = p * _sig(p) if silu else p
        sT[b] = v[n:]
    return y, sT


def backward(x, lengths, w, bias, s0, silu, dy, dsT):
    """Returns dx, dw, dbias, ds0."""
    T, B, D = x.shape
    K = w.shape[1]
    w = np.asarray(w, np.float64)
    dx, dw, db, ds0 = np.zeros((T, B, D)), np.zeros((D, K)), np.zeros(D), np.zeros((B, K - 1, D))
    for b in range(B):
        n = T if lengths is None else int(lengths[b])
        v = _seq(x, s0, b, n, K)
        dv = np.zeros_like(v)
        if dsT is not None:
            dv[n:] += dsT[b]
        for t in range(n):
            g = np.asarray(dy[t, b], np.float64)
            if silu:
                p = (w.T * v[t:t + K]).sum(0) + (0.0 if bias is None else bias)
                q = _sig(p)
                g = g * q * (1.0 + p * (1.0 - q))
            dv[t:t + K] += w.T * g
            dw += (v[t:t + K] * g).T
            db += g
        ds0[b], dx[:n, b] = dv[:K - 1], dv[K - 1:]
    return dx, dw, db, ds0


def step(x, w, bias, state, slots, silu):
    """One row per sequence: x [B, D], state [n_slots, K-1, D] (not changed).
    Returns y [B, D] and the new state."""
    state = np.array(state, np.float64)
    new, y = state.copy(), np.zeros(x.shape)
    for b, s in enumerate(slots):
        if 0 <= s < state.shape[0]:
            yb, sb = forward(x[None, b:b + 1], None, w, bias, state[s][None], silu)
            y[b], new[s] = yb[0, 0], sb[0]
    return y, new
