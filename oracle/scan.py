"""Selective scan over variable-length sequences, float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

    e = log(1 + exp(dt + dt_bias))  or  dt + dt_bias
    h_t[d, n] = exp(e A[d, n]) h_{t-1}[d, n] + e B_t[g, n] x_t[d]
    y_t[d] = (sum_n C_t[g, n] h_t[d, n] + Dskip[d] x_t[d]) z_t[d] s(z_t[d])

for t < len_b (g the group of channel d), y = 0 after, the state carried; one
step after the other as the imperative program would, the backward derived by
hand and run in reverse.
"""
from __future__ import annotations

import numpy as np


def _sig(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def _f(a):
    return None if a is None else np.asarray(a, np.float64)


def _wide(m, D):
    return np.repeat(m, D // m.shape[-2], axis=-2)


def _cells(x, dt, A, Bm, Cm, dt_bias, softplus, h, lengths):
    """States before every step and after the last, step sizes, running flags."""
    T, B, D = x.shape
    v = dt + (0.0 if dt_bias is None else dt_bias)
    e = np.logaddexp(0.0, v) if softplus else v
    de_dv = _sig(v) if softplus else np.ones_like(v)
    on = np.ones((T, B), bool) if lengths is None else np.arange(T)[:, None] < np.asarray(lengths)[None]
    hs = [h]
    for t in range(T):
        live = on[t][:, None, None]
        with np.errstate(invalid="ignore", over="ignore"):
            new = np.exp(e[t][..., None] * A) * h + (e[t] * x[t])[..., None] * _wide(Bm[t], D)
        h = np.where(live, new, h)
        hs.append(h)
    return hs, e, de_dv, on


def forward(x, dt, A, Bm, Cm, Dskip=None, z=None, dt_bias=None, lengths=None, h0=None, softplus=True):
    """Returns y [T, B, D], hT [B, D, N]."""
    x, dt, A, Bm, Cm, Dskip, z, dt_bias, h0 = map(_f, (x, dt, A, Bm, Cm, Dskip, z, dt_bias, h0))
    T, B, D = x.shape
    h0 = np.zeros((B, D, A.shape[1])) if h0 is None else h0
    hs, _, _, on = _cells(x, dt, A, Bm, Cm, dt_bias, softplus, h0, lengths)
    y = np.zeros((T, B, D))
    for t in range(T):
        r = (hs[t + 1] * _wide(Cm[t], D)).sum(-1) + (0.0 if Dskip is None else Dskip * x[t])
        y[t] = np.where(on[t][:, None], r if z is None else r * z[t] * _sig(z[t]), 0.0)
    return y, hs[-1]


def backward(x, dt, A, Bm, Cm, dy, Dskip=None, z=None, dt_bias=None, lengths=None, h0=None, dhT=None, softplus=True):
    """Returns a dict dx, ddt, dA, dBm, dCm, dDskip, dz, ddt_bias, dh0."""
    x, dt, A, Bm, Cm, dy, Dskip, z, dt_bias, h0, dhT = map(_f, (x, dt, A, Bm, Cm, dy, Dskip, z, dt_bias, h0, dhT))
    T, B, D = x.shape
    N, G = A.shape[1], Bm.shape[2]
    h0 = np.zeros((B, D, N)) if h0 is None else h0
    hs, e, de_dv, on = _cells(x, dt, A, Bm, Cm, dt_bias, softplus, h0, lengths)
    g = np.zeros((B, D, N)) if dhT is None else dhT
    o = dict(dx=np.zeros_like(x), ddt=np.zeros_like(x), dA=np.zeros_like(A), dBm=np.zeros_like(Bm),
             dCm=np.zeros_like(Cm), dDskip=np.zeros(D), ddt_bias=np.zeros(D),
             dz=None if z is None else np.zeros_like(x))
    for t in reversed(range(T)):
        r = on[t]
        if not r.any():
            continue
        c, b, xt, et = _wide(Cm[t], D)[r], _wide(Bm[t], D)[r], x[t][r], e[t][r]
        h, prev = hs[t + 1][r], hs[t][r]
        gy = dy[t][r]
        if z is not None:
            zt = z[t][r]
            q = _sig(zt)
            raw = (h * c).sum(-1) + (0.0 if Dskip is None else Dskip * xt)
            o["dz"][t][r] = gy * raw * q * (1.0 + zt * (1.0 - q))
            gy = gy * zt * q
        G_ = g[r] + gy[..., None] * c
        k = G_.shape[0]
        o["dCm"][t][r] = (gy[..., None] * h).reshape(k, G, D // G, N).sum(2)
        o["dBm"][t][r] = (G_ * (et * xt)[..., None]).reshape(k, G, D // G, N).sum(2)
        s = (G_ * b).sum(-1)
        w = G_ * np.exp(et[..., None] * A)
        q = w * prev
        o["dx"][t][r] = et * s + (0.0 if Dskip is None else Dskip * gy)
        ddt = (xt * s + (q * A).sum(-1)) * de_dv[t][r]
        o["ddt"][t][r] = ddt
        o["dA"] += (q * et[..., None]).sum(0)
        o["dDskip"] += (gy * xt).sum(0)
        o["ddt_bias"] += ddt.sum(0)
        g = g.copy()
        g[r] = w
    o["dh0"] = g
    return o


def step(x, dt, A, Bm, Cm, state, slots, Dskip=None, z=None, dt_bias=None, softplus=True):
    """One row per sequence ([B, D], [B, G, N]); state [n_slots, D, N] (not
    changed).  Returns y [B, D] and the new state."""
    state = np.array(state, np.float64)
    new, y = state.copy(), np.zeros(x.shape)
    for i, s in enumerate(slots):
        if 0 <= s < state.shape[0]:
            one = lambda a: None if a is None else a[None, i:i + 1]
            yi, hi = forward(one(x), one(dt), A, one(Bm), one(Cm), Dskip, one(z), dt_bias, None, state[s][None],
                             softplus)
            y[i], new[s] = yi[0, 0], hi[0]
    return y, new
