"""Layer norm with a residual sum before it, float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).

    h = x + r,  mean = sum h / D,  rstd = 1 / sqrt(sum (h - mean)^2 / D + eps)
    y = (h - mean) rstd gamma + beta
    xh = (h - mean) rstd,  g = dy gamma
    dx = rstd (g - sum g / D - xh sum(g xh) / D) + dh
    dgamma = sum dy xh,  dbeta = sum dy    (over rows)

h is taken as given: the caller rounds the sum to the rows' type.
"""
from __future__ import annotations

import numpy as np


def forward(h, gamma=None, beta=None, eps=1e-5):
    h = np.asarray(h, np.float64)
    mean = h.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    y = (h - mean) * rstd
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return y, mean[:, 0], rstd[:, 0]


def backward(h, dy, gamma=None, dh=None, eps=1e-5):
    """dx, dgamma, dbeta."""
    dy = np.asarray(dy, np.float64)
    xh, _, rstd = forward(h, eps=eps)
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    if dh is not None:
        dx = dx + np.asarray(dh, np.float64)
    return dx, (dy * xh).sum(0), dy.sum(0)
