"""AdamW with a global-norm limit, and its states in 8 bits.

TEST INFRASTRUCTURE ONLY (see the package docstring).

    t = step + 1,  g <- s g,  m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2
    p <- p - lr decay p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)

with s as in ``sgd``; nothing changes when the norm is not finite.  ``update`` is
float64.  ``encode`` and ``moments32`` are the definition of the 8-bit states to the
bit: each operation in float32 rounded by itself, the power of two of 256 elements,
the random bits of an element and the rounding with them.  ``least_root`` is what a
root that 8 bits kept as 0 counts as at least in the next step of its parameter.
"""
from __future__ import annotations

import math

import numpy as np

from . import sgd

F = np.float32


def update(p, g, m, v, step, lr, b1, b2, eps, decay, s, least=0.0):
    """One tensor in float64: new p, m, v.  ``least``: sqrt(v) in the parameter's step
    is this at least."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * s
    m = b1 * m + (1.0 - b1) * g
    v = b2 * v + (1.0 - b2) * g * g
    t = step + 1
    root = np.maximum(np.sqrt(v), least)
    p = p - lr * decay * p - lr / (1.0 - b1 ** t) * m / (root / np.sqrt(1.0 - b2 ** t) + eps)
    return p, m, v


def scale_of(grads, max_norm):
    """The norm and the scale of the gradients."""
    norm = sgd.global_norm(grads)
    return norm, sgd.clip_scale(norm, max_norm)


def mix(a):
    """32 random bits a number (uint32 arrays)."""
    a = np.asarray(a, np.uint32)
    with np.errstate(over="ignore"):
        a = a ^ (a >> np.uint32(16))
        a = a * np.uint32(0x6A09E667)
        a = a ^ (a >> np.uint32(15))
        a = a * np.uint32(0xBB67AE85)
        return a ^ (a >> np.uint32(16))


def random16(seed, t, tensor, n):
    """Two 16-bit numbers for each of n elements."""
    key = mix(mix(mix(np.uint32(seed)) ^ np.uint32(t & 0xffffffff)) ^ np.uint32(tensor))
    x = mix(np.arange(n, dtype=np.uint32) ^ key)
    return x & np.uint32(0xffff), x >> np.uint32(16)


def blocks(x):
    x = np.asarray(x, F)
    return np.pad(x, (0, -x.size % 256)).reshape(-1, 256)


def encode(x, rnd16):
    """float32 x [n] as e4m3 codes [n] and the powers of two of its blocks."""
    n = np.asarray(x).size
    b, rnd = blocks(x), np.pad(np.asarray(rnd16, np.uint32), (0, -n % 256)).reshape(-1, 256)
    a = np.minimum(np.abs(b), F(1.75 * 2.0 ** 127))
    E = np.maximum((a.max(1).view(np.uint32) + np.uint32(0x1FFFFF)) >> np.uint32(23), 9)
    scale = ((E - 8).astype(np.uint32) << np.uint32(23)).view(F)
    t = (a.astype(np.float64) / scale[:, None].astype(np.float64)).astype(F)   # exact, or below 2^-126
    bits, r = t.view(np.uint32), rnd << np.uint32(4)
    big = ((bits + r) >> np.uint32(20)) - np.uint32(960)
    small = ((t.astype(np.float64) * 2.0 ** 29).astype(np.uint64).astype(np.uint32) + r) >> np.uint32(20)
    code = np.where(bits >= np.uint32(121 << 23), big, small)
    code = code | np.where(b < 0, np.uint32(128), np.uint32(0))
    return code.astype(np.uint8).reshape(-1)[:n], scale


def decode(codes, scale):
    """float32 values of codes."""
    c = np.asarray(codes, np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0)) * np.where(c & 128, -1.0, 1.0)
    return (v * np.repeat(np.asarray(scale, np.float64), 256)[:c.size]).astype(F)


def least_root(codes, scale, b2):
    """float64, for each element: sqrt(b2) times the least root above 0 that its block can
    hold where the code of its own, before the step, is 0; else 0."""
    c = np.asarray(codes)
    return np.where(c == 0, math.sqrt(b2) * 2.0 ** -9 * np.repeat(np.asarray(scale, np.float64), 256)[:c.size], 0.0)


def moments32(g, m, v, b1, b2, s):
    """m and v after the step in float32, rounded after every operation."""
    g, m, v, b1, b2 = (np.asarray(a, F) for a in (g, m, v, b1, b2))
    c1, c2 = F(1.0 - float(b1)), F(1.0 - float(b2))
    with np.errstate(over="ignore"):
        g = g * F(s)
        return m * b1 + g * c1, v * b2 + (g * g) * c2
