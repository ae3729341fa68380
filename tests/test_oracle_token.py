"""Pins of the layer norm, sampling and AdamW oracles, each against something
that shares no code with it."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import adamw, norm, sample


@pytest.mark.parametrize("rows,D", [(1, 1), (3, 5), (4, 33)])
def test_norm_against_autograd_and_differences(rows, D):
    rng = np.random.default_rng(rows)
    h, dy, dh = (rng.normal(size=(rows, D)) for _ in range(3))
    ga, be = rng.normal(size=D), rng.normal(size=D)
    t = [torch.tensor(a, requires_grad=True) for a in (h, ga, be)]
    y = torch.nn.functional.layer_norm(t[0], (D,), t[1], t[2], 1e-5)
    ((y * torch.tensor(dy)).sum() + (t[0] * torch.tensor(dh)).sum()).backward()
    np.testing.assert_allclose(norm.forward(h, ga, be)[0], y.detach().numpy(), rtol=1e-12, atol=1e-12)
    got = norm.backward(h, dy, ga, dh)
    for a, b in zip(got, t):
        np.testing.assert_allclose(a, b.grad.numpy(), rtol=1e-9, atol=1e-9 * (1 + (D == 1) * 1e3))
    if D > 1:
        f = lambda: float((norm.forward(h, ga, be)[0] * dy).sum() + (h * dh).sum())
        e = 1e-6
        for i in itertools.product(range(rows), range(D)):
            h[i] += e
            up = f()
            h[i] -= 2 * e
            down = f()
            h[i] += e
            assert abs((up - down) / (2 * e) - got[0][i]) < 1e-6 * max(1.0, np.abs(got[0]).max())


def test_sample_frequencies_are_the_kept_ones_shares():
    """Over a fine grid of u each token comes up for its share of it."""
    x = np.array([0.3, 2.0, -np.inf, 2.0, -1.0, 1.1])
    n = 20000
    us = (np.arange(n) + 0.5) / n
    for T, k, p, minp in [(1.0, 0, 1.0, 0.0), (0.7, 3, 1.0, 0.0), (1.3, 0, 0.6, 0.0), (1.0, 0, 1.0, 0.3), (2.0, 4, 0.9, 0.2)]:
        w = np.exp((x - 2.0) / T)
        order = sorted(range(len(x)), key=lambda i: (-x[i], i))[:-1]
        if k:
            order = order[:k]
        share = np.cumsum([w[i] for i in order]) / sum(w[i] for i in order)
        order = [i for j, i in enumerate(order) if j == 0 or share[j - 1] < p]
        order = [i for i in order if w[i] >= minp]
        q = np.zeros(len(x))
        q[order] = w[order] / w[order].sum()
        got = [sample.draw(x, u, T, k, p, minp) for u in us]
        count = np.bincount([g[0] for g in got], minlength=len(x)) / n
        assert np.abs(count - q).max() <= 1.0 / n + 1e-12
        assert {g[3] for g in got} == {len(order)}
        for tok, lp, dl, _ in got[::997]:
            assert dl == pytest.approx(math.log(q[tok]), abs=1e-12)
            assert lp == pytest.approx(float(torch.log_softmax(torch.tensor(x), 0)[tok]), abs=1e-12)


def test_sample_ties_limits_and_bad_rows():
    x = np.zeros(10)
    assert sample.kept(x, k=3)[0].tolist() == [0, 1, 2]
    assert sample.kept(x, p=0.5)[0].tolist() == [0, 1, 2, 3, 4]
    assert sample.kept(x, p=0.0)[0].tolist() == [0]
    assert sample.kept(x, minp=7.0)[0].tolist() == list(range(10))
    assert sample.draw(x, 0.0)[0] == 0 and sample.draw(x, 1.0)[0] == 9 and sample.draw(x, -3.0)[0] == 0
    assert sample.draw([1.0, 3.0, 3.0], 0.9, T=0.0) == (1, pytest.approx(-math.log(2 + math.exp(-2))), 0.0, 1)
    assert sample.draw([1.0, 5.0, -np.inf], 0.999, T=math.inf)[0] == 1
    assert sample.draw([-np.inf] * 3, 0.5) == (-1, -math.inf, -math.inf, 0)
    for bad in ([0.0, np.nan], [np.inf, 0.0]):
        assert sample.draw(bad, 0.5)[0] == -1 and math.isnan(sample.draw(bad, 0.5)[1])
    assert sample.draw(x, math.nan)[0] == -1 and sample.draw(x, 0.5, T=-1.0)[0] == -1


@pytest.mark.parametrize("max_norm", [0.0, 0.5])
def test_adamw_against_torch(max_norm):
    rng = np.random.default_rng(1)
    p = [rng.normal(size=s) for s in (7, 20)]
    t = [torch.tensor(a, requires_grad=True) for a in p]
    opt = torch.optim.AdamW(t, lr=0.01, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    m, v = [np.zeros_like(a) for a in p], [np.zeros_like(a) for a in p]
    for step in range(5):
        g = [rng.normal(size=a.shape) for a in p]
        for a, b in zip(t, g):
            a.grad = torch.tensor(b)
        if max_norm:
            torch.nn.utils.clip_grad_norm_(t, max_norm)
        opt.step()
        s = adamw.scale_of(g, max_norm)[1]
        for i in range(2):
            p[i], m[i], v[i] = adamw.update(p[i], g[i], m[i], v[i], step, 0.01, 0.9, 0.99, 1e-8, 0.1, s)
            np.testing.assert_allclose(p[i], t[i].detach().numpy(), rtol=1e-10)


def test_codes_are_torchs_and_keep_what_they_hold():
    """Every code decodes to torch's e4m3 value; a value that a code holds comes
    back as that code whatever the random bits are, and the largest is at most 448."""
    every = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(every.copy()).view(torch.float8_e4m3fn).float().numpy()
    ok = (every & 127) != 127
    np.testing.assert_array_equal(adamw.decode(every, np.ones(1, np.float32))[ok], ref[ok])
    held = np.where(ok, ref, 0.0).astype(np.float32)
    for rnd in (0, 1, 0x7fff, 0xffff):
        for k in (-40, 0, 33):
            code, scale = adamw.encode(held * np.float32(2.0 ** k), np.full(256, rnd))
            assert scale[0] == 2.0 ** k
            np.testing.assert_array_equal(adamw.decode(code, scale), held * np.float32(2.0 ** k))
    x = np.random.default_rng(0).normal(size=4096).astype(np.float32)
    for rnd in (0, 0xffff):
        code, scale = adamw.encode(x, np.full(4096, rnd))
        assert np.isfinite(torch.from_numpy(code).view(torch.float8_e4m3fn).float().numpy()).all()
        top = np.abs(x).reshape(-1, 256).max(1) / scale
        assert (top <= 448).all() and (top > 224 * 0.999).all()
    for tiny in (0.0, 1e-45):   # nothing, and less than 2^-9 of the least power, 2^-126
        code, scale = adamw.encode(np.full(256, tiny, np.float32), np.zeros(256))
        assert scale[0] == np.float32(2.0 ** -126) and not code.any()


def test_rounding_keeps_the_mean():
    """The mean over 4096 draws is within five deviations of x (a code step d apart
    the deviation of one is at most d / 2), normal and subnormal codes."""
    x = np.float32(448.0) * np.array([1.0, 0.3137, 0.0171, 3e-4, 5.3e-5, 1.1e-5, 2.1e-6], np.float32)
    row = np.zeros(256, np.float32)
    row[:7] = x
    row[7:14] = -x
    total, n = np.zeros(256), 4096
    for t in range(1, n + 1):
        for r in (adamw.random16(9, t, 3, 256)[0],):
            total += adamw.decode(*adamw.encode(row, r))
    step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(row), 1e-30))) - 3), 2.0 ** -9)
    assert (np.abs(total / n - row) <= 5 * 0.5 * step / math.sqrt(n) + step * 2.0 ** -16).all()


def test_random_bits_are_spread_and_unrelated():
    """Counts of the top 6 bits of both numbers over elements, and of their pairs
    over neighbours: chi-square within 6 deviations of its mean."""
    a, b = adamw.random16(1, 77, 2, 1 << 16)
    def chi(v, k):
        c = np.bincount(v, minlength=k)
        e = len(v) / k
        return (((c - e) ** 2 / e).sum() - (k - 1)) / math.sqrt(2 * (k - 1))
    for v in (a, b):
        assert abs(chi(v >> 10, 64)) < 6
        assert abs(chi((v[1:] >> 12) * 16 + (v[:-1] >> 12), 256)) < 6
    assert abs(chi((a >> 12) * 16 + (b >> 12), 256)) < 6
    c = adamw.random16(1, 78, 2, 1 << 16)[0]
    assert abs(chi((a >> 12) * 16 + (c >> 12), 256)) < 6


def test_eight_bit_root_of_v_decays():
    """With no gradient, 700 steps of beta2 0.999 take sqrt(v) to 0.999^350 of itself:
    within 3 % over 4096 elements (a step rounds by up to 12 %, as a random walk
    of 17 % an element at rest; a block's 256 share no random bits: 17 % / 64, and
    the power of two's change takes nothing off)."""
    n = 4096
    v = np.full(n, 4.0, np.float32) * np.random.default_rng(3).uniform(0.5, 2, n).astype(np.float32)
    first = np.sqrt(v.astype(np.float64)).mean()
    code, scale = adamw.encode(np.sqrt(v), adamw.random16(0, 0, 0, n)[1])
    for t in range(1, 701):
        r = adamw.decode(code, scale)
        _, v = adamw.moments32(np.zeros(n), np.zeros(n), r * r, 0.9, 0.999, 1.0)
        code, scale = adamw.encode(np.sqrt(v), adamw.random16(0, t, 0, n)[1])
    assert abs(adamw.decode(code, scale).astype(np.float64).mean() / first / 0.999 ** 350 - 1) < 0.03
