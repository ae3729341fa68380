"""Pins of the convolution, scan and policy-loss oracles (oracle/conv.py,
oracle/scan.py, oracle/policy.py) against what does not depend on them:
central differences of their own forwards, torch's automatic differentiation
in float64, and steps chained one by one."""
import numpy as np
import pytest
import torch

from oracle import conv, policy, scan


def _diff(f, a, i, h=1e-6):
    """Central difference of the scalar f() in entry i of the array a."""
    old = a[i]
    a[i] = old + h
    up = f()
    a[i] = old - h
    down = f()
    a[i] = old
    return (up - down) / (2 * h)


def _some(rng, a, n=6):
    return [tuple(int(rng.integers(0, s)) for s in a.shape) for _ in range(n)] if a.size else []


@pytest.mark.parametrize("silu", [False, True])
@pytest.mark.parametrize("K", [1, 2, 4])
def test_conv_gradient_is_the_difference(K, silu):
    rng = np.random.default_rng(K + 10 * silu)
    T, B, D, lengths = 7, 4, 3, [7, 0, 2, 5]
    v = dict(x=rng.normal(size=(T, B, D)), w=rng.normal(size=(D, K)), bias=rng.normal(size=D),
             s0=rng.normal(size=(B, K - 1, D)))
    dy, dsT = rng.normal(size=(T, B, D)), rng.normal(size=(B, K - 1, D))

    def f():
        y, sT = conv.forward(v["x"], lengths, v["w"], v["bias"], v["s0"], silu)
        return (y * dy).sum() + (sT * dsT).sum()

    got = dict(zip(("x", "w", "bias", "s0"), conv.backward(v["x"], lengths, v["w"], v["bias"], v["s0"], silu, dy, dsT)))
    for k in v:
        for i in _some(rng, v[k]):
            assert got[k][i] == pytest.approx(_diff(f, v[k], i), rel=1e-6, abs=1e-7), (k, i)


def test_conv_is_torch_conv1d():
    rng = np.random.default_rng(1)
    T, B, D, K = 9, 2, 5, 4
    x, w, bias = rng.normal(size=(T, B, D)), rng.normal(size=(D, K)), rng.normal(size=D)
    y, _ = conv.forward(x, None, w, bias, None, True)
    tx = torch.nn.functional.pad(torch.from_numpy(x).permute(1, 2, 0), (K - 1, 0))
    ref = torch.nn.functional.silu(torch.nn.functional.conv1d(tx, torch.from_numpy(w)[:, None], torch.from_numpy(bias),
                                                              groups=D))
    np.testing.assert_allclose(y, ref.permute(2, 0, 1).numpy(), atol=1e-12)


@pytest.mark.parametrize("softplus", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("G", [1, 2])
def test_scan_gradient_is_the_difference(G, gate, softplus):
    rng = np.random.default_rng(G + 2 * gate + 4 * softplus)
    T, B, D, N, lengths = 5, 3, 4, 3, [5, 0, 3]
    v = dict(x=rng.normal(size=(T, B, D)), dt=rng.uniform(0.1, 1.0, (T, B, D)), A=-rng.uniform(0.2, 2, (D, N)),
             Bm=rng.normal(size=(T, B, G, N)), Cm=rng.normal(size=(T, B, G, N)), Dskip=rng.normal(size=D),
             dt_bias=rng.uniform(0, 0.5, D), h0=rng.normal(size=(B, D, N)))
    if gate:
        v["z"] = rng.normal(size=(T, B, D))
    dy, dhT = rng.normal(size=(T, B, D)), rng.normal(size=(B, D, N))

    def f():
        y, hT = scan.forward(lengths=lengths, softplus=softplus, **v)
        return (y * dy).sum() + (hT * dhT).sum()

    got = scan.backward(dy=dy, dhT=dhT, lengths=lengths, softplus=softplus, **v)
    for k in v:
        for i in _some(rng, v[k]):
            assert got["d" + k][i] == pytest.approx(_diff(f, v[k], i), rel=1e-6, abs=1e-7), (k, i)


def test_steps_chained_are_the_sequence():
    rng = np.random.default_rng(2)
    T, B, D, N, K = 6, 3, 4, 5, 3
    x, dt, z = (rng.normal(size=(T, B, D)) for _ in range(3))
    A, Bm, Cm = -rng.uniform(0.2, 2, (D, N)), rng.normal(size=(T, B, 1, N)), rng.normal(size=(T, B, 1, N))
    w = rng.normal(size=(D, K))
    y, hT = scan.forward(x, dt, A, Bm, Cm, z=z)
    c, sT = conv.forward(x, None, w, None, None, True)
    slots = [4, 0, 2]
    h, s = np.zeros((5, D, N)), np.zeros((5, K - 1, D))
    for t in range(T):
        yt, h = scan.step(x[t], dt[t], A, Bm[t], Cm[t], h, slots, z=z[t])
        ct, s = conv.step(x[t], w, None, s, slots, True)
        np.testing.assert_allclose(yt, y[t], atol=1e-13)
        np.testing.assert_allclose(ct, c[t], atol=1e-13)
    np.testing.assert_allclose(h[slots], hT, atol=1e-13)
    np.testing.assert_allclose(s[slots], sT, atol=1e-13)
    assert not h[[1, 3]].any()


@pytest.mark.parametrize("beta,eta", [(0.0, 0.0), (0.3, 0.0), (0.2, 0.05)])
def test_policy_gradient_is_automatic_differentiation(beta, eta):
    rng = np.random.default_rng(int(100 * beta + 1000 * eta))
    R, V = 40, 17
    x = rng.normal(size=(R, V)) * 2
    actions = rng.integers(0, V, R)
    actions[3] = -1
    w = (rng.random(R) < 0.8) * rng.uniform(0.5, 2, R)
    old, ref, adv = rng.normal(-2.5, 0.7, R), rng.normal(-2.5, 0.7, R), rng.normal(size=R)
    got = policy.loss(x, actions, old, adv, ref, w, 0.1, 0.3, beta, eta)
    tx = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(tx, 1)
    l = lp[torch.arange(R), torch.from_numpy(actions).clamp(min=0)]
    H = -(lp.exp() * lp).sum(1)
    ratio, ta = torch.exp(l - torch.from_numpy(old)), torch.from_numpy(adv)
    u = torch.from_numpy(ref) - l
    row = -torch.minimum(ratio * ta, ratio.clamp(0.9, 1.3) * ta) + beta * (torch.exp(u) - 1 - u) - eta * H
    tw = torch.from_numpy(w * (actions >= 0))
    loss = (tw * row).sum() / tw.sum()
    loss.backward()
    assert got["stats"][0] == pytest.approx(loss.item(), rel=1e-12)
    assert got["stats"][5] == pytest.approx(float(tw.sum()), rel=1e-12)
    np.testing.assert_allclose(got["dlogits"], tx.grad.numpy(), atol=1e-14)


def test_policy_rows_that_do_not_count_or_have_no_choice():
    x = np.array([[0.0, 1.0, -np.inf], [np.nan, np.inf, 0.0], [-np.inf] * 3, [0.0, 0.0, 0.0]])
    got = policy.loss(x, np.array([1, -1, 0, 2]), np.zeros(4), np.ones(4), None, None, 0.2, 0.2)
    assert got["stats"][5] == 3 and np.isfinite(got["stats"]).all()
    assert np.isfinite(got["dlogits"]).all() and not got["dlogits"][1:3].any() and got["dlogits"][0, 2] == 0
    assert np.isneginf(got["logp"][2]) and got["entropy"][2] == 0
    none = policy.loss(x, np.array([-1] * 4), np.zeros(4), np.ones(4), None, None, 0.2, 0.2)
    assert not none["stats"].any() and not none["dlogits"].any()
    bad = policy.loss(x, np.array([1, 0, 0, 2]), np.zeros(4), np.ones(4), None, None, 0.2, 0.2)
    assert np.isnan(bad["stats"][0])
