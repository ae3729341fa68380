"""Pins of the policy oracle's KL term where it is switched off or infinite: with
a coefficient of 0 a reference changes neither loss nor gradient, whatever its
values are, and its mean is still the mean of exp(u) - 1 - u."""
import numpy as np
import pytest

from oracle import policy


@pytest.mark.parametrize("eta", [0.0, 0.1])
def test_reference_without_a_coefficient(eta):
    rng = np.random.default_rng(1)
    R, V = 6, 5
    x, a = rng.normal(size=(R, V)), rng.integers(0, V, R)
    x[1, a[1]] = -np.inf                       # forbidden, and taken all the same: u = inf
    old, adv = rng.normal(-1.5, 0.3, R), rng.normal(size=R)
    ref = rng.normal(-1.5, 0.3, R)
    plain = policy.loss(x, a, old, adv, None, None, eta=eta)
    assert np.isfinite(plain["stats"]).all() and np.isfinite(plain["dlogits"]).all()
    for at, value in ((2, 200.0), (3, -np.inf)):
        r = ref.copy()
        r[at] = value
        got = policy.loss(x, a, old, adv, r, None, beta=0.0, eta=eta)
        np.testing.assert_array_equal(got["dlogits"], plain["dlogits"])
        np.testing.assert_array_equal(got["stats"][[0, 1, 3, 4, 5]], plain["stats"][[0, 1, 3, 4, 5]])
        assert got["stats"][2] == np.inf
    x[1, a[1]] = 0.3
    l = policy.loss(x, a, old, adv)["logp"]
    got = policy.loss(x, a, old, adv, ref, None, beta=0.0)["stats"]
    assert got[2] == pytest.approx(np.mean(np.exp(ref - l) - 1 - (ref - l)), rel=1e-12)


def test_infinite_kl_with_a_coefficient():
    rng = np.random.default_rng(2)
    x, a = rng.normal(size=(3, 4)), np.array([1, 0, 3])
    ref = np.array([-1.0, -np.inf, -1.0])
    got = policy.loss(x, a, np.full(3, -1.4), np.ones(3), ref, None, beta=0.5)
    assert got["stats"][0] == np.inf and got["stats"][2] == np.inf
    assert np.isfinite(got["dlogits"]).all()   # exp(-inf) - 1 = -1
    x[0, 1] = -np.inf
    with np.errstate(invalid="ignore"):   # inf * 0 in the row's gradient
        got = policy.loss(x, a, np.full(3, -1.4), np.ones(3), np.full(3, -1.0), None, beta=0.5)
    assert got["stats"][0] == np.inf and not np.isfinite(got["dlogits"][0, 1])
    assert np.isfinite(got["dlogits"][1:]).all()
