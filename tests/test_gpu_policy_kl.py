"""GPU parity of the policy loss where its KL term is switched off or infinite:
a reference with a coefficient of 0 leaves loss and gradient bit for bit as
without one, also where ref - l is infinite or exp of it passes float32; with a
coefficient the loss says so.

Tolerances as in the policy loss's other parity tests."""
import numpy as np
import pytest
import torch

from oracle import policy as oracle
from test_gpu_policy import Case, near

pytestmark = pytest.mark.gpu


def case(dtype, V, eta, beta):
    """Eight rows: an action that is forbidden (l = -inf), references far above
    l and at -inf, a row of nothing but -inf, padding full of NaN."""
    c = Case(31, 8, V, dtype, ref=True, weights=False, beta=beta, eta=eta)
    c.x[0], c.a[0] = np.nan, -1
    c.x[1] = -np.inf
    c.x[2, c.a[2]] = -np.inf
    l = oracle.rows(c.x, c.a)[0]
    c.ref[0], c.ref[1], c.ref[2] = np.nan, -2.0, -3.0
    c.old[1:3] = -2.0
    c.ref[3], c.ref[4] = l[3] + 120.0, -np.inf
    return c


@pytest.mark.parametrize("eta", [0.0, 0.05])
@pytest.mark.parametrize("dtype,V", [("f32", 300), ("bf16", 301), ("f32", 66000)])
def test_reference_without_a_coefficient(dtype, V, eta):
    print(f"[policy kl] {dtype} V={V} eta={eta}", flush=True)
    c = case(dtype, V, eta, 0.0)
    got = c.run()[0]
    none = case(dtype, V, eta, 0.0)
    none.ref = None
    plain = none.run()[0]
    assert bool(plain["dlogits"].isfinite().all()) and bool(plain["stats"].isfinite().all())
    for k in ("dlogits", "logp", "entropy"):
        assert torch.equal(got[k], plain[k]), k
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(got["stats"][keep], plain["stats"][keep])
    assert float(got["stats"][2]) == np.inf
    ref = oracle.loss(c.x, c.a, c.old, c.adv, c.ref, None, 0.2, 0.25, 0.0, eta)
    near("dlogits", got["dlogits"], ref["dlogits"], 2.0 ** -8 if dtype == "bf16" else 2e-5)
    near("stats", got["stats"], ref["stats"], 2e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_mean_of_an_ordinary_reference_without_a_coefficient(dtype):
    c = Case(32, 300, 515, dtype, beta=0.0, eta=0.01)
    c.check(c.run())


@pytest.mark.parametrize("which", [2, 3, 4])
def test_infinite_kl_with_a_coefficient(which):
    """The loss is infinite; the gradient of the other rows stays finite, and of
    the row itself too where the reference is -inf."""
    c = case("f32", 300, 0.0, 0.5)
    for r in (2, 3, 4):
        if r != which:
            c.a[r] = -1
    got = c.run()[0]
    assert float(got["stats"][0]) == np.inf and float(got["stats"][2]) == np.inf
    rows = [r for r in range(8) if r != which or which == 4]
    assert bool(got["dlogits"][rows].isfinite().all())
    if which != 4:
        assert not bool(got["dlogits"][which].isfinite().all())
