"""GPU parity of the policy loss where its rows are many (the weights' sum comes
from a launch of its own past 2048 rows) and at vocabularies of the workgroup
sizes between those of the other parity tests, with rows that start anywhere.

Tolerances as in the policy loss's other parity tests."""
import numpy as np
import pytest

from test_gpu_policy import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [2048, 2049, 9001])
def test_rows(rows, dtype):
    """Fractional weights, padding by weight and by action, NaN in the padding."""
    print(f"[policy many] rows={rows} {dtype}", flush=True)
    c = Case(rows, rows, 33, dtype, pad=1, beta=0.2, eta=0.05)
    out = np.random.default_rng(rows).random(rows) < 0.1
    c.a[out] = -1
    c.x[out] = np.nan
    c.check(c.run())
    c.w = None
    c.check(c.run(in_place=True))


@pytest.mark.parametrize("dtype,V", [("f32", 17500), ("f32", 28001), ("f32", 40003), ("bf16", 36001), ("bf16", 80005),
                                     ("f32", 65529), ("bf16", 131065)])
def test_vocabularies_between(V, dtype):
    print(f"[policy many] V={V} {dtype}", flush=True)
    for pad in (0, 1):
        c = Case(V, 5, V, dtype, pad=pad, eta=0.05, masked=True)
        c.check(c.run())
    c.check(c.run(in_place=True))
