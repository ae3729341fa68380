"""Min-p alone on float32 rows too long for LDS, whose marks are still one element each
(32769 to 65536 elements, dense or from any start): few kept, which are listed, and many,
which are added up where they are; settings as in the sampler's other tests."""
import numpy as np
import pytest

from tests.test_gpu_sample import check, run

pytestmark = pytest.mark.gpu

COUNTS = [1, 2, 63, 127, 128, 129, 200, 256, 257, 1024, 1025, 5000]


@pytest.mark.parametrize("V,pad,shift", [(32769, 0, 0), (50257, 0, 0), (50257, 7, 1), (65536, 0, 0), (65536, 3, 3)])
def test_kept_by_min_p_alone(V, pad, shift):
    """A row for each count of kept elements, at places from the first to the last; the first
    and the last of them drawn, and one between."""
    print(f"[sample unheld] V={V} {pad} {shift}", flush=True)
    rng = np.random.default_rng(V + pad)
    rows = [(n, u) for n in COUNTS for u in (0.0, 0.37, 0.9999999)]
    x = np.minimum(rng.normal(size=(len(rows), V)) * 2, 6.0).astype(np.float32)
    x[:, 1:][rng.random((len(rows), V - 1)) < 0.05] = -np.inf
    for r, (n, _) in enumerate(rows):
        at = rng.choice(V, n, replace=False)
        if n > 1:
            at[:2] = 0, V - 1
            at[2:] = rng.choice(np.arange(1, V - 1), n - 2, replace=False)
        x[r, at] = 10 + rng.random(n)
    u = np.array([v for _, v in rows], np.float32)
    for per_row in (False, True):
        got = run(x, u, "f32", pad, shift, minp=0.2, per_row=per_row)   # (10 is at least 0.2 of 11: 1.61)
        assert got[3].tolist() == [n for n, _ in rows]
        check(x, u, got, minp=0.2)
