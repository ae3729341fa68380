"""AdamW with states of 8 bits beside AdamW with states of 64, step by step on the
same gradients: blocks of 256 whose elements lie far apart, where m is kept and
sqrt(v), next to a larger one, comes out as 0.

Bounds.  AdamW's own step is at most (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)) = 7.3 lr; with m
an eighth too large and the root an eighth too small it is 9.4: 10 lr.  A root between
one and two least codes may be kept as one: steps of double length; with the noise of
the rounding a walk is at most three times as long as the one of 64 bits."""
import numpy as np
import pytest

from oracle import adamw

F = np.float32
LR, B1, B2 = 1e-3, float(F(0.9)), float(F(0.999))


def walks(gradient, steps, eps, seed=3):
    """Largest step in units of lr and furthest parameter, by both kinds of states."""
    n = 256
    cm, cv = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    sm, sv = np.zeros(1, F), np.zeros(1, F)
    p8, p64, m64, v64 = (np.zeros(n) for _ in range(4))
    far8 = far64 = 0.0
    for t in range(1, steps + 1):
        g = gradient(t).astype(F)
        m, r = adamw.decode(cm, sm), adamw.decode(cv, sv)
        least = adamw.least_root(cv, sv, B2)
        new = adamw.update(p8, g, m, r.astype(np.float64) ** 2, t - 1, LR, B1, B2, eps, 0.0, 1.0, least)[0]
        far8, p8 = max(far8, np.abs(new - p8).max() / LR), new
        m, v = adamw.moments32(g, m, r * r, B1, B2, 1.0)
        rm, rv = adamw.random16(seed, t, 0, n)
        (cm, sm), (cv, sv) = adamw.encode(m, rm), adamw.encode(np.sqrt(v), rv)
        new, m64, v64 = adamw.update(p64, g, m64, v64, t - 1, LR, B1, B2, eps, 0.0, 1.0)
        far64, p64 = max(far64, np.abs(new - p64).max() / LR), new
    return far8, far64, np.abs(p8).max(), np.abs(p64).max()


@pytest.mark.parametrize("eps,top", [(1e-8, 1.0), (1e-12, 1.0), (1e-12, 1e-3)])
@pytest.mark.parametrize("ratio", [1e-3, 1e-4, 1e-5, 1e-6, 1e-7])
def test_one_large_element_among_small_ones(ratio, eps, top):
    rng = np.random.default_rng(0)
    s = np.full(256, ratio * top)
    s[0] = top
    far8, far64, walk8, walk64 = walks(lambda t: rng.normal(size=256) * s, 600, eps)
    assert far64 <= 7.3 and far8 <= 10.0 and walk8 <= 3 * walk64, (far8, far64, walk8, walk64)


@pytest.mark.parametrize("ratio", [1e-2, 1e-3, 1e-4, 1e-5, 1e-6])
def test_a_gradient_that_comes_once(ratio):
    """Half of the block has gradients for 100 steps, the other half a smaller one in step 200
    and none after: m, whose power of two has fallen, is kept, and the root is not."""
    rng = np.random.default_rng(1)

    def gradient(t):
        g = np.zeros(256)
        if t <= 100:
            g[:128] = rng.normal(size=128)
        if t == 200:
            g[128:] = ratio * rng.normal(size=128)
        return g
    far8, far64, walk8, walk64 = walks(gradient, 300, 1e-8)
    assert far64 <= 7.3 and far8 <= 10.0 and walk8 <= 3 * walk64, (far8, far64, walk8, walk64)


@pytest.mark.parametrize("ratio", [1e-1, 1e-3, 1e-5])
def test_rare_rows_that_share_a_block(ratio):
    """Eight rows of 32 parameters, each with a gradient in one step of twenty, of sizes
    from 1 to `ratio`."""
    rng = np.random.default_rng(2)
    size = np.repeat(ratio ** (np.arange(8) / 7), 32)
    far8, far64, walk8, walk64 = walks(lambda t: np.repeat(rng.random(8) < 0.05, 32) * size * rng.normal(size=256), 800, 1e-8)
    assert far64 <= 7.3 and far8 <= 10.0 and walk8 <= 3 * walk64, (far8, far64, walk8, walk64)


def test_the_least_root_is_that_of_code_1_and_only_of_code_0():
    codes = np.zeros(300, np.uint8)
    codes[5], codes[299] = 1, 0x7e
    scale = np.array([0.25, 8.0], F)
    got = adamw.least_root(codes, scale, 0.81)
    want = np.repeat(0.9 * adamw.decode(np.ones(512, np.uint8), scale).astype(np.float64)[[0, 256]], 256)[:300]
    want[[5, 299]] = 0.0
    np.testing.assert_allclose(got, want, rtol=1e-15)
    assert not adamw.least_root(codes, np.zeros(2, F), 0.999).any()
    assert not adamw.least_root(codes, scale, 0.0).any()
