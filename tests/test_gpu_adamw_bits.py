"""States of 8 bits where the root is kept as 0 and m is not (janus_adamw_update):
blocks of 256 whose gradients lie far apart, step by step against the oracle, and
no step longer than AdamW's.

Tolerances: a parameter's step has, as in the other tests of the update, at most 2^-19
of itself and 2^-22 of the parameter; where the two terms of m cancel, three roundings of
them, each at most 2^-24 of terms that would be 12 lr by themselves (7.3 of the old m, 3.2
of g, an eighth of the codes' rounding): 2^-22 of 12 lr.  No step longer than 10 lr, as
derived for the oracle."""
import numpy as np
import pytest

from oracle import adamw as oracle

pytestmark = pytest.mark.gpu

F = np.float32
LR, B1, B2 = float(F(1e-3)), float(F(0.9)), float(F(0.999))


@pytest.mark.parametrize("n,shift", [(512, 0), (512, 1), (777, 0), (200, 3)])
@pytest.mark.parametrize("kind", ["large", "once"])
def test_steps_with_roots_kept_as_0(kind, n, shift):
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[adamw bits] {kind} {n} {shift}", flush=True)
    eps = float(F(1e-12))
    rng = np.random.default_rng(n)
    put = lambda dt: torch.zeros(n + shift, dtype=dt, device="cuda")[shift:]
    p, g, m, v = put(torch.float32), put(torch.float32), put(torch.uint8), put(torch.uint8)
    scale = torch.zeros(-(-n // 256), 2, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = J.AdamWDesc(1, J.ADAMW_8BIT, LR, B1, B2, eps, 0.0, 7)
    ws = torch.empty(J.janus_adamw_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    tensors = J.adamw_tensors([p], [g], [m], [v], [scale])
    size = np.where(np.arange(n) % 256 == 3, 1.0, 10.0 ** rng.uniform(-7, -3, n))
    cm, cv, sm, sv = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(-(-n // 256), F), np.zeros(-(-n // 256), F)
    w, met = np.zeros(n), 0
    for t in range(1, 61):
        grad = rng.normal(size=n) * size
        if kind == "once":   # the first gradients of half of the block come late, and once
            grad[::2] *= t == 30
            grad[1::2] *= t <= 20
        grad = grad.astype(F)
        g.copy_(torch.from_numpy(grad))
        J.janus_adamw_update(d, tensors, step, ws=ws)
        m0, r0 = oracle.decode(cm, sm), oracle.decode(cv, sv)
        least = oracle.least_root(cv, sv, B2)
        want, _, _ = oracle.update(w, grad, m0, r0.astype(np.float64) ** 2, t - 1, LR, B1, B2, eps, 0.0, 1.0, least)
        met += int(((cv == 0) & (cm & 127 != 0) & (least > 0)).sum())
        mt, vt = oracle.moments32(grad, m0, r0 * r0, F(B1), F(B2), 1.0)
        rm, rv = oracle.random16(7, t, 0, n)
        (cm, sm), (cv, sv) = oracle.encode(mt, rm), oracle.encode(np.sqrt(vt), rv)
        np.testing.assert_array_equal(m.cpu().numpy(), cm, err_msg=f"step {t}")
        np.testing.assert_array_equal(v.cpu().numpy(), cv, err_msg=f"step {t}")
        np.testing.assert_array_equal(scale.cpu().numpy(), np.stack([sm, sv], 1), err_msg=f"step {t}")
        got = p.double().cpu().numpy()
        assert np.abs(got - w).max() <= 10 * LR, f"step {t}: {np.abs(got - w).max() / LR} lr"
        assert (np.abs(got - want) <= 2.0 ** -22 * np.abs(want) + 2.0 ** -19 * np.abs(want - w) + 2.0 ** -22 * 12 * LR).all(), f"step {t}"
        w = got
    assert met > 100   # (what this is about did happen)
