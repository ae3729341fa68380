"""GPU parity of the policy loss past the rows that one launch holds threads
for (2^24 at 256 threads a row): rows on both sides of every launch's edge and
the statistics of all of them, against float64 on the device.

Tolerances as in the policy loss's other parity tests; the statistics are means
of 2^24 such terms added in float64."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _reference(x, a, old, adv, w, lo, hi):
    lp = torch.log_softmax(x.double(), 1)
    l = lp.gather(1, a.clamp(min=0).long()[:, None])[:, 0]
    w = w.double() * (a >= 0)
    r = torch.exp(l - old.double())
    free, cut = r * adv.double(), r.clamp(1 - lo, 1 + hi) * adv.double()
    H = -(lp.exp() * lp).sum(1)
    c = torch.where(free > cut, 0.0, -free) * w / w.sum()
    g = -lp.exp() * c[:, None]
    g.scatter_add_(1, a.clamp(min=0).long()[:, None], c[:, None])
    mean = lambda v: float((w * v).sum() / w.sum())
    first = mean(-torch.minimum(free, cut))
    return l, H, g, [first, first, 0.0, mean(H), mean((free > cut).double()), float(w.sum())]


def test_more_rows_than_a_launch():
    from paper_1812_01329_amd import janus as J
    rows, V = (1 << 24) + 5, 2
    print(f"[policy rows] {rows}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((rows, V), generator=g, device="cuda")
    a = torch.randint(-1, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    a[-1] = 1
    adv = torch.randn(rows, generator=g, device="cuda")
    w = torch.rand(rows, generator=g, device="cuda")
    # ratios off the clip's corners, where the gradient jumps
    step = torch.randint(0, 4, (rows,), generator=g, device="cuda")
    old = torch.log_softmax(x, 1).gather(1, a.clamp(min=0).long()[:, None])[:, 0] \
        - torch.tensor([-0.5, -0.1, 0.1, 0.5], device="cuda")[step]
    d = J.PolicyDesc(rows, V, J.F32, 0, 0.2, 0.25, 0.0, 0.0)
    ws = torch.empty(J.janus_policy_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    out, logp, H, stats = torch.full_like(x, float("nan")), torch.empty_like(adv), torch.empty_like(adv), \
        torch.empty(6, device="cuda")
    J.janus_policy_loss(d, x, a, old_logp=old, adv=adv, weights=w, dlogits=out, logp=logp, entropy=H, stats=stats, ws=ws)
    l2 = torch.full_like(adv, float("nan"))
    J.janus_policy_loss(d, x, a, logp=l2)
    torch.cuda.synchronize()
    rl, rH, rg, rs = _reference(x, a, old, adv, w, 0.2, 0.25)
    rl, rH = rl * (a >= 0), rH * (a >= 0)

    def near(name, got, ref, tol):
        err = float((got.double() - ref).abs().max()) / float(ref.abs().max())
        assert err <= tol, f"{name}: {err:.3e}"

    near("logp", logp, rl, 1e-5)
    near("scored", l2, rl, 1e-5)
    near("entropy", H, rH, 1e-5)
    near("dlogits", out, rg, 2e-5)
    np.testing.assert_allclose(stats.double().cpu().numpy(), rs, rtol=2e-5, atol=2e-5)
