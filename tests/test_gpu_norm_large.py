"""Layer norm's backward where a row's values are so large that even 0 is out of reach of its
mean: constant rows, whose deviation is eps alone, of every length of a last access.

Sums of equal powers of two are exact, so xh is 0 and dx = rstd (g - sum g / D): as the
other tests of the gradient, within 2e-5 of its largest and one rounding to bf16, 2^-8;
dgamma is 0 and dbeta within (64 + 1) * 2^-24 + 1e-5 of its terms' magnitudes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [1, 3, 33, 301, 302, 303, 1027, 2047, 8195, 12001, 20001, 40003])
def test_constant_rows_of_large_values(D, dtype):
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[norm large] {D} {dtype}", flush=True)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(D)
    rows, eps = 5, 1e-12
    value = 2.0 ** 110   # (its product with rstd = 1e6 is past float32, its sum over a row is not)
    x = torch.from_numpy(rng.normal(size=(rows, D)).astype(np.float32)).cuda().to(dt)
    x[1] = value
    x[3] = -value
    dy = torch.from_numpy(rng.normal(size=(rows, D)).astype(np.float32)).cuda().to(dt)
    gamma = torch.from_numpy(rng.uniform(0.5, 1.5, D).astype(np.float32)).cuda()
    d = J.NormDesc(rows, D, J.F32 if dtype == "f32" else J.BF16, eps, 0, 0, 0)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dgamma, dbeta = (torch.empty(n, device="cuda") for n in (rows, rows, D, D))
    ws = torch.empty(J.janus_layer_norm_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    J.janus_layer_norm_fwd(d, x, gamma, None, y, mean=mean, rstd=rstd)
    J.janus_layer_norm_bwd(d, x, gamma, mean, rstd, dy, dx, ws, dgamma=dgamma, dbeta=dbeta)
    big, others = [1, 3], [0, 2, 4]
    assert not bool(y[big].any()) and mean[big].tolist() == [value, -value]
    np64 = lambda t: t.double().cpu().numpy()
    g = np64(dy[big]) * np64(gamma)
    want = 1e6 * (g - g.mean(1, keepdims=True))
    bf = 2.0 ** -8 if dtype == "bf16" else 0.0
    got = np64(dx[big])
    assert (np.abs(got - want) <= bf * np.abs(want) + 2e-5 * 1e6 * np.abs(g).max()).all()
    # nothing of it is in the other rows, in dgamma or in dbeta
    few, dx2, dg2 = x[others].contiguous(), torch.empty_like(x[others]), torch.empty_like(dgamma)
    d.rows = 3
    J.janus_layer_norm_bwd(d, few, gamma, mean[others].contiguous(), rstd[others].contiguous(), dy[others].contiguous(), dx2, ws,
                           dgamma=dg2)
    assert torch.equal(dx[others], dx2)
    xh = (np64(few) - np64(mean[others])[:, None]) * np64(rstd[others])[:, None]
    assert (np.abs(np64(dgamma) - np64(dg2)) <= 2.0 ** -22 * (np.abs(np64(dy[others]) * xh)).sum(0) + 1e-30).all()
    assert (np.abs(np64(dbeta) - np64(dy).sum(0)) <= (65 * 2.0 ** -24 + 1e-5) * np.abs(np64(dy)).sum(0)).all()
