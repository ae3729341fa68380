"""GPU parity of the selective scan at its documented limits of channels and
states, 2^22 and 64, where the sums over the parts of the parameters' gradients
need more threads than a launch holds.  One step, against float64 on the device.

Tolerances as in the scan's other parity tests: 1e-4 of a tensor's largest entry."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_most_channels_and_states():
    from paper_1812_01329_amd import janus as J
    D, N, Dg = 1 << 22, 64, 128
    G = D // Dg
    print(f"[scan wide] D={D} N={N} G={G}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, dt, dy, Dskip, dtb = (r(D) for _ in range(5))
    A, h0, dhT = -torch.rand((D, N), generator=g, device="cuda") * 3, r(D, N), r(D, N)
    Bm, Cm = r(G, N), r(G, N)
    d = J.ScanDesc(D, N, G, 1, 1, J.F32, J.SCAN_SOFTPLUS | J.SCAN_KEEP, 0, 0, 0, 0, 0, 0)
    ws = torch.empty(J.janus_selective_scan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    nan = lambda t: torch.full_like(t, float("nan"))
    o = dict(y=nan(x), hT=nan(h0), dx=nan(x), ddt=nan(x), dA=nan(A), dBm=nan(Bm), dCm=nan(Cm), dDskip=nan(x),
             ddt_bias=nan(x), dh0=nan(h0))
    J.janus_selective_scan_fwd(d, x, dt, A, Bm, Cm, None, o["y"], ws, Dskip=Dskip, dt_bias=dtb, h0=h0, hT=o["hT"])
    J.janus_selective_scan_bwd(d, x, dt, A, Bm, Cm, None, dy, ws, o["dx"], o["ddt"], o["dA"], o["dBm"], o["dCm"],
                               Dskip=Dskip, dt_bias=dtb, h0=h0, dhT=dhT, dDskip=o["dDskip"], ddt_bias=o["ddt_bias"],
                               dh0=o["dh0"])
    torch.cuda.synchronize()
    step = 1 << 17
    worst, top = dict.fromkeys(o, 0.0), dict.fromkeys(o, 0.0)
    for c in range(0, D, step):
        s, gs = slice(c, c + step), slice(c // Dg, (c + step) // Dg)
        f = lambda t: t[s].double()
        wide = lambda m: m[gs].double().repeat_interleave(Dg, 0)
        v = f(dt) + f(dtb)
        e = torch.nn.functional.softplus(v)
        a, b, cm = torch.exp(e[:, None] * f(A)), wide(Bm), wide(Cm)
        h = a * f(h0) + (e * f(x))[:, None] * b
        G_ = f(dhT) + f(dy)[:, None] * cm
        q, s_b = G_ * a * f(h0), (G_ * b).sum(1)
        de = f(x) * s_b + (q * f(A)).sum(1)
        fold = lambda m: m.view(-1, Dg, N).sum(1)
        ref = dict(y=(cm * h).sum(1) + f(Dskip) * f(x), hT=h, dx=f(dy) * f(Dskip) + e * s_b, ddt=de * torch.sigmoid(v),
                   dA=q * e[:, None], dBm=fold(G_ * (e * f(x))[:, None]), dCm=fold(f(dy)[:, None] * h),
                   dDskip=f(dy) * f(x), ddt_bias=de * torch.sigmoid(v), dh0=G_ * a)
        for k, t in ref.items():
            got = o[k][gs if k in ("dBm", "dCm") else s].double()
            assert bool(got.isfinite().all()), (k, c)
            worst[k] = max(worst[k], float((got - t).abs().max()))
            top[k] = max(top[k], float(t.abs().max()))
    for k in o:
        assert worst[k] <= 1e-4 * top[k], f"{k}: {worst[k] / top[k]:.3e}"
