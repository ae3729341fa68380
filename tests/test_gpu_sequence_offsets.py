"""The convolution, the scan and the policy loss where rows and slots lie more
than 2^32 elements apart: states of single tokens in the first and the last slot
of a large cache, and rows with strides of 2^29 and 2^31 elements.

Only the addressing is at stake: every result is the bits of the same call on
small, dense buffers."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _gen():
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    return lambda *s, dt=torch.float32: torch.randn(s, generator=g, device="cuda").to(dt)


def test_scan_step_in_a_large_cache():
    from paper_1812_01329_amd import janus as J
    D, N, n = 4096, 16, (1 << 16) + 3
    print(f"[offsets] scan step, {n * D * N} elements of state", flush=True)
    r = _gen()
    x, dt, z, Bm, Cm, A, h = r(2, D), r(2, D), r(2, D), r(2, 1, N), r(2, 1, N), -r(D, N).abs(), r(2, D, N)
    d = J.ScanDesc(D, N, 1, 2, 1, J.F32, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
    state = torch.empty((n, D, N), device="cuda")
    slots = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    state[n - 1], state[0] = h[0], h[1]
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    J.janus_selective_scan_step(d, x, dt, A, Bm, Cm, state, y, z=z, slots=slots)
    J.janus_selective_scan_step(d, x, dt, A, Bm, Cm, h, y2, z=z)
    assert torch.equal(y, y2) and torch.equal(state[n - 1], h[0]) and torch.equal(state[0], h[1])


def test_conv_step_in_a_large_cache():
    from paper_1812_01329_amd import janus as J
    D, K = 4096, 4
    n = (1 << 32) // (D * (K - 1)) + 2
    print(f"[offsets] conv step, {n * D * (K - 1)} elements of state", flush=True)
    r, dt = _gen(), torch.bfloat16
    x, w, s = r(2, D, dt=dt), r(D, K, dt=dt), r(2, K - 1, D, dt=dt)
    d = J.ConvDesc(D, K, 2, 1, J.BF16, J.CONV_SILU, 0, 0)
    state = torch.empty((n, K - 1, D), dtype=dt, device="cuda")
    slots = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    state[n - 1], state[0] = s[0], s[1]
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    J.janus_causal_conv_step(d, x, w, None, state, y, slots=slots)
    J.janus_causal_conv_step(d, x, w, None, s, y2)
    assert torch.equal(y, y2) and torch.equal(state[n - 1], s[0]) and torch.equal(state[0], s[1])


def _spread(a, ld, buf):
    """The rows of a [rows, D], ld elements apart from the start of buf."""
    v = torch.as_strided(buf, a.shape, (ld, 1))
    v.copy_(a)
    return v


def test_conv_rows_far_apart():
    from paper_1812_01329_amd import janus as J
    T, D, K, ld = 4, 136, 3, 1 << 31
    print("[offsets] conv rows", flush=True)
    r, dt = _gen(), torch.bfloat16
    xs, dys, w, bias = r(T, D, dt=dt), r(T, D, dt=dt), r(D, K, dt=dt), r(D, dt=dt)
    out = {}
    for far in (False, True):
        step = ld if far else D
        d = J.ConvDesc(D, K, 1, T, J.BF16, J.CONV_SILU, step, step)
        new = lambda: torch.empty((T - 1) * step + D, dtype=dt, device="cuda")
        ws = torch.empty(J.janus_causal_conv_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        dw, db, by, bdx = torch.empty(D, K, device="cuda"), torch.empty(D, device="cuda"), new(), new()
        x, dy = _spread(xs, step, new()), _spread(dys, step, new())
        J.janus_causal_conv_fwd(d, x, None, w, bias, None, by)
        J.janus_causal_conv_bwd(d, x, None, w, bias, None, dy, None, bdx, dw, db, None, ws)
        out[far] = [torch.as_strided(t, (T, D), (step, 1)).clone() for t in (by, bdx)] + [dw, db]
    assert all(torch.equal(a, b) for a, b in zip(out[False], out[True]))


def test_scan_rows_far_apart():
    from paper_1812_01329_amd import janus as J
    T, D, N, ld = 10, 136, 16, 1 << 29
    print("[offsets] scan rows", flush=True)
    r, dt = _gen(), torch.bfloat16
    xs, dts, dys, Bs, Cs = r(T, D, dt=dt), r(T, D, dt=dt), r(T, D, dt=dt), r(T, N, dt=dt), r(T, N, dt=dt)
    A, Dskip = -r(D, N).abs(), r(D)
    out = {}
    for far in (False, True):
        sd, sn = (ld, ld) if far else (D, N)
        d = J.ScanDesc(D, N, 1, 1, T, J.BF16, J.SCAN_SOFTPLUS | J.SCAN_KEEP, sd, sd, sn, sn, 0, sd)
        new = lambda n=D, step=None: torch.empty((T - 1) * (step or sd) + n, dtype=dt, device="cuda")
        ws = torch.empty(J.janus_selective_scan_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        x, dtv, dy = (_spread(a, sd, new()) for a in (xs, dts, dys))
        Bm, Cm = (_spread(a, sn, new(N, sn)) for a in (Bs, Cs))
        y, dx, ddt, dB, dC = new(), new(), new(), new(N, sn), new(N, sn)
        dA, dD = torch.empty(D, N, device="cuda"), torch.empty(D, device="cuda")
        J.janus_selective_scan_fwd(d, x, dtv, A, Bm, Cm, None, y, ws, Dskip=Dskip)
        J.janus_selective_scan_bwd(d, x, dtv, A, Bm, Cm, None, dy, ws, dx, ddt, dA, dB, dC, Dskip=Dskip, dDskip=dD)
        out[far] = [torch.as_strided(t, (T, D), (sd, 1)).clone() for t in (y, dx, ddt)] + \
            [torch.as_strided(t, (T, N), (sn, 1)).clone() for t in (dB, dC)] + [dA, dD]
    assert all(torch.equal(a, b) for a, b in zip(out[False], out[True]))


@pytest.mark.parametrize("V", [1003, 70001])
def test_policy_rows_far_apart(V):
    from paper_1812_01329_amd import janus as J
    rows, ld = 4, 1 << 31
    print(f"[offsets] policy rows V={V}", flush=True)
    r = _gen()
    xs = r(rows, V, dt=torch.bfloat16)
    a = torch.arange(rows, dtype=torch.int32, device="cuda") * 200
    old, adv, ref = r(rows) - 7, r(rows), r(rows) - 7
    out = {}
    for far in (False, True):
        step = ld if far else -(-V // 8) * 8   # (both cut at the same bytes)
        d = J.PolicyDesc(rows, V, J.BF16, step, 0.2, 0.2, 0.1, 0.01)
        ws = torch.empty(J.janus_policy_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        x = _spread(xs, step, torch.empty((rows - 1) * step + V, dtype=torch.bfloat16, device="cuda"))
        stats, logp = torch.empty(6, device="cuda"), torch.empty(rows, device="cuda")
        J.janus_policy_loss(d, x, a, old_logp=old, adv=adv, ref_logp=ref, dlogits=x, logp=logp, stats=stats, ws=ws)
        out[far] = [x.clone(), stats, logp]
    assert all(torch.equal(p, q) for p, q in zip(out[False], out[True]))
