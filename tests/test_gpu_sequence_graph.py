"""The convolution, the scan and the policy loss inside a captured HIP graph,
and on a stream of their own: every replay, with new inputs copied in and eager
work between the replays, gives the bits of the eager calls."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _program(torch, J):
    """One step of conv -> scan -> loss -> backward on fixed buffers; returns
    (inputs that may be overwritten, outputs, the calls)."""
    T, B, D, N, K, V = 70, 3, 136, 16, 4, 136
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    e = lambda *s: torch.empty(s, device="cuda")
    lengths = np.array([70, 11, 64], np.int32)
    cd = J.ConvDesc(D, K, B, T, J.F32, J.CONV_SILU, 0, 0)
    sd = J.ScanDesc(D, N, 1, B, T, J.F32, J.SCAN_SOFTPLUS | J.SCAN_KEEP, 0, 0, 0, 0, 0, 0)
    pd = J.PolicyDesc(T * B, V, J.F32, 0, 0.2, 0.2, 0.1, 0.01)
    ws = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    cw, sw, pw = (ws(J.janus_causal_conv_workspace_bytes(cd)), ws(J.janus_selective_scan_workspace_bytes(sd)),
                  ws(J.janus_policy_workspace_bytes(pd)))
    # (x small: with y as logits, exp(ref - l) of float32 has to stay finite)
    x, dt, z, Bm, Cm = 0.02 * r(T, B, D), r(T, B, D), r(T, B, D), r(T, B, 1, N), r(T, B, 1, N)
    w, bias, A, Dskip = r(D, K), 0.02 * r(D), -r(D, N).abs() - 0.1, r(D)
    old, adv, ref = r(T * B) - 5, r(T * B), r(T * B) - 5
    act = torch.randint(0, V, (T * B,), generator=g, device="cuda", dtype=torch.int32)
    o = dict(u=e(T, B, D), y=e(T, B, D), dl=e(T, B, D), stats=e(6), du=e(T, B, D), ddt=e(T, B, D), dz=e(T, B, D),
             dB=e(T, B, 1, N), dC=e(T, B, 1, N), dA=e(D, N), dD=e(D), dx=e(T, B, D), dw=e(D, K), db=e(D))

    def run():
        J.janus_causal_conv_fwd(cd, x, lengths, w, bias, None, o["u"])
        J.janus_selective_scan_fwd(sd, o["u"], dt, A, Bm, Cm, lengths, o["y"], sw, Dskip=Dskip, z=z)
        J.janus_policy_loss(pd, o["y"], act, old_logp=old, adv=adv, ref_logp=ref, dlogits=o["dl"], stats=o["stats"],
                            ws=pw)
        J.janus_selective_scan_bwd(sd, o["u"], dt, A, Bm, Cm, lengths, o["dl"], sw, o["du"], o["ddt"], o["dA"], o["dB"],
                                   o["dC"], Dskip=Dskip, z=z, dDskip=o["dD"], dz=o["dz"])
        J.janus_causal_conv_bwd(cd, x, lengths, w, bias, None, o["du"], None, o["dx"], o["dw"], o["db"], None, cw)

    return [x, dt, z, Bm, Cm], o, run


def test_graph_replays_are_the_eager_calls():
    import torch
    from paper_1812_01329_amd import janus as J
    inputs, out, run = _program(torch, J)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(4):
        print(f"[sequence graph] replay {k}", flush=True)
        for i, t in enumerate(inputs):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(10 * k + i)) * (0.02 if i == 0 else 1.0))
        run()
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in out.items()}
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for n, t in out.items():
            assert bool(t.isfinite().all()), n
            assert torch.equal(t, eager[n]), n
