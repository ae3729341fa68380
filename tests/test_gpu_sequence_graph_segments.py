"""The selective scan with its time axis cut into segments inside a captured HIP
graph: the local passes and the chains of both directions, and a prompt whose
state is carried in place; every replay, with new inputs copied in and eager
work between the replays, gives the bits of the eager calls."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _program(torch, J):
    T, B, D, N = 300, 3, 136, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    e = lambda *s: torch.empty(s, device="cuda")
    lengths = np.array([300, 11, 264], np.int32)
    sd = J.ScanDesc(D, N, 1, B, T, J.F32, J.SCAN_SOFTPLUS | J.SCAN_KEEP, 0, 0, 0, 0, 0, 0)
    pd = J.ScanDesc(D, N, 1, B, T, J.F32, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
    sw, pw = (torch.empty(J.janus_selective_scan_workspace_bytes(d), dtype=torch.uint8, device="cuda") for d in (sd, pd))
    assert pw.numel() > 0, "the time axis is not cut"
    x, dt, z, dy, Bm, Cm = r(T, B, D), r(T, B, D), r(T, B, D), r(T, B, D), r(T, B, 1, N), r(T, B, 1, N)
    h0, dhT, A, Dskip = r(B, D, N), r(B, D, N), -r(D, N).abs() - 0.1, r(D)
    o = dict(y=e(T, B, D), y2=e(T, B, D), hT=e(B, D, N), state=e(B, D, N), dx=e(T, B, D), ddt=e(T, B, D), dz=e(T, B, D),
             dB=e(T, B, 1, N), dC=e(T, B, 1, N), dA=e(D, N), dD=e(D), dh0=e(B, D, N))

    def run():
        J.janus_selective_scan_fwd(sd, x, dt, A, Bm, Cm, lengths, o["y"], sw, Dskip=Dskip, z=z, h0=h0, hT=o["hT"])
        J.janus_selective_scan_bwd(sd, x, dt, A, Bm, Cm, lengths, dy, sw, o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"],
                                   Dskip=Dskip, z=z, h0=h0, dhT=dhT, dDskip=o["dD"], dz=o["dz"], dh0=o["dh0"])
        o["state"].copy_(h0)
        J.janus_selective_scan_fwd(pd, x, dt, A, Bm, Cm, lengths, o["y2"], pw, Dskip=Dskip, z=z, h0=o["state"],
                                   hT=o["state"])

    return [x, dt, z, dy, Bm, Cm, h0, dhT], o, run


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
        print(f"[segments graph] replay {k}", flush=True)
        for i, t in enumerate(inputs):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(10 * k + i)))
        run()
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in out.items()}
        assert torch.equal(eager["y"], eager["y2"]) and torch.equal(eager["hT"], eager["state"])
        for t in out.values():
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for n, t in out.items():
            assert bool(t.isfinite().all()), n
            assert torch.equal(t, eager[n]), n
