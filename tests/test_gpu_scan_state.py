"""GPU parity of the selective scan where a sequence's state is handed on while
the time axis is cut into segments: the final state in the place of the initial
one, segments past one round of the chain's loads, more than 32 states,
batches past one launch's lengths, training over many segments, prompts
continued by single tokens.

The first segment of a prompt reads its initial state while the last one, in
another workgroup of the same launch, writes the final state.  A sequence that
ends inside an early segment leaves the last one without steps, which then
writes at once.  So in place is compared bit for bit with out of place.

Tolerances as in the scan's other parity tests, and by the same reasoning: 1e-4
of a tensor's largest entry in float32, one rounding of 2^-8 in bf16."""
import numpy as np
import pytest

from oracle import scan as oracle
from test_gpu_scan import TOL, Scan, near

pytestmark = pytest.mark.gpu


def prompt(s, in_place):
    """The forward without KEEP; returns y and the final state."""
    torch, J = s.torch, s.J
    f32 = torch.float32
    code = J.BF16 if s.dtype == "bf16" else J.F32
    d = J.ScanDesc(s.D, s.N, s.G, s.B, s.T, code, J.SCAN_SOFTPLUS if s.softplus else 0, 0, 0, 0, 0, 0, 0)
    ws = torch.full((J.janus_selective_scan_workspace_bytes(d),), 0xff, dtype=torch.uint8, device="cuda")
    assert ws.numel() > 0, "the time axis is not cut"
    h0 = s.dev(s.h0, f32)
    hT = h0 if in_place else torch.full_like(h0, float("nan"))
    y = torch.full((s.T, s.B, s.D), float("nan"), dtype=s.tdt, device="cuda")
    J.janus_selective_scan_fwd(d, s.dev(s.x), s.dev(s.dt), s.dev(s.A, f32), s.dev(s.Bm), s.dev(s.Cm), s.lengths, y, ws,
                               Dskip=s.dev(s.Dskip, f32), z=s.dev(s.z), dt_bias=s.dev(s.dt_bias, f32), h0=h0, hT=hT)
    torch.cuda.synchronize()
    return y, hT


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,D,N,G,lengths", [
    (128, 1, 64, 16, 1, None),                    # two segments
    (256, 1, 64, 16, 1, [40]),                    # the last segments have no steps
    (600, 3, 300, 13, 3, [5, 600, 0]),
    (1280, 2, 70, 16, 1, [1280, 64]),             # twenty segments: the chain's second round of loads
    (300, 2, 66, 40, 1, [300, 17]),               # past 32 states
    (130, 300, 40, 4, 1, "ragged"),               # more sequences than one launch carries lengths for
])
def test_final_state_in_the_initial_ones_place(T, B, D, N, G, lengths, dtype):
    print(f"[scan state] T={T} B={B} D={D} N={N} G={G} {dtype}", flush=True)
    if lengths == "ragged":
        lengths = np.random.default_rng(T).integers(0, T + 1, B)
    s = Scan(21, T, B, D, N, G, dtype, None if lengths is None else np.array(lengths, np.int32))
    y, hT = prompt(s, False)
    y2, h2 = prompt(s, True)
    assert s.torch.equal(y, y2) and s.torch.equal(hT, h2)
    ry, rh = oracle.forward(s.x, s.dt, s.A, s.Bm, s.Cm, Dskip=s.Dskip, z=s.z, dt_bias=s.dt_bias, lengths=s.lengths,
                            h0=s.h0, softplus=s.softplus)
    near("y", y2, ry, TOL[dtype])
    near("hT", h2, rh, TOL["f32"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,B,D,N,G,lengths", [
    (1280, 1, 70, 16, 1, None),                   # twenty segments, both directions
    (1280, 2, 40, 8, 2, [1280, 700]),
    (2048, 1, 33, 13, 1, [1990]),                 # thirty-two
    (300, 2, 66, 40, 1, [300, 17]),               # past 32 states: states kept every four steps
    (260, 1, 130, 64, 1, None),
    (257, 1, 200, 33, 2, [231]),
    (130, 300, 40, 4, 1, "ragged"),
])
def test_training_over_segments(T, B, D, N, G, lengths, dtype):
    print(f"[scan segments] T={T} B={B} D={D} N={N} G={G} {dtype}", flush=True)
    if lengths == "ragged":
        lengths = np.random.default_rng(T).integers(0, T + 1, B)
    s = Scan(22, T, B, D, N, G, dtype, None if lengths is None else np.array(lengths, np.int32))
    s.check(s.run())


@pytest.mark.parametrize("dtype,T,D,N,G", [("f32", 150, 40, 16, 1), ("bf16", 150, 66, 13, 2), ("f32", 20, 70, 64, 1),
                                           ("bf16", 20, 64, 16, 1), ("f32", 20, 33, 12, 1), ("bf16", 20, 36, 20, 3),
                                           ("bf16", 20, 40, 36, 1)])
def test_a_prompt_continued_by_single_tokens(dtype, T, D, N, G):
    """The final states of ragged prompts (with the time axis cut and not), put
    into slots of a larger state and moved on token by token, give what the
    whole sequences give."""
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[scan continued] T={T} D={D} N={N} G={G} {dtype}", flush=True)
    more = 5
    lengths = np.array([T, 0, 1, 17, T - 3], np.int32)
    B = len(lengths)
    s = Scan(23, T + more, B, D, N, G, dtype)
    f32 = torch.float32
    code = s.desc.dtype
    kw = dict(Dskip=s.dev(s.Dskip, f32), dt_bias=s.dev(s.dt_bias, f32))
    A = s.dev(s.A, f32)
    d = J.ScanDesc(D, N, G, B, T, code, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
    need = J.janus_selective_scan_workspace_bytes(d)
    assert (need > 0) == (T >= 128)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    y, h = torch.empty((T, B, D), dtype=s.tdt, device="cuda"), s.dev(s.h0, f32)
    J.janus_selective_scan_fwd(d, s.dev(s.x[:T]), s.dev(s.dt[:T]), A, s.dev(s.Bm[:T]), s.dev(s.Cm[:T]), lengths, y, ws,
                               z=s.dev(s.z[:T]), h0=h, hT=h, **kw)
    slots = torch.tensor([6, 2, 0, 5, 3], dtype=torch.int32, device="cuda")
    state = torch.full((8, D, N), float("nan"), device="cuda")
    state[slots.long()] = h
    one = J.ScanDesc(D, N, G, B, 1, code, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
    rows = np.arange(B)
    for k in range(more):
        at = lambda a: s.dev(a[lengths + k, rows])
        yk = torch.full((B, D), float("nan"), dtype=s.tdt, device="cuda")
        J.janus_selective_scan_step(one, at(s.x), at(s.dt), A, at(s.Bm), at(s.Cm), state, yk, z=at(s.z), slots=slots, **kw)
        ref, end = oracle.forward(s.x, s.dt, s.A, s.Bm, s.Cm, Dskip=s.Dskip, z=s.z, dt_bias=s.dt_bias,
                                  lengths=lengths + k + 1, h0=s.h0)
        near(f"y of token {k}", yk, ref[lengths + k, rows], TOL[dtype])
        near(f"state after token {k}", state[slots.long()], end, TOL["f32"])
    assert bool(torch.isnan(state[[1, 4, 7]]).all())
