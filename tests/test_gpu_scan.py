"""GPU parity of the selective scan (janus_selective_scan_fwd, _bwd, _step)
against the float64 oracle: state counts with and without padding, groups,
lengths from 0, time cut into segments, several workgroups along the channels,
strided rows of packed buffers, garbage past the sequences' ends.

Tolerances (relative to the largest entry of a tensor): decays are at most 1, so
a float32 state gathers one rounding of 2^-24 and an exponential off by about
2^-22 of itself a step, over the few hundred steps that it remembers; the sums
over channels and time add their roundings: 1e-4.  A bf16 result is one rounding
of such a value: 2^-8."""
import numpy as np
import pytest

from oracle import scan as oracle
from paper_1812_01329_amd import workloads as wl

pytestmark = pytest.mark.gpu
TOL = {"f32": 1e-4, "bf16": 2.0 ** -8}


def near(name, got, ref, tol):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, name
    err = np.abs(got - ref).max() / max(np.abs(ref).max(), 1e-30) if ref.size else 0.0
    assert err <= tol, f"{name}: {err:.3e} > {tol:.1e}"


class Scan:
    def __init__(self, seed, T, B, D, N, G, dtype, lengths=None, gate=True, skip=True, bias=True, state=True,
                 softplus=True, pads=(0,) * 6):
        import torch
        from paper_1812_01329_amd import janus as J
        self.J, self.torch = J, torch
        rng = np.random.default_rng(seed)
        r = lambda a: wl.bf16_round(a.astype(np.float32)) if dtype == "bf16" else a.astype(np.float32)
        f = lambda a: a.astype(np.float32)
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.T, self.B, self.D, self.N, self.G, self.dtype, self.lengths = T, B, D, N, G, dtype, lengths
        self.softplus, self.pads = softplus, pads
        self.x, self.dy = r(rng.normal(size=(T, B, D))), r(rng.normal(size=(T, B, D)))
        self.dt = r(rng.normal(size=(T, B, D)) * 0.5 if softplus else rng.uniform(0.01, 0.2, (T, B, D)))
        self.Bm, self.Cm = r(rng.normal(size=(T, B, G, N))), r(rng.normal(size=(T, B, G, N)))
        self.z = r(rng.normal(size=(T, B, D))) if gate else None
        self.A = f(-rng.uniform(0.3, 1.2, (D, N)) * np.arange(1, N + 1))
        self.Dskip = f(rng.normal(size=D)) if skip else None
        self.dt_bias = f(rng.uniform(-5, -1, D) if softplus else rng.uniform(0, 0.1, D)) if bias else None
        self.h0 = f(rng.normal(size=(B, D, N))) if state else None
        self.dhT = f(rng.normal(size=(B, D, N))) if state else None
        code = J.BF16 if dtype == "bf16" else J.F32
        rows = (D, D, G * N, G * N, D, D)
        self.desc = J.ScanDesc(D, N, G, B, T, code, (J.SCAN_SOFTPLUS if softplus else 0) | J.SCAN_KEEP,
                               *(n + p for n, p in zip(rows, pads)))

    def dev(self, a, dt=None):
        return None if a is None else self.torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dt or self.tdt)

    def rows(self, shape, a, which, dead=False):
        """Rows inside a wider buffer, NaN outside and (dead) past the ends."""
        n = int(np.prod(shape[2:]))
        wide = self.torch.full((*shape[:2], n + self.pads[which]), float("nan"), dtype=self.tdt, device="cuda")
        if a is not None:
            wide[:, :, :n] = self.dev(a).view(*shape[:2], n)
        if dead and self.lengths is not None:
            for b, m in enumerate(self.lengths):
                wide[m:, b] = float("nan")
        self.wide.append(wide)
        return wide

    def run(self, h0=True):
        torch, J = self.torch, self.J
        self.wide = []
        rd, rn = (self.T, self.B, self.D), (self.T, self.B, self.G, self.N)
        f32 = torch.float32
        x, dt = self.rows(rd, self.x, 0, True), self.rows(rd, self.dt, 1, True)
        Bm, Cm = self.rows(rn, self.Bm, 2, True), self.rows(rn, self.Cm, 3, True)
        z = None if self.z is None else self.rows(rd, self.z, 4, True)
        dy = self.rows(rd, self.dy, 5, True)
        y, dx, ddt = self.rows(rd, None, 5), self.rows(rd, None, 0), self.rows(rd, None, 1)
        dB, dC = self.rows(rn, None, 2), self.rows(rn, None, 3)
        dz = None if z is None else self.rows(rd, None, 4)
        new = lambda *s: torch.full(s, float("nan"), device="cuda")
        hT, dh0 = new(self.B, self.D, self.N), new(self.B, self.D, self.N)
        dA, dD, dtb = new(self.D, self.N), new(self.D), new(self.D)
        ws = torch.full((J.janus_selective_scan_workspace_bytes(self.desc),), 0xff, dtype=torch.uint8, device="cuda")
        kw = dict(Dskip=self.dev(self.Dskip, f32), z=z, dt_bias=self.dev(self.dt_bias, f32), h0=self.dev(self.h0, f32))
        A = self.dev(self.A, f32)
        J.janus_selective_scan_fwd(self.desc, x, dt, A, Bm, Cm, self.lengths, y, ws, hT=hT, **kw)
        J.janus_selective_scan_bwd(self.desc, x, dt, A, Bm, Cm, self.lengths, dy, ws, dx, ddt, dA, dB, dC,
                                   dhT=self.dev(self.dhT, f32), dDskip=dD, dz=dz, ddt_bias=dtb, dh0=dh0, **kw)
        torch.cuda.synchronize()
        cut = lambda t, n, s: t[:, :, :n].reshape(s)
        o = dict(y=cut(y, self.D, rd), hT=hT, dx=cut(dx, self.D, rd), ddt=cut(ddt, self.D, rd), dA=dA,
                 dBm=cut(dB, self.G * self.N, rn), dCm=cut(dC, self.G * self.N, rn), dDskip=dD, ddt_bias=dtb, dh0=dh0)
        if z is not None:
            o["dz"] = cut(dz, self.D, rd)
        # nothing is written between the rows
        for wide, n in ((y, self.D), (dx, self.D), (ddt, self.D), (dB, self.G * self.N), (dC, self.G * self.N)):
            assert bool(torch.isnan(wide[:, :, n:]).all())
        return o

    def reference(self):
        kw = dict(Dskip=self.Dskip, z=self.z, dt_bias=self.dt_bias, lengths=self.lengths, h0=self.h0,
                  softplus=self.softplus)
        y, hT = oracle.forward(self.x, self.dt, self.A, self.Bm, self.Cm, **kw)
        o = oracle.backward(self.x, self.dt, self.A, self.Bm, self.Cm, self.dy, dhT=self.dhT, **kw)
        return dict(o, y=y, hT=hT)

    def check(self, got):
        ref = self.reference()
        for k in got:
            near(k, got[k], ref[k], TOL["f32" if k in ("hT", "dA", "dDskip", "ddt_bias", "dh0") else self.dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 4, 8, 13, 16, 20, 32, 33, 64])
def test_states(N, dtype):
    print(f"[scan] N={N} {dtype}", flush=True)
    s = Scan(N, 21, 4, 70, N, 1, dtype, np.array([21, 0, 1, 17], np.int32))
    s.check(s.run())


@pytest.mark.parametrize("gate,skip,bias,state,softplus", [(False, True, True, True, True), (True, False, False, False, True),
                                                           (False, False, False, False, False), (True, True, True, True, False)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_optional_parts(dtype, gate, skip, bias, state, softplus):
    print(f"[scan] parts {dtype} {gate} {skip} {bias} {state} {softplus}", flush=True)
    s = Scan(5, 19, 3, 66, 16, 1, dtype, None, gate, skip, bias, state, softplus)
    s.check(s.run())


@pytest.mark.parametrize("T,B,D,N,G", [
    (1, 1, 1, 16, 1), (1, 5, 130, 16, 2), (8, 2, 64, 16, 1), (40, 3, 600, 16, 1), (33, 2, 516, 8, 2),
    (400, 1, 96, 16, 1),      # one sequence: time in segments
    (301, 2, 300, 13, 3), (260, 1, 700, 4, 1),
    (3, 300, 65, 16, 1),      # more sequences than one launch carries lengths for
])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes(dtype, T, B, D, N, G):
    print(f"[scan] T={T} B={B} D={D} N={N} G={G} {dtype}", flush=True)
    rng = np.random.default_rng(T + B)
    for lengths in (None, rng.integers(0, T + 1, B).astype(np.int32)):
        s = Scan(11, T, B, D, N, G, dtype, lengths)
        s.check(s.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pads", [(7, 1, 3, 5, 2, 9), (8, 16, 8, 24, 8, 8)])
def test_strided_rows(dtype, pads):
    print(f"[scan] pads={pads} {dtype}", flush=True)
    s = Scan(12, 30, 3, 72, 16, 1, dtype, np.array([30, 9, 25], np.int32), pads=pads)
    s.check(s.run())


def test_no_steps():
    s = Scan(13, 0, 2, 20, 16, 1, "f32")
    got = s.run()
    near("hT", got["hT"], s.h0.astype(np.float64), 0.0)
    near("dh0", got["dh0"], s.dhT.astype(np.float64), 0.0)
    assert not got["dA"].any()


@pytest.mark.parametrize("T,B", [(200, 1), (24, 6)])
def test_repeats_bit_for_bit(T, B):
    s = Scan(14, T, B, 530, 16, 1, "bf16")
    a, b = s.run(), s.run()
    for k in a:
        assert s.torch.equal(a[k], b[k]), k


def test_prompt_needs_no_kept_states_and_continues():
    """Without KEEP the same y and hT; two halves with the state carried are
    the whole (the forward may overwrite its own initial state)."""
    import torch
    from paper_1812_01329_amd import janus as J
    s = Scan(15, 64, 2, 100, 16, 1, "f32")
    whole = s.run()
    f32 = torch.float32
    h = s.dev(s.h0, f32)
    ys = []
    for lo, hi in ((0, 24), (24, 64)):
        d = J.ScanDesc(100, 16, 1, 2, hi - lo, J.F32, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
        y = torch.empty((hi - lo, 2, 100), device="cuda")
        need = J.janus_selective_scan_workspace_bytes(d)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        J.janus_selective_scan_fwd(d, s.dev(s.x[lo:hi]), s.dev(s.dt[lo:hi]), s.dev(s.A), s.dev(s.Bm[lo:hi]),
                                   s.dev(s.Cm[lo:hi]), None, y, ws, Dskip=s.dev(s.Dskip), z=s.dev(s.z[lo:hi]),
                                   dt_bias=s.dev(s.dt_bias), h0=h, hT=h)
        ys.append(y)
    ref = s.reference()
    near("y", torch.cat(ys), ref["y"], TOL["f32"])
    near("hT", h, ref["hT"], TOL["f32"])
    near("whole", whole["y"], ref["y"], TOL["f32"])


def test_extreme_step_sizes():
    """Very large and very small step sizes: the state is replaced or kept, and
    nothing turns into NaN."""
    s = Scan(16, 12, 2, 64, 16, 1, "f32")
    s.dt[:, :, 0::4], s.dt[:, :, 1::4], s.dt[:, :, 2::4] = 60.0, -60.0, -100.0
    s.dt_bias[:] = 0.0
    got, ref = s.run(), s.reference()
    for k in got:
        assert bool(got[k].isfinite().all()), k
    near("y", got["y"], ref["y"], TOL["f32"])
    near("hT", got["hT"], ref["hT"], TOL["f32"])
    near("ddt", got["ddt"], ref["ddt"], TOL["f32"])


@pytest.mark.parametrize("dtype,D,N,G", [("f32", 33, 16, 1), ("bf16", 64, 16, 2), ("bf16", 130, 13, 1), ("f32", 12, 1, 3),
                                         ("f32", 20, 64, 1), ("bf16", 70, 32, 1)])
def test_step(dtype, D, N, G):
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[scan step] {dtype} D={D} N={N} G={G}", flush=True)
    s = Scan(17, 3, 5, D, N, G, dtype)
    state = np.random.default_rng(3).normal(size=(9, D, N)).astype(np.float32)
    slots = np.array([8, -1, 0, 3, 9], np.int32)
    f32 = torch.float32
    ds, ref = s.dev(state, f32), state
    d = J.ScanDesc(D, N, G, 5, 1, s.desc.dtype, J.SCAN_SOFTPLUS, 0, 0, 0, 0, 0, 0)
    for t in range(3):
        y = torch.full((5, D), float("nan"), dtype=s.tdt, device="cuda")
        J.janus_selective_scan_step(d, s.dev(s.x[t]), s.dev(s.dt[t]), s.dev(s.A, f32), s.dev(s.Bm[t]), s.dev(s.Cm[t]),
                                    ds, y, Dskip=s.dev(s.Dskip, f32), z=s.dev(s.z[t]), dt_bias=s.dev(s.dt_bias, f32),
                                    slots=torch.from_numpy(slots).cuda())
        yr, ref = oracle.step(s.x[t], s.dt[t], s.A, s.Bm[t], s.Cm[t], ref, slots, s.Dskip, s.z[t], s.dt_bias)
        near("y", y, yr, TOL[dtype])
        near("state", ds, ref, TOL["f32"])
    # no gate, no skip, no bias, rows to slots of their own number
    s5, y = s.dev(state[:5], f32), torch.empty((5, D), dtype=s.tdt, device="cuda")
    J.janus_selective_scan_step(d, s.dev(s.x[0]), s.dev(s.dt[0]), s.dev(s.A, f32), s.dev(s.Bm[0]), s.dev(s.Cm[0]), s5, y)
    yr, hr = oracle.step(s.x[0], s.dt[0], s.A, s.Bm[0], s.Cm[0], state[:5], range(5))
    near("y", y, yr, TOL[dtype])
    near("state", s5, hr, TOL["f32"])
