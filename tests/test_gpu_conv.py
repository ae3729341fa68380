"""GPU parity of the short causal convolution (janus_causal_conv_fwd, _bwd,
_step) against the float64 oracle: every tap count, lengths from 0, carried
states, strides that are no multiple of 16 bytes, batches past one launch's
lengths, garbage past the sequences' ends, infinite inputs.

Tolerances (relative to the largest entry of a tensor): float32 results are
sums of at most a few thousand float32 products, rounded to 2^-24 each and with
the logistic function off by a few ulp: 2e-5.  A bf16 result is one rounding of
such a value, 2^-9 of it at most: 2^-8 leaves room for the sums."""
import numpy as np
import pytest

from oracle import conv as oracle
from paper_1812_01329_amd import workloads as wl

pytestmark = pytest.mark.gpu
TOL = {"f32": 2e-5, "bf16": 2.0 ** -8}


def near(name, got, ref, tol):
    got = got.detach().double().cpu().numpy()
    assert got.shape == ref.shape, name
    err = np.abs(got - ref).max() / max(np.abs(ref).max(), 1e-30) if ref.size else 0.0
    assert err <= tol, f"{name}: {err:.3e} > {tol:.1e}"


class Conv:
    """Seeded inputs on the host (bf16-exact for bf16) and on the device."""

    def __init__(self, seed, T, B, D, K, dtype, silu=True, lengths=None, state=True, bias=True, pad=(0, 0)):
        import torch
        from paper_1812_01329_amd import janus as J
        self.J, self.torch = J, torch
        rng = np.random.default_rng(seed)
        r = lambda a: wl.bf16_round(a.astype(np.float32)) if dtype == "bf16" else a.astype(np.float32)
        self.tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.T, self.B, self.D, self.K, self.silu, self.dtype, self.lengths = T, B, D, K, silu, dtype, lengths
        self.x, self.dy = r(rng.normal(size=(T, B, D))), r(rng.normal(size=(T, B, D)))
        self.w, self.bias = r(rng.normal(size=(D, K)) * 0.5), r(rng.normal(size=D)) if bias else None
        self.s0 = r(rng.normal(size=(B, K - 1, D))) if state else None
        self.dsT = rng.normal(size=(B, K - 1, D)).astype(np.float32)
        self.pad = pad
        self.desc = J.ConvDesc(D, K, B, T, J.BF16 if dtype == "bf16" else J.F32,
                               J.CONV_SILU if silu else J.CONV_LINEAR, D + pad[0], D + pad[1])

    def dev(self, a, dt=None):
        return None if a is None else self.torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dt or self.tdt)

    def rows(self, a, which):
        """[T, B, D] rows inside a wider buffer (NaN outside), or an empty one."""
        wide = self.torch.full((self.T, self.B, self.D + self.pad[which]), float("nan"), dtype=self.tdt, device="cuda")
        v = wide[:, :, :self.D]
        if a is not None:
            v.copy_(self.dev(a))
        return v

    def run(self):
        torch, J = self.torch, self.J
        x, dy = self.rows(self.x, 0), self.rows(self.dy, 1)
        if self.lengths is not None:   # nothing past an end is read
            for b, n in enumerate(self.lengths):
                x[n:, b] = float("nan")
                dy[n:, b] = float("nan")
        w, bias, s0 = self.dev(self.w), self.dev(self.bias), self.dev(self.s0)
        y, dx = self.rows(None, 1), self.rows(None, 0)
        new = lambda *s, dt=torch.float32: torch.full(s, float("nan"), dtype=dt, device="cuda")
        sT = new(self.B, self.K - 1, self.D, dt=self.tdt)
        dw, db, ds0 = new(self.D, self.K), new(self.D), new(self.B, self.K - 1, self.D)
        ws = torch.empty(J.janus_causal_conv_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")
        J.janus_causal_conv_fwd(self.desc, x, self.lengths, w, bias, s0, y, sT)
        J.janus_causal_conv_bwd(self.desc, x, self.lengths, w, bias, s0, dy, self.dev(self.dsT, torch.float32), dx,
                                dw, db, ds0, ws)
        torch.cuda.synchronize()
        return dict(y=y, sT=sT, dx=dx, dw=dw, dbias=db, ds0=ds0)

    def check(self, got):
        y, sT = oracle.forward(self.x, self.lengths, self.w, self.bias, self.s0, self.silu)
        dx, dw, db, ds0 = oracle.backward(self.x, self.lengths, self.w, self.bias, self.s0, self.silu, self.dy, self.dsT)
        t, f = TOL[self.dtype], TOL["f32"]
        near("y", got["y"], y, t)
        near("sT", got["sT"], sT, 0.0)
        near("dx", got["dx"], dx, t)
        near("dw", got["dw"], dw, f)
        near("dbias", got["dbias"], db, f)
        near("ds0", got["ds0"], ds0, f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", range(1, 9))
def test_taps(K, dtype):
    print(f"[conv] K={K} {dtype}", flush=True)
    lengths = np.array([11, 0, 1, K - 1, K, 13], np.int32)
    for silu, pad in ((True, (0, 0)), (False, (3, 5))):
        c = Conv(K, 13, 6, 40, K, dtype, silu, lengths, pad=pad)
        c.check(c.run())


@pytest.mark.parametrize("dtype,D,pad", [("bf16", 650, (2, 0)), ("bf16", 513, (0, 0)), ("bf16", 1032, (8, 16)),
                                         ("f32", 301, (0, 1)), ("f32", 260, (4, 0)), ("bf16", 1, (0, 0))])
@pytest.mark.parametrize("T,B", [(1, 1), (2, 3), (150, 2), (5, 300)])
def test_sizes_and_strides(T, B, dtype, D, pad):
    """Widths that take each access width, one step, long sequences in several
    segments, and more sequences than one launch carries lengths for."""
    print(f"[conv] T={T} B={B} D={D} {dtype} pad={pad}", flush=True)
    if B == 300 and D > 700:
        D = 520
    lengths = np.random.default_rng(T + B).integers(0, T + 1, B).astype(np.int32)
    c = Conv(7, T, B, D, 4, dtype, True, lengths, pad=pad)
    c.check(c.run())
    c = Conv(8, T, B, D, 3, dtype, False, None, state=False, bias=False, pad=pad)
    c.check(c.run())


def test_no_steps():
    """T = 0: the state goes through, its gradient comes back."""
    c = Conv(3, 0, 2, 24, 4, "f32")
    got = c.run()
    near("sT", got["sT"], c.s0.astype(np.float64), 0.0)
    near("ds0", got["ds0"], c.dsT.astype(np.float64), 0.0)
    assert not got["dw"].any() and not got["dbias"].any()


def test_infinite_input_stays_within_its_taps():
    c = Conv(4, 12, 1, 8, 3, "f32", False)
    c.x[5, 0, 2] = np.inf
    y = c.run()["y"].cpu().numpy()
    assert np.isinf(y[5:8, 0, 2]).all()
    y[5:8, 0, 2] = 0
    assert np.isfinite(y).all()


def test_repeats_bit_for_bit():
    c = Conv(5, 90, 40, 130, 4, "bf16", lengths=np.arange(40, dtype=np.int32) * 2)
    a, b = c.run(), c.run()
    for k in a:
        assert c.torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype,D,K", [("f32", 33, 4), ("bf16", 64, 3), ("bf16", 650, 4), ("f32", 8, 1)])
def test_step(dtype, D, K):
    """Single tokens on slots of a larger state: a row without a slot gives 0
    and moves nothing; a prompt's final state continues."""
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[conv step] {dtype} D={D} K={K}", flush=True)
    c = Conv(6, 3, 5, D, K, dtype)
    rng = np.random.default_rng(9)
    state = rng.normal(size=(9, K - 1, D)).astype(np.float32)
    state = wl.bf16_round(state) if dtype == "bf16" else state
    slots = np.array([8, -1, 0, 3, 9], np.int32)
    ds, w, bias, ref = c.dev(state), c.dev(c.w), c.dev(c.bias), state
    d = J.ConvDesc(D, K, 5, 1, c.desc.dtype, c.desc.act, D, D)
    for t in range(3):
        y = torch.full((5, D), float("nan"), dtype=c.tdt, device="cuda")
        J.janus_causal_conv_step(d, c.dev(c.x[t]), w, bias, ds, y, slots=torch.from_numpy(slots).cuda())
        yr, ref = oracle.step(c.x[t], c.w, c.bias, ref, slots, True)
        near("y", y, yr, TOL[dtype])
        near("state", ds, ref, 0.0)
    # rows to slots of their own number
    s5 = c.dev(state[:5])
    y = torch.empty((5, D), dtype=c.tdt, device="cuda")
    J.janus_causal_conv_step(d, c.dev(c.x[0]), w, bias, s5, y)
    yr, _ = oracle.step(c.x[0], c.w, c.bias, state[:5], range(5), True)
    near("y", y, yr, TOL[dtype])
