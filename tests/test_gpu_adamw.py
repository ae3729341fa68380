"""GPU parity of the AdamW update (janus_adamw_update): 32-bit states against the
float64 oracle, 8-bit states against its bit-by-bit definition; tensors of any size
and alignment, many of them, empty ones, float32 among bf16, masters; steps that are
held; the training steps that end in it.

Tolerances: m and v are sums of two terms with three or four roundings: 2^-22 of the
terms' magnitudes; a parameter adds six roundings of its step (twice the root's and the
quotient's): 2^-23 of itself and 2^-19 of the step; bf16 parameters are rounded once
more: 2^-8."""
import math

import numpy as np
import pytest

from oracle import adamw as oracle
from paper_1812_01329_amd import workloads as wl

pytestmark = pytest.mark.gpu

F = np.float32
HYPER = dict(lr=F(0.01), b1=F(0.9), b2=F(0.99), eps=F(1e-8))


class Case:
    """Tensors of the given sizes; f32: which are float32; shift: elements that a
    tensor starts off a 256-byte boundary."""

    def __init__(self, sizes, bits=32, f32=None, masters=False, shift=0, max_norm=0.0, decay=0.1, seed=0, gscale=1.0):
        import torch
        from paper_1812_01329_amd import janus as J
        self.torch, self.J, self.sizes, self.bits, self.max_norm = torch, J, sizes, bits, max_norm
        rng = np.random.default_rng(seed + len(sizes))
        n = len(sizes)
        self.f32 = [True] * n if f32 is None else f32
        self.decay = [F(decay if i % 2 == 0 else 0.0) for i in range(n)]

        def put(a, dt):
            t = torch.empty(len(a) + shift + 1, dtype=dt, device="cuda")[shift:shift + len(a)]
            t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
            return t
        bf = lambda a: torch.from_numpy(a).bfloat16().float().numpy()
        self.w = [rng.normal(size=s).astype(F) for s in sizes]
        if not masters:
            self.w = [a if f else bf(a) for a, f in zip(self.w, self.f32)]
        self.g = [(rng.normal(size=s) * gscale * np.exp(rng.normal(size=s))).astype(F) for s in sizes]
        self.m = [(rng.normal(size=s) * 0.3 * gscale).astype(F) for s in sizes]
        self.v = [(rng.uniform(0.01, 2, s) * gscale ** 2).astype(F) for s in sizes]
        dts = [torch.float32 if f else torch.bfloat16 for f in self.f32]
        self.P = [put(a, d) for a, d in zip(self.w, dts)]
        self.G = [put(a, torch.float32) for a in self.g]
        self.W = [put(a, torch.float32) if masters and not f else None for a, f in zip(self.w, self.f32)]
        self.S = None
        if bits == 8:
            half = [np.full(s, 0x8000) for s in sizes]
            em = [oracle.encode(a, h) for a, h in zip(self.m, half)]
            ev = [oracle.encode(np.sqrt(a), h) for a, h in zip(self.v, half)]
            self.em, self.ev = em, ev
            self.M, self.V = [put(c, torch.uint8) for c, _ in em], [put(c, torch.uint8) for c, _ in ev]
            self.S = [torch.from_numpy(np.stack([a, b], 1).copy()).cuda() for (_, a), (_, b) in zip(em, ev)]
            self.m = [oracle.decode(*e) for e in em]
            self.v = [oracle.decode(*e) ** 2 for e in ev]
        else:
            self.M, self.V = [put(a, torch.float32) for a in self.m], [put(a, torch.float32) for a in self.v]
        self.step = torch.tensor([4], dtype=torch.int64, device="cuda")
        self.stats = torch.full((2,), 7.0, device="cuda")
        h = HYPER
        self.desc = J.AdamWDesc(n, J.ADAMW_8BIT if bits == 8 else J.ADAMW_F32, h["lr"], h["b1"], h["b2"], h["eps"], max_norm, 77)
        self.tensors = J.adamw_tensors(self.P, self.G, self.M, self.V, self.S, self.W, self.decay)
        self.ws = torch.empty(J.janus_adamw_workspace_bytes(self.desc), dtype=torch.uint8, device="cuda")

    def run(self, **kw):
        self.J.janus_adamw_update(self.desc, self.tensors, self.step, stats=self.stats, ws=self.ws, **kw)

    def all(self):
        return [t for t in (*self.P, *self.M, *self.V, *(self.S or []), *self.W, self.step) if t is not None]

    def check(self, lr=None):
        h, torch = HYPER, self.torch
        lr = float(h["lr"] if lr is None else lr)
        norm, s = oracle.scale_of(self.g, self.max_norm)
        st = self.stats.double().cpu().numpy()
        assert abs(st[0] - norm) <= 2.0 ** -23 * norm and abs(st[1] - s) <= 2.0 ** -23
        assert int(self.step) == 5
        np64 = lambda t: t.detach().double().cpu().numpy()
        for i, n in enumerate(self.sizes):
            p, m, v = oracle.update(self.w[i], self.g[i], self.m[i], self.v[i], 4, lr, float(h["b1"]), float(h["b2"]),
                                    float(h["eps"]), float(self.decay[i]), s)
            if self.bits == 8:
                m32, v32 = oracle.moments32(self.g[i], self.m[i], self.v[i], h["b1"], h["b2"], F(s))
                rm, rv = oracle.random16(77, 5, i, n)
                for got, val, rnd, k in ((self.M[i], m32, rm, 0), (self.V[i], np.sqrt(v32), rv, 1)):
                    code, scale = oracle.encode(val, rnd)
                    np.testing.assert_array_equal(got.cpu().numpy(), code, err_msg=f"tensor {i} of {n}, state {k}")
                    np.testing.assert_array_equal(self.S[i][:, k].cpu().numpy(), scale)
            else:
                assert (np.abs(np64(self.M[i]) - m) <= 2.0 ** -22 * (np.abs(self.m[i]) + np.abs(self.g[i]))).all()
                assert (np.abs(np64(self.V[i]) - v) <= 2.0 ** -22 * v + 1e-40).all()
            tol = 2.0 ** -23 * (np.abs(p) + np.abs(self.w[i])) + 2.0 ** -19 * np.abs(p - self.w[i])
            bf = 0.0 if self.f32[i] else 2.0 ** -8 * np.abs(p)
            if self.W[i] is not None:
                assert (np.abs(np64(self.W[i]) - p) <= tol).all(), f"master {i} of {n}"
                assert torch.equal(self.P[i], self.W[i].bfloat16())
            assert (np.abs(np64(self.P[i]) - p) <= tol + bf).all(), f"tensor {i} of {n}"


SIZES = [1, 2, 3, 4, 5, 63, 64, 255, 256, 257, 1000, 4095, 4096, 4097, 8191, 70001]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 4])
def test_sizes_and_alignments(bits, shift):
    print(f"[adamw] sizes {bits} {shift}", flush=True)
    for f32, masters in ((None, False), ([i % 3 == 0 for i in range(len(SIZES))], True), ([False] * len(SIZES), False)):
        c = Case(SIZES, bits, f32, masters, shift, max_norm=1.0, seed=shift)
        c.run()
        c.check()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("n", [1, 39, 51, 52, 53, 105, 200, 1025])
def test_many_tensors_some_empty(bits, n):
    """More tensors than a launch takes, every seventh of them empty."""
    print(f"[adamw] {n} tensors {bits}", flush=True)
    rng = np.random.default_rng(n)
    sizes = [0 if i % 7 == 3 else int(rng.integers(1, 6000 if n < 1000 else 700)) for i in range(n)]
    c = Case(sizes, bits, [i % 2 == 0 for i in range(n)], True, max_norm=0.5)
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("max_norm", [0.0, -1.0, math.inf, 1e-3, 1e6])
def test_norm_limit(bits, max_norm):
    c = Case([5000, 300], bits, max_norm=max_norm)
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_large_call(bits):
    """More tiles than a launch has workgroups."""
    c = Case([9000001, 3, 700000], bits, [False, True, False], True, max_norm=1.0)
    c.run()
    c.check()


@pytest.mark.parametrize("bits", [32, 8])
def test_held_steps_change_nothing(bits):
    """A gradient that is not finite, a learning rate that is not, a raised hold word:
    no parameter, state, scale or count moves, in any launch."""
    import torch
    sizes = [300] * 50 + [5000]
    c = Case(sizes, bits, [i % 2 == 0 for i in range(51)], True, max_norm=1.0)
    before = [t.clone() for t in c.all()]
    word = torch.ones(1, dtype=torch.int32, device="cuda")
    same = lambda: all(torch.equal(a, b) for a, b in zip(before, c.all()))
    c.run(hold=word.data_ptr())
    assert same() and float(c.stats[1]) == 0.0
    for lr in (math.nan, math.inf):
        c.run(lr=torch.tensor([lr], device="cuda"))
        assert same() and float(c.stats[1]) == 0.0
    for bad in (math.nan, math.inf, -math.inf):
        for i in (0, 17, 50):
            keep = c.G[i][7].clone()
            c.G[i][7] = bad
            c.run()
            assert same() and float(c.stats[1]) == 0.0 and not math.isfinite(float(c.stats[0]))
            c.G[i][7] = keep
    word.zero_()
    c.run(hold=word.data_ptr(), lr=torch.tensor([0.25], device="cuda"))
    c.check(lr=0.25)


def test_far_values_of_eight_bits():
    """States from 2^-100 to 2^50 in blocks of their own, blocks of zeros, one large
    value among tiny ones: codes as defined."""
    import torch
    c = Case([256 * 9], 8, max_norm=0.0)
    g = c.g[0].reshape(9, 256)
    for b, k in enumerate((-100, -60, -30, -8, 8, 30, 50)):
        g[b] *= F(2.0 ** k)
    g[7] = 0.0
    g[8] = F(1e-20)
    g[8, 3] = F(1e19)
    for codes in (c.M[0], c.V[0]):
        codes.view(9, 256)[7:] = 0
    c.m[0].reshape(9, 256)[7:] = 0
    c.v[0].reshape(9, 256)[7:] = 0
    c.G[0].copy_(torch.from_numpy(c.g[0]))
    c.run()
    c.check()


def test_states_from_nothing_follow_the_oracle():
    """Twenty steps from zero states, a new gradient each: the codes are the oracle's to
    the bit, the masters follow it."""
    import torch
    c = Case([777], 8, [False], True)
    for t in (c.M[0], c.V[0], c.S[0], c.step):
        t.zero_()
    h = HYPER
    w = c.w[0].astype(np.float64)
    cm, sm = np.zeros(777, np.uint8), np.zeros(4, F)
    cv, sv = cm.copy(), sm.copy()
    rng = np.random.default_rng(8)
    for t in range(1, 21):
        g = (rng.normal(size=777) * 0.1).astype(F)
        c.G[0].copy_(torch.from_numpy(g))
        c.run()
        m0, r0 = oracle.decode(cm, sm), oracle.decode(cv, sv)
        w, _, _ = oracle.update(w, g, m0, r0.astype(np.float64) ** 2, t - 1, float(h["lr"]), float(h["b1"]), float(h["b2"]),
                                float(h["eps"]), float(c.decay[0]), 1.0)
        m, v = oracle.moments32(g, m0, r0 * r0, h["b1"], h["b2"], 1.0)
        rm, rv = oracle.random16(77, t, 0, 777)
        (cm, sm), (cv, sv) = oracle.encode(m, rm), oracle.encode(np.sqrt(v), rv)
        np.testing.assert_array_equal(c.M[0].cpu().numpy(), cm, err_msg=f"step {t}")
        np.testing.assert_array_equal(c.V[0].cpu().numpy(), cv, err_msg=f"step {t}")
    # (twenty steps of at most about lr each, every one with six roundings)
    assert np.abs(c.W[0].double().cpu().numpy() - w).max() <= 20 * (2.0 ** -22 * np.abs(w).max() + 2.0 ** -19 * 0.02)


def test_a_tensor_of_more_than_2_to_32_elements():
    import torch
    from paper_1812_01329_amd import janus as J
    n = (1 << 32) + 4097
    print("[adamw offsets]", flush=True)
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    at = [0, 1 << 31, (1 << 32) - 1, 1 << 32, n - 1]
    for i in at:
        g[i] = 1.0
    d = J.AdamWDesc(1, J.ADAMW_F32, 0.5, 0.9, 0.99, 1e-8, 0.0, 0)
    step, stats = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(2, device="cuda")
    ws = torch.empty(J.janus_adamw_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    J.janus_adamw_update(d, J.adamw_tensors([p], [g], [m], [v]), step, stats=stats, ws=ws)
    assert float(stats[0]) == pytest.approx(math.sqrt(5.0), rel=1e-6)
    assert [float(p[i]) for i in at] == [-0.5] * 5       # the first step is lr, whatever the gradient
    p.index_fill_(0, torch.tensor(at, device="cuda"), 0.0)
    assert not any(bool(c.any()) for c in p.split(1 << 30))


@pytest.mark.parametrize("bits,masters", [(32, False), (8, False), (32, True)])
@pytest.mark.parametrize("kind", ["lstm", "tree"])
def test_training_steps_end_in_it(kind, bits, masters):
    """A training step with an AdamW update: every parameter moves as the oracle's
    does by the step's own gradients; a state dict resumes to the same bits."""
    import torch
    from paper_1812_01329_amd import train_step as ts
    w = wl.tiny_lstm() if kind == "lstm" else wl.sst_treelstm()
    spec = ts.AdamW(1e-3, max_norm=1.0, decay=0.05, bits=bits, masters=masters)
    step = ts.make_step(w, update=spec)
    up = step.update
    before = [p.double().cpu().numpy() for p in up.params]
    step.run()
    torch.cuda.synchronize()
    grads = [g.double().cpu().numpy() for g in up.grads]
    norm, s = oracle.scale_of(grads, 1.0)
    assert float(up.stats[0]) == pytest.approx(norm, rel=1e-6) and int(up.step) == 1
    for i, (a, g) in enumerate(zip(before, grads)):
        p = oracle.update(a, g, 0 * g, 0 * g, 0, float(F(1e-3)), float(F(0.9)), float(F(0.999)), float(F(1e-8)),
                          float(F(up.tensors[i].decay)), s)[0]
        bf = 2.0 ** -8 if up.params[i].dtype == torch.bfloat16 else 0.0
        # (a gradient next to eps has all of its rounding in the step: 2^-19 of lr at most)
        assert (np.abs(up.params[i].double().cpu().numpy() - p) <= (2.0 ** -22 + bf) * np.abs(a) + 2.0 ** -18 * 1e-3).all(), i
    saved, params = up.state_dict(), [p.clone() for p in up.params]
    step.run()
    torch.cuda.synchronize()
    want = [p.clone() for p in up.params]
    for p, q in zip(up.params, params):
        p.copy_(q)
    up.load_state_dict(saved)
    up.apply()
    # (the gradients are those of the second step; it has to land on the same bits)
    assert all(torch.equal(p, q) for p, q in zip(up.params, want)) and int(up.step) == 2


def test_roots_are_rounded_correctly():
    """With beta2 0 and no states sqrt(v) is |g| itself: gradients that lie, by the element's
    random bits, on the border between two codes and one bit below it come out as
    defined, which a root that is off by its last bit would not."""
    import torch
    from paper_1812_01329_amd import janus as J
    n = 256 * 256
    rng = np.random.default_rng(12)
    rnd = oracle.random16(77, 1, 0, n)[1].astype(np.int64)
    low = ((1 << 20) - (rnd << 4)) % (1 << 20) - np.arange(n) % 2 * (rnd > 0)
    bits = (rng.integers(121, 134, n) << 23) + (rng.integers(0, 8, n) << 20) + low
    g = bits.astype(np.uint32).view(F)
    p, m, v = (torch.zeros(n, dtype=t, device="cuda") for t in (torch.float32, torch.uint8, torch.uint8))
    scale = torch.zeros(n // 256, 2, device="cuda")
    d = J.AdamWDesc(1, J.ADAMW_8BIT, 0.1, 0.9, 0.0, 1e-8, 0.0, 77)
    ws = torch.empty(J.janus_adamw_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    grad = torch.from_numpy(g.copy()).cuda()
    J.janus_adamw_update(d, J.adamw_tensors([p], [grad], [m], [v], [scale]), step, ws=ws)
    code, s = oracle.encode(np.sqrt(g.astype(np.float64) ** 2).astype(F), rnd)
    np.testing.assert_array_equal(scale[:, 1].cpu().numpy(), s)
    np.testing.assert_array_equal(v.cpu().numpy(), code)


@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** -75])
def test_gradients_whose_squares_are_nearly_nothing(eps):
    """A first step from p = m = v = 0 is -lr g / (|g| + eps).  Gradients are powers of
    two whose halved squares a float32 still holds, subnormal ones among them; 0
    gives 0.  (2^-19 of the step, as above: nothing else is rounded here.)"""
    import torch
    from paper_1812_01329_amd import janus as J
    g = np.concatenate([[0.0], 2.0 ** -np.arange(1.0, 75.0)])
    g = np.where(np.arange(g.size) % 3 == 0, -g, g)
    dev = lambda a: torch.from_numpy(a.astype(F)).cuda()
    p, m, v, grad = *(dev(np.zeros(g.size)) for _ in range(3)), dev(g)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = J.AdamWDesc(1, J.ADAMW_F32, 1.0, 0.5, 0.5, eps, 0.0, 0)
    ws = torch.empty(J.janus_adamw_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    J.janus_adamw_update(d, J.adamw_tensors([p], [grad], [m], [v]), step, ws=ws)
    want = -g / (np.abs(g) + eps)
    got = p.cpu().numpy().astype(np.float64)
    assert np.array_equal(v.cpu().numpy().astype(np.float64), g * g / 2)
    assert (np.abs(got - want) <= 2.0 ** -19 * np.abs(want)).all(), (g, got, want)
