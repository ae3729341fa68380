"""GPU parity of the token sampler (janus_sample) against the float64 oracle:
tokens and counts equal, over vocabularies from 1 to past what a workgroup holds,
every filter and their combinations, ties, forbidden tokens, rows with nothing to
choose and rows that are not numbers.

Tolerances: logp is a difference of float32 values of up to about 30 (ulp 2^-19),
with a sum of up to 2^18 exponentials in a tree: 2e-5; draw_logp is rounded once from
64 bits: 2^-23 of itself, and 1e-11 of a weight's rounding."""
import math

import numpy as np
import pytest

from oracle import sample as oracle

pytestmark = pytest.mark.gpu


def bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).bfloat16().float().numpy()


def run(x, u, dtype="f32", pad=0, shift=0, T=1.0, k=0, p=1.0, minp=0.0, per_row=True, want=True):
    """Tokens, logp, draw_logp and kept of the rows x; settings numbers or lists."""
    import torch
    from paper_1812_01329_amd import janus as J
    R, V = x.shape
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    flat = torch.full((R * (V + pad) + shift,), float("nan"), dtype=dt, device="cuda")
    logits = flat[shift:].view(R, V + pad)[:, :V]
    logits.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)))
    dev = lambda v, d: torch.from_numpy(np.broadcast_to(np.asarray(v, d), (R,)).copy()).cuda()
    kw = {}
    d = [1.0, 0, 1.0, 0.0]
    if per_row:
        kw = dict(temperature=dev(T, np.float32), top_k=dev(k, np.int32), top_p=dev(p, np.float32), min_p=dev(minp, np.float32))
    else:
        d = [T, k, p, minp]
    desc = J.SampleDesc(R, V, J.F32 if dtype == "f32" else J.BF16, V + pad if pad else 0, *d)
    tokens = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    if want:
        kw.update(logp=torch.full((R,), 7.0, device="cuda"), draw_logp=torch.full((R,), 7.0, device="cuda"),
                  kept=torch.full((R,), -7, dtype=torch.int32, device="cuda"))
    ws = torch.empty(max(1, J.janus_sample_workspace_bytes(desc)), dtype=torch.uint8, device="cuda")
    J.janus_sample(desc, logits, dev(u, np.float32), tokens, ws=ws, **kw)
    torch.cuda.synchronize()
    return tuple(t.cpu().numpy() for t in ([tokens, kw["logp"], kw["draw_logp"], kw["kept"]] if want else [tokens]))


def check(x, u, got, T=1.0, k=0, p=1.0, minp=0.0):
    R = len(x)
    f = lambda v: np.broadcast_to(np.asarray(v, np.float32), (R,)).astype(np.float64)
    T, k, p, minp, u = f(T), np.broadcast_to(k, (R,)), f(p), f(minp), f(u)
    for r in range(R):
        ref = oracle.draw(x[r], u[r], T[r], int(k[r]), p[r], minp[r])
        ref = (ref[0], *(float(np.float32(v)) if abs(v) > 3e38 else v for v in ref[1:3]), ref[3])   # (past float32: -inf)
        one = [g[r] for g in got]
        at = f"row {r}: T={T[r]} k={k[r]} p={p[r]} minp={minp[r]} u={u[r]!r}: {one} against {ref}"
        assert one[0] == ref[0] and one[3] == ref[3], at
        for a, b, tol in ((one[1], ref[1], 2e-5 * max(1.0, abs(ref[1]) / 8)), (one[2], ref[2], 2.0 ** -23 * abs(ref[2]) + 1e-10)):
            assert (math.isnan(a) and math.isnan(b)) or a == b or abs(a - b) <= tol, at


SETTINGS = [dict(), dict(T=0.6), dict(T=0.0), dict(k=1), dict(k=5, T=1.3), dict(k=50), dict(p=0.9), dict(p=0.3, T=0.7),
            dict(minp=0.1), dict(k=40, p=0.8, T=0.8), dict(k=300, p=0.95, minp=0.02), dict(p=0.999, minp=0.001, T=2.0)]
SIZES = [1, 2, 3, 7, 8, 63, 64, 65, 500, 1000, 2049, 4096, 10007, 32768, 65529, 131075]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_filters(V, dtype):
    """Every setting on rows of its own: normal logits, a tenth of them forbidden."""
    print(f"[sample] V={V} {dtype}", flush=True)
    rng = np.random.default_rng(V)
    R = len(SETTINGS) * (2 if V > 20000 else 4)
    x = (rng.normal(size=(R, V)) * 2.5).astype(np.float32)
    x[:, 1:][rng.random((R, V - 1)) < 0.1] = -np.inf
    x = bf16(x) if dtype == "bf16" else x
    s = {n: [SETTINGS[r % len(SETTINGS)].get(n, v) for r in range(R)] for n, v in dict(T=1.0, k=0, p=1.0, minp=0.0).items()}
    u = rng.random(R).astype(np.float32)
    check(x, u, run(x, u, dtype, **s), **s)


@pytest.mark.parametrize("dtype,pad,shift", [("f32", 1, 0), ("f32", 3, 2), ("bf16", 5, 3), ("bf16", 8, 1), ("bf16", 0, 7)])
@pytest.mark.parametrize("V", [37, 1001, 9973])
def test_rows_that_start_anywhere(V, dtype, pad, shift):
    """Row strides and starts off 16 bytes; NaN between the rows is not read; the
    descriptor's settings instead of the rows'."""
    rng = np.random.default_rng(V + pad)
    x = rng.normal(size=(7, V)).astype(np.float32) * 2
    x = bf16(x) if dtype == "bf16" else x
    u = rng.random(7).astype(np.float32)
    for s in (dict(), dict(T=0.9, k=20, p=0.9), dict(minp=0.2)):
        check(x, u, run(x, u, dtype, pad, shift, per_row=False, **s), **s)
        assert (run(x, u, dtype, pad, shift, per_row=False, want=False, **s)[0] == run(x, u, dtype, pad, shift, **s)[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [10, 600, 5000, 70000])
def test_ties(V, dtype):
    """Few different logits, so that the filters cut among hundreds of equal ones:
    the lowest indices stay."""
    print(f"[sample ties] V={V} {dtype}", flush=True)
    rng = np.random.default_rng(V)
    for levels in ([0.0], [0.0, -0.0, 1.0], [-1.0, 0.5, 3.0], list(np.arange(8) * 0.25)):
        x = rng.choice(np.array(levels, np.float32), size=(12, V))
        s = dict(T=[1.0, 0.5, 2.0, 0.0] * 3, k=[0, 3, V // 2, 0] * 3, p=[1.0, 0.7, 0.35, 1.0, 0.9, 1.0] * 2,
                 minp=[0.0, 0.0, 0.0, 0.5] * 3)
        u = rng.random(12).astype(np.float32)
        check(x, u, run(x, u, dtype, **s), **s)


@pytest.mark.parametrize("V", [5, 3000, 40000])
def test_masks_and_far_values(V):
    """The type's lowest value, large negative masks and -inf beside ordinary logits;
    nothing but such masks; very far and very near values; extreme temperatures."""
    print(f"[sample masks] V={V}", flush=True)
    rng = np.random.default_rng(V)
    low = float(np.finfo(np.float32).min)
    base = rng.normal(size=V).astype(np.float32)
    rows = []
    for mask in (low, -1e4, -1e9, -np.inf):
        a = base.copy()
        a[rng.random(V) < 0.7] = mask
        a[V // 2] = 0.25
        rows.append(a)
    rows += [np.full(V, low), np.full(V, -1e4), np.linspace(-3e38, 3e38, V), base * 1e-30, base * 1e-42, base * 1e30,
             np.where(np.arange(V) == V - 1, 1.0, -np.inf)]
    rows = [np.asarray(a, np.float32) for a in rows]
    x, s, us = [], dict(T=[], k=[], p=[], minp=[]), []
    for a in rows:
        for T, k, p, minp in ((1.0, 0, 1.0, 0.0), (1.0, 7, 0.9, 0.0), (0.5, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.3), (math.inf, 0, 0.5, 0.0),
                              (1e-30, 3, 1.0, 0.0), (1e30, 0, 1.0, 0.0), (0.0, 5, 0.5, 0.5)):
            x.append(a)
            for n, v in zip(s, (T, k, p, minp)):
                s[n].append(v)
            us.append(rng.random())
    x, u = np.stack(x), np.array(us, np.float32)
    check(x, u, run(x, u, "f32", **s), **s)


def test_limits_of_settings_and_chances():
    rng = np.random.default_rng(5)
    x = rng.normal(size=(1, 999)).astype(np.float32).repeat(24, 0)
    u = np.array([0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -1.0, np.inf, -np.inf, 0.5] * 3, np.float32)
    for s in (dict(k=999), dict(k=5000), dict(k=-3), dict(p=0.0), dict(p=-1.0), dict(p=2.0), dict(p=1.0 - 2.0 ** -24),
              dict(minp=1.0), dict(minp=9.0), dict(minp=-1.0), dict(minp=math.inf), dict(p=math.inf), dict(p=-math.inf)):
        check(x, u, run(x, u, "f32", **s), **s)


def test_bad_rows():
    """Nothing to choose from, and what is not a number, beside good rows."""
    rng = np.random.default_rng(6)
    for V in (9, 20000):
        x = rng.normal(size=(12, V)).astype(np.float32)
        x[0] = -np.inf
        x[1, V - 1] = np.nan
        x[2] = -np.inf
        x[2, 4] = np.nan
        x[3, 0] = np.inf
        x[4] = np.nan
        s = dict(T=[1.0] * 5 + [-1.0, math.nan, 1.0, 1.0, 1.0, 0.0, 1.0], k=[0] * 11 + [4],
                 p=[1.0] * 7 + [math.nan] + [1.0] * 4, minp=[0.0] * 8 + [math.nan] + [0.0] * 3)
        u = rng.random(12).astype(np.float32)
        u[9] = np.nan
        got = run(x, u, "f32", **s)
        check(x, u, got, **s)
        assert (got[0][:10] == -1).all() and (got[0][10:] >= 0).all()


def test_frequencies():
    """100000 draws from one row: each token's count within six deviations of its share."""
    import torch
    rng = np.random.default_rng(7)
    row = rng.normal(size=300).astype(np.float32) * 1.5
    n = 100000
    x = np.broadcast_to(row, (n, 300))
    u = torch.rand(n, generator=torch.Generator().manual_seed(1)).numpy()
    tok = run(x, u, "f32", T=1.2, k=100, p=0.9, want=False)[0]
    at, w = oracle.kept(row, 1.2000000476837158, 100, 0.8999999761581421)
    q = np.zeros(300)
    q[at] = w / w.sum()
    c = np.bincount(tok, minlength=300)
    assert (np.abs(c - n * q) <= 6 * np.sqrt(n * q * (1 - q)) + 1e-9).all()


def test_rows_more_than_2_to_32_elements_apart():
    import torch
    from paper_1812_01329_amd import janus as J
    ld, V = (1 << 32) + 3, 1000
    print("[sample offsets]", flush=True)
    big = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((3, V), (ld, 1))
    x.copy_(torch.randn(3, V, generator=torch.Generator().manual_seed(1)))
    u, tok = torch.tensor([0.1, 0.5, 0.9], device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    want = torch.empty_like(tok)
    J.janus_sample(J.SampleDesc(3, V, J.BF16, ld, 1.0, 0, 0.9, 0.0), x, u, tok)
    J.janus_sample(J.SampleDesc(3, V, J.BF16, 0, 1.0, 0, 0.9, 0.0), x.contiguous(), u, want)
    assert torch.equal(tok, want)


@pytest.mark.parametrize("dtype,V,shift", [("bf16", 4096, 0), ("bf16", 4097, 0), ("bf16", 16384, 0), ("bf16", 16384, 3), ("bf16", 65536, 0),
                                           ("bf16", 65536, 5), ("bf16", 65544, 0), ("f32", 2048, 1), ("f32", 8192, 0),
                                           ("f32", 32768, 2), ("f32", 32772, 0), ("f32", 100000, 0)])
def test_every_way_to_the_token(dtype, V, shift):
    """Around the sizes at which a row goes to more threads, or no longer to LDS: lists of a few
    entries, of hundreds, past what a workgroup lists; bins alone; peaked rows beside flat ones."""
    print(f"[sample ways] {dtype} {V} {shift}", flush=True)
    rng = np.random.default_rng(V)
    settings = [dict(), dict(k=2), dict(k=130), dict(k=500), dict(k=900), dict(k=3000, p=0.9), dict(p=0.97, T=1.5), dict(p=0.4),
                dict(minp=0.3), dict(minp=0.01, T=1.5), dict(minp=1e-4, T=2.0), dict(minp=0.02, p=0.6), dict(T=0.0), dict(T=1e-3, p=0.99)]
    flat = rng.normal(size=(len(settings), V)) * 2.5
    peaked = rng.normal(size=(len(settings), V)) * 1.5
    peaked[:, rng.integers(0, V, 8)] += 15.0
    x = np.concatenate([flat, peaked]).astype(np.float32)
    x = bf16(x) if dtype == "bf16" else x
    s = {n: [c.get(n, v) for c in settings] * 2 for n, v in dict(T=1.0, k=0, p=1.0, minp=0.0).items()}
    u = rng.random(len(x)).astype(np.float32)
    check(x, u, run(x, u, dtype, shift=shift, **s), **s)


@pytest.mark.parametrize("dtype,V", [("f32", 301), ("bf16", 5000), ("bf16", 20008), ("bf16", 20001), ("f32", 40000)])
def test_more_rows_than_workgroups(dtype, V):
    """A workgroup takes several rows one after another: each is what it is alone (logp, a
    float32 sum whose order follows the row's start in memory, within its tolerance)."""
    rng = np.random.default_rng(V)
    R = 1100
    x = (rng.normal(size=(R, V)) * 2).astype(np.float32)
    x[::7, 1] = np.nan
    x[::11] = -np.inf
    s = dict(T=[1.0, 0.0, 0.8, 1.3] * 275, k=[0, 0, 40, 0, 400] * 220, p=[1.0, 0.9, 1.0, 0.8] * 275, minp=[0.0, 0.0, 0.05, 0.0] * 275)
    u = rng.random(R).astype(np.float32)
    got = run(x, u, dtype, **s)
    for r0 in range(0, R, 100):
        part = {n: v[r0:r0 + 100] for n, v in s.items()}
        alone = run(x[r0:r0 + 100], u[r0:r0 + 100], dtype, **part)
        for i, (a, b) in enumerate(zip(got, alone)):
            np.testing.assert_allclose(a[r0:r0 + 100], b, rtol=0, atol=2e-5 if i == 1 else 0, equal_nan=True)
    pick = list(range(0, R, 97))
    part = {n: [v[i] for i in pick] for n, v in s.items()}
    check(bf16(x[pick]) if dtype == "bf16" else x[pick], u[pick], [g[pick] for g in got], **part)
