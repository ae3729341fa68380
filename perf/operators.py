"""Performance cases of the sequence-policy operators: the short causal
convolution, the selective scan and the clipped policy loss.

A case is a dict of plain values; ``kind`` names the operator and ``mode``
what a program does with it:

  conv  prompt   janus_causal_conv_fwd from a carried state: y and the new state
        train    the same and janus_causal_conv_bwd: y and every gradient
        step     janus_causal_conv_step: one token for each row, states in slots
  scan  prompt   janus_selective_scan_fwd from a carried state: y and the new state
        train    the same and janus_selective_scan_bwd: y and every gradient
        step     janus_selective_scan_step: one token for each row
  policy train   janus_policy_loss: the statistics, the rows' log-probabilities
                 and entropies and the gradient of the logits
        score    the same without a gradient (the old or the reference policy's
                 log-probabilities of given actions)

Sequences are time-major, [T, B, *], with host lengths or all of length T.
``run`` computes the plain form, from elementary torch operations in float32,
unless ``own`` is set; ``exact`` has the definitions in float64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"


def listed():
    return [
        # one token for each of 20 running sequences, channels twice 650: launch and latency
        dict(name="conv_step_20", kind="conv", mode="step", dtype="bf16", B=20, D=1300, K=4, act=True, slots=32),
        # three float32 prompts continued from a carried state, no size a multiple of a tile
        dict(name="conv_prompt_odd_f32", kind="conv", mode="prompt", dtype="f32", T=511, B=3, D=1301, K=3, act=False,
             ragged=True),
        # training over sequences of 1..200 steps, batch 128, the convolution of a 1024-unit layer
        dict(name="conv_train_varlen", kind="conv", mode="train", dtype="bf16", T=200, B=128, D=1024, K=4, act=True,
             ragged=True),
        # one token for each of 20 running sequences
        dict(name="scan_step_20", kind="scan", mode="step", dtype="bf16", B=20, D=1300, N=16, G=1, slots=32),
        # one token for each of 256 running sequences of a wide layer: the states' bytes
        dict(name="scan_step_256", kind="scan", mode="step", dtype="bf16", B=256, D=4096, N=16, G=1, slots=256),
        # one long prompt: little to share out but the time axis
        dict(name="scan_prompt_8192", kind="scan", mode="prompt", dtype="bf16", T=8192, B=1, D=2048, N=16, G=1,
             ragged=False),
        # a small float32 layer over short sentences, odd sizes
        dict(name="scan_train_odd_f32", kind="scan", mode="train", dtype="f32", T=50, B=32, D=301, N=13, G=1,
             ragged=True),
        # training over sequences of 1..200 steps, batch 128
        dict(name="scan_train_varlen", kind="scan", mode="train", dtype="bf16", T=200, B=128, D=1024, N=16, G=1,
             ragged=True),
        # the largest training call: batch 256, 256 steps, 2048 channels
        dict(name="scan_train_2048", kind="scan", mode="train", dtype="bf16", T=256, B=256, D=2048, N=16, G=1,
             ragged=False),
        # a policy step over 20 sequences of 35 tokens, vocabulary 10000
        dict(name="policy_700", kind="policy", mode="train", dtype="bf16", rows=700, V=10000, kl=0.1, ent=0.0,
             masked=False),
        # float32 logits of an odd vocabulary with forbidden actions, entropy and KL terms
        dict(name="policy_odd_f32", kind="policy", mode="train", dtype="f32", rows=1021, V=20001, kl=0.05, ent=0.01,
             masked=True),
        # the largest: a batch of rollouts over a large vocabulary
        dict(name="policy_16384", kind="policy", mode="train", dtype="bf16", rows=16384, V=32768, kl=0.1, ent=0.0,
             masked=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["conv", "scan", "scan", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "policy":
        rows = _log(rng, 1, 16384)
        V = min(_log(rng, 500, 131072), 268435456 // rows)
        return dict(kind=kind, mode=rng.choice(["train", "train", "score"]), dtype=dtype, rows=rows, V=V,
                    kl=rng.choice([0.0, 0.1]), ent=rng.choice([0.0, 0.01]), masked=rng.random() < 0.3)
    mode = rng.choice(["step", "prompt", "train", "train"])
    D = _log(rng, 64, 4096)
    c = dict(kind=kind, mode=mode, dtype=dtype)
    if kind == "conv":
        c.update(K=rng.choice([2, 3, 4, 4]), act=rng.random() < 0.7)
        width, most = 1, 1 << 26
    else:
        N = rng.choice([8, 13, 16, 16, 16, 32])
        G = 2 if D % 2 == 0 and rng.random() < 0.25 else 1
        c.update(N=N, G=G)
        width, most = N, 1 << 30
    if mode == "step":
        B = _log(rng, 1, 256)
        c.update(B=B, D=D, slots=B + rng.randrange(16))
        return c
    B = _log(rng, 1, 256)
    T = _log(rng, 1, 4096 if mode == "prompt" else 1024)
    B = max(1, min(B, most // (width * T * D)))
    c.update(T=T, B=B, D=D, ragged=rng.random() < 0.5)
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, s, *shape):
    return torch.randn(shape, generator=g, device=DEV) * s


def _rand(g, lo, hi, *shape):
    return torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo


def _lengths(case, seed):
    """Host lengths U{1..T} (the longest always T), or None for all T."""
    if not case.get("ragged"):
        return None
    n = np.random.default_rng(seed).integers(1, case["T"] + 1, size=case["B"]).astype(np.int32)
    n[int(n.argmax())] = case["T"]
    return n


def _slots(case, seed):
    p = np.random.default_rng(seed).permutation(case["slots"])[:case["B"]].astype(np.int32)
    return torch.from_numpy(p).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = dict(case=case, dt=dt)
    if case["kind"] == "policy":
        return _prepare_policy(case, s, g, dt)
    B, D, step, train = case["B"], case["D"], case["mode"] == "step", case["mode"] == "train"
    T = 1 if step else case["T"]
    s["lengths"] = _lengths(case, seed)
    if step:
        s["slots"] = _slots(case, seed)
    if case["kind"] == "conv":
        K = case["K"]
        s["x"] = _normal(g, 1.0, T, B, D).to(dt)
        s["w"] = _rand(g, -1 / math.sqrt(K), 1 / math.sqrt(K), D, K).to(dt)
        s["bias"] = _rand(g, -1 / math.sqrt(K), 1 / math.sqrt(K), D).to(dt)
        s["state"] = _normal(g, 1.0, case["slots"] if step else B, K - 1, D).to(dt)
        if train:
            s["dy"] = _normal(g, 1.0, T, B, D).to(dt)
            s["dsT"] = _normal(g, 1.0, B, K - 1, D)
        return s
    N, G = case["N"], case["G"]
    s["x"] = _normal(g, 1.0, T, B, D).to(dt)
    s["dtin"] = _normal(g, 0.5, T, B, D).to(dt)
    s["z"] = _normal(g, 1.0, T, B, D).to(dt)
    s["Bm"] = _normal(g, 1.0, T, B, G, N).to(dt)
    s["Cm"] = _normal(g, 1.0, T, B, G, N).to(dt)
    # decay rates 1..N, spread a little; step sizes of about 0.001 to 0.1
    s["A"] = -torch.arange(1, N + 1, device=DEV).float() * _rand(g, 0.8, 1.2, D, N)
    s["Dskip"] = _rand(g, 0.5, 1.5, D)
    d0 = torch.exp(_rand(g, math.log(1e-3), math.log(1e-1), D))
    s["dt_bias"] = d0 + torch.log(-torch.expm1(-d0))
    s["state"] = _normal(g, 0.5, case["slots"] if step else B, D, N)
    if train:
        s["dy"] = _normal(g, 1.0, T, B, D).to(dt)
        s["dhT"] = _normal(g, 0.5, B, D, N)
    return s


def _prepare_policy(case, s, g, dt):
    rows, V = case["rows"], case["V"]
    s["logits"] = _normal(g, 2.0, rows, V).to(dt)
    s["actions"] = torch.randint(0, V, (rows,), generator=g, device=DEV, dtype=torch.int32)
    at = s["actions"].long()[:, None]
    if case["masked"]:   # one action in ten is forbidden, never the one taken
        kept = s["logits"].gather(1, at)
        s["logits"].masked_fill_(torch.rand((rows, V), generator=g, device=DEV) < 0.1, -math.inf)
        s["logits"].scatter_(1, at, kept)
    # old and reference policies a little away from the present one; the ratio
    # keeps off the clip's two corners, where the gradient jumps
    lse = torch.cat([r.float().logsumexp(1) for r in s["logits"].split(2048)])
    lp = s["logits"].gather(1, at)[:, 0].float() - lse
    r = _normal(g, 0.2, rows)
    for corner in (math.log(0.8), math.log(1.2)):
        r = torch.where((r - corner).abs() < 1e-3, r + 4e-3, r)
    s["old_logp"] = lp - r
    s["ref_logp"] = lp - _normal(g, 0.3, rows)
    s["adv"] = _normal(g, 1.0, rows)
    s["weights"] = (torch.rand(rows, generator=g, device=DEV) < 0.9).float()   # the rest is padding
    s["weights"][0] = 1.0
    return s


# ------------------------------------------------------------- plain forms
def _active(lengths, T, B):
    """[T, B] truth values: t < len_b."""
    if lengths is None:
        return torch.ones(T, B, dtype=torch.bool, device=DEV)
    n = torch.from_numpy(np.asarray(lengths)).to(DEV)
    return torch.arange(T, device=DEV)[:, None] < n[None, :]


def _conv_taps(s):
    """Inputs with the carried ones in front, float32 [K - 1 + T, B, D]."""
    return torch.cat([s["state"].float().transpose(0, 1), s["x"].float()])


def _conv_pre(s, xs, T):
    w = s["w"].float()
    return sum(xs[k:k + T] * w[:, k] for k in range(w.shape[1])) + s["bias"].float()


def _plain_conv_step(s):
    c, slots = s["case"], s["slots"].long()
    xs = torch.cat([s["state"][slots].float(), s["x"][0].float()[:, None]], 1)       # [B, K, D]
    p = (xs * s["w"].float().t()).sum(1) + s["bias"].float()
    y = p * torch.sigmoid(p) if c["act"] else p
    s["state"][slots] = xs[:, 1:].to(s["dt"])
    return dict(y=y.to(s["dt"])[None], state=s["state"])


def _plain_conv(s):
    c, dt = s["case"], s["dt"]
    T, B, K = c["T"], c["B"], c["K"]
    on = _active(s["lengths"], T, B)
    xs = _conv_taps(s)
    p = _conv_pre(s, xs, T)
    y = p * torch.sigmoid(p) if c["act"] else p
    n = on.sum(0)                                                                    # [B]
    at = n[:, None] + torch.arange(K - 1, device=DEV)                                # rows of xs in the final state
    rows = torch.arange(B, device=DEV)[:, None]
    out = dict(y=torch.where(on[..., None], y, 0.0).to(dt), sT=xs[at, rows].to(dt))
    if c["mode"] == "prompt":
        return out
    g = torch.where(on[..., None], s["dy"].float(), 0.0)
    if c["act"]:
        q = torch.sigmoid(p)
        g = g * (q * (1.0 + p * (1.0 - q)))
    w = s["w"].float()
    dxs = torch.zeros_like(xs)
    for k in range(K):
        dxs[k:k + T] += g * w[:, k]
    dxs[at, rows] += s["dsT"]
    out.update(dx=dxs[K - 1:].to(dt), ds0=dxs[:K - 1].transpose(0, 1).contiguous(),
               dw=torch.stack([(g * xs[k:k + T]).sum((0, 1)) for k in range(K)], 1), dbias=g.sum((0, 1)))
    return out


def _softplus(v):
    return v.clamp(min=0.0) + torch.log1p(torch.exp(-v.abs()))


def _wide(m, D):
    """[..., G, N] -> [..., D, N]: the channels of a group share its row."""
    return m.float().repeat_interleave(D // m.shape[-2], dim=-2)


def _plain_scan_step(s):
    slots, D = s["slots"].long(), s["case"]["D"]
    x, z = s["x"][0].float(), s["z"][0].float()
    d = _softplus(s["dtin"][0].float() + s["dt_bias"])
    h = s["state"][slots] * torch.exp(d[..., None] * s["A"]) + (d * x)[..., None] * _wide(s["Bm"][0], D)
    y = ((h * _wide(s["Cm"][0], D)).sum(-1) + s["Dskip"] * x) * z * torch.sigmoid(z)
    s["state"][slots] = h
    return dict(y=y.to(s["dt"])[None], state=s["state"])


def _plain_scan(s):
    c, dt = s["case"], s["dt"]
    T, B, D, N, G = (c[k] for k in "TBDNG")
    train = c["mode"] == "train"
    on = _active(s["lengths"], T, B)
    x, z, A = s["x"].float(), s["z"].float(), s["A"]
    v = s["dtin"].float() + s["dt_bias"]
    d = _softplus(v)
    h = s["state"]
    hs, ys = [h], []
    for t in range(T):
        new = h * torch.exp(d[t][..., None] * A) + (d[t] * x[t])[..., None] * _wide(s["Bm"][t], D)
        h = new if s["lengths"] is None else torch.where(on[t][:, None, None], new, h)
        if train:
            hs.append(h)
        ys.append((h * _wide(s["Cm"][t], D)).sum(-1))
    raw = torch.stack(ys) + s["Dskip"] * x
    sz = torch.sigmoid(z)
    live = on[..., None]
    out = dict(y=torch.where(live, raw * z * sz, 0.0).to(dt), hT=h)
    if not train:
        return out
    dy = torch.where(live, s["dy"].float(), 0.0)
    gy = dy * z * sz
    dz = dy * raw * (sz * (1.0 + z * (1.0 - sz)))
    g, dA = s["dhT"], torch.zeros_like(A)
    dx, dd = s["Dskip"] * gy, torch.zeros_like(x)
    dB, dC = torch.zeros(T, B, G, N, device=DEV), torch.zeros(T, B, G, N, device=DEV)
    for t in reversed(range(T)):
        a = torch.exp(d[t][..., None] * A)
        now = g + gy[t][..., None] * _wide(s["Cm"][t], D)
        if s["lengths"] is not None:
            now = torch.where(on[t][:, None, None], now, 0.0)
        dC[t] = (gy[t][..., None] * hs[t + 1]).view(B, G, D // G, N).sum(2)
        dB[t] = (now * (d[t] * x[t])[..., None]).view(B, G, D // G, N).sum(2)
        nb = (now * _wide(s["Bm"][t], D)).sum(-1)
        back = now * a
        q = back * hs[t]
        dx[t] += d[t] * nb
        dd[t] = x[t] * nb + (q * A).sum(-1)
        dA += (q * d[t][..., None]).sum(0)
        g = back if s["lengths"] is None else torch.where(on[t][:, None, None], back, g)
    ddt = dd * torch.sigmoid(v)
    out.update(dx=dx.to(dt), ddt=ddt.to(dt), dz=dz.to(dt), dBm=dB.to(dt), dCm=dC.to(dt), dA=dA,
               dDskip=(gy * x).sum((0, 1)), ddt_bias=ddt.sum((0, 1)), dh0=g)
    return out


LOW, HIGH = 0.2, 0.2


def _plain_policy(s):
    c = s["case"]
    x, w, at = s["logits"].float(), s["weights"], s["actions"].long()[:, None]
    m = x.max(1, keepdim=True).values
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    p = e / total
    lse = m + torch.log(total)
    logp = (x.gather(1, at) - lse)[:, 0]
    plogp = torch.where(p > 0, p * (x - lse), 0.0)
    H = -plogp.sum(1)
    if c["mode"] == "score":
        return dict(logp=logp, entropy=H)
    r = torch.exp(logp - s["old_logp"])
    free, cut = r * s["adv"], r.clamp(1.0 - LOW, 1.0 + HIGH) * s["adv"]
    d = s["ref_logp"] - logp
    kl = torch.expm1(d) - d
    W = w.sum()
    mean = lambda v: (w * v).sum() / W   # noqa: E731
    pol, klm, ent = mean(-torch.minimum(free, cut)), mean(kl), mean(H)
    clipped = mean((free > cut).float())
    c1 = torch.where(free <= cut, -free, 0.0) - c["kl"] * torch.expm1(d)
    grad = -c1[:, None] * p + c["ent"] * (plogp + p * H[:, None])
    grad.scatter_add_(1, at, c1[:, None])
    return dict(stats=torch.stack([pol + c["kl"] * klm - c["ent"] * ent, pol, klm, ent, clipped, W]), logp=logp,
                entropy=H, dlogits=(grad * (w / W)[:, None]).to(s["dt"]))


# ------------------------------------------------- the library's operators
def _plan(s):
    """Descriptors, outputs and workspaces that a program keeps between calls."""
    from paper_1812_01329_amd import janus as J
    c, dt = s["case"], s["dt"]
    code = J.BF16 if dt == torch.bfloat16 else J.F32
    new = lambda like: torch.empty_like(like)   # noqa: E731
    p = dict(J=J)
    if c["kind"] == "policy":
        d = J.PolicyDesc(c["rows"], c["V"], code, 0, LOW, HIGH, c["kl"], c["ent"])
        p.update(logp=new(s["adv"]), entropy=new(s["adv"]), stats=torch.empty(6, device=DEV),
                 dlogits=new(s["logits"]) if c["mode"] == "train" else None)
        need = J.janus_policy_workspace_bytes(d)
    elif c["kind"] == "conv":
        d = J.ConvDesc(c["D"], c["K"], c["B"], c.get("T", 1), code, J.CONV_SILU if c["act"] else J.CONV_LINEAR, 0, 0)
        p.update(y=new(s["x"]), sT=new(s["state"]))
        need = 0
        if c["mode"] == "train":
            p.update(dx=new(s["x"]), dw=torch.empty(c["D"], c["K"], device=DEV), dbias=torch.empty(c["D"], device=DEV),
                     ds0=torch.empty(s["state"].shape, device=DEV))
            need = J.janus_causal_conv_workspace_bytes(d)
    else:
        flags = J.SCAN_SOFTPLUS | (J.SCAN_KEEP if c["mode"] == "train" else 0)
        d = J.ScanDesc(c["D"], c["N"], c["G"], c["B"], c.get("T", 1), code, flags, 0, 0, 0, 0, 0, 0)
        p.update(y=new(s["x"]), hT=new(s["state"]))
        need = 0 if c["mode"] == "step" else J.janus_selective_scan_workspace_bytes(d)
        if c["mode"] == "train":
            p.update(dx=new(s["x"]), ddt=new(s["x"]), dz=new(s["x"]), dBm=new(s["Bm"]), dCm=new(s["Cm"]),
                     dA=new(s["A"]), dDskip=new(s["Dskip"]), ddt_bias=new(s["Dskip"]), dh0=new(s["state"]))
    p.update(desc=d, ws=torch.empty(max(need, 1), dtype=torch.uint8, device=DEV))
    return p


def _own(s):
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    J, c, d = p["J"], s["case"], p["desc"]
    if c["kind"] == "policy":
        train = c["mode"] == "train"
        if not train:
            J.janus_policy_loss(d, s["logits"], s["actions"], logp=p["logp"], entropy=p["entropy"], ws=p["ws"])
            return dict(logp=p["logp"], entropy=p["entropy"])
        J.janus_policy_loss(d, s["logits"], s["actions"], old_logp=s["old_logp"], adv=s["adv"],
                            ref_logp=s["ref_logp"], weights=s["weights"], dlogits=p["dlogits"], logp=p["logp"],
                            entropy=p["entropy"], stats=p["stats"], ws=p["ws"])
        return {k: p[k] for k in ("stats", "logp", "entropy", "dlogits")}
    if c["kind"] == "conv":
        if c["mode"] == "step":
            J.janus_causal_conv_step(d, s["x"], s["w"], s["bias"], s["state"], p["y"], slots=s["slots"])
            return dict(y=p["y"], state=s["state"])
        J.janus_causal_conv_fwd(d, s["x"], s["lengths"], s["w"], s["bias"], s["state"], p["y"], p["sT"])
        if c["mode"] == "prompt":
            return dict(y=p["y"], sT=p["sT"])
        J.janus_causal_conv_bwd(d, s["x"], s["lengths"], s["w"], s["bias"], s["state"], s["dy"], s["dsT"], p["dx"],
                                p["dw"], p["dbias"], p["ds0"], p["ws"])
        return {k: p[k] for k in ("y", "sT", "dx", "ds0", "dw", "dbias")}
    if c["mode"] == "step":
        J.janus_selective_scan_step(d, s["x"], s["dtin"], s["A"], s["Bm"], s["Cm"], s["state"], p["y"],
                                    Dskip=s["Dskip"], z=s["z"], dt_bias=s["dt_bias"], slots=s["slots"])
        return dict(y=p["y"], state=s["state"])
    J.janus_selective_scan_fwd(d, s["x"], s["dtin"], s["A"], s["Bm"], s["Cm"], s["lengths"], p["y"], p["ws"],
                               Dskip=s["Dskip"], z=s["z"], dt_bias=s["dt_bias"], h0=s["state"], hT=p["hT"])
    if c["mode"] == "prompt":
        return dict(y=p["y"], hT=p["hT"])
    J.janus_selective_scan_bwd(d, s["x"], s["dtin"], s["A"], s["Bm"], s["Cm"], s["lengths"], s["dy"], p["ws"],
                               p["dx"], p["ddt"], p["dA"], p["dBm"], p["dCm"], Dskip=s["Dskip"], z=s["z"],
                               dt_bias=s["dt_bias"], h0=s["state"], dhT=s["dhT"], dDskip=p["dDskip"], dz=p["dz"],
                               ddt_bias=p["ddt_bias"], dh0=p["dh0"])
    return {k: p[k] for k in ("y", "hT", "dx", "ddt", "dz", "dBm", "dCm", "dA", "dDskip", "ddt_bias", "dh0")}


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["kind"] == "policy":
        return _plain_policy(state)
    if c["kind"] == "conv":
        return _plain_conv_step(state) if c["mode"] == "step" else _plain_conv(state)
    return _plain_scan_step(state) if c["mode"] == "step" else _plain_scan(state)


# ------------------------------------------------------------ what it takes
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "policy":
        n, r = case["rows"] * case["V"], case["rows"]
        if case["mode"] == "score":
            return dict(bytes=n * es + r * 12, flops=5 * n)
        return dict(bytes=2 * n * es + r * 28, flops=9 * n)
    B, D = case["B"], case["D"]
    R = B * case.get("T", 1)
    mode, K = case["mode"], case.get("K", 1)
    if case["kind"] == "conv":
        edge, per = B * (K - 1) * D, 2 * K + (4 if case["act"] else 0)
        if mode == "step":
            return dict(bytes=2 * B * D * es + 2 * edge * es + D * (K + 1) * es, flops=B * D * per)
        fwd = dict(bytes=2 * R * D * es + 2 * edge * es + D * (K + 1) * es, flops=R * D * per)
        if mode == "prompt":
            return fwd
        # x and dy in, y and dx out, each once
        return dict(bytes=4 * R * D * es + edge * (2 * es + 8) + D * (K + 1) * (es + 4), flops=R * D * (3 * per + 6))
    N, G = case["N"], case["G"]
    params = D * (N + 2) * 4
    if mode == "step":
        return dict(bytes=4 * B * D * es + 2 * B * G * N * es + 2 * B * D * N * 4 + params, flops=B * D * (7 * N + 20))
    rows, state = R * (D * es), B * D * N * 4
    if mode == "prompt":
        return dict(bytes=4 * rows + 2 * R * G * N * es + 2 * state + params, flops=R * D * (7 * N + 20))
    # x, dt, z, dy in, y, dx, ddt, dz out, B, C in, their gradients out
    return dict(bytes=8 * rows + 4 * R * G * N * es + 4 * state + 2 * params, flops=R * D * (24 * N + 60))


# ------------------------------------------------------- 64-bit definitions
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "policy":
        return _exact_policy(case, s)
    if case["kind"] == "conv":
        return _exact_conv(case, s)
    return _exact_scan(case, s)


def _leaf(t, grad=True):
    return t.detach().double().requires_grad_(grad)


def _exact_conv(case, s):
    """Sequences one after another, each a correlation of its own inputs; the
    gradients by automatic differentiation."""
    step, train, K = case["mode"] == "step", case["mode"] == "train", case["K"]
    w, bias = _leaf(s["w"], train), _leaf(s["bias"], train)
    x, state = _leaf(s["x"], train), _leaf(s["state"], train)
    T, B, D = x.shape
    rows = s["slots"].tolist() if step else list(range(B))
    lens = [T] * B if s["lengths"] is None else [int(n) for n in s["lengths"]]
    ys, ends = [], []
    for b in range(B):
        seq = torch.cat([state[rows[b]], x[:lens[b], b]])                     # [K - 1 + len, D]
        p = (seq.unfold(0, K, 1) * w[None]).sum(-1) + bias                    # [len, D]
        y = torch.nn.functional.silu(p) if case["act"] else p
        ys.append(torch.cat([y, torch.zeros(T - lens[b], D, dtype=y.dtype, device=DEV)]))
        ends.append(seq[seq.shape[0] - (K - 1):])
    y, sT = torch.stack(ys, 1), torch.stack(ends)
    if step:
        new = state.clone()
        new[rows] = sT
        return dict(y=y, state=new)
    if not train:
        return dict(y=y, sT=sT)
    ((y * s["dy"].double()).sum() + (sT * s["dsT"].double()).sum()).backward()
    return dict(y=y.detach(), sT=sT.detach(), dx=x.grad, ds0=state.grad, dw=w.grad, dbias=bias.grad)


def _exact_scan(case, s):
    """The recurrence in float64, a few sequences at a time; the gradients by
    automatic differentiation."""
    step, train = case["mode"] == "step", case["mode"] == "train"
    T, B, D = s["x"].shape
    N, G = case["N"], case["G"]
    P = {k: _leaf(s[k], train) for k in ("A", "Dskip", "dt_bias")}
    slots = s["slots"].long() if step else None
    lens = torch.full((B,), T, device=DEV) if s["lengths"] is None else torch.from_numpy(s["lengths"]).to(DEV)
    few = max(1, int(48e9 // (T * D * N * 8 * 8))) if train else B
    parts = []
    for b0 in range(0, B, few):
        b1 = min(B, b0 + few)
        I = {k: _leaf(s[k][:, b0:b1], train) for k in ("x", "dtin", "z", "Bm", "Cm")}
        first = _leaf((s["state"][slots] if step else s["state"])[b0:b1], train)
        h, ys = first, []
        for t in range(T):
            d = torch.nn.functional.softplus(I["dtin"][t] + P["dt_bias"])
            b = I["Bm"][t][:, :, None].expand(b1 - b0, G, D // G, N).reshape(b1 - b0, D, N)
            c = I["Cm"][t][:, :, None].expand(b1 - b0, G, D // G, N).reshape(b1 - b0, D, N)
            new = torch.exp(d[:, :, None] * P["A"]) * h + d[:, :, None] * b * I["x"][t][:, :, None]
            run_on = (t < lens[b0:b1])[:, None]
            h = torch.where(run_on[:, :, None], new, h)
            y = ((h * c).sum(2) + P["Dskip"] * I["x"][t]) * torch.nn.functional.silu(I["z"][t])
            ys.append(torch.where(run_on, y, torch.zeros_like(y)))
        y = torch.stack(ys)
        got = dict(y=y.detach(), hT=h.detach())
        if train:
            ((y * s["dy"][:, b0:b1].double()).sum() + (h * s["dhT"][b0:b1].double()).sum()).backward()
            got.update(dx=I["x"].grad, ddt=I["dtin"].grad, dz=I["z"].grad, dBm=I["Bm"].grad, dCm=I["Cm"].grad,
                       dh0=first.grad)
        parts.append(got)
    out = {k: torch.cat([p[k] for p in parts], 0 if k in ("hT", "dh0") else 1) for k in parts[0]}
    if step:
        new = s["state"].double()
        new[slots] = out.pop("hT")
        out["state"] = new
    if train:
        out.update(dA=P["A"].grad, dDskip=P["Dskip"].grad, ddt_bias=P["dt_bias"].grad)
    return out


def _exact_policy(case, s):
    """The loss from log_softmax in float64, a few rows at a time; the gradient
    by automatic differentiation."""
    train = case["mode"] == "train"
    W = s["weights"].double().sum()
    sums, logps, ents, grads = 0.0, [], [], []
    few = max(1, (1 << 27) // case["V"])
    for r0 in range(0, case["rows"], few):
        part = {k: s[k][r0:r0 + few].double() for k in ("old_logp", "ref_logp", "adv", "weights")}
        x = _leaf(s["logits"][r0:r0 + few], train)
        lp = torch.log_softmax(x, 1)
        logp = lp.gather(1, s["actions"][r0:r0 + few].long()[:, None])[:, 0]
        gone = torch.isinf(lp)
        H = -torch.where(gone, torch.zeros_like(lp), torch.exp(lp) * torch.where(gone, torch.zeros_like(lp), lp)).sum(1)
        logps.append(logp.detach())
        ents.append(H.detach())
        if not train:
            continue
        ratio = torch.exp(logp - part["old_logp"])
        free, cut = ratio * part["adv"], ratio.clamp(1.0 - LOW, 1.0 + HIGH) * part["adv"]
        d = part["ref_logp"] - logp
        terms = torch.stack([-torch.minimum(free, cut), torch.expm1(d) - d, H, (free > cut).double()])
        part_sums = (terms * part["weights"]).sum(1) / W
        (part_sums[0] + case["kl"] * part_sums[1] - case["ent"] * part_sums[2]).backward()
        sums = sums + part_sums.detach()
        grads.append(x.grad)
    out = dict(logp=torch.cat(logps), entropy=torch.cat(ents))
    if train:
        pol, kl, ent, clipped = sums
        out["stats"] = torch.stack([pol + case["kl"] * kl - case["ent"] * ent, pol, kl, ent, clipped, W])
        out["dlogits"] = torch.cat(grads)
    return out
