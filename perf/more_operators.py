"""Performance cases of what surrounds a token model's layers: layer norm, the
drawing of tokens from logits, and the AdamW update of many tensors.

A case is a dict of plain values; ``kind`` names the operator and ``mode``
what a program does with it:

  norm    infer   janus_layer_norm_fwd: y (and h = x + r with a residual)
          train   the same with statistics, and janus_layer_norm_bwd: y, h, the
                  statistics and every gradient
  sample          janus_sample: tokens from given uniform numbers under
                  temperature, top-k, top-p and min-p, the log-probability of
                  each under the policy and under the filtered distribution, and
                  how many tokens the filters kept
  adamw           janus_adamw_update: one step of many tensors with their
                  gradients' global norm; states of 32 bits, or of 8 bits with a
                  scale for every 256 elements

``run`` computes the plain form, from elementary torch operations, unless
``own`` is set; ``exact`` has the definitions in float64.  States of 8 bits come
back as float8 tensors, whose values times their block's scale (returned too)
are the states.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"


def listed():
    return [
        # one token for each of 20 running sequences, width twice 650: launch and latency
        dict(name="norm_infer_20", kind="norm", mode="infer", dtype="bf16", rows=20, D=1300, residual=True, wide=False),
        # a small float32 layer, odd sizes, rows that are column slices of a wider matrix
        dict(name="norm_train_odd_f32", kind="norm", mode="train", dtype="f32", rows=1021, D=301, residual=False,
             wide=True),
        # training over 128 sequences of 200 steps, a 1024-unit layer
        dict(name="norm_train_1024", kind="norm", mode="train", dtype="bf16", rows=25600, D=1024, residual=False,
             wide=False),
        # the largest: batch 256, 256 steps, 2048 units, a residual stream and its gradient
        dict(name="norm_train_2048", kind="norm", mode="train", dtype="bf16", rows=65536, D=2048, residual=True,
             wide=False),
        # a rollout's step: 20 sequences over a vocabulary of 10000, all of the usual filters
        dict(name="sample_20", kind="sample", dtype="bf16", rows=20, V=10000, pad=0, T=0.8, k=50, p=0.9, minp=0.0,
             per_row=False, masked=False),
        # float32 logits of an odd vocabulary in padded rows, forbidden actions, min-p alone
        dict(name="sample_odd_f32", kind="sample", dtype="f32", rows=37, V=20001, pad=31, T=1.0, k=0, p=1.0, minp=0.05,
             per_row=False, masked=True),
        # 256 running sequences with settings of their own, some greedy
        dict(name="sample_256", kind="sample", dtype="bf16", rows=256, V=32768, pad=0, T=1.0, k=40, p=0.95, minp=0.02,
             per_row=True, masked=False),
        # the largest: draws from the policy itself, nothing filtered
        dict(name="sample_1024", kind="sample", dtype="bf16", rows=1024, V=65536, pad=0, T=1.0, k=0, p=1.0, minp=0.0,
             per_row=False, masked=False),
        # the tensors of a small token policy: launches and latency
        dict(name="adamw_policy", kind="adamw", dtype="f32", bits=32, master=False, max_norm=1.0,
             sizes="128000,65536,1024,256,10240,2048,256000,4096,256,256", n=10, total=467712),
        # a two-layer 650-unit language model over 10000 words, float32
        dict(name="adamw_ptb", kind="adamw", dtype="f32", bits=32, master=False, max_norm=5.0,
             sizes="6500000,1690000,1690000,2600,1690000,1690000,2600,6500000,10000", n=9, total=19775200),
        # 300 tensors of odd sizes, float32 among bf16, states of 8 bits
        dict(name="adamw_many_8bit", kind="adamw", dtype="mixed", bits=8, master=False, max_norm=1.0, sizes="", n=300,
             total=10000019),
        # the largest: two layers of 2048 units and the head, bf16 with float32 masters, states of 8 bits
        dict(name="adamw_2048_8bit", kind="adamw", dtype="bf16", bits=8, master=True, max_norm=1.0,
             sizes="16777216,16777216,8192,16777216,16777216,8192,4194304,2048", n=8, total=71321600),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above."""
    kind = rng.choice(["norm", "sample", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norm":
        D = _log(rng, 16, 8192)
        rows = min(_log(rng, 1, 65536), (1 << 27) // D)
        return dict(kind=kind, mode=rng.choice(["infer", "train", "train"]), dtype=dtype, rows=rows, D=D,
                    residual=rng.random() < 0.5, wide=rng.random() < 0.3)
    if kind == "sample":
        V = _log(rng, 500, 131072)
        rows = min(_log(rng, 1, 1024), (1 << 26) // V)
        return dict(kind=kind, dtype=dtype, rows=rows, V=V, pad=rng.choice([0, 0, rng.randrange(64)]),
                    T=rng.choice([0.6, 0.8, 1.0, 1.0, 1.3]), k=rng.choice([0, 0, 20, 50, 400]),
                    p=rng.choice([1.0, 1.0, 0.8, 0.95]), minp=rng.choice([0.0, 0.0, 0.05]),
                    per_row=rng.random() < 0.25, masked=rng.random() < 0.3)
    n = _log(rng, 1, 300)
    bits = rng.choice([32, 8, 8])
    dtype = rng.choice(["f32", "bf16", "mixed"])
    return dict(kind=kind, dtype=dtype, bits=bits, master=dtype != "f32" and rng.random() < 0.5,
                max_norm=rng.choice([0.0, 1.0]), sizes="", n=n, total=max(4 * n, _log(rng, 10000, 60000000)))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, s, *shape):
    return torch.randn(shape, generator=g, device=DEV) * s


def _rand(g, lo, hi, *shape):
    return torch.rand(shape, generator=g, device=DEV) * (hi - lo) + lo


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case, dt=torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
    return {"norm": _prepare_norm, "sample": _prepare_sample, "adamw": _prepare_adamw}[case["kind"]](case, s, g)


EPS_NORM = 1e-5


def _prepare_norm(case, s, g):
    R, D, dt = case["rows"], case["D"], s["dt"]
    x = _normal(g, 1.0, R, 2 * D if case["wide"] else D).to(dt)
    s["x"] = x[:, :D]
    if case["residual"]:   # a stream that has grown over some layers
        s["r"] = (_normal(g, 2.0, R, D) + 0.3).to(dt)
    s["gamma"], s["beta"] = _rand(g, 0.5, 1.5, D), _normal(g, 0.1, D)
    if case["mode"] == "train":
        s["dy"] = _normal(g, 1.0, R, D).to(dt)
        if case["residual"]:
            s["dh"] = _normal(g, 1.0, R, D).to(dt)
    return s


def _prepare_sample(case, s, g):
    R, V = case["rows"], case["V"]
    x = _normal(g, 2.5, R, V + case["pad"]).to(s["dt"])
    s["logits"] = x[:, :V]
    if case["masked"]:   # one action in ten is forbidden, never all of a row
        gone = torch.rand((R, V), generator=g, device=DEV) < 0.1
        gone[:, 0] = False
        s["logits"].masked_fill_(gone, -math.inf)
    s["u"] = torch.rand(R, generator=g, device=DEV)
    if case["per_row"]:
        pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(0, len(v), (R,), generator=g, device=DEV)]   # noqa: E731
        s["T"] = pick(0.0, 0.7 * case["T"], case["T"], case["T"], 1.2 * case["T"])
        s["k"] = pick(0, case["k"], case["k"], 2 * case["k"]).int()
        s["p"] = pick(1.0, case["p"], case["p"], 0.5)
        s["minp"] = pick(0.0, case["minp"], case["minp"])
    return s


# The update's constants: every case's, as a program sets them once.
LR, BETA1, BETA2, EPS, DECAY, SEED, DONE = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1234, 100
BLOCK = 256


def _sizes(case):
    if case["sizes"]:
        return [int(v) for v in case["sizes"].split(",")]
    n, total = case["n"], case["total"]
    w = np.exp(np.random.default_rng(n * 7919 + total).normal(0.0, 1.5, n))
    out = np.maximum(1, np.floor(w / w.sum() * (total - n))).astype(int)
    out[int(out.argmax())] += total - int(out.sum())
    return [int(v) for v in out]


def _prepare_adamw(case, s, g):
    """Tensors are views of one buffer a kind and type, each from a multiple of
    64 elements on, but those of an odd place in cases without given sizes, which
    follow the one before."""
    sizes, mixed = _sizes(case), case["dtype"] == "mixed"
    f32 = [case["dtype"] == "f32" or (mixed and i % 3 == 0) for i in range(len(sizes))]
    at, end = [], {True: 0, False: 0}
    for i, n in enumerate(sizes):
        start = end[f32[i]]
        if case["sizes"] or i % 2 == 0:
            start = -(-start // 64) * 64
        at.append(start)
        end[f32[i]] = start + n
    bats, b_end = [], 0   # blocks of the 8-bit states
    for n in sizes:
        bats.append(b_end)
        b_end += -(-n // BLOCK)
    total = sum(sizes)
    outs, s["tensors"] = {}, []
    for k in {k for k in f32}:
        outs["p32" if k else "p16"] = _normal(g, 0.05, end[k]).to(torch.float32 if k else torch.bfloat16)
    grads = _normal(g, 1e-3, total) * torch.exp(_normal(g, 1.0, total))
    m, r = 0.3 * grads.roll(17), 1.1 * grads.abs().roll(31) + 1e-5
    cut = list(np.cumsum([0] + sizes))
    if case["bits"] == 8:
        wide = [_pad(m[a:b]) for a, b in zip(cut, cut[1:])], [_pad(r[a:b]) for a, b in zip(cut, cut[1:])]
        half = torch.tensor(0x8000, device=DEV)
        done = [[_quantise(t, half) for t in w] for w in wide]
        outs["m"], outs["r"] = (torch.cat([c.view(-1)[:n] for (c, _), n in zip(d, sizes)]) for d in done)
        outs["scale"] = torch.stack([torch.cat([sc for _, sc in d]) for d in done], 1)
    else:
        outs["m"], outs["v"] = m, r * r
    if case["master"]:
        outs["w16"] = outs["p16"].float()
    outs["step"] = torch.tensor([DONE], dtype=torch.int64, device=DEV)
    outs["stats"] = torch.zeros(2, device=DEV)
    for i, n in enumerate(sizes):
        a, b = cut[i], cut[i + 1]
        k = "p32" if f32[i] else "p16"
        t = dict(p=outs[k][at[i]:at[i] + n], g=grads[a:b], m=outs["m"][a:b], decay=0.0 if n < 16384 else DECAY)
        t["v"] = outs["r" if case["bits"] == 8 else "v"][a:b]
        if case["bits"] == 8:
            t["scale"] = outs["scale"][bats[i]:bats[i] + -(-n // BLOCK)]
        t["master"] = outs["w16"][at[i]:at[i] + n] if case["master"] and not f32[i] else None
        s["tensors"].append(t)
    s["outs"] = outs
    return s


# ------------------------------------------------------------- plain forms
def _plain_norm(s):
    c, dt, D = s["case"], s["dt"], s["case"]["D"]
    out = {}
    h = s["x"].float()
    if c["residual"]:
        out["h"] = (h + s["r"].float()).to(dt)
        h = out["h"].float()
    mean = h.sum(1, keepdim=True) / D
    d = h - mean
    rstd = 1.0 / torch.sqrt((d * d).sum(1, keepdim=True) / D + EPS_NORM)
    xh = d * rstd
    out["y"] = (xh * s["gamma"] + s["beta"]).to(dt)
    if c["mode"] == "infer":
        return out
    dy = s["dy"].float()
    g = dy * s["gamma"]
    dx = (g - g.sum(1, keepdim=True) / D - xh * ((g * xh).sum(1, keepdim=True) / D)) * rstd
    if c["residual"]:
        dx = dx + s["dh"].float()
    out.update(mean=mean[:, 0], rstd=rstd[:, 0], dx=dx.to(dt), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    return out


def _settings(s):
    """Temperature, k, p and min-p as columns."""
    c, R = s["case"], s["case"]["rows"]
    if c["per_row"]:
        return [s[n][:, None] for n in ("T", "k", "p", "minp")]
    return [torch.full((R, 1), c[n], device=DEV, dtype=torch.int32 if n == "k" else torch.float32)
            for n in ("T", "k", "p", "minp")]


def _plain_sample(s):
    """In 64 bits: a token next to a border is decided by sums' last bits."""
    c, V = s["case"], s["case"]["V"]
    x = s["logits"].double()
    T, k, p, minp = (v.double() for v in _settings(s))
    greedy = T == 0.0
    k = torch.where(greedy, 1.0, torch.where((k <= 0) | (k > V), float(V), k))
    m = x.amax(1, keepdim=True)
    d = x - m
    live = x > -math.inf
    w = torch.where(live, torch.exp(d / torch.where(greedy, 1.0, T)), 0.0)
    kept = live & (torch.where(minp > 0, w >= minp, True) | greedy)
    if c["per_row"] or c["k"] or c["p"] < 1.0:
        order = x.sort(dim=1, descending=True, stable=True).indices
        inside = torch.arange(V, device=DEV) < k
        ws = torch.where(inside, w.gather(1, order), 0.0)
        mass = ws.cumsum(1)
        inside &= (p >= 1.0) | (mass - ws < p.clamp(min=0.0) * mass[:, -1:]) | (torch.arange(V, device=DEV) == 0)
        kept &= torch.zeros_like(kept).scatter_(1, order, inside)
    wk = torch.where(kept, w, 0.0)
    mass = wk.cumsum(1)
    W = mass[:, -1:]
    token = (mass <= s["u"].double()[:, None] * W).sum(1, keepdim=True)
    last = torch.where(wk > 0, torch.arange(V, device=DEV), 0).amax(1, keepdim=True)
    token = torch.minimum(token, last)
    lse = torch.log(torch.exp(d).sum(1, keepdim=True))
    return dict(token=token[:, 0].int(), kept=kept.sum(1).int(), logp=(d.gather(1, token) - lse)[:, 0].float(),
                draw_logp=torch.log(wk.gather(1, token) / W)[:, 0].float())


LOW32 = 0xffffffff


def _mix(a):
    """32 random bits a number: shifts and products modulo 2^32."""
    a = a ^ (a >> 16)
    a = (a * 0x6A09E667) & LOW32
    a = a ^ (a >> 15)
    a = (a * 0xBB67AE85) & LOW32
    return a ^ (a >> 16)


def _random(step, tensor, n):
    """Two numbers of 16 bits for each of n elements of a tensor at a step."""
    key = _mix(_mix(_mix(torch.full_like(step, SEED)) ^ (step & LOW32)) ^ tensor)
    x = _mix(torch.arange(n, device=DEV) ^ key)
    return x & 0xffff, x >> 16


def _pad(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _quantise(x, rnd16):
    """Blocks [n, 256] as float8 codes and a power of two for each, so that the
    largest is at most 448; ``rnd16`` decides between the two codes around."""
    a = x.abs().clamp(max=1.75 * 2.0 ** 127)
    top = ((a.amax(1).view(torch.int32) + 0x1FFFFF) >> 23).clamp(min=9)
    scale = ((top - 8) << 23).view(torch.float32)
    t = a * ((262 - top) << 23).view(torch.float32)[:, None]
    bits, rnd = t.view(torch.int32), (rnd16 << 4).int()
    code = torch.where(bits >= 121 << 23, ((bits + rnd) >> 20) - 960, ((t * 2.0 ** 29).int() + rnd) >> 20)
    code = code | torch.where(x < 0, 128, 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _f32(v):
    return float(np.float32(v))


def _plain_adamw(s):
    c, o = s["case"], s["outs"]
    norm = torch.sqrt(sum((t["g"].double() ** 2).sum() for t in s["tensors"]))
    scale = torch.clamp(c["max_norm"] / (norm + 1e-6), max=1.0) if c["max_norm"] > 0 else torch.ones_like(norm)
    o["stats"].copy_(torch.stack([norm, scale]))
    o["step"] += 1
    t64 = o["step"].double()
    b1, b2 = _f32(BETA1), _f32(BETA2)
    rate = (_f32(LR) / (1.0 - b1 ** t64)).float()
    root = (1.0 / torch.sqrt(1.0 - b2 ** t64)).float()
    for i, t in enumerate(s["tensors"]):
        n, old = t["g"].numel(), t["master"] if t["master"] is not None else t["p"].float()
        g = t["g"] * scale.float()
        if c["bits"] == 8:
            m, r = _pad(t["m"].float()), _pad(t["v"].float())
            m, r = (m * t["scale"][:, :1]).view(-1)[:n], (r * t["scale"][:, 1:]).view(-1)[:n]
            v = r * r
        else:
            m, v = t["m"], t["v"]
        m = m * b1 + g * _f32(1.0 - b1)
        v = v * b2 + (g * g) * _f32(1.0 - b2)
        r = torch.sqrt(v.double()).float()   # (rounded once, whatever torch's root of 32 bits is)
        p = old - old * _f32(_f32(LR) * _f32(t["decay"])) - rate * m / (r * root + _f32(EPS))
        if c["bits"] == 8:
            for k, (x, rnd) in enumerate(zip((m, r), _random(o["step"], i, -(-n // BLOCK) * BLOCK))):
                code, sc = _quantise(_pad(x), rnd.view(-1, BLOCK))
                (t["v"] if k else t["m"]).view(torch.uint8).copy_(code.view(torch.uint8).view(-1)[:n])
                t["scale"][:, k] = sc
        else:
            t["m"].copy_(m)
            t["v"].copy_(v)
        if t["master"] is not None:
            t["master"].copy_(p)
        t["p"].copy_(p)
    return o


# ------------------------------------------------- the library's operators
def _plan(s):
    """Descriptors, outputs and workspaces that a program keeps between calls."""
    from paper_1812_01329_amd import janus as J
    c = s["case"]
    new = lambda *n, dt=torch.float32: torch.empty(*n, dtype=dt, device=DEV)   # noqa: E731
    p = dict(J=J)
    code = J.F32 if c["dtype"] == "f32" else J.BF16
    if c["kind"] == "norm":
        R, D = c["rows"], c["D"]
        ldx = s["x"].stride(0) if R > 1 else 0
        d = J.NormDesc(R, D, code, EPS_NORM, ldx, 0 if c["residual"] else ldx, 0)
        p.update(y=new(R, D, dt=s["dt"]), h=new(R, D, dt=s["dt"]) if c["residual"] else None, mean=None, rstd=None)
        need = 0
        if c["mode"] == "train":
            dx = new(R, 2 * D if c["wide"] else D, dt=s["dt"])[:, :D]
            p.update(mean=new(R), rstd=new(R), dx=dx, dgamma=new(D), dbeta=new(D))
            need = J.janus_layer_norm_workspace_bytes(d)
    elif c["kind"] == "sample":
        R = c["rows"]
        one = not c["per_row"]
        d = J.SampleDesc(R, c["V"], code, s["logits"].stride(0) if R > 1 else 0, c["T"] if one else 1.0,
                         c["k"] if one else 0, c["p"] if one else 1.0, c["minp"] if one else 0.0)
        p.update(token=new(R, dt=torch.int32), kept=new(R, dt=torch.int32), logp=new(R), draw_logp=new(R))
        need = J.janus_sample_workspace_bytes(d)
    else:
        T = s["tensors"]
        get = lambda k: [t[k] for t in T]   # noqa: E731
        d = J.AdamWDesc(len(T), J.ADAMW_8BIT if c["bits"] == 8 else J.ADAMW_F32, LR, BETA1, BETA2, EPS,
                        c["max_norm"], SEED)
        p["tensors"] = J.adamw_tensors(get("p"), get("g"), get("m"), get("v"), get("scale") if c["bits"] == 8 else None,
                                       get("master"), get("decay"))
        need = J.janus_adamw_workspace_bytes(d)
    p.update(desc=d, ws=torch.empty(max(need, 1), dtype=torch.uint8, device=DEV))
    return p


def _own(s):
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    J, c, d = p["J"], s["case"], p["desc"]
    if c["kind"] == "norm":
        J.janus_layer_norm_fwd(d, s["x"], s["gamma"], s["beta"], p["y"], r=s.get("r"), h=p["h"], mean=p["mean"],
                               rstd=p["rstd"])
        out = dict(y=p["y"]) if p["h"] is None else dict(y=p["y"], h=p["h"])
        if c["mode"] == "infer":
            return out
        J.janus_layer_norm_bwd(d, s["x"] if p["h"] is None else p["h"], s["gamma"], p["mean"], p["rstd"], s["dy"],
                               p["dx"], p["ws"], dgamma=p["dgamma"], dbeta=p["dbeta"], dh=s.get("dh"))
        out.update({k: p[k] for k in ("mean", "rstd", "dx", "dgamma", "dbeta")})
        return out
    if c["kind"] == "sample":
        kw = dict(temperature=s["T"], top_k=s["k"], top_p=s["p"], min_p=s["minp"]) if c["per_row"] else {}
        J.janus_sample(d, s["logits"], s["u"], p["token"], logp=p["logp"], draw_logp=p["draw_logp"], kept=p["kept"],
                       ws=p["ws"], **kw)
        return {k: p[k] for k in ("token", "kept", "logp", "draw_logp")}
    o = s["outs"]
    J.janus_adamw_update(d, p["tensors"], o["step"], stats=o["stats"], ws=p["ws"])
    return o


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"norm": _plain_norm, "sample": _plain_sample, "adamw": _plain_adamw}[kind](state)


# ------------------------------------------------------------ what it takes
def work(case):
    if case["kind"] == "adamw":
        sizes = _sizes(case)
        n, n32 = sum(sizes), sum(z for i, z in enumerate(sizes) if case["dtype"] == "f32" or
                                 (case["dtype"] == "mixed" and i % 3 == 0))
        states = n * 4 + sum(-(-z // BLOCK) for z in sizes) * 16 if case["bits"] == 8 else n * 16
        # gradients in, parameters in and out (only out where there is a master, which goes in and out)
        half = (n - n32) * (2 + 8 if case["master"] else 4)
        return dict(bytes=n * 4 + n32 * 8 + half + states, flops=16 * n)
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "sample":
        return dict(bytes=case["rows"] * (case["V"] * es + 20), flops=6 * case["rows"] * case["V"])
    R, D = case["rows"], case["D"]
    fwd = R * D * es * (4 if case["residual"] else 2) + 8 * D
    if case["mode"] == "infer":
        return dict(bytes=fwd, flops=8 * R * D)
    # x (and r), dy (and dh) in; y (and h) and dx out
    return dict(bytes=R * D * es * (7 if case["residual"] else 4) + 16 * D + 8 * R, flops=22 * R * D)


# ------------------------------------------------------- 64-bit definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "sample": _exact_sample, "adamw": _exact_adamw}[case["kind"]](case, s)


def _exact_norm(case, s):
    """torch's layer norm in float64, a few thousand rows at a time; the
    gradients by automatic differentiation."""
    D, train = case["D"], case["mode"] == "train"
    gamma, beta = (s[k].double().requires_grad_(train) for k in ("gamma", "beta"))
    few, parts = max(1, (1 << 26) // D), []
    for a in range(0, case["rows"], few):
        at = slice(a, a + few)
        h = s["x"][at]
        if case["residual"]:
            h = (h.float() + s["r"][at].float()).to(s["dt"])   # (the sum is kept in the rows' type)
        got = dict(h=h.double()) if case["residual"] else {}
        h = h.double().requires_grad_(train)
        y = torch.nn.functional.layer_norm(h, (D,), gamma, beta, EPS_NORM)
        got["y"] = y.detach()
        if train:
            (y * s["dy"][at].double()).sum().backward()
            var, mean = torch.var_mean(h.detach(), 1, correction=0)
            got.update(mean=mean, rstd=torch.rsqrt(var + EPS_NORM), dx=h.grad)
            if case["residual"]:
                got["dx"] = got["dx"] + s["dh"][at].double()
        parts.append(got)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if train:
        out.update(dgamma=gamma.grad, dbeta=beta.grad)
    return out


def _exact_sample(case, s):
    """Row by row on the host, from each row's own sorted list."""
    x = s["logits"].double().cpu().numpy()
    u = s["u"].double().cpu().numpy()
    T, k, p, minp = (v[:, 0].double().cpu().numpy() for v in _settings(s))
    R, V = x.shape
    token, kept, logp, drawn = np.zeros(R, np.int32), np.zeros(R, np.int32), np.zeros(R), np.zeros(R)
    for r in range(R):
        row = x[r]
        top = row.max()
        if T[r] == 0:
            keep = np.array([int(row.argmax())])
            w = np.ones(1)
        elif 0 < k[r] < V or p[r] < 1 or minp[r] > 0:
            order = np.argsort(-row, kind="stable")[:int(k[r]) if 0 < k[r] < V else V]
            order = order[row[order] > -np.inf]
            w = np.exp((row[order] - top) / T[r])
            n = len(order)
            if p[r] < 1:
                n = min(n, int(np.searchsorted(np.cumsum(w), p[r] * w.sum())) + 1)
            if minp[r] > 0:
                n = min(n, int((w >= minp[r]).sum()))
            keep = np.sort(order[:n])
            w = np.exp((row[keep] - top) / T[r])
        else:
            keep = np.flatnonzero(row > -np.inf)
            w = np.exp((row[keep] - top) / T[r])
        c = np.cumsum(w)
        j = min(int(np.searchsorted(c, u[r] * c[-1], side="right")), len(keep) - 1)
        token[r], kept[r] = keep[j], len(keep)
        drawn[r] = math.log(w[j] / c[-1])
        logp[r] = row[keep[j]] - top - math.log(np.exp(row - top).sum())
    dev = lambda a: torch.from_numpy(a).to(DEV)   # noqa: E731
    return dict(token=dev(token), kept=dev(kept), logp=dev(logp), draw_logp=dev(drawn))


def _exact_adamw(case, s):
    """The update of the stored states in float64; quantised states have no such
    value."""
    o, norm2 = s["outs"], sum(float(t["g"].double().pow(2).sum()) for t in s["tensors"])
    out = {k: v.double() if v.dtype in (torch.float32, torch.bfloat16) else None for k, v in o.items()}
    if case["bits"] == 8:
        out["scale"] = None
    norm = math.sqrt(norm2)
    clip = min(1.0, case["max_norm"] / (norm + 1e-6)) if case["max_norm"] > 0 else 1.0
    out["stats"] = torch.tensor([norm, clip], dtype=torch.float64, device=DEV)
    out["step"] = o["step"] + 1
    lr, b1, b2, eps = _f32(LR), _f32(BETA1), _f32(BETA2), _f32(EPS)
    step = DONE + 1

    def put(k, view, value):
        first = (view.data_ptr() - o[k].data_ptr()) // view.element_size()
        out[k][first:first + value.numel()] = value

    for t in s["tensors"]:
        n, g = t["g"].numel(), t["g"].double() * clip
        m, v = t["m"].double(), t["v"].double()
        if case["bits"] == 8:
            of = torch.arange(n, device=DEV) // BLOCK
            m, v = m * t["scale"][of, 0].double(), (v * t["scale"][of, 1].double()) ** 2
        m = torch.lerp(g, m, b1)
        v = torch.lerp(g.square(), v, b2)
        w = (t["p"] if t["master"] is None else t["master"]).double()
        w = w * (1.0 - lr * _f32(t["decay"])) - lr * (m / (1.0 - b1 ** step)) / ((v / (1.0 - b2 ** step)).sqrt() + eps)
        put("p32" if t["p"].dtype == torch.float32 else "p16", t["p"], w)
        if t["master"] is not None:
            put("w16", t["master"], w)
        if case["bits"] == 32:
            put("m", t["m"], m)
            put("v", t["v"], v)
    return out
