"""A token policy with one convolution and selective-scan layer: rollouts by the
single-token forms, and a clipped policy-gradient step by the sequence forms.

    x0 = E[token]                          (EMBED_FWD)
    [x | z] = x0 Win^T
    u = silu(conv(x))                      (janus_causal_conv_*)
    [r | B | C] = u Wx^T,  dt = r Wdt^T
    y = scan(u, dt, A, B, C, Dskip, z)     (janus_selective_scan_*)
    logits = y Wout^T
    loss, dlogits                          (janus_policy_loss)

and back through the same calls to every parameter, then the SGD update.  This
module allocates buffers and orders the calls; the plain products between them
are torch's.  The packed products are never split: x, z, B and C, and their
gradients, are column slices that the calls address by row strides.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import numpy as np
import torch

from . import janus as J
from . import workloads as wl
from .train_step import SgdUpdate, _cdt, _dev, _tdt


class SelectivePolicy:
    """Parameters, rollouts and the training step of a PolicyWorkload.

    ``update`` = (lr, max_norm) appends the parameter update to the step (the
    float32 parameters of a bf16 model are updated by a call of their own, with
    their own norm)."""

    def __init__(self, w: wl.PolicyWorkload, device="cuda", clip=(0.2, 0.2), kl_coef=0.0, ent_coef=0.0,
                 update: Optional[Tuple[float, float]] = None):
        self.w, self.device, self.tdt = w, device, _tdt(w.dtype)
        self.coefs = (*clip, kl_coef, ent_coef)
        f32 = torch.float32
        scan = ("A", "Dskip", "dt_bias")
        self.P = {k: _dev(a, f32 if k in scan else self.tdt, device) for k, a in w.params.items()}
        self.G = {k: torch.zeros_like(p, dtype=f32) for k, p in self.P.items()}
        code = _cdt(w.dtype)
        T, B, D, N = w.T, w.B, w.D, w.N
        p_cols = w.R + 2 * N
        self.conv = J.ConvDesc(D, w.K, B, T, code, J.CONV_SILU, 2 * D, 0)
        strides = dict(ldx=0, ldt=0, ldb=p_cols, ldc=p_cols, ldz=2 * D, ldy=0)
        self.scan = J.ScanDesc(D, N, 1, B, T, code, J.SCAN_SOFTPLUS | J.SCAN_KEEP, **strides)
        self.scan_score = J.ScanDesc(D, N, 1, B, T, code, J.SCAN_SOFTPLUS, **strides)
        self.embed = J.XentDesc(w.V, w.M, T * B, code)
        self.loss = J.PolicyDesc(T * B, w.V, code, 0, *self.coefs)
        ws = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=device)
        self.conv_ws = ws(J.janus_causal_conv_workspace_bytes(self.conv))
        self.scan_ws = ws(J.janus_selective_scan_workspace_bytes(self.scan))
        self.embed_ws = ws(J.janus_xent_workspace_bytes(w.V, w.M, T * B, code, J.EMBED_BWD))
        self.loss_ws = ws(J.janus_policy_workspace_bytes(self.loss))
        new = lambda *s, dt=self.tdt: torch.empty(*s, dtype=dt, device=device)
        self.rows = new   # (allocator of row buffers)
        self.dxz, self.dp = new(T * B, 2 * D), new(T * B, p_cols)
        self.du, self.ddt, self.dx0 = new(T * B, D), new(T * B, D), new(T * B, w.M)
        self.stats = torch.zeros(6, dtype=f32, device=device)
        self.updates = []
        if update is not None:
            groups = [[k for k in self.P if self.P[k].dtype == dt] for dt in dict.fromkeys(p.dtype for p in self.P.values())]
            self.updates = [SgdUpdate([self.P[k] for k in g], [self.G[k] for k in g], *update) for g in groups]

    # ------------------------------------------------------------- forward
    def _mid(self, ids_host, ids, desc):
        """Rows before the scan: x0, [x | z], and the embedding lookup."""
        x0 = self.rows(len(ids_host), self.w.M)
        J.janus_embed_softmax_xent(desc, J.EMBED_FWD, ids_host, ids, table=self.P["E"], out=x0)
        return x0, x0 @ self.P["Win"].t()

    def _project(self, u):
        """Step sizes, B and C of the rows u: (packed product, dt, B, C)."""
        R, N = self.w.R, self.w.N
        p = u @ self.P["Wx"].t()
        return p, p[:, :R] @ self.P["Wdt"].t(), p[:, R:R + N], p[:, R + N:]

    def logits(self, tokens: np.ndarray, lengths, keep: bool = False):
        """Logits [T * B, V] of the sequences (rows past an end are those of a
        zero row), and what the backward reads."""
        w, P = self.w, self.P
        ids_host = np.ascontiguousarray(tokens[:w.T].reshape(-1), np.int32)
        ids = torch.from_numpy(ids_host).to(self.device)
        x0, xz = self._mid(ids_host, ids, self.embed)
        z = xz[:, w.D:]
        u = self.rows(w.T * w.B, w.D)
        J.janus_causal_conv_fwd(self.conv, xz, lengths, P["conv_w"], P["conv_b"], None, u)
        p, dt, Bm, Cm = self._project(u)
        y = self.rows(w.T * w.B, w.D)
        J.janus_selective_scan_fwd(self.scan if keep else self.scan_score, u, dt, P["A"], Bm, Cm, lengths, y,
                                   self.scan_ws, Dskip=P["Dskip"], z=z, dt_bias=P["dt_bias"])
        return y @ P["Wout"].t(), (ids_host, ids, x0, xz, z, u, p, dt, Bm, Cm, y)

    def actions(self, tokens: np.ndarray, lengths) -> torch.Tensor:
        """Action of each row: the next token, -1 past the sequence's end."""
        T, B = self.w.T, self.w.B
        a = np.array(tokens[1:T + 1], np.int32)
        if lengths is not None:
            a[np.arange(T)[:, None] >= np.asarray(lengths)[None]] = -1
        return torch.from_numpy(a.reshape(-1)).to(self.device)

    def score(self, tokens: np.ndarray, lengths) -> torch.Tensor:
        """Log-probabilities [T * B] of the sequences' actions (0 past an end)."""
        logits, _ = self.logits(tokens, lengths)
        logp = torch.empty(self.w.T * self.w.B, dtype=torch.float32, device=self.device)
        J.janus_policy_loss(self.loss, logits, self.actions(tokens, lengths), logp=logp)
        return logp

    # ------------------------------------------------------------ training
    def step(self, tokens: np.ndarray, lengths, old_logp: torch.Tensor, adv: torch.Tensor,
             ref_logp: Optional[torch.Tensor] = None):
        """One policy-gradient step on rollouts: the statistics of
        janus_policy_loss and the gradients in ``G``; with ``update``, new
        parameters.  ``old_logp``, ``adv``, ``ref_logp``: [T * B] float32."""
        w, P, G = self.w, self.P, self.G
        logits, (ids_host, ids, x0, xz, z, u, p, dt, Bm, Cm, y) = self.logits(tokens, lengths, keep=True)
        R, N, D = w.R, w.N, w.D
        J.janus_policy_loss(self.loss, logits, self.actions(tokens, lengths), old_logp=old_logp, adv=adv,
                            ref_logp=ref_logp, dlogits=logits, stats=self.stats, ws=self.loss_ws)
        dlogits = logits   # formed in place
        G["Wout"].copy_(dlogits.t() @ y)
        dy = dlogits @ P["Wout"]
        dp, dxz = self.dp, self.dxz
        J.janus_selective_scan_bwd(self.scan, u, dt, P["A"], Bm, Cm, lengths, dy, self.scan_ws, self.du, self.ddt,
                                   G["A"], dp[:, R:R + N], dp[:, R + N:], Dskip=P["Dskip"], z=z, dt_bias=P["dt_bias"],
                                   dDskip=G["Dskip"], dz=dxz[:, D:], ddt_bias=G["dt_bias"])
        G["Wdt"].copy_(self.ddt.t() @ p[:, :R])
        dp[:, :R] = self.ddt @ P["Wdt"]
        G["Wx"].copy_(dp.t() @ u)
        self.du += dp @ P["Wx"]
        # the convolution's rows: y of its descriptor is u, dx goes beside dz
        J.janus_causal_conv_bwd(self.conv, xz, lengths, P["conv_w"], P["conv_b"], None, self.du, None, dxz,
                                G["conv_w"], G["conv_b"], None, self.conv_ws)
        G["Win"].copy_(dxz.t() @ x0)
        torch.mm(dxz, P["Win"], out=self.dx0)
        J.janus_embed_softmax_xent(self.embed, J.EMBED_BWD, ids_host, ids, inp=self.dx0, dtable=G["E"],
                                   ws=self.embed_ws)
        for up in self.updates:
            up.apply()
        return self.stats

    # ------------------------------------------------------------ rollouts
    def rollout(self, first: np.ndarray, steps: int, seed: int = 0):
        """Samples ``steps`` tokens after each of the tokens ``first`` [B], one
        token at a time from carried states.  Returns tokens [steps + 1, B] and
        the log-probabilities [steps, B] under this policy."""
        w, P, B = self.w, self.P, len(first)
        code = _cdt(w.dtype)
        g = torch.Generator(device=self.device)
        g.manual_seed(seed)
        conv = J.ConvDesc(w.D, w.K, B, 1, code, J.CONV_SILU, 2 * w.D, 0)
        p_cols = w.R + 2 * w.N
        scan = J.ScanDesc(w.D, w.N, 1, B, 1, code, J.SCAN_SOFTPLUS, 0, 0, p_cols, p_cols, 2 * w.D, 0)
        embed = J.XentDesc(w.V, w.M, B, code)
        loss = J.PolicyDesc(B, w.V, code, 0, *self.coefs)
        taps = torch.zeros(B, w.K - 1, w.D, dtype=self.tdt, device=self.device)
        state = torch.zeros(B, w.D, w.N, dtype=torch.float32, device=self.device)
        ids = torch.from_numpy(np.ascontiguousarray(first, np.int32)).to(self.device)
        tokens, logps = [np.asarray(first, np.int32)], []
        u, y = self.rows(B, w.D), self.rows(B, w.D)
        for _ in range(steps):
            _, xz = self._mid(tokens[-1], ids, embed)
            J.janus_causal_conv_step(conv, xz, P["conv_w"], P["conv_b"], taps, u)
            _, dt, Bm, Cm = self._project(u)
            J.janus_selective_scan_step(scan, u, dt, P["A"], Bm, Cm, state, y, Dskip=P["Dskip"], z=xz[:, w.D:],
                                        dt_bias=P["dt_bias"])
            logits = y @ P["Wout"].t()
            ids = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=g)[:, 0].int()
            logp = torch.empty(B, dtype=torch.float32, device=self.device)
            J.janus_policy_loss(loss, logits, ids, logp=logp)
            logps.append(logp)
            tokens.append(ids.cpu().numpy())
        return np.stack(tokens), torch.stack(logps)


def results(policy: SelectivePolicy) -> Dict[str, np.ndarray]:
    torch.cuda.synchronize()
    out = {k: g.double().cpu().numpy() for k, g in policy.G.items()}
    out["stats"] = policy.stats.double().cpu().numpy()
    return out
