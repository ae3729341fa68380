"""The token policy that runs the convolution, the scan and the policy loss
together (policy_step.SelectivePolicy): the step's loss and every gradient
against float64 automatic differentiation of the same model on the CPU, and the
single-token rollouts against the sequence forms.

Tolerances (relative to the largest entry): the products and the scan add a few
hundred float32 roundings: 1e-3 on gradients, as for the framework's other
training steps; bf16 rounds every activation to 2^-9 and the gradients pass four
products of such values: 6e-2."""
import numpy as np
import pytest
import torch

from paper_1812_01329_amd import workloads as wl

pytestmark = pytest.mark.gpu


def reference(w, tokens, lengths, old, adv, ref, beta, eta):
    """Loss and gradients in float64, step by step."""
    P = {k: torch.tensor(np.asarray(a, np.float64), requires_grad=True) for k, a in w.params.items()}
    T, B, D, N, K, R = w.T, w.B, w.D, w.N, w.K, w.R
    loss, count, logps = 0.0, 0, np.zeros((T, B))
    for b in range(B):
        n = int(lengths[b])
        xz = P["E"][torch.tensor(tokens[:n, b].astype(np.int64))] @ P["Win"].t()
        x, z = xz[:, :D], xz[:, D:]
        seq = torch.cat([torch.zeros(K - 1, D, dtype=torch.float64), x])
        u = torch.nn.functional.silu((seq.unfold(0, K, 1) * P["conv_w"]).sum(-1) + P["conv_b"])
        p = u @ P["Wx"].t()
        e = torch.nn.functional.softplus(p[:, :R] @ P["Wdt"].t() + P["dt_bias"])
        h, ys = torch.zeros(D, N, dtype=torch.float64), []
        for t in range(n):
            h = torch.exp(e[t][:, None] * P["A"]) * h + (e[t] * u[t])[:, None] * p[t, R:R + N]
            ys.append((h * p[t, R + N:]).sum(1) + P["Dskip"] * u[t])
        y = torch.stack(ys) * torch.nn.functional.silu(z)
        lp = torch.log_softmax(y @ P["Wout"].t(), 1)
        l = lp[torch.arange(n), torch.tensor(tokens[1:n + 1, b].astype(np.int64))]
        logps[:n, b] = l.detach().numpy()
        o, a, r = (torch.tensor(np.asarray(v, np.float64)[:n, b]) for v in (old, adv, ref))
        ratio = torch.exp(l - o)
        k = r - l
        row = -torch.minimum(ratio * a, ratio.clamp(0.8, 1.2) * a) + beta * (torch.exp(k) - 1 - k) \
            + eta * (lp.exp() * lp).sum(1)
        loss, count = loss + row.sum(), count + n
    (loss / count).backward()
    return float((loss / count).detach()), {k: v.grad.numpy() for k, v in P.items()}, logps


@pytest.mark.parametrize("dtype,tol", [("f32", 1e-3), ("bf16", 6e-2)])
def test_step_against_float64(dtype, tol):
    from paper_1812_01329_amd.policy_step import SelectivePolicy, results
    w = wl.sequence_policy(V=101, M=24, D=40, N=16, R=6, B=5, T=13, dtype=dtype)
    print(f"[policy step] {dtype} lengths={w.lengths}", flush=True)
    rng = np.random.default_rng(4)
    pol = SelectivePolicy(w, kl_coef=0.1, ent_coef=0.01)
    logp = pol.score(w.tokens, w.lengths).cpu().numpy().reshape(w.T, w.B)
    # ratios inside and outside the clip, off its corners
    old = (logp - rng.choice([-0.5, -0.1, 0.05, 0.4], size=logp.shape)).astype(np.float32)
    ref = (logp - rng.normal(0, 0.3, logp.shape)).astype(np.float32)
    adv = np.broadcast_to(w.adv, logp.shape).astype(np.float32).copy()
    dev = lambda a: torch.from_numpy(a.reshape(-1)).cuda()
    pol.step(w.tokens, w.lengths, dev(old), dev(adv), dev(ref))
    got = results(pol)
    loss, grads, logps = reference(w, w.tokens, w.lengths, old, adv, ref, 0.1, 0.01)
    assert np.abs(logp - logps).max() <= tol * np.abs(logps).max()
    assert abs(got["stats"][0] - loss) <= tol * max(1.0, abs(loss))
    assert got["stats"][5] == w.lengths.sum()
    for k, g in grads.items():
        err = np.abs(got[k] - g).max() / np.abs(g).max()
        print(f"  {k}: {err:.2e}", flush=True)
        assert err <= tol, (k, err)


def test_rollout_is_the_sequence_form():
    """The log-probabilities of sampled tokens, from single-token steps, are
    those that the sequence forms give for the same tokens."""
    from paper_1812_01329_amd.policy_step import SelectivePolicy
    w = wl.sequence_policy(V=301, M=32, D=72, B=6, T=20)
    pol = SelectivePolicy(w)
    tokens, logp = pol.rollout(w.tokens[0], w.T, seed=3)
    assert tokens.shape == (w.T + 1, w.B) and (tokens >= 0).all() and (tokens < w.V).all()
    again = pol.score(tokens, None).view(w.T, w.B)
    assert float((again - logp).abs().max()) <= 1e-4 * float(logp.abs().max())


def test_update_goes_down_the_loss():
    """On fixed rollouts a small step changes the loss by -lr |g|^2 to first
    order (the ratio is 1 there, inside the clip)."""
    from paper_1812_01329_amd.policy_step import SelectivePolicy
    w = wl.sequence_policy(V=50, M=32, D=64, B=32, T=12)
    lr = 10.0
    pol = SelectivePolicy(w, update=(lr, 0.0))
    tokens, logp = pol.rollout(w.tokens[0], w.T, seed=1)
    adv = torch.from_numpy(np.broadcast_to(w.adv, (w.T, w.B)).copy()).cuda().reshape(-1)
    old = logp.reshape(-1)
    before = pol.step(tokens, w.lengths, old, adv).double().cpu().numpy().copy()
    norm2 = sum(float((g.double() ** 2).sum()) for g in pol.G.values())
    after = pol.step(tokens, w.lengths, old, adv).double().cpu().numpy()
    assert before[5] == after[5] == w.lengths.sum()
    drop = before[0] - after[0]
    print(f"[policy update] loss {before[0]:.6f} -> {after[0]:.6f}, drop {drop:.3e}, first order {lr * norm2:.3e}", flush=True)
    assert 0.5 * lr * norm2 < drop < 1.5 * lr * norm2
