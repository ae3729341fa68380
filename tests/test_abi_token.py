"""Refusals of the layer norm, sampling and AdamW entry points (no GPU needed):
bad descriptors and arguments are rejected with their status before any device
work, and no buffer is touched."""
import ctypes as C
import math

import pytest

from paper_1812_01329_amd import janus as J
from tests.test_abi_sequence import INV, UNS, WS, Buf, refused


def norm(**k):
    return J.NormDesc(*(k.get(n, v) for n, v in dict(rows=3, D=8, dtype=J.F32, eps=1e-5, ldx=0, ldh=0, ldy=0).items()))


def fwd(d, **k):
    v = dict(d=d, x=Buf(), gamma=Buf(), beta=Buf(), y=Buf(), r=Buf(), h=Buf(), mean=Buf(), rstd=Buf())
    v.update(k)
    return list(v.values())


def bwd(d, **k):
    v = dict(d=d, h=Buf(), gamma=Buf(), mean=Buf(), rstd=Buf(), dy=Buf(), dx=Buf(),
             ws=Buf(J.janus_layer_norm_workspace_bytes(d) or 1), dgamma=Buf(), dbeta=Buf(), dh=Buf())
    v.update(k)
    return list(v.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INV), (dict(D=0), INV), (dict(ldx=7), INV), (dict(ldh=7), INV), (dict(ldy=-8), INV),
    (dict(eps=-1e-5), INV), (dict(eps=math.inf), INV), (dict(eps=math.nan), INV), (dict(dtype=2), UNS),
    (dict(D=(1 << 24) + 1), UNS), (dict(rows=(1 << 30) + 1), UNS)])
def test_norm_descriptors(change, status):
    d = norm(**change)
    assert J.janus_layer_norm_workspace_bytes(d) == 0
    refused(status, J.janus_layer_norm_fwd, fwd(d))
    refused(status, J.janus_layer_norm_bwd, bwd(d))


def test_norm_arguments():
    d = norm()
    for k in ("x", "y"):
        refused(INV, J.janus_layer_norm_fwd, fwd(d, **{k: None}))
    for k in ("h", "mean", "rstd", "dy"):
        refused(INV, J.janus_layer_norm_bwd, bwd(d, **{k: None}))
    refused(INV, J.janus_layer_norm_fwd, fwd(d, r=None))                 # a sum of nothing
    for k in ("x", "y", "r", "h", "gamma", "beta", "mean", "rstd"):
        refused(INV, J.janus_layer_norm_fwd, fwd(d, **{k: Buf(shift=2)}))
    for k in ("h", "dy", "dx", "dh", "gamma", "mean", "rstd", "dgamma", "dbeta"):
        refused(INV, J.janus_layer_norm_bwd, bwd(d, **{k: Buf(shift=2)}))
    b = Buf()
    for k in ("x", "r", "h"):
        refused(INV, J.janus_layer_norm_fwd, fwd(d, y=b, **{k: b}))
    refused(INV, J.janus_layer_norm_fwd, fwd(norm(ldx=16), x=b, h=b))    # in place with another stride
    refused(INV, J.janus_layer_norm_bwd, bwd(norm(ldx=16), dx=b, dh=b))
    for k in ("h", "dy"):
        refused(INV, J.janus_layer_norm_bwd, bwd(d, dx=b, **{k: b}))
    need = J.janus_layer_norm_workspace_bytes(d)
    assert need > 0
    for ws in (None, Buf(need - 1), Buf(need, shift=128)):
        refused(WS, J.janus_layer_norm_bwd, bwd(d, ws=ws))


def test_norm_of_no_rows():
    """No rows: a forward has nothing to do and needs no buffer."""
    J.janus_layer_norm_fwd(norm(rows=0), None, None, None, None, stream=0)
    J.janus_layer_norm_bwd(norm(rows=0), None, None, None, None, None, None, stream=0)
    assert J.janus_layer_norm_workspace_bytes(norm(rows=0)) == 0


def sample(**k):
    return J.SampleDesc(*(k.get(n, v) for n, v in dict(rows=3, V=10, dtype=J.F32, ld=0, temperature=1.0, top_k=0, top_p=1.0,
                                                       min_p=0.0).items()))


def sample_args(d, **k):
    v = dict(d=d, logits=Buf(), u=Buf(), tokens=Buf(), temperature=Buf(), top_k=Buf(), top_p=Buf(), min_p=Buf(),
             logp=Buf(), draw_logp=Buf(), kept=Buf(), ws=Buf(J.janus_sample_workspace_bytes(d) or 1))
    v.update(k)
    return list(v.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), INV), (dict(V=0), INV), (dict(ld=9), INV), (dict(temperature=-0.5), INV),
    (dict(temperature=math.nan), INV), (dict(top_p=math.nan), INV), (dict(min_p=math.nan), INV), (dict(dtype=9), UNS),
    (dict(V=(1 << 24) + 1), UNS), (dict(rows=(1 << 30) + 1), UNS)])
def test_sample_descriptors(change, status):
    d = sample(**change)
    assert J.janus_sample_workspace_bytes(d) == 0
    refused(status, J.janus_sample, sample_args(d))


def test_sample_arguments():
    d = sample()
    for k in ("logits", "u", "tokens"):
        refused(INV, J.janus_sample, sample_args(d, **{k: None}))
    for k in ("logits", "u", "tokens", "temperature", "top_k", "top_p", "min_p", "logp", "draw_logp", "kept"):
        refused(INV, J.janus_sample, sample_args(d, **{k: Buf(shift=2)}))


def adamw(**k):
    return J.AdamWDesc(*(k.get(n, v) for n, v in dict(n=2, states=J.ADAMW_8BIT, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                                                      max_norm=1.0, seed=0).items()))


class Tensors:
    """Two tensors of 100 elements; `change` is of the second."""

    def __init__(self, **change):
        self.bufs = []
        self.array = (J.AdamWTensor * 2)()
        for i in range(2):
            f = dict(p=Buf(), g=Buf(), m=Buf(), v=Buf(), scale=Buf(), master=None, size=100, decay=0.0, dtype=J.F32)
            if i:
                f.update(change)
            self.bufs += [b for b in f.values() if isinstance(b, Buf)]
            self.array[i] = J.AdamWTensor(*[b.data_ptr() if isinstance(b, Buf) else b for b in f.values()])


def call(status, d, t=None, step="there", ws="there", lr=None, stats=None, hold=None):
    t = t or Tensors()
    step = Buf() if step == "there" else step
    ws = Buf(J.janus_adamw_workspace_bytes(d) or 1) if ws == "there" else ws
    with pytest.raises(J.JanusError) as e:
        J.janus_adamw_update(d, t.array if t != "none" else C.cast(None, C.POINTER(J.AdamWTensor)), step, lr=lr, stats=stats,
                             ws=ws, hold=hold, stream=0)
    assert e.value.status == status
    for b in ([] if t == "none" else t.bufs) + [b for b in (step, ws, lr, stats) if isinstance(b, Buf)]:
        assert b.untouched()


@pytest.mark.parametrize("change,status", [
    (dict(n=0), INV), (dict(lr=math.nan), INV), (dict(lr=math.inf), INV), (dict(beta1=1.0), INV), (dict(beta1=-0.1), INV),
    (dict(beta2=1.0), INV), (dict(beta2=math.nan), INV), (dict(eps=0.0), INV), (dict(eps=math.inf), INV),
    (dict(max_norm=math.nan), INV), (dict(states=2), UNS)])
def test_adamw_descriptors(change, status):
    d = adamw(**change)
    assert J.janus_adamw_workspace_bytes(d) == 0
    call(status, d)


def test_adamw_eps_is_a_normal_number():
    """The reciprocal of a smaller one leaves float32: 0 / (0 + eps) would be NaN."""
    assert J.janus_adamw_workspace_bytes(adamw(eps=2.0 ** -127)) == 0
    assert J.janus_adamw_workspace_bytes(adamw(eps=2.0 ** -126)) > 0


def test_adamw_arguments():
    d = adamw()
    call(INV, d, "none")
    call(INV, d, step=None)
    call(INV, d, step=Buf(shift=4))
    call(INV, d, lr=Buf(shift=2))
    call(INV, d, stats=Buf(shift=2))
    call(INV, d, hold=Buf(shift=2).data_ptr())
    for k in ("p", "g", "m", "v", "scale"):
        call(INV, d, Tensors(**{k: None}))
    for k in ("p", "g", "master"):
        call(INV, d, Tensors(**{k: Buf(shift=2), "dtype": J.BF16 if k == "master" else J.F32}))
    call(INV, d, Tensors(p=Buf(shift=1), dtype=J.BF16))
    call(INV, d, Tensors(scale=Buf(shift=4)))
    call(INV, adamw(states=J.ADAMW_F32), Tensors(m=Buf(shift=2)))
    call(INV, d, Tensors(master=Buf()))            # of float32 parameters
    call(INV, d, Tensors(size=-1))
    call(INV, d, Tensors(decay=math.nan))
    call(UNS, d, Tensors(dtype=4))
    call(UNS, d, Tensors(size=(1 << 32) + 1))
    call(UNS, adamw(states=J.ADAMW_F32), Tensors(size=(1 << 40) + 1))
    need = J.janus_adamw_workspace_bytes(d)
    for ws in (None, Buf(need - 1), Buf(need, shift=64)):
        call(WS, d, ws=ws)


def test_update_classes_refuse():
    import torch
    from paper_1812_01329_amd import train_step as ts
    p = [torch.zeros(4), torch.zeros(3, dtype=torch.bfloat16)]
    g = [torch.zeros(4), torch.zeros(3)]
    with pytest.raises(ValueError):
        ts.make_update(p, g, ts.AdamW(1e-3, bits=4))
    with pytest.raises(ValueError):
        ts.make_update(p, [g[0], g[1].bfloat16()], ts.AdamW(1e-3))
    with pytest.raises(ValueError):
        ts.make_update([p[0].half()], g[:1], ts.AdamW(1e-3))
    up = ts.make_update(p, g, ts.AdamW(1e-3, bits=8, masters=True))
    assert up.master[0] is None and up.master[1].dtype == torch.float32
    state = up.state_dict()
    up.load_state_dict(state)
    state["m"][0] = state["m"][0][:2]
    with pytest.raises(ValueError):
        up.load_state_dict(state)


def test_host_tensors_are_refused():
    """A tensor in host memory is refused before the call (its address would fault on the GPU)."""
    import torch
    x = torch.zeros(3, 8)
    with pytest.raises(ValueError, match="not on the GPU"):
        J.janus_layer_norm_fwd(norm(), x, None, None, x.clone())
    with pytest.raises(ValueError, match="not on the GPU"):
        J.janus_layer_norm_bwd(norm(), x, None, x[0], x[0], x, x.clone())
    with pytest.raises(ValueError, match="not on the GPU"):
        J.janus_sample(sample(V=8), x, x[0, :3], torch.zeros(3, dtype=torch.int32))
    from paper_1812_01329_amd import train_step as ts
    with pytest.raises(ValueError, match="not on the GPU"):
        ts.make_update([x], [x.clone()], ts.AdamW(1e-3)).apply()


def test_tensors_that_do_not_go_together():
    import torch
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)
    good = dict(params=[z(300)], grads=[z(300)], m=[z(300, torch.uint8)], v=[z(300, torch.uint8)], scale=[torch.zeros(2, 2)])
    J.adamw_tensors(**good)
    for name, bad in (("grads", z(299)), ("grads", z(300, torch.bfloat16)), ("params", z(300, torch.float16)), ("m", z(300)),
                      ("v", z(301, torch.uint8)), ("scale", torch.zeros(1, 2)), ("params", z(600)[::2]), ("master", z(3))):
        with pytest.raises(ValueError, match="adamw_tensors"):
            J.adamw_tensors(**{**good, name: [bad]})
    with pytest.raises(ValueError, match="adamw_tensors"):
        J.adamw_tensors([z(3)], [z(3)], [z(3, torch.uint8)], [z(3)])   # no scale: states of 32 bits
