"""GPU parity of the short causal convolution with every tap count at every
access width (one, two and four channels a lane), over several segments of time
with sequences that end at their edges; and prompts whose final states single
tokens continue.

Tolerances as in the convolution's other parity tests."""
import numpy as np
import pytest

from oracle import conv as oracle
from test_gpu_conv import TOL, Conv, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D", [("bf16", 260), ("bf16", 130), ("bf16", 131), ("f32", 260), ("f32", 130)])
@pytest.mark.parametrize("K", range(1, 9))
def test_taps(K, dtype, D):
    print(f"[conv wide] K={K} D={D} {dtype}", flush=True)
    # 70 steps in segments of 18
    lengths = np.array([70, 15, 16, 17, 18, 19, K - 1, 0, 35, 36, 37, 36 + K - 1, 36 - (K - 1), 69], np.int32)
    for silu in (True, False):
        c = Conv(40 + K, 70, len(lengths), D, K, dtype, silu, lengths)
        c.check(c.run())


@pytest.mark.parametrize("dtype,D", [("bf16", 260), ("bf16", 130), ("bf16", 33), ("f32", 260), ("f32", 33)])
@pytest.mark.parametrize("K", [1, 2, 3, 5, 6, 7, 8])
def test_a_prompt_continued_by_single_tokens(K, dtype, D):
    """The final states of ragged prompts, put into slots of a larger state and
    moved on token by token, give what the whole sequences give."""
    import torch
    from paper_1812_01329_amd import janus as J
    print(f"[conv continued] K={K} D={D} {dtype}", flush=True)
    T, more = 20, 5
    lengths = np.array([20, 0, 1, K, 13], np.int32)
    B = len(lengths)
    c = Conv(60 + K, T + more, B, D, K, dtype)
    w, bias, s0 = c.dev(c.w), c.dev(c.bias), c.dev(c.s0)
    d = J.ConvDesc(D, K, B, T, c.desc.dtype, c.desc.act, 0, 0)
    y = torch.empty((T, B, D), dtype=c.tdt, device="cuda")
    sT = torch.empty((B, K - 1, D), dtype=c.tdt, device="cuda")
    J.janus_causal_conv_fwd(d, c.dev(c.x[:T]), lengths, w, bias, s0, y, sT)
    slots = np.array([6, 2, 0, 5, 3], np.int32)
    state = torch.full((8, K - 1, D), float("nan"), dtype=c.tdt, device="cuda")
    state[torch.from_numpy(slots).long().cuda()] = sT
    one = J.ConvDesc(D, K, B, 1, c.desc.dtype, c.desc.act, 0, 0)
    rows = np.arange(B)
    for k in range(more):
        yk = torch.full((B, D), float("nan"), dtype=c.tdt, device="cuda")
        J.janus_causal_conv_step(one, c.dev(c.x[lengths + k, rows]), w, bias, state, yk,
                                 slots=torch.from_numpy(slots).cuda())
        ref, end = oracle.forward(c.x, lengths + k + 1, c.w, c.bias, c.s0, True)
        near(f"y of token {k}", yk, ref[lengths + k, rows], TOL[dtype])
    near("state", state[torch.from_numpy(slots).long().cuda()], end, 0.0)
    if K > 1:
        assert bool(torch.isnan(state[[1, 4, 7]]).all())
