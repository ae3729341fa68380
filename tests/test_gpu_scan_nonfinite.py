"""The selective scan with an infinite or NaN input, state or gradient in one
channel of one sequence: rows past that sequence's end stay 0, other sequences
and what does not depend on the value keep their bits, and the results are
finite exactly where the float64 oracle's are.

Tolerances as in the scan's other parity tests, over the finite entries."""
import numpy as np
import pytest

from test_gpu_scan import TOL, Scan

pytestmark = pytest.mark.gpu


def poison(s, where, value, b, t, d):
    if where == "x":
        s.x[t, b, d] = value
    elif where == "h0":
        s.h0[b, d, 1] = value
    else:
        s.dhT[b, d, 1] = value


@pytest.mark.parametrize("T,N,gate,dtype", [(13, 16, True, "f32"), (13, 13, True, "f32"), (21, 16, False, "bf16"),
                                            (150, 16, True, "f32"), (19, 40, True, "f32"), (16, 3, True, "bf16")])
@pytest.mark.parametrize("where,value", [("x", np.inf), ("x", np.nan), ("h0", np.inf), ("dhT", np.inf), ("dhT", np.nan)])
def test_stays_within_its_sequence(where, value, T, N, gate, dtype):
    print(f"[scan nonfinite] {where} {value} T={T} N={N} {dtype}", flush=True)
    B, D, b, d = 3, 70, 1, 5
    lengths = np.array([T, T - 2, T - 3], np.int32)
    clean, s = (Scan(51, T, B, D, N, 1, dtype, lengths, gate=gate) for _ in range(2))
    n = int(lengths[b])
    poison(s, where, value, b, n - 1, d)          # the last step that runs
    got, ok = s.run(), clean.run()
    for k in ("y", "dx", "ddt", "dz", "dBm", "dCm"):
        if k not in got:
            continue
        for i, m in enumerate(lengths):
            assert not bool(got[k][m:, i].any()), f"{k} past the end of sequence {i}"
        others = [i for i in range(B) if i != b]
        assert s.torch.equal(got[k][:, others], ok[k][:, others]), k
    for k in ("hT", "dh0"):
        others = [i for i in range(B) if i != b]
        assert s.torch.equal(got[k][others], ok[k][others]), k
    with np.errstate(invalid="ignore", over="ignore"):
        ref = s.reference()
    for k in got:
        g, r = got[k].double().cpu().numpy(), ref[k]
        fine = np.isfinite(r)
        np.testing.assert_array_equal(np.isfinite(g), fine, err_msg=k)
        if fine.any():
            tol = TOL["f32" if k in ("hT", "dA", "dDskip", "ddt_bias", "dh0") else dtype]
            err = np.abs(g[fine] - r[fine]).max() / np.abs(r[fine]).max()
            assert err <= tol, f"{k}: {err:.3e}"
