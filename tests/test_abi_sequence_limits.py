"""Limits of the convolution's and the scan's entry points (no GPU needed): what
the kernels' 32-bit offsets or the order of their reads and writes cannot hold
is refused before any device work."""
import pytest

from paper_1812_01329_amd import janus as J
from test_abi_sequence import INV, UNS, Buf, conv, refused, scan, scan_bwd, scan_fwd


@pytest.mark.parametrize("name", ["ldx", "ldt", "ldz", "ldy"])
@pytest.mark.parametrize("B,ld", [(4, 1 << 62), (4, (1 << 62) + 8), (2, 1 << 62), (16, 1 << 60), (2, (1 << 28) + 1)])
def test_scan_strides_whose_product_with_the_batch_overflows(name, B, ld):
    d = scan(B=B, **{name: ld})
    assert J.janus_selective_scan_workspace_bytes(d) == 0
    refused(UNS, J.janus_selective_scan_fwd, *scan_fwd(d, ws=Buf()))
    refused(UNS, J.janus_selective_scan_bwd, *scan_bwd(d, ws=Buf()))
    refused(UNS, J.janus_selective_scan_step, (d, *[Buf() for _ in range(7)]))


def test_scan_strides_at_the_limit_are_taken():
    assert J.janus_selective_scan_workspace_bytes(scan(B=2, ldx=1 << 28)) > 0


@pytest.mark.parametrize("T", [0, 5, 100])
def test_conv_state_gradient_in_place(T):
    """ds0 is written before dsT is read, in long sequences by another workgroup."""
    d, b, g = conv(T=T), [Buf() for _ in range(9)], Buf()
    ws = Buf(J.janus_causal_conv_workspace_bytes(d))
    refused(INV, J.janus_causal_conv_bwd, (d, b[0], None, b[1], b[2], b[3], b[4], g, b[5], b[6], b[7], g, ws))
