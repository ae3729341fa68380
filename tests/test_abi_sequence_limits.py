"""Size limits of the scan's entry points (no GPU needed): what the kernels'
32-bit offsets cannot hold is refused before any device work."""
import pytest

from paper_1812_01329_amd import janus as J
from test_abi_sequence import UNS, Buf, refused, scan, scan_bwd, scan_fwd


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
