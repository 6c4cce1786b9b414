"""One batch element or row alone of 2^32 threads and more is refused by its status (no pointer given here is ever read)."""
import ctypes

from test_block_abi_cpu import A16, ssdi8  # noqa: F401


def test_refusals(ssdi8):  # noqa: F811
    s, L = ssdi8, ssdi8.lib()
    norm = s.NormArgs(dtype=s.F16, eps=1e-5)
    call = lambda channels, groups: L.ssdi8_gated_norm(1, channels, groups, ctypes.byref(norm), None)
    assert call(1 << 26, 1 << 26) == call(1 << 27, 1 << 26) == s.ERR_UNSUPPORTED
    assert call((1 << 26) - 1, (1 << 26) - 1) == s.ERR_NULL
    scan = s.SelScanArgs(dtype=s.F16, dt_dtype=s.F32)
    for f in (L.ssdi8_selective_scan, L.ssdi8_selective_scan_step):
        call = lambda ch, n: f(ctypes.byref(s.SelScanDims(batch=1, seqlen=1, nheads=ch, headdim=1, ngroups=1, dstate=n)),
                               ctypes.byref(scan), None)
        assert call(1 << 26, 256) == call(1 << 27, 100) == call(1 << 29, 16) == s.ERR_UNSUPPORTED
        assert call((1 << 26) - 8, 256) == call((1 << 29) - 64, 16) == s.ERR_NULL
