"""The operators around the SSD layer where their forms differ, against the 64-bit forms and bounds of
block_ref.py."""
import pytest
import torch

import block_ref as R
from test_gpu_block import BF16, F16, F32, Draw, dev, scan_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


# ------------------------------------------------------------------------------ selective scan
@pytest.mark.parametrize("L,H,P,G,N,tied,dtype", [
    (40, 24, 1, 1, 16, False, F16), (40, 24, 1, 1, 8, False, F16), (70, 24, 1, 1, 12, False, BF16),
    (300, 40, 1, 1, 24, False, F32),                                    # cut into spans
    (40, 24, 1, 1, 5, False, F32), (40, 12, 3, 2, 18, False, F16),      # the general form
    (70, 3, 8, 1, 36, True, F16), (300, 3, 16, 1, 100, True, BF16), (40, 3, 5, 1, 100, True, F32),
    (300, 2, 8, 1, 200, True, F16)])
def test_scan_infinite_inputs(ssdi8, L, H, P, G, N, tied, dtype):
    """An infinite input or time step makes its channel's states infinite from there on, of the sign that the
    formula gives, whatever the number of states: those that only fill up the lanes add nothing."""
    r = Draw(L + N)
    positive = lambda *s: r.normal(*s).abs() + 0.125
    i = {"u": positive(1, L, H * P).to(dtype), "dt": r.normal(1, L, H) * 0.5 - 4.0,
         "A": -torch.exp(r.uniform(0.0, 1.0, *((H,) if tied else (H * P, N)))),
         "B": positive(1, L, G, N).to(dtype), "C": positive(1, L, G, N).to(dtype), "D": positive(H),
         "dt_bias": None, "z": None, "state": positive(1, H * P, N)}
    t0 = L // 2 + 1
    i["u"][0, t0, 2], i["u"][0, t0 + 3, 3] = float("inf"), -float("inf")
    i["dt"][0, t0 + 1, H - 1] = float("inf")
    y, e, h, he = scan_ref(i)
    last = slice((H - 1) * P, H * P)
    assert (y[0, t0:, 2] == float("inf")).all() and (y[0, t0 + 3:, 3] == -float("inf")).all()
    assert (y[0, t0 + 1:, last] == float("inf")).all() and torch.isfinite(y[0, :t0]).all()
    g = {k: dev(v) for k, v in i.items()}
    out = ssdi8.selective_scan(g["u"], g["dt"], g["A"], g["B"], g["C"], D=g["D"], init_state=g["state"])
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    R.assert_within(out["final_state"], h, he + R.TINY[F32], "final_state")


@pytest.mark.parametrize("H,P,G,N,tied,dtype", [(40, 1, 1, 16, False, F16), (40, 1, 1, 24, False, F32),
                                                (3, 16, 1, 100, True, BF16), (9, 5, 1, 16, False, F32)])
def test_scan_infinite_state_over_spans(ssdi8, H, P, G, N, tied, dtype):
    """No finite decay ends an infinite state, however many tokens it comes from: not where a scan is cut and
    the decay of a whole span, a product of many, is 0 in fp32."""
    r, L = Draw(N), 640
    positive = lambda *s: r.normal(*s).abs() + 0.125
    i = {"u": positive(1, L, H * P).to(dtype), "dt": r.normal(1, L, H) * 0.5 - 1.0,
         "A": -torch.exp(r.uniform(1.0, 2.7, *((H,) if tied else (H * P, N)))),
         "B": positive(1, L, G, N).to(dtype), "C": positive(1, L, G, N).to(dtype), "D": positive(H),
         "dt_bias": None, "z": None, "state": positive(1, H * P, N)}
    i["state"][0, 1, 0], i["state"][0, 2, N - 1] = float("inf"), -float("inf")
    i["u"][0, 3, 7] = float("inf")
    y, e, h, he = scan_ref(i)
    assert (y[0, :, 1] == float("inf")).all() and (y[0, :, 2] == -float("inf")).all()
    assert (y[0, 3:, 7] == float("inf")).all()
    g = {k: dev(v) for k, v in i.items()}
    sizes = ssdi8.SelScanDims(1, L, H, P, G, N)
    assert ssdi8.selective_scan_workspace_size(sizes) > 0      # cut
    out = ssdi8.selective_scan(g["u"], g["dt"], g["A"], g["B"], g["C"], D=g["D"], init_state=g["state"])
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    R.assert_within(out["final_state"], h, he + R.TINY[F32], "final_state")
