"""The int8 codes of the quantizing norm, code by code."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,D", [(300, 1000), (200, 81), (40, 2560), (40, 8195)])
def test_codes(M, D):
    """A code is its value times the rounded inverse of its row's step, rounded to even, as quantize_act's; fp32's y is what
    is quantized."""
    from paper_2608_21952_amd import ssdi8
    x = torch.randn(M, D, generator=torch.Generator().manual_seed(M)).cuda()
    w = (1 + 0.1 * torch.randn(D, generator=torch.Generator().manual_seed(D))).cuda()
    out = ssdi8.norm_quantize(x, w, format="int8", with_y=True)
    y = out["y"].cpu()
    step = y.abs().amax(1) / 127
    assert torch.equal(out["scales"].cpu(), step)
    assert torch.equal(out["codes"].cpu().float(), torch.round(y * (1 / step)[:, None]))
    codes, steps = ssdi8.quantize_act(out["y"].view(1, M, 1, D), "token")
    assert torch.equal(codes.view(M, D), out["codes"]) and torch.equal(steps, out["scales"])
