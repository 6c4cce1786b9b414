"""Linear attention where few of a chunk's terms count: sparse keys, decays of many bits within a chunk, values of
very different sizes in a column.  Every element of the state keeps fp32's accuracy relative to its own terms (mixer_ref.py),
over a prompt as over its tokens one by one.

Of y (16-bit types) the terms are held to the type's rounding.  fp16 values below the normal range are off by 2^-25
instead; p of a row and S of a column are brought to where their largest is at least 2^14, so that the terms' own bounds
grow by 2^-39 of the largest p of the row's chunk, of the largest S of the column (`floor`)."""
import pytest
import torch

import mixer_ref as R
from test_gpu_attention import BF16, F16, F32, draw, ssdi8  # noqa: F401

pytestmark = pytest.mark.gpu
# Of the state, beyond its relative bound: terms below fp32's normal range are lost, 2^-126 times keys of up to 8 for each of
# up to 2200 tokens.
LOST = 2.0 ** -110


def floor(t, dtype):
    """What fp16's smallest steps add to y's bound; 0 for other types."""
    q, k, v, g, init = (None if t[n] is None else t[n].double() for n in ("q", "k", "v", "g", "init"))
    b, L, Hv, V = v.shape
    H = max(q.shape[2], Hv)
    if dtype != F16:
        return torch.zeros(b, L, H, V, dtype=torch.float64, device=v.device)
    qh, kv = R.spread(q, 2, H).transpose(1, 2), R.spread(k, 2, Hv).transpose(1, 2)
    kh, vh = R.spread(kv, 1, H), R.spread(v, 2, H).transpose(1, 2)
    g = g.expand(b, L, Hv)
    c = R.spread(g, 2, H).cumsum(1).transpose(1, 2)
    at = torch.arange(L, device=v.device)
    near = (at[:, None] >= at) & (at[:, None] // 64 == at // 64)
    diff = torch.where(near, c[..., :, None] - c[..., None, :], 0.0)
    p = torch.where(near, torch.exp(diff) * (qh @ kh.mT).abs(), 0.0)
    out = p.amax(-1, keepdim=True) * (near.double() @ vh.abs())
    S = torch.zeros(b, Hv, k.shape[-1], V, dtype=torch.float64, device=v.device) if init is None else init.abs()
    for i in range(L):
        if i % 64 == 0:
            most, behind = R.spread(S.amax(2), 1, H), torch.zeros(b, H, device=v.device, dtype=torch.float64)
        behind = behind + R.spread(g[:, i], 1, H)
        out[:, :, i] += (qh[:, :, i].abs().sum(-1) * torch.exp(behind))[..., None] * most
        S = torch.exp(g[:, i])[..., None, None] * S + kv[:, :, i].abs()[..., None] * v[:, i].abs()[:, :, None]
    return 2.0 ** -39 * q.shape[-1] ** -0.5 * out.transpose(1, 2)


def sparse(t):
    t["k"].relu_()
    t["g"].fill_(-2.0)


def no_last_key(decay):
    def change(t):
        t["k"][:, -1] = 0
        t["g"][:, -1] = decay
    return change


def no_last_values(t):
    t["v"][:, -4:] = 0
    t["g"].fill_(-3.0)


def large_then(later):
    def change(t):
        t["g"].fill_(-0.4)
        t["v"][:, :90] *= 1000
        t["v"][:, 90:] *= later
    return change


CASES = {"sparse": sparse, "-10": no_last_key(-10.0), "-20": no_last_key(-20.0), "-60": no_last_key(-60.0),
         "no_last_values": no_last_values, "large_then_small": large_then(0.001), "large_then_none": large_then(0.0)}
SIZES = [(2, 128, 2, 2, 2, 64, 64), (1, 130, 1, 1, 4, 128, 64), (1, 120, 2, 1, 2, 100, 130), (2, 128, 1, 1, 1, 200, 72),
         (40, 100, 8, 8, 8, 40, 128)]


def make(seed, sizes, dtype, case):
    t = draw(seed, *sizes, dtype, init=False)
    CASES[case](t)
    return t


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("sizes", SIZES)
def test_state_keeps_what_is_left(ssdi8, sizes, case, dtype):  # noqa: F811
    t = make(sum(sizes), sizes, dtype, case)
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"])
    _, _, S, es = R.attention(*(t[n].double() for n in ("q", "k", "v")), t["g"], dtype=dtype)
    bound = R.rounded(F32, S, es).cpu() + LOST
    R.assert_within(out["final_state"], S.cpu(), bound, "final_state")
    state = torch.zeros_like(S, dtype=F32)
    for i in range(sizes[1]):
        ssdi8.linear_attention_step(*(t[n][:, i] for n in ("q", "k", "v")), state, t["g"][:, i])
    R.assert_within(state, S.cpu(), bound, "state behind the tokens")


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_state_of_a_long_prompt_keeps_what_is_left(ssdi8, dtype):  # noqa: F811
    """Cut into spans: their own states, too."""
    t = draw(5, 1, 2200, 2, 2, 2, 64, 64, dtype)
    sparse(t)
    t["g"][:, 700:720] = -20.0
    t["v"][:, 2100:] = 0
    t["g"][:, 2100:] = -0.5
    assert ssdi8.linear_attention_workspace_size(ssdi8.AttnDims(1, 2200, 2, 2, 2, 64, 64), dtype) > 0
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    _, _, S, es = R.attention(*(t[n].double() for n in ("q", "k", "v")), t["g"], None, t["init"], dtype=dtype)
    R.assert_within(out["final_state"], S.cpu(), R.rounded(F32, S, es).cpu() + LOST, "final_state")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("case", list(CASES))
@pytest.mark.parametrize("sizes", SIZES)
def test_outputs_of_terms_of_different_sizes(ssdi8, sizes, case, dtype):  # noqa: F811
    t = make(sum(sizes) + 1, sizes, dtype, case)
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"])
    y, e, _, _ = R.attention(*(t[n].double() for n in ("q", "k", "v")), t["g"], dtype=dtype)
    R.assert_within(out["y"], y.cpu(), R.rounded(dtype, y, e + floor(t, dtype)).cpu(), "y")
