"""Calls of more workgroups than one launch has threads for (2^32): the results are those of calls on parts, at both ends and
on either side of every launch's border."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


def parts(n, border):
    """Some rows at each end and around each multiple of border."""
    at = [0, *range(border, n, border), n]
    return [slice(max(0, a - 70), min(n, a + 70)) for a in at]


def normal(*shape):
    return torch.randn(*shape, device="cuda", dtype=F16)


def test_attention_step(ssdi8):
    n = 2 ** 24 + 5
    q, k, v = normal(n, 1, 1), normal(n, 1, 1), normal(n, 1, 1)
    g, state = -torch.rand(n, 1, device="cuda"), torch.randn(n, 1, 1, 1, device="cuda")
    want = [state[s].clone() for s in parts(n, 2 ** 23)]
    y = ssdi8.linear_attention_step(q, k, v, state, g)
    for s, w in zip(parts(n, 2 ** 23), want):
        assert torch.equal(ssdi8.linear_attention_step(q[s], k[s], v[s], w, g[s]), y[s])
        assert torch.equal(state[s], w)


def test_attention(ssdi8):
    n = 2 ** 24 + 5
    q, k, v = normal(n, 1, 1, 1), normal(n, 1, 1, 1), normal(n, 1, 1, 1)
    out = ssdi8.linear_attention(q, k, v)
    for s in parts(n, 2 ** 23):
        part = ssdi8.linear_attention(q[s], k[s], v[s])
        assert torch.equal(part["y"], out["y"][s]) and torch.equal(part["final_state"], out["final_state"][s])


# rows of a workgroup: one where the values go through LDS, sixteen of eight values each
@pytest.mark.parametrize("n,D,border", [(2 ** 26 + 5, 1, 2 ** 25), (2 ** 28 + 37, 8, 2 ** 27)])
def test_norm_quantize(ssdi8, n, D, border):
    x, w = torch.empty(n, D, device="cuda", dtype=F16).normal_(), torch.full((D,), 2.0, device="cuda")
    out = ssdi8.norm_quantize(x, w)
    for s in parts(n, border):
        part = ssdi8.norm_quantize(x[s], w)
        assert torch.equal(part["codes"], out["codes"][s]) and torch.equal(part["scales"], out["scales"][s])


def test_linear_mx(ssdi8):
    n = 2 ** 27 + 53
    codes = torch.randint(0, 256, (n, 16), device="cuda", dtype=torch.uint8)
    scales = torch.randint(120, 131, (n, 1), device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)
    X = ssdi8.quantize_mx(normal(1, 32), "mxfp8")
    y = ssdi8.linear_mx(X, ssdi8.Mx(codes, scales))
    for s in parts(n, 2 ** 26):
        assert torch.equal(ssdi8.linear_mx(X, ssdi8.Mx(codes[s], scales[s])), y[:, s])
