"""Calls of more workgroups than one launch has threads for (2^32): the results are those of calls on halves, which one launch
could hold, and of a call on a few."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F16 = torch.float16


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


def parts(n):
    return slice(0, n // 2), slice(n // 2, n), slice(n - 70, n)


def normal(*shape):
    return torch.randn(*shape, device="cuda", dtype=F16)


def test_attention_step(ssdi8):
    n = 2 ** 24 + 5
    q, k, v = normal(n, 1, 1), normal(n, 1, 1), normal(n, 1, 1)
    g, state = -torch.rand(n, 1, device="cuda"), torch.randn(n, 1, 1, 1, device="cuda")
    want = [state[s].clone() for s in parts(n)]
    y = ssdi8.linear_attention_step(q, k, v, state, g)
    for s, w in zip(parts(n), want):
        assert torch.equal(ssdi8.linear_attention_step(q[s], k[s], v[s], w, g[s]), y[s])
        assert torch.equal(state[s], w)


def test_attention(ssdi8):
    n = 2 ** 24 + 5
    q, k, v = normal(n, 1, 1, 1), normal(n, 1, 1, 1), normal(n, 1, 1, 1)
    out = ssdi8.linear_attention(q, k, v)
    for s in parts(n):
        part = ssdi8.linear_attention(q[s], k[s], v[s])
        assert torch.equal(part["y"], out["y"][s]) and torch.equal(part["final_state"], out["final_state"][s])


# rows of a workgroup: one where the values go through LDS, sixteen of eight values each
@pytest.mark.parametrize("n,D", [(2 ** 26 + 5, 1), (2 ** 28 + 37, 8)])
def test_norm_quantize(ssdi8, n, D):
    x, w = torch.empty(n, D, device="cuda", dtype=F16).normal_(), torch.full((D,), 2.0, device="cuda")
    out = ssdi8.norm_quantize(x, w)
    for s in parts(n):
        part = ssdi8.norm_quantize(x[s], w)
        assert torch.equal(part["codes"], out["codes"][s]) and torch.equal(part["scales"], out["scales"][s])


def test_linear_mx(ssdi8):
    n = 2 ** 27 + 53
    codes = torch.randint(0, 256, (n, 16), device="cuda", dtype=torch.uint8)
    scales = torch.randint(120, 131, (n, 1), device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)
    X = ssdi8.quantize_mx(normal(1, 32), "mxfp8")
    y = ssdi8.linear_mx(X, ssdi8.Mx(codes, scales))
    for s in parts(n):
        assert torch.equal(ssdi8.linear_mx(X, ssdi8.Mx(codes[s], scales[s])), y[:, s])


def test_conv(ssdi8):
    n = 2 ** 24 + 5
    x, w, init = normal(n, 1, 8), torch.randn(8, 4, device="cuda"), normal(n, 3, 8)
    out = ssdi8.causal_conv(x, w, init_state=init)
    for s in parts(n):
        part = ssdi8.causal_conv(x[s].clone(), w, init_state=init[s].clone())
        assert torch.equal(part["y"], out["y"][s]) and torch.equal(part["final_state"], out["final_state"][s])


def test_conv_step(ssdi8):
    n = 2 ** 26 + 5
    x, w, state = normal(n, 8), torch.randn(8, 2, device="cuda"), normal(n, 1, 8)
    want = [state[s].clone() for s in parts(n)]
    y = ssdi8.causal_conv_step(x, w, state, split=(3, 5))
    for s, st in zip(parts(n), want):
        a, b = ssdi8.causal_conv_step(x[s].clone(), w, st, split=(3, 5))
        assert torch.equal(a, y[0][s]) and torch.equal(b, y[1][s]) and torch.equal(state[s], st)


def scan_inputs(n, *tokens):
    u, B, C, z = normal(n, *tokens, 1), normal(n, *tokens, 1, 1), normal(n, *tokens, 1, 1), normal(n, *tokens, 1)
    return u, normal(n, *tokens, 1), B, C, z, torch.full((1, 1), -1.0, device="cuda"), torch.randn(n, 1, 1, device="cuda")


def test_selective_scan(ssdi8):
    n = 2 ** 24 + 5
    u, dt, B, C, z, A, init = scan_inputs(n, 1)
    out = ssdi8.selective_scan(u, dt, A, B, C, z=z, init_state=init)
    for s in parts(n):
        part = ssdi8.selective_scan(*(t[s].clone() for t in (u, dt)), A, *(t[s].clone() for t in (B, C)), z=z[s].clone(),
                                    init_state=init[s].clone())
        assert torch.equal(part["y"], out["y"][s]) and torch.equal(part["final_state"], out["final_state"][s])


def test_selective_scan_step(ssdi8):
    n = 2 ** 24 + 5
    u, dt, B, C, z, A, state = scan_inputs(n)
    want = [state[s].clone() for s in parts(n)]
    y = ssdi8.selective_scan_step(u, dt, A, B, C, state, z=z)
    for s, st in zip(parts(n), want):
        got = ssdi8.selective_scan_step(*(t[s].clone() for t in (u, dt)), A, *(t[s].clone() for t in (B, C)), st, z=z[s].clone())
        assert torch.equal(got, y[s]) and torch.equal(state[s], st)


def test_selective_scan_step_of_many_channels(ssdi8):
    """A batch element of 2^26 threads: fewer than 64 of them are a launch's."""
    n, D, N = 67, 2 ** 20, 129
    u, z, dt, B, C = normal(n, D), normal(n, D), normal(n, 1), normal(n, 1, N), normal(n, 1, N)
    A, state = torch.full((1,), -1.0, device="cuda"), torch.empty(n, D, N, device="cuda").uniform_()
    some = slice(n - 3, n)
    want = state[some].clone()
    y = ssdi8.selective_scan_step(u, dt, A, B, C, state, z=z)
    assert torch.equal(ssdi8.selective_scan_step(*(t[some].clone() for t in (u, dt)), A, *(t[some].clone() for t in (B, C)), want,
                                                 z=z[some].clone()), y[some])
    assert torch.equal(state[some], want)


def test_gated_norm(ssdi8):
    n, D = 2 ** 28 + 37, 8
    x, w = torch.empty(n, D, device="cuda", dtype=F16).normal_(), torch.full((D,), 2.0, device="cuda")
    y = ssdi8.gated_norm(x, w)["y"]
    for s in parts(n):
        assert torch.equal(ssdi8.gated_norm(x[s].clone(), w)["y"], y[s])


@pytest.mark.parametrize("m,n,k", [(3, 2 ** 27 + 53, 8), (2 ** 30 + 77, 1, 1)])
def test_linear(ssdi8, m, n, k):
    x, w, bias = normal(m, k), normal(n, k), torch.randn(n, device="cuda")
    y = ssdi8.linear(x, w, bias=bias)
    for s in parts(n) if n > m else parts(m):
        got = ssdi8.linear(x, w[s].clone(), bias=bias[s].clone()) if n > m else ssdi8.linear(x[s].clone(), w, bias=bias)
        assert torch.equal(got, y[:, s] if n > m else y[s])


def test_quantize_act(ssdi8):
    n = 2 ** 26 + 5
    x = normal(1, n, 1, 8)
    codes, steps = ssdi8.quantize_act(x, "token")
    for s in parts(n):
        part = ssdi8.quantize_act(x[:, s].clone(), "token")
        assert torch.equal(part[0], codes[:, s]) and torch.equal(part[1], steps[s])
