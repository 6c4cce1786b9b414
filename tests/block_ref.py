"""The operators around the SSD layer in 64 bits, term by term, with bounds on what fp32 arithmetic and the
rounding of the results may add.  u = 2^-24 is half an ulp of fp32 (relative).

The bounds count roundings.  An exponential of v in base 2 costs the rounding of v log2(e), |v| u
relative in the result for each of the two (constant and product), and one ulp of the instruction, 2 u: the
factor (2 |v| + 2) u.  silu = v / (1 + exp(-v)): the exponential's part, a sum, a reciprocal of one ulp and a
product; softplus: exponential, logarithm and reciprocal of one ulp each, three products and sums.
"""
import torch

U = 2.0 ** -24
HALF_ULP = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}


def silu(v):
    return v * torch.sigmoid(v)


def silu_bound(v, e):
    """Of silu(v + an error of at most e): the slope is at most 1.1; 2 |v| + 8 roundings."""
    return 1.1 * e + (2 * v.abs() + 8) * U * silu(v).abs()


def softplus(v):
    return torch.where(v > 20, v, torch.log1p(torch.exp(v.clamp(max=20.0))))


def rounded(dtype, v, e):
    """The bound of a value with error e once it is stored."""
    return e + HALF_ULP[dtype] * (v.abs() + e) + TINY[dtype]


def assert_within(got, want, bound, what=""):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= bound) & ~(got == want)
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond their bound, first at {i}: "
                             f"{got[i].item()!r} for {want[i].item()!r} +- {bound[i].item():.3g}")


def conv(x, w, bias, act, init, lengths):
    """y, its bound before storing, and the final state; x (B,L,D) and init in 64 bits."""
    B, L, D = x.shape
    W = w.shape[1]
    w = w.double()
    line = torch.zeros(B, L + W - 1, D, dtype=torch.float64)
    line[:, W - 1:] = x
    if init is not None:
        line[:, :W - 1] = init
    y = torch.zeros(B, L, D, dtype=torch.float64) + (0 if bias is None else bias.double())
    size = y.abs()
    for j in range(W):
        y = y + line[:, j:j + L] * w[:, j]
        size = size + (line[:, j:j + L] * w[:, j]).abs()
    e = (W + 1) * U * size
    if act:
        y, e = silu(y), silu_bound(y, e)
    last = torch.zeros(B, W - 1, D, dtype=torch.float64)
    for b in range(B):
        n = L if lengths is None else min(max(int(lengths[b]), 0), L)
        y[b, n:], e[b, n:] = 0, 0
        last[b] = line[b, n:n + W - 1]
    return y, e, last


def scan(u, dt, A, Bm, Cm, D, z, dt_bias, softplus_on, init, lengths):
    """y and its bound before storing, final state and its bound; inputs in 64 bits."""
    B, L, ch = u.shape
    H, (G, N) = dt.shape[2], Bm.shape[2:]
    per = ch // H
    Bm, Cm = (t.repeat_interleave(ch // G, 2) for t in (Bm, Cm))               # (B, L, ch, N)
    delta = dt + (0 if dt_bias is None else dt_bias)
    # of delta: the sum's rounding moves softplus by at most as much, then 2 |v| + 10 roundings
    de = U * delta.abs()
    if softplus_on:
        d0 = delta
        delta = softplus(d0)
        de = de * torch.sigmoid(d0) + (2 * d0.abs() + 10) * U * delta.abs()
    delta, de = (t.repeat_interleave(per, 2) for t in (delta, de))
    A = A.repeat_interleave(per, 0)[:, None].expand(ch, N) if A.dim() == 1 else A
    Dh = (torch.zeros(H, dtype=torch.float64) if D is None else D).repeat_interleave(per, 0)
    h = torch.zeros(B, ch, N, dtype=torch.float64) if init is None else init.clone()
    E = torch.zeros_like(h)
    y, ye = torch.zeros(B, L, ch, dtype=torch.float64), torch.zeros(B, L, ch, dtype=torch.float64)
    n = torch.full((B,), L) if lengths is None else lengths.clamp(0, L)
    for t in range(L):
        live = (t < n)[:, None, None]
        d, e = delta[:, t, :, None], de[:, t, :, None]
        a = torch.exp(d * A)
        ae = a * ((d * A).abs() * 4 * U + e * A.abs() + 2 * U)
        add = d * u[:, t, :, None] * Bm[:, t]
        adde = add.abs() * 2 * U + e * (u[:, t, :, None] * Bm[:, t]).abs()
        new = a * h + add
        newE = a * E + ae * (h.abs() + E) + adde + U * new.abs()
        h, E = torch.where(live, new, h), torch.where(live, newE, E)
        size = (new * Cm[:, t]).abs().sum(-1) + (Dh * u[:, t]).abs()
        v = (new * Cm[:, t]).sum(-1) + Dh * u[:, t]
        ve = (newE * Cm[:, t].abs()).sum(-1) + (N + 2) * U * size
        if z is not None:
            g = silu(z[:, t])
            v, ve = v * g, ve * g.abs() + (2 * z[:, t].abs() + 10) * U * (v * g).abs()
        y[:, t], ye[:, t] = torch.where(live[..., 0], v, 0.0), torch.where(live[..., 0], ve, 0.0)
    return y, ye, h, E


def norm(x, w, z, residual, eps, groups, before):
    """y and its bound before storing, and the sum; rows in 64 bits."""
    s = x if residual is None else x + residual
    e = U * s.abs() if residual is not None else torch.zeros_like(s)
    g = torch.ones_like(s) if z is None else silu(z)
    ge = torch.zeros_like(s) if z is None else (2 * z.abs() + 8) * U * g.abs()
    v, ve = s, e
    if not before and z is not None:
        v, ve = s * g, e * g.abs() + ge * s.abs() + U * (s * g).abs()
    M, D = s.shape
    rows = v.reshape(M, groups, D // groups)
    ms = rows.pow(2).mean(-1, keepdim=True)
    scale = 1 / torch.sqrt(ms + eps)
    # the mean square's relative error: twice the values' (through their absolute sum), its additions'
    # (per lane, then a tree: at most width / 64 + 10), then square root, reciprocal, products
    rel = 2 * (ve.reshape(rows.shape) * rows.abs()).mean(-1, keepdim=True) / (ms + eps + 1e-300)
    rel = 0.5 * (rel + (D // groups / 64 + 12) * U) + 3 * U
    y = (rows * scale).reshape(M, D) * w
    ye = ve * (scale.expand_as(rows).reshape(M, D) * w).abs() + (rel.expand_as(rows).reshape(M, D) + 3 * U) * y.abs()
    if before and z is not None:
        y, ye = y * g, ye * g.abs() + ge * y.abs() + U * (y * g).abs()
    return y, ye, s


def linear(x, w, bias, act, residual, xs, ws):
    """y and its bound before storing; x, w in 64 bits, xs and ws the steps of int8 codes or None."""
    y = x @ w.t()
    # fp32 sums of exact products: as many roundings as terms, of the absolute sum; int32 sums are exact
    e = x.shape[1] * U * (x.abs() @ w.abs().t()) if xs is None else U * y.abs()
    if xs is not None:
        s = xs.double()[:, None] * ws.double()
        y, e = y * s, e * s.abs() + 2 * U * (y * s).abs()
    if bias is not None:
        y = y + bias.double()
        e = e + U * y.abs()
    if act == "silu":
        y, e = silu(y), silu_bound(y, e)
    elif act == "gelu":
        # slope at most 1.13; erf within 4 ulp, 1 + erf may cancel: 8 u of |y|
        g = 0.5 * y * torch.erfc(-y / 2 ** 0.5)
        y, e = g, 1.13 * e + 8 * U * y.abs()
    elif act == "softplus":
        g = softplus(y)
        y, e = g, e + (2 * y.abs() + 10) * U * g
    if residual is not None:
        y = y + residual
        e = e + U * y.abs()
    return y, e
