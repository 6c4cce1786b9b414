"""Linear attention, blocks of few bits and products of them in 64 bits, with bounds on what the kernels' arithmetic
may add.  U = 2^-24 is half an ulp of fp32 (relative)."""
import torch

from block_ref import HALF_ULP, TINY, U, assert_within, rounded, silu, silu_bound, softplus  # noqa: F401

# Of a value that enters the matrix unit rounded to the type: half an ulp; as the sum of two of fp16 or three of bf16:
# what a rounding leaves of 1 is at most half an ulp h, whose own half ulp is h^2 / 2, and so on.
ONE = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SPLIT = {torch.float32: 0.0, torch.float16: 2.0 ** -23, torch.bfloat16: 2.0 ** -26}


def spread(t, dim, n):
    return t.repeat_interleave(n // t.shape[dim], dim)


def attention(q, k, v, g, scale=None, init=None, lengths=None, dtype=torch.float32):
    """y (b,L,H,V) and its bound before storing, the final state (b,Hv,K,V) and its bound; 64-bit inputs, any device.

    The quadratic form: y_i = scale (sum_{j<=i} exp(c_i - c_j) (q_i . k_j) v_j + exp(c_i) S0^T q_i).  What the
    kernel's arithmetic may add is counted against the same sums of magnitudes: K + 1 + (chunks + 1) * 2 fp32 sums
    and products on a way through the states, L more along the tokens; an exponential in base 2 of a difference
    that fp64 holds costs (|v| + 2) U, one for every chunk that a term passes (their |v| add up).  Of 16-bit
    types v with its decay enters as two or three of the type, for S: off by SPLIT; p, or S, as one, for y: off by ONE."""
    b, L, Hq, K = q.shape
    Hk, Hv, V = k.shape[2], v.shape[2], v.shape[3]
    H = max(Hq, Hv)
    scale = K ** -0.5 if scale is None else scale
    dev, f64 = q.device, torch.float64
    g = torch.zeros(b, L, Hv, dtype=f64, device=dev) if g is None else g.double().expand(b, L, Hv).clone()
    live = torch.ones(b, L, dtype=torch.bool, device=dev)
    if lengths is not None:
        live = torch.arange(L, device=dev) < lengths.to(dev)[:, None]
    g[~live] = 0
    q, k, v = (torch.where(live[..., None, None], t, torch.zeros((), dtype=f64, device=dev)) for t in (q, k, v))
    c = spread(g, 2, H).cumsum(1).transpose(1, 2)                     # b H L
    qh, vh = spread(q, 2, H).transpose(1, 2), spread(v, 2, H).transpose(1, 2)
    kv = spread(k, 2, Hv)
    kh = spread(kv, 2, H).transpose(1, 2)
    S0 = torch.zeros(b, Hv, K, V, dtype=f64, device=dev) if init is None else init.double()
    S0h = spread(S0, 1, H)
    chunks = -(-L // 32) + 1
    roundings = (K + L + 4 * chunks + 16) * U + SPLIT[dtype]
    of_y = roundings + ONE[dtype]
    diff = c[..., :, None] - c[..., None, :]
    past = torch.ones(L, L, dtype=torch.bool, device=dev).tril()
    W = torch.where(past, torch.exp(torch.where(past, diff, torch.zeros_like(diff))), torch.zeros_like(diff))
    extra = (diff.abs() + 2 * chunks + 2) * U
    y = (W * (qh @ kh.mT)) @ vh + torch.exp(c)[..., None] * (qh @ S0h)
    big = W * (qh.abs() @ kh.abs().mT)
    e = (big * (of_y + extra)) @ vh.abs()
    e = e + (torch.exp(c) * (of_y + (c.abs() + 2 * chunks + 2) * U))[..., None] * (qh.abs() @ S0h.abs())
    y, e = (scale * y).transpose(1, 2), (abs(scale) * e).transpose(1, 2)
    y[~live] = 0
    cv = g.cumsum(1).transpose(1, 2)                                  # b Hv L
    last = cv[..., -1] if L else torch.zeros(b, Hv, dtype=f64, device=dev)
    w = torch.exp(last[..., None] - cv)
    kt, vt = kv.transpose(1, 2), v.transpose(1, 2)
    S = (kt * w[..., None]).mT @ vt + torch.exp(last)[..., None, None] * S0
    es = (kt.abs() * (w * (roundings + ((last[..., None] - cv).abs() + 2 * chunks + 2) * U))[..., None]).mT @ vt.abs()
    es = es + (torch.exp(last) * (roundings + (last.abs() + 2 * chunks + 2) * U))[..., None, None] * S0.abs()
    return y, e, S, es


# ------------------------------------------------------------------------------ blocks
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
E4M3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
EMAX = {"mxfp8": 8, "mxfp4": 2}


def blocks(x):
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))


def nearest(m, table):
    """The index of the element nearest to m >= 0, ties to the even index, behind the last one the last."""
    hi = torch.searchsorted(table, m.contiguous()).clamp(max=len(table) - 1)
    lo = (hi - 1).clamp(min=0)
    a, b = m - table[lo], table[hi] - m
    return torch.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def quantize_mx(x, format):
    """Codes and scale bytes of x (64-bit values of at most 32 bits, CPU)."""
    v = blocks(x)
    big = v.abs().amax(-1)
    fine = torch.isfinite(v).all(-1)
    m, e = torch.frexp(torch.where(fine, big, torch.ones_like(big)))
    e = (torch.where(big > 0, e.long() - 1, torch.full_like(e.long(), -200)) - EMAX[format]).clamp(min=-127)
    q = torch.where(fine[..., None], v, torch.zeros_like(v)) * torch.exp2(-e.double())[..., None]
    code = nearest(q.abs(), E4M3 if format == "mxfp8" else E2M1)
    sign = torch.signbit(q) & fine[..., None]
    code = (code | (sign.long() << (7 if format == "mxfp8" else 3))).to(torch.uint8).flatten(-2)
    scales = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    if format == "mxfp4":
        code = code[..., 0::2] | (code[..., 1::2] << 4)
    return code, scales


def values(codes, scales, format):
    """The values that codes and scales stand for, in 64 bits (scales float8_e8m0fnu or their bytes)."""
    s = scales.view(torch.uint8).long()
    s = torch.where(s == 255, torch.full((), float("nan"), dtype=torch.float64, device=s.device),
                    torch.exp2(s.double() - 127))
    if format == "mxfp8":
        v = codes.view(torch.float8_e4m3fn).float().double()
    else:
        c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
        v = E2M1.to(c.device)[c & 7] * (1 - 2 * (c >> 3))
    return v * s.repeat_interleave(32, -1)


def half_step(y, s, format):
    """How far the nearest element may be from y under scale s: half the distance of the neighbours at |y| / s, above
    the largest element the distance to that."""
    m = y.abs() / s
    if format == "mxfp8":
        step = torch.exp2(torch.floor(torch.log2(m.clamp(min=2.0 ** -6))) - 3)
        top = 448.0
    else:
        step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0)).double()
        top = 6.0
    return torch.where(m > top, m - top, step / 2) * s


def linear_mx(xv, wv, xs, ws, x_format, bias=None, act=None, residual=None):
    """y and its bound before storing of values xv (..., K), wv (O, K) in 64 bits.

    Products of e2m1 elements are added up exactly within an instruction.  With e4m3 elements the unit adds them up in
    groups of eight neighbours, whose terms it cuts to a whole multiple of 2^-13 of the power of two below the largest
    (256 + 1.875 2^-3 - 256 gives 1.75 2^-3 where the three are in one group of eight, all of it where they are
    not): the seven others are off by less than 2^-13 of the largest each.  Between instructions fp32 sums, of eight
    waves' parts at most."""
    y = xv @ wv.T
    size = xv.abs() @ wv.abs().T
    e = (xv.shape[-1] // 64 + 10) * U * size
    if x_format == "mxfp8":
        big = lambda v: torch.nn.functional.pad(v.abs(), (0, -v.shape[-1] % 8)).unflatten(-1, (-1, 8)).amax(-1)
        e = e + 7 * 2.0 ** -13 * (big(xv) @ big(wv).T)   # no group's largest is above the product of these
    if bias is not None:
        y = y + bias.double()
        e = e + U * y.abs()
    if act == "silu":
        y, e = silu(y), silu_bound(y, e)
    elif act == "gelu":
        v = y
        y = 0.5 * v * torch.erfc(-v * 0.5 ** 0.5)
        e = 1.2 * e + (1.5 * v * v + 28) * U * y.abs()
    elif act == "softplus":
        y = softplus(y)
        e = e + (2 * y.abs() + 8) * U * (y.abs() + 1)
    if residual is not None:
        y = y + residual.double()
        e = e + U * y.abs()
    return y, e


def norm(x, w, z, residual, eps, groups, before):
    """The norm of rows in 64 bits, its bound before storing, and the sum with the residual."""
    s = x if residual is None else x + residual
    es = torch.zeros_like(s) if residual is None else U * s.abs()
    gate, eg = torch.ones_like(s), torch.zeros_like(s)
    if z is not None:
        gate = silu(z)
        eg = (2 * z.abs() + 8) * U * gate.abs()
    v, ev = (s, es) if before else (s * gate, es * gate.abs() + (eg + U * gate.abs()) * s.abs())
    D = s.shape[-1]
    rows, er = v.unflatten(-1, (groups, -1)), ev.unflatten(-1, (groups, -1))
    W = D // groups
    mean = rows.pow(2).mean(-1, keepdim=True)
    root = torch.sqrt(mean + eps)
    # of the mean: every value's own error, twice, and W roundings of the sum; half of that of its root
    off = ((2 * rows.abs() * er).mean(-1, keepdim=True) + (W + 4) * U * mean) / (2 * (mean + eps)) + 6 * U
    y = (rows / root).flatten(-2) * w
    ey = ((er + rows.abs() * (off + 2 * U)) / root).flatten(-2) * w.abs() + 2 * U * y.abs()
    if before:
        ey = ey * gate.abs() + y.abs() * (eg + U * gate.abs())
        y = y * gate
    return y, ey, s
