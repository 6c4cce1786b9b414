"""Values in few bits: the quantizing norm, the microscaled formats and the products with 4-bit weights, against 64-bit
forms and, where the arithmetic is exact, code by code (mixer_ref.py)."""
import pytest
import torch

import mixer_ref as R

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


def gen(seed):
    return torch.Generator().manual_seed(seed)


def cut(t, before, after=3):
    """t on the device as columns of wider rows whose other columns are NaN."""
    wide = torch.full((*t.shape[:-1], before + t.shape[-1] + after), float("nan")).to(t.dtype).cuda()
    wide[..., before:before + t.shape[-1]] = t.cuda()
    return wide[..., before:before + t.shape[-1]]


def bytes_of(t):
    return t.view(torch.uint8).cpu()


# ------------------------------------------------------------------------------ blocks
@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M,K,before", [(1, 1, 0), (3, 31, 1), (2, 32, 0), (5, 33, 7), (64, 2560, 0), (7, 1000, 5), (300, 96, 3)])
def test_quantize_mx(ssdi8, M, K, before, dtype, format):
    g = gen(M + K)
    x = torch.randn(M, K, generator=g) * torch.exp2(torch.randint(-6, 7, (M, 1), generator=g).float())
    x = x.to(dtype)
    got = ssdi8.quantize_mx(cut(x, before), format)
    codes, scales = R.quantize_mx(x.double(), format)
    assert torch.equal(bytes_of(got.codes), codes) and torch.equal(bytes_of(got.scales), scales)
    assert got.codes.dtype == (torch.uint8 if format == "mxfp4" else torch.float8_e4m3fn)
    assert got.scales.dtype == torch.float8_e8m0fnu


@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_quantize_mx_at_the_borders(ssdi8, dtype, format):
    """Every tie and its neighbours, zeros, the smallest and largest values, values that are no numbers."""
    table = R.E4M3 if format == "mxfp8" else R.E2M1
    top = float(table[-1])
    mid = (table[1:] + table[:-1]) / 2
    rows = []
    for v in (table, mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -8)):
        for s in (1.0, 2.0 ** -5, -(2.0 ** 4)):
            for part in v.split(31):
                rows.append(torch.cat([torch.tensor([top * s]), part * s, torch.zeros(31 - len(part))]))
    tiny, huge = torch.finfo(dtype).tiny, torch.finfo(dtype).max
    sub = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    for first in (0.0, tiny, sub, huge, -huge, float("inf"), float("-inf"), float("nan"), 1.9999, 7.99, 511.0):
        rows.append(torch.cat([torch.tensor([first, -0.0]), torch.zeros(30)]).double())
    x = torch.stack([r.double() for r in rows]).to(dtype)
    got = ssdi8.quantize_mx(x.cuda(), format)
    codes, scales = R.quantize_mx(x.double(), format)
    assert torch.equal(bytes_of(got.scales), scales)
    fine = (scales != 255)[:, 0]
    assert torch.equal(bytes_of(got.codes)[fine], codes[fine])
    assert (bytes_of(got.codes)[~fine] == 0).all() and (~fine).sum() == 3


def test_quantize_mx_rows(ssdi8):
    x = torch.randn(2, 3, 5, 40, device="cuda").half()
    a, b = ssdi8.quantize_mx(x), ssdi8.quantize_mx(x.view(30, 40))
    assert a.codes.shape == (2, 3, 5, 32) and a.scales.shape == (2, 3, 5, 2)
    assert torch.equal(a.codes.view(30, 32), b.codes)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = ssdi8.quantize_mx(x, "mxfp4", stream=side)
    side.synchronize()
    assert torch.equal(a.codes, c.codes) and torch.equal(bytes_of(a.scales), bytes_of(c.scales))
    none = ssdi8.quantize_mx(x[:, :0])
    assert none.codes.shape == (2, 0, 5, 32) and none.scales.shape == (2, 0, 5, 2)
    for bad in (lambda: ssdi8.quantize_mx(x, "int8"), lambda: ssdi8.quantize_mx(x.cpu()),
                lambda: ssdi8.quantize_mx(x.transpose(-1, -2)), lambda: ssdi8.quantize_mx(x.int()),
                lambda: ssdi8.quantize_mx(x[:, :, ::2, :].transpose(0, 1))):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------------------ the norm
NORM = [  # M, D, groups, gate, residual, before, columns before x, columns before z
    (1, 1, 1, False, False, False, 0, 0), (8, 768, 1, False, True, False, 0, 0), (3, 31, 1, True, False, False, 1, 2),
    (5, 33, 1, True, True, True, 3, 0), (4, 648, 8, True, False, False, 0, 5), (4, 640, 8, True, True, False, 0, 0),
    (2, 1025, 1, True, False, False, 0, 9), (9, 2560, 1, False, True, False, 0, 0), (3, 5120, 8, True, False, True, 0, 7),
    (2, 8192, 1, True, True, False, 0, 0), (2, 8200, 1, True, True, False, 0, 0), (2, 8193, 1, False, False, False, 1, 0),
    (2, 10000, 4, True, False, True, 0, 0), (1, 32768, 1, True, True, False, 0, 0), (2, 12, 12, False, False, False, 0, 0),
    (2, 20001, 3, True, True, False, 0, 0), (20000, 64, 1, True, False, False, 0, 0),
]


@pytest.mark.parametrize("format", ["int8", "mxfp8", "mxfp4"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("M,D,groups,gate,residual,before,px,pz", NORM)
def test_norm_quantize(ssdi8, M, D, groups, gate, residual, before, px, pz, dtype, format):
    g = gen(M + D)
    n = lambda: torch.randn(M, D, generator=g).to(dtype)
    x, z, r = n(), n() if gate else None, n() if residual else None
    w = 1 + 0.2 * torch.randn(D, generator=g)
    d64 = lambda t: None if t is None else t.double().cuda()
    y, e, s = R.norm(d64(x), w.double().cuda(), d64(z), d64(r), 1e-5, groups, before)
    out = ssdi8.norm_quantize(cut(x, px), w.cuda(), z=None if z is None else cut(z, pz),
                              residual=None if r is None else r.cuda(), groups=groups, norm_before_gate=before,
                              format=format, with_y=True)
    assert set(out) == {"codes", "scales", "y"} | ({"residual"} if residual else set())
    R.assert_within(out["y"], y.cpu(), R.rounded(dtype, y, e).cpu(), "y")
    if residual:
        assert torch.equal(out["residual"].cpu(), (x.float() + r.float()).to(dtype))
    if format == "int8":
        steps = out["scales"].double()[:, None]
        want = y.abs().amax(-1, keepdim=True) / 127
        off = e.amax(-1, keepdim=True) / 127 + 2 * R.U * want
        assert ((steps - torch.where(want == 0, 1.0, want)).abs() <= off).all()
        got = out["codes"].double() * steps
        # half a step, and what the inverse of the step and the product with it are off by: 127 steps of 3 U
        bound = e + steps * (0.5 + 127 * 4 * R.U)
    else:
        assert out["codes"].shape[-1] == -(-D // 32) * (32 if format == "mxfp8" else 16)
        scales = out["scales"].float().double().repeat_interleave(32, -1)[:, :D]
        big = R.blocks(y.abs()).amax(-1)
        slack = R.blocks(e).amax(-1)
        step = lambda v: torch.exp2(torch.floor(torch.log2(v)) - R.EMAX[format]).clamp(min=2.0 ** -127)
        s64 = out["scales"].float().double()
        assert ((s64 == step(big - slack)) | (s64 == step(big + slack)) | (big <= slack)).all()
        got = R.values(out["codes"], out["scales"], format)
        assert (got[:, D:] == 0).all()
        got = got[:, :D]
        # a value beside a border may go either way, off by as much as it is from the border
        bound = R.half_step(y.abs() + e, scales, format) + 2 * e
    R.assert_within(got, y.cpu(), bound.cpu(), "values")


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_norm_quantize_is_gated_norm_and_a_quantizer(ssdi8, dtype):
    """The codes are those of the unrounded y; in fp32, where y is not rounded, those of the written one."""
    g = gen(3)
    x = torch.randn(37, 1000, generator=g).to(dtype).cuda()
    z = torch.randn(37, 1000, generator=g).to(dtype).cuda()
    w = (1 + 0.1 * torch.randn(1000, generator=g)).cuda()
    for format in ("mxfp8", "mxfp4"):
        out = ssdi8.norm_quantize(x, w, z=z, format=format, with_y=True)
        if dtype == F32:
            again = ssdi8.quantize_mx(out["y"], format)
            assert torch.equal(bytes_of(again.codes), bytes_of(out["codes"]))
            assert torch.equal(bytes_of(again.scales), bytes_of(out["scales"]))
    # rows shaped as a batch, in place of the residual, on a stream, and without y
    r = torch.randn(37, 1000, generator=g).to(dtype).cuda()
    a = ssdi8.norm_quantize(x, w, residual=r, format="int8")
    side = torch.cuda.Stream()
    r2 = r.clone()
    side.wait_stream(torch.cuda.current_stream())
    b = ssdi8.norm_quantize(x.view(1, 37, 1000), w, residual=r2.view(1, 37, 1000), residual_out=r2.view(1, 37, 1000),
                            format="int8", stream=side)
    side.synchronize()
    assert torch.equal(a["codes"], b["codes"][0]) and torch.equal(a["scales"], b["scales"][0])
    assert torch.equal(a["residual"], r2) and "y" not in a
    c = ssdi8.norm_quantize(x[:0], w, residual=r[:0], format="mxfp4", with_y=True)
    assert c["codes"].shape == (0, 512) and c["scales"].shape == (0, 32) and c["y"].shape == (0, 1000)


@pytest.mark.parametrize("D", [512, 2000, 9000])
def test_norm_quantize_of_what_is_no_number(ssdi8, D):
    """An infinity or a NaN takes its row's norm, and with it every scale of the row, and no other row's; a row of
    zeros gives zeros."""
    x = torch.randn(6, D).half()
    x[1, 3], x[2, D - 1], x[4] = float("nan"), float("inf"), 0.0
    w = torch.ones(D).cuda()
    for format in ("int8", "mxfp8", "mxfp4"):
        out = ssdi8.norm_quantize(x.cuda(), w, format=format)
        scales = out["scales"].float().cpu().view(6, -1)
        codes = bytes_of(out["codes"]).view(6, -1)
        assert torch.isnan(scales[1]).all() and (codes[[1, 4]] == 0).all()
        assert torch.isfinite(scales[[0, 3, 4, 5]]).all()
        assert torch.isnan(scales[2]).any()       # the infinity's own block; the others are 0
        assert (scales[4] == (1.0 if format == "int8" else 2.0 ** -127)).all()


def test_norm_quantize_refusals(ssdi8):
    x, w = torch.randn(4, 64).half().cuda(), torch.ones(64).cuda()
    for bad in (dict(format="fp8"), dict(z=x.float()), dict(z=x[:2]), dict(residual=x[:, :32]), dict(residual_out=x),
                dict(residual=x.float())):
        with pytest.raises((ValueError, ssdi8.SSDi8Error)):
            ssdi8.norm_quantize(x, w, **bad)
    for xx, ww in ((x.cpu(), w), (x, w.half()), (x, w[:32]), (x.int(), w), (x.t(), torch.ones(4).cuda())):
        with pytest.raises(ValueError):
            ssdi8.norm_quantize(xx, ww)
    for bad in (dict(groups=3), dict(groups=0), dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(ssdi8.SSDi8Error):
            ssdi8.norm_quantize(x, w, **bad)
    with pytest.raises(ssdi8.SSDi8Error):
        ssdi8.norm_quantize(torch.zeros(1, 32769).cuda(), torch.zeros(32769).cuda())


# ------------------------------------------------------------------------------ products
def operand(g, M, K, format):
    """Random codes (every one of them but e4m3's NaN) and scales of a few powers of two."""
    blocks = -(-K // 32)
    scales = torch.randint(120, 131, (M, blocks), generator=g).to(torch.uint8)
    codes = torch.randint(0, 256, (M, blocks * (32 if format == "mxfp8" else 16)), generator=g).to(torch.uint8)
    if format == "mxfp8":
        codes[(codes & 127) == 127] = 0
        codes = codes.view(torch.float8_e4m3fn)
    return codes.cuda(), scales.cuda().view(torch.float8_e8m0fnu)


LINEAR = [  # M, O, K, act, bias, residual, y
    (1, 1, 32, None, False, False, F32), (8, 200, 256, None, True, True, F16), (16, 33, 288, "silu", True, False, F32),
    (17, 64, 1024, "gelu", False, True, BF16), (32, 50, 2560, None, False, False, F32), (33, 65, 512, None, True, True, F32),
    (64, 128, 96, "softplus", True, False, F16), (65, 130, 1056, None, False, False, F32), (300, 257, 768, "silu", True, True, F16),
    (2100, 2100, 320, None, True, True, F32), (4096, 512, 1536, None, False, True, BF16), (129, 8, 64, None, False, False, F32),
    (2, 4100, 8192, None, False, False, F32),
]


@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("M,O,K,act,bias,residual,ydt", LINEAR)
def test_linear_mx(ssdi8, M, O, K, act, bias, residual, ydt, format):
    g = gen(M + O + K)
    x, w = operand(g, M, K, format), operand(g, O, K, "mxfp4")
    shift = -7   # products of about 1
    b = torch.randn(O, generator=g).cuda() if bias else None
    r = cut(torch.randn(M, O, generator=g).to(ydt), 4) if residual else None
    down = torch.clamp(w[1].view(torch.uint8).int() + shift, 0).to(torch.uint8).view(torch.float8_e8m0fnu)
    w = (w[0], down)
    xv, wv = R.values(*x, format), R.values(*w, "mxfp4")
    y, e = R.linear_mx(xv, wv, x[1], w[1], format, b, act, r)
    got = ssdi8.linear_mx(ssdi8.Mx(*x), ssdi8.Mx(*w), bias=b, activation=act, residual=r, y_dtype=ydt)
    assert got.dtype == ydt
    R.assert_within(got, y.cpu(), R.rounded(ydt, y, e).cpu(), "y")


@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("M", [3, 100])
def test_linear_mx_is_a_sum_of_integers(ssdi8, M, format):
    """Small whole numbers: every product and sum is one, so that each lane's place shows."""
    g = gen(M)
    K, O = 1312, 300
    w = torch.randint(-3, 4, (O, K), generator=g).float()
    x = torch.randint(-3, 4, (M, K), generator=g).float()
    w[:, ::32], x[:, ::32] = 4.0, 4.0   # every block's scale is 1 (e2m1); e4m3: 2^-6, codes times 64
    W, X = ssdi8.quantize_mx(w.cuda()), ssdi8.quantize_mx(x.cuda(), format)
    got = ssdi8.linear_mx(X, W, y_dtype=F32)
    assert torch.equal(got.cpu().double(), x.double() @ w.double().T)


# Sizes that take the large tiles, each with a last tile and a last k-tile that are cut.
@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("M,O,K,act,bias,residual,ydt", [(2107, 2011, 992, "gelu", True, True, F16),
                                                         (2107, 2011, 4128, None, False, False, F32),
                                                         (4001, 1100, 32, "silu", True, False, BF16)])
def test_linear_mx_large(ssdi8, M, O, K, act, bias, residual, ydt, format):
    test_linear_mx(ssdi8, M, O, K, act, bias, residual, ydt, format)


@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("K", [1312, 4192])
def test_linear_mx_large_is_a_sum_of_integers(ssdi8, K, format):
    g = gen(K)
    w = torch.randint(-3, 4, (2050, K), generator=g).float()
    x = torch.randint(-3, 4, (2080, K), generator=g).float()
    w[:, ::32], x[:, ::32] = 4.0, 4.0
    W, X = ssdi8.quantize_mx(w.cuda()), ssdi8.quantize_mx(x.cuda(), format)
    assert torch.equal(ssdi8.linear_mx(X, W, y_dtype=F32).double(), x.cuda().double() @ w.cuda().double().T)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("format", ["mxfp8", "mxfp4"])
@pytest.mark.parametrize("M,K", [(5, 1000), (90, 512)])
def test_linear_mx_of_a_tensor(ssdi8, M, K, dtype, format):
    """x that is no Mx is quantized first: the same bits as in two calls; K filled up to whole blocks."""
    x = torch.randn(M, K).to(dtype).cuda()
    W = ssdi8.quantize_mx(torch.randn(200, K).cuda() / K ** 0.5)
    a = ssdi8.linear_mx(cut(x.cpu(), 5), W, x_format=format, activation="silu")
    b = ssdi8.linear_mx(ssdi8.quantize_mx(x, format), W, activation="silu", y_dtype=dtype)
    assert a.dtype == dtype and torch.equal(a, b)
    xv, wv = (R.values(*t, f) for t, f in ((ssdi8.quantize_mx(x, format), format), (W, "mxfp4")))
    y, e = R.linear_mx(xv, wv, None, None, format, act="silu")
    R.assert_within(a, y.cpu(), R.rounded(dtype, y, e).cpu(), "y")


def test_linear_mx_rows_outputs_and_streams(ssdi8):
    x = torch.randn(2, 3, 640, device="cuda").half()
    W = ssdi8.quantize_mx(torch.randn(100, 640, device="cuda"))
    X = ssdi8.quantize_mx(x, "mxfp8")
    a = ssdi8.linear_mx(X, W)
    assert a.shape == (2, 3, 100) and a.dtype == F16
    wide = torch.full((2, 3, 120), 7.0, dtype=F16, device="cuda")
    b = ssdi8.linear_mx(X, W, y=wide[..., 10:110])
    assert torch.equal(a, b) and (wide[..., :10] == 7).all() and (wide[..., 110:] == 7).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c = ssdi8.linear_mx(x, W, stream=side)
    side.synchronize()
    assert torch.equal(a, c)
    r = torch.randn(2, 3, 100, device="cuda").half()
    d = ssdi8.linear_mx(X, W, residual=r)
    e = r.clone()
    ssdi8.linear_mx(X, W, residual=e, y=e)       # y may be the residual
    assert torch.equal(d, e)
    none = ssdi8.linear_mx(ssdi8.Mx(X.codes[:0], X.scales[:0]), W)
    assert none.shape == (0, 3, 100)


def test_linear_mx_of_what_is_no_number(ssdi8):
    """A scale of NaN takes its row of y (of x's) or its column (of the weight's), and no other."""
    x, w = torch.randn(70, 256), torch.randn(90, 256)
    x[3, 40], w[7, 250] = float("inf"), float("nan")
    for M in (70, 5):
        for format in ("mxfp8", "mxfp4"):
            y = ssdi8.linear_mx(ssdi8.quantize_mx(x[:M].cuda(), format), ssdi8.quantize_mx(w.cuda()), y_dtype=F32).cpu()
            bad = torch.isnan(y)
            want = torch.zeros_like(bad)
            want[3], want[:, 7] = True, True
            assert torch.equal(bad, want)


def test_captured(ssdi8):
    """Norm and product in a graph, with eager calls between its replays."""
    x = torch.randn(40, 512, device="cuda").half()
    w = torch.ones(512, device="cuda")
    W = ssdi8.quantize_mx(torch.randn(300, 512, device="cuda"))

    def run():
        n = ssdi8.norm_quantize(x, w, format="mxfp8")
        a = ssdi8.linear_mx(ssdi8.Mx(n["codes"], n["scales"]), W)
        i = ssdi8.norm_quantize(x, w)
        return a, ssdi8.linear_mx(a, ssdi8.quantize_mx(a[:64].float(), "mxfp4")), i["codes"], i["scales"]

    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for k in range(3):
        x.copy_(torch.randn(40, 512, device="cuda"))
        g.replay()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_linear_mx_refusals(ssdi8):
    x = torch.randn(4, 64, device="cuda").half()
    X, W = ssdi8.quantize_mx(x, "mxfp8"), ssdi8.quantize_mx(torch.randn(10, 64, device="cuda"))
    f = ssdi8.linear_mx
    for bad in (lambda: f(x[:, :32], W), lambda: f(X, X), lambda: f(X, W, x_format="int8"), lambda: f(X, W, activation="relu"),
                lambda: f(X, W, residual=x), lambda: f(X, W, bias=x[0, :10]), lambda: f(X, W, y_dtype=torch.int8),
                lambda: f(ssdi8.Mx(X.codes, W.scales), W), lambda: f(ssdi8.Mx(X.codes, X.scales.view(torch.uint8)), W),
                lambda: f(X, ssdi8.Mx(W.codes[:, ::2], W.scales)), lambda: f(X.codes, W), lambda: f(X, W.codes),
                lambda: f(ssdi8.Mx(X.codes.cpu(), X.scales), W), lambda: f(x.cpu(), W),
                lambda: f(X, ssdi8.Mx(W.codes.cpu(), W.scales)),
                lambda: f(X, W, y=torch.empty(4, 11, dtype=F16, device="cuda"))):
        with pytest.raises((ValueError, TypeError, AttributeError)):
            bad()
