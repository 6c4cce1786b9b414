"""The operators around the SSD layer at the sizes that choose their other forms: the convolution's walks of
32 and 64 tokens, the norm's walks of two and four rows, the few-row products' unrolled lines and wider
tiles, int8 sums shared by sets of waves, the selective scan's compile-time forms.  Against the 64-bit
forms and bounds of block_ref.py, or, for products, whole value by whole value."""
import ctypes

import pytest
import torch

import block_ref as R
from test_gpu_block import BF16, F16, F32, Draw, cut, d64, dev, scan_inputs, scan_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


# ------------------------------------------------------------------------------ convolution
# B waves lie along the channels here: 256 of them with two workgroups each take walks of 32 tokens, 512
# take walks of 64
WALKS = [(256, 130, 8, 4, F16, None, 0), (256, 130, 21, 3, BF16, (9, 8, 4), 5),
         (512, 70, 8, 4, F16, None, 3), (512, 300, 19, 4, F32, (1, 10, 8), 0),
         (512, 257, 24, 2, BF16, (8, 16), 8)]


def walk_inputs(B, L, D, W, dtype):
    r = Draw(B + L + D)
    x, w, s0 = r.normal(B, L, D, dtype=dtype), r.uniform(-0.7, 0.7, D, W), r.normal(B, W - 1, D, dtype=dtype)
    n = torch.tensor([(L, 0, 1, L - 1, 64, 65, 32, 3)[b % 8] for b in range(B)], dtype=torch.int32)
    return x, w, r.normal(D), s0, n


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,L,D,W,dtype,split,before", WALKS)
def test_conv_walks(ssdi8, B, L, D, W, dtype, split, before, ragged):
    x, w, b, s0, n = walk_inputs(B, L, D, W, dtype)
    y, e, last = R.conv(x.double(), w, b, "silu", s0.double(), n if ragged else None)
    xd = x.clone()
    if ragged:
        xd[torch.arange(L)[None] >= n[:, None]] = float("nan")
    out = ssdi8.causal_conv(cut(xd, before), dev(w), bias=dev(b), split=split, init_state=dev(s0),
                            lengths=dev(n) if ragged else None)
    got = out["y"] if split is None else torch.cat(out["y"], -1)
    R.assert_within(got, y, R.rounded(dtype, y, e), "y")
    assert torch.equal(out["final_state"].double().cpu(), last)


def test_conv_walk_with_the_state_in_place(ssdi8):
    B, L, D, W = 512, 300, 19, 4
    x, w, b, s0, n = walk_inputs(B, L, D, W, F16)
    y, e, last = R.conv(x.double(), w, None, "silu", s0.double(), n)
    xd, wd, st, nd = dev(x), dev(w), dev(s0), dev(n)
    a, out = ssdi8._conv(xd, wd, None, "silu", None, None, B, L, None)
    a.x_token_stride = xd.stride(1)
    a.init_state = a.final_state = st.data_ptr()
    a.lengths = nd.data_ptr()
    stream = torch.cuda.current_stream().cuda_stream
    assert ssdi8.lib().ssdi8_causal_conv(B, L, D, ctypes.byref(a), stream) == ssdi8.OK
    R.assert_within(out[0], y, R.rounded(F16, y, e), "y")
    assert torch.equal(st.double().cpu(), last)


# ------------------------------------------------------------------------------ gated norm
# Walks of two rows from 4096 groups of a workgroup or 16384 of a wave each, of four from twice as many
ROWS = [(8195, 1032, 1, F16, True, True, False), (4099, 1032, 1, BF16, True, False, True),
        (8197, 1029, 1, F32, False, True, False), (16390, 1000, 1, F16, True, True, True),
        (33001, 40, 1, F16, True, True, False), (17001, 82, 2, BF16, True, False, False),
        (33003, 7, 1, F16, True, True, False), (33003, 15, 1, F32, False, False, False)]


@pytest.mark.parametrize("M,D,groups,dtype,z,res,before", ROWS)
def test_norm_walks(ssdi8, M, D, groups, dtype, z, res, before):
    r = Draw(M + D)
    x, w = dev(r.normal(M, D, dtype=dtype)), dev(1 + 0.1 * r.normal(D))
    zz = dev(r.normal(M, D, dtype=dtype, scale=3.0)) if z else None
    rr = dev(r.normal(M, D, dtype=dtype)) if res else None
    x[M - 1] = 0
    y, e, s = R.norm(x.double(), w.double(), d64(zz), d64(rr), 1e-5, groups, before)
    y, e, s = y.cpu(), e.cpu(), s.cpu()
    kw = dict(groups=groups, norm_before_gate=before)
    out = ssdi8.gated_norm(x, w, z=zz, residual=rr, **kw)
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    if res:
        R.assert_within(out["residual"], s, R.rounded(dtype, s, R.U * s.abs()), "residual")
    # columns of wider rows
    wide = torch.full((M, D + 5), float("nan"), dtype=dtype, device="cuda")
    wide[:, 3:3 + D] = x
    again = ssdi8.gated_norm(wide[:, 3:3 + D], w, z=zz, residual=rr, **kw)
    assert torch.equal(again["y"], out["y"])
    # y over x, the sum over the residual
    place = ssdi8.gated_norm(x, w, z=zz, residual=rr, y=x, residual_out=rr, **kw)
    assert place["y"] is x and torch.equal(x, out["y"])
    if res:
        assert place["residual"] is rr and torch.equal(rr, out["residual"])


# ------------------------------------------------------------------------------ projections
FEW = [(8, 70, 2600), (16, 4100, 2100), (24, 4100, 300), (32, 4111, 2600), (30, 70, 2600), (50, 100, 2600),
       (64, 8190, 320), (40, 8200, 330), (64, 8190, 2600), (33, 4111, 1700), (63, 300, 6800), (48, 4096, 640)]
SPLIT = [(65, 70, 3211), (1000, 1000, 3211), (130, 700, 6500)]


@pytest.mark.parametrize("M,O,K", FEW + SPLIT)
@pytest.mark.parametrize("dtype", [F16, BF16, torch.int8])
def test_linear_forms(ssdi8, M, O, K, dtype):
    """Small integers, whose products and sums every type holds exactly."""
    r = Draw(M + O)
    x, w = (r.uniform(-2.5, 2.5, *s).round() for s in ((M, K), (O, K)))
    b, rr = r.uniform(-9, 9, O).round(), r.uniform(-9, 9, M, O).round()
    kw = dict(x_scale=torch.ones(M, device="cuda"), w_scale=torch.ones(O, device="cuda")) \
        if dtype == torch.int8 else {}
    got = ssdi8.linear(x.to(dtype).cuda(), w.to(dtype).cuda(), bias=dev(b), residual=dev(rr), y_dtype=F32, **kw)
    want = x.cuda().double() @ w.cuda().double().t() + dev(b) + dev(rr)
    assert torch.equal(got.double(), want)


@pytest.mark.parametrize("M", [3, 80])
def test_gelu_of_negative_values(ssdi8, M):
    """v (1 + erf(v / sqrt(2))) / 2 has relative accuracy for negative v too, where 1 + erf cancels.  The
    exponential of -v^2 / 2 costs three roundings of its argument, 1.5 v^2 u in the result; the rest (a
    reciprocal and a polynomial in it, whose slopes in the logarithm stay below 2.5, and the products) 28 u."""
    v = torch.cat([torch.linspace(-12.0, 12.0, 4001), torch.tensor([0.0, -1e-20, 1e-6, -14.0, -40.0, -1e30, 1e30])])
    y = 0.5 * v.double() * torch.erfc(-v.double() / 2 ** 0.5)
    e = (1.5 * v.double().clamp(-20, 20) ** 2 + 28) * R.U * y.abs() + 16 * R.TINY[F32]
    zero = lambda *s: torch.zeros(*s, dtype=F16, device="cuda")
    got = ssdi8.linear(zero(M, 16), zero(v.numel(), 16), bias=dev(v), activation="gelu", y_dtype=F32)
    R.assert_within(got, y.expand(M, -1), e.expand(M, -1), "y")
    ends = ssdi8.linear(zero(M, 16), zero(2, 16), bias=torch.tensor([float("inf"), float("nan")], device="cuda"),
                        activation="gelu", y_dtype=F32).cpu()
    assert (ends[:, 0] == float("inf")).all() and torch.isnan(ends[:, 1]).all()


# ------------------------------------------------------------------------------ selective scan
FORMS = [  # B, L, heads, headdim, groups, N, tied, dtype, dt fp32, z, init, lengths
    (2, 70, 66, 1, 2, 24, False, F16, False, True, True, [70, 3]),
    (1, 300, 40, 1, 1, 32, False, BF16, True, True, True, None),        # cut into spans
    (1, 40, 24, 1, 1, 20, False, F32, True, False, True, None),
    (3, 129, 35, 1, 1, 32, False, F16, True, True, False, [0, 129, 64]),
    (2, 65, 3, 64, 1, 64, True, F16, True, True, True, [64, 65]),
    (1, 400, 4, 16, 2, 40, True, BF16, False, True, False, [390]),      # cut into spans
    (2, 33, 2, 8, 1, 36, True, F32, True, False, True, None),
    (1, 70, 5, 8, 1, 64, True, F16, False, False, False, None),
    (2, 90, 40, 1, 1, 12, False, BF16, False, True, True, [90, 11]),
]


@pytest.mark.parametrize("B,L,H,P,G,N,tied,dtype,dt32,z,init,lengths", FORMS)
def test_scan_forms(ssdi8, B, L, H, P, G, N, tied, dtype, dt32, z, init, lengths):
    i = scan_inputs(Draw(L + H + N), B, L, H, P, G, N, tied, dtype, dt32, z, init)
    n = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    y, e, h, he = scan_ref(i, lengths=n)
    t = {k: None if v is None else v.clone() for k, v in i.items()}
    if n is not None:
        for k in ("u", "dt", "B", "C", "z"):
            if t[k] is not None:
                t[k][torch.arange(L)[None] >= n[:, None]] = float("nan")
    g = {k: dev(v) for k, v in t.items()}
    out = ssdi8.selective_scan(g["u"], g["dt"], g["A"], g["B"], g["C"], D=g["D"], z=g["z"],
                               dt_bias=g["dt_bias"], init_state=g["state"], lengths=dev(n))
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    R.assert_within(out["final_state"], h, he + R.TINY[F32], "final_state")


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


# ------------------------------------------------------------------------------ the followed calls
SMALL = [{"op": "conv", "B": 2, "L": 70, "D": 21, "d1": 9, "d2": 8, "ragged": True, "state": True, "pad": 3},
         {"op": "conv", "B": 3, "D": 40, "W": 3, "state": True, "step": True, "dtype": "bf16"},
         {"op": "scan", "B": 2, "L": 40, "H": 16, "gate": True, "state": True, "ragged": True},
         {"op": "scan", "B": 2, "L": 33, "H": 2, "P": 64, "N": 128, "tied": True, "dtype": "bf16"},
         {"op": "scan", "B": 3, "H": 4, "P": 32, "G": 2, "N": 100, "tied": True, "state": True, "step": True},
         {"op": "norm", "M": 5, "D": 96, "groups": 2, "gate": True, "residual": True, "pad": 7},
         {"op": "norm", "M": 3, "D": 77, "gate": True, "before": True, "dtype": "fp32"},
         {"op": "linear", "M": 9, "O": 33, "K": 200, "act": "gelu", "bias": True, "residual": True},
         {"op": "linear", "M": 70, "O": 40, "K": 130, "dtype": "int8", "act": "softplus", "bias": True}]


@pytest.mark.parametrize("case", SMALL, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_the_calls_64_bit_forms(ssdi8, case):
    """The 64-bit results beside the calls whose speed is followed are those of block_ref.py: both are
    64-bit sums of at most a few hundred terms, 2^-40 relative of the largest is far above either's
    rounding and far below any other formula's."""
    import perf.operators as P
    got = P.exact(case, 5)
    s = P.prepare(case, 5)
    c = s["c"]
    f = {k: v.double().cpu() if isinstance(v, torch.Tensor) and k != "lengths" else
         v.cpu() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    one = lambda k: f[k] if f[k] is None or not c["step"] else f[k][:, None]
    if c["op"] == "conv":
        y, _, last = R.conv(one("x"), f["w"], f["bias"], "silu", f["state"], f["lengths"])
        want = (y[:, 0] if c["step"] else y), last
        got = (got[0] if s["split"] is None else torch.cat(got[0], -1)), got[1]
    elif c["op"] == "scan":
        y, _, h, _ = R.scan(one("u"), one("dt"), f["A"], one("B"), one("C"), f["D"], one("z"), f["dt_bias"], True,
                            f["state"], f["lengths"])
        want = (y[:, 0] if c["step"] else y), h
    elif c["op"] == "norm":
        y, _, total = R.norm(f["x"], f["w"], f["z"], f["residual"], 1e-5, c["groups"], c["before"])
        want = y, (total if f["residual"] is not None else None)
    else:
        want = R.linear(f["x"], f["w"], f["bias"], c["act"], f["residual"], f.get("x_scale"), f.get("w_scale"))[:1]
        got = (got,)
    for a, b in zip(got, want, strict=True):
        assert (a is None) == (b is None)
        if a is not None:
            assert (a.cpu() - b).abs().max() <= 2.0 ** -40 * b.abs().max()
