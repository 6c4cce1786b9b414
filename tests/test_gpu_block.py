"""The operators around the SSD layer against their 64-bit forms: the convolution, the selective scan,
their single-token forms, the gated norm and the projections.  Every bound counts the roundings of the
formula (block_ref.py)."""
import pytest
import torch

import block_ref as R

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    s.lib()
    return s


class Draw:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)

    def normal(self, *s, dtype=F32, scale=1.0):
        return (scale * torch.randn(*s, generator=self.g)).to(dtype)

    def uniform(self, lo, hi, *s):
        return lo + (hi - lo) * torch.rand(*s, generator=self.g)


def dev(t):
    return None if t is None else t.cuda()


def cut(t, before, after=3):
    """t on the device as columns of wider rows whose other columns are NaN."""
    if t is None:
        return None
    wide = torch.full((*t.shape[:-1], before + t.shape[-1] + after), float("nan")).to(t.dtype).cuda()
    wide[..., before:before + t.shape[-1]] = t.cuda()
    return wide[..., before:before + t.shape[-1]]


d64 = lambda t: None if t is None else t.double()


# ------------------------------------------------------------------------------ convolution
CONV = [  # B, L, D, W, dtype, split, bias, act, init, lengths, columns before x
    (1, 1, 8, 4, F16, None, True, "silu", False, None, 0),
    (2, 2, 24, 4, F16, None, True, "silu", True, None, 8),
    (3, 67, 1792, 4, F16, (1536, 128, 128), True, "silu", False, [67, 0, 1], 0),
    (2, 130, 517, 3, BF16, (5, 500, 12), False, None, True, [2, 130], 7),
    (2, 64, 1, 2, F32, None, True, None, True, [63, 64], 0),
    (1, 65, 1030, 4, F32, (1030,), True, "silu", True, [5000], 1),
    (2, 129, 40, 3, F16, (0, 33, 7), True, "silu", True, [-4, 3], 5),
    (1, 0, 16, 4, F16, None, True, "silu", True, None, 0),
    (1, 3, 600, 4, BF16, None, True, "silu", False, None, 0),
]


@pytest.mark.parametrize("B,L,D,W,dtype,split,bias,act,init,lengths,before", CONV)
def test_conv(ssdi8, B, L, D, W, dtype, split, bias, act, init, lengths, before):
    r = Draw(L + D)
    x, w = r.normal(B, L, D, dtype=dtype), r.uniform(-0.7, 0.7, D, W)
    b = r.normal(D) if bias else None
    s0 = r.normal(B, W - 1, D, dtype=dtype) if init else None
    n = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    y, e, last = R.conv(x.double(), w, b, act, d64(s0), n)
    xd = x.clone()
    if n is not None:   # what lies behind a sequence's end is not read
        for i in range(B):
            xd[i, max(0, int(n[i])):] = float("nan")
    out = ssdi8.causal_conv(cut(xd, before), dev(w), bias=dev(b), activation=act, split=split,
                            init_state=dev(s0), lengths=dev(n))
    got = out["y"] if split is None else torch.cat(out["y"], -1)
    if split is not None:
        assert [t.shape[-1] for t in out["y"]] == list(split)
        assert all(t.is_contiguous() for t in out["y"])
    R.assert_within(got, y, R.rounded(dtype, y, e), "y")
    assert torch.equal(out["final_state"].double().cpu(), last)


@pytest.mark.parametrize("B,D,W,dtype,split", [(1, 8, 4, F16, None), (5, 1792, 4, F16, (1536, 128, 128)),
                                               (3, 517, 3, BF16, (1, 516)), (2, 33, 2, F32, None)])
def test_conv_token_by_token(ssdi8, B, D, W, dtype, split):
    """Tokens one at a time leave what the prompt leaves."""
    r = Draw(D)
    L = 7
    x, w, b = r.normal(B, L, D, dtype=dtype), r.uniform(-0.7, 0.7, D, W), r.normal(D)
    y, e, last = R.conv(x.double(), w, b, "silu", None, None)
    state = torch.zeros(B, W - 1, D, dtype=dtype, device="cuda")
    xd, got = cut(x, 3), []
    for t in range(L):
        o = ssdi8.causal_conv_step(xd[:, t], dev(w), state, bias=dev(b), split=split)
        got.append(o if split is None else torch.cat(o, -1))
    R.assert_within(torch.stack(got, 1), y, R.rounded(dtype, y, e), "y")
    assert torch.equal(state.double().cpu(), last)


@pytest.mark.parametrize("B,L,D,W,split,lengths", [(2, 70, 1540, 4, (1029, 260, 251), [70, 1]),
                                                   (3, 5, 20, 3, None, [0, 2, 1]), (1, 0, 9, 4, None, None)])
def test_conv_state_in_place(ssdi8, B, L, D, W, split, lengths):
    """The state of a resumed sequence may be its own final state."""
    import ctypes
    r = Draw(D)
    x, w, s0 = r.normal(B, L, D, dtype=F16), r.uniform(-0.7, 0.7, D, W), r.normal(B, W - 1, D, dtype=F16)
    n = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    y, e, last = R.conv(x.double(), w, None, "silu", s0.double(), n)
    xd, wd, st, nd = dev(x), dev(w), dev(s0), dev(n)
    a, out = ssdi8._conv(xd, wd, None, "silu", split, None, B, L, None)
    a.x_token_stride = xd.stride(1)
    a.init_state = a.final_state = st.data_ptr()
    a.lengths = nd.data_ptr() if n is not None else None
    stream = torch.cuda.current_stream().cuda_stream
    assert ssdi8.lib().ssdi8_causal_conv(B, L, D, ctypes.byref(a), stream) == ssdi8.OK
    R.assert_within(torch.cat(out, -1), y, R.rounded(F16, y, e), "y")
    assert torch.equal(st.double().cpu(), last)


# ------------------------------------------------------------------------------ selective scan
SCAN = [  # B, L, heads, headdim, groups, N, tied, dtype, dt fp32, z, init, lengths, columns before
    (1, 1, 64, 1, 1, 16, False, F16, False, True, False, None, 0),
    (2, 33, 130, 1, 1, 16, False, F16, False, True, True, None, 3),
    (3, 77, 66, 1, 2, 16, False, BF16, True, False, True, [77, 0, 1], 0),
    (2, 50, 7, 1, 1, 5, False, F32, True, True, False, [20, 50], 1),
    (1, 31, 10, 3, 3, 24, False, F16, False, True, True, None, 0),
    (2, 65, 3, 64, 1, 128, True, F16, True, False, True, [64, 65], 0),
    (1, 40, 4, 24, 4, 100, True, BF16, False, True, False, None, 5),
    (2, 36, 2, 20, 1, 64, True, F32, True, True, True, [-1, 99], 0),
    (1, 34, 2, 8, 1, 256, False, F16, True, False, True, None, 0),
    (1, 17, 1, 1, 1, 1, True, F32, True, False, False, None, 0),
    (1, 1025, 70, 1, 1, 16, False, F16, False, True, True, None, 0),        # cut into spans
    (2, 700, 2, 64, 2, 128, True, F32, True, True, True, [700, 130], 0),
    (2, 515, 9, 5, 1, 16, False, BF16, False, True, False, [0, 400], 2),
    (1, 0, 4, 8, 1, 16, True, F16, True, False, True, None, 0),
]


def scan_inputs(r, B, L, H, P, G, N, tied, dtype, dt32, z, init):
    lead = (B,) if L is None else (B, L)
    i = {"u": r.normal(*lead, H * P, dtype=dtype), "dt": r.normal(*lead, H) * 1.5 - 2.0,
         "A": -torch.exp(r.uniform(0.0, 2.77, *((H,) if tied else (H * P, N)))),
         "B": r.normal(*lead, G, N, dtype=dtype), "C": r.normal(*lead, G, N, dtype=dtype),
         "D": r.normal(H), "dt_bias": r.normal(H, scale=0.1),
         "z": r.normal(*lead, H * P, dtype=dtype) if z else None,
         "state": r.normal(B, H * P, N) if init else None}
    if H > 2:
        i["dt"][..., 0] = 25.0    # above the threshold of softplus
        i["dt"][..., 1] = -14.0
    if not dt32:
        i["dt"] = i["dt"].to(dtype)
    return i


def scan_ref(i, softplus_on=True, lengths=None):
    return R.scan(i["u"].double(), i["dt"].double(), i["A"].double(), i["B"].double(), i["C"].double(),
                  i["D"].double(), d64(i["z"]), d64(i["dt_bias"]), softplus_on, d64(i["state"]), lengths)


@pytest.mark.parametrize("B,L,H,P,G,N,tied,dtype,dt32,z,init,lengths,before", SCAN)
def test_scan(ssdi8, B, L, H, P, G, N, tied, dtype, dt32, z, init, lengths, before):
    i = scan_inputs(Draw(L + H), B, L, H, P, G, N, tied, dtype, dt32, z, init)
    n = torch.tensor(lengths, dtype=torch.int32) if lengths else None
    y, e, h, he = scan_ref(i, lengths=n)
    u, dt, Bm, Cm, zz = (None if i[k] is None else i[k].clone() for k in ("u", "dt", "B", "C", "z"))
    if n is not None:
        for b in range(B):
            for t in (u, dt, Bm, Cm, zz):
                if t is not None:
                    t[b, max(0, int(n[b])):] = float("nan")
    out = ssdi8.selective_scan(cut(u, before), cut(dt, before), dev(i["A"]),
                               cut(Bm.flatten(2), before).unflatten(2, (G, N)),
                               cut(Cm.flatten(2), before).unflatten(2, (G, N)), D=dev(i["D"]),
                               z=cut(zz, before), dt_bias=dev(i["dt_bias"]),
                               init_state=dev(i["state"]), lengths=dev(n))
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    R.assert_within(out["final_state"], h, he + R.TINY[F32], "final_state")


@pytest.mark.parametrize("L", [40, 1300])
def test_scan_in_place_and_without_options(ssdi8, L):
    """The state of a resumed sequence may be its own final state, cut into spans or not."""
    i = scan_inputs(Draw(5), 1, L, 40, 1, 1, 16, False, F16, True, False, True)
    i["D"], i["dt_bias"], i["dt"] = torch.zeros(40), None, i["dt"].abs().clamp(max=0.5)
    y, e, h, he = scan_ref(i, softplus_on=False)
    d, a, out = ssdi8._sel_scan(dev(i["u"]), dev(i["dt"]), dev(i["A"]), dev(i["B"]), dev(i["C"]), None,
                                None, None, False, None, None)
    keep = [dev(i[k]) for k in ("u", "dt", "A", "B", "C", "state")]
    for k, t in zip(("u", "dt", "A", "B", "C", "init_state"), keep):
        setattr(a, k, t.data_ptr())
    a.final_state = keep[-1].data_ptr()
    need = ssdi8.selective_scan_workspace_size(d)
    assert (need > 0) == (L > 1000)
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), need
    st = torch.cuda.current_stream().cuda_stream
    import ctypes
    assert ssdi8.lib().ssdi8_selective_scan(ctypes.byref(d), ctypes.byref(a), st) == ssdi8.OK
    R.assert_within(out, y, R.rounded(F16, y, e), "y")
    R.assert_within(keep[-1], h, he + R.TINY[F32], "final_state")


def test_scan_infinite_decay_and_empty_step(ssdi8):
    """A decay rate of -inf forgets at every token with a positive step and keeps the state at a step of 0."""
    u = torch.ones(1, 3, 8, device="cuda")
    dt = torch.tensor([0.0, 0.5, 0.0], device="cuda")[None, :, None].repeat(1, 1, 8)
    A = torch.full((8, 16), -float("inf"), device="cuda")
    B = torch.ones(1, 3, 1, 16, device="cuda")
    out = ssdi8.selective_scan(u, dt, A, B, B, dt_softplus=False,
                               init_state=torch.full((1, 8, 16), 3.0, device="cuda"))
    assert torch.equal(out["y"][0, :, 0].cpu(), torch.tensor([48.0, 8.0, 8.0]))
    assert torch.equal(out["final_state"].cpu(), torch.full((1, 8, 16), 0.5))


def test_scan_continues_the_chunked_layer(ssdi8):
    """Whole chunks by the FP16 layer, the rest by the scan from its final state: one sequence of the
    recurrence, within the FP16 layer's own error (operands rounded to fp16: 2^-11 each)."""
    r, L, H = Draw(9), 300, 4
    i = scan_inputs(r, 1, L, H, 64, 1, 128, True, F16, True, False, False)
    i["dt"] = r.normal(1, L, H, scale=0.5) - 2.0
    i["dt_bias"] = torch.zeros(H)
    y, e, h, he = scan_ref(i)
    g = {k: dev(v) for k, v in i.items()}
    x = g["u"].view(1, L, H, 64)
    head = ssdi8.ssd_chunk_scan_fp16(x[:, :256].contiguous(), g["dt"][:, :256].contiguous(), g["A"],
                                     g["B"][:, :256].contiguous(), g["C"][:, :256].contiguous(), D=g["D"])
    rest = ssdi8.selective_scan(g["u"][:, 256:], g["dt"][:, 256:], g["A"], g["B"][:, 256:],
                                g["C"][:, 256:], D=g["D"],
                                init_state=head["final_state"].view(1, H * 64, 128))
    want = y[:, 256:]
    rel = ((rest["y"].double().cpu() - want).norm() / want.norm()).item()
    assert rel < 4 * 2.0 ** -11, rel
    rel = ((rest["final_state"].double().cpu() - h).norm() / h.norm()).item()
    assert rel < 4 * 2.0 ** -11, rel


@pytest.mark.parametrize("B,H,P,G,N,tied,dtype,dt32,z", [
    (1, 64, 1, 1, 16, False, F16, False, True), (3, 130, 1, 2, 16, False, BF16, True, False),
    (2, 7, 3, 1, 5, False, F32, True, True), (2, 3, 64, 1, 128, True, F16, True, True),
    (5, 4, 24, 4, 100, True, BF16, False, True), (1, 2, 20, 1, 63, True, F32, True, False),
    (2, 2, 8, 1, 256, False, F16, True, True), (1, 1, 1, 1, 1, True, F32, True, False),
    (70, 80, 64, 1, 32, True, F16, True, False)])
def test_scan_step(ssdi8, B, H, P, G, N, tied, dtype, dt32, z):
    i = scan_inputs(Draw(H + N), B, None, H, P, G, N, tied, dtype, dt32, z, True)
    one = {k: v[:, None] if k in ("u", "dt", "B", "C", "z") and v is not None else v for k, v in i.items()}
    y, e, h, he = scan_ref(one)
    state = dev(i["state"])
    got = ssdi8.selective_scan_step(cut(i["u"], 2), cut(i["dt"], 1), dev(i["A"]),
                                    cut(i["B"].flatten(1), 5).unflatten(1, (G, N)),
                                    dev(i["C"]), state, D=dev(i["D"]), z=cut(i["z"], 9),
                                    dt_bias=dev(i["dt_bias"]))
    R.assert_within(got, y[:, 0], R.rounded(dtype, y, e)[:, 0], "y")
    R.assert_within(state, h, he + R.TINY[F32], "state")


# ------------------------------------------------------------------------------ gated norm
@pytest.mark.parametrize("M,D,groups,dtype,z,res,before,cols", [
    (1, 1, 1, F32, False, False, False, 0), (3, 7, 1, F16, True, False, False, 1),
    (5, 768, 1, F16, False, True, False, 0), (9, 1536, 8, BF16, True, True, False, 0),
    (2, 5120, 1, F16, True, False, True, 77), (4, 2049, 1, F32, True, True, True, 3),
    (2, 8193, 1, BF16, True, False, False, 0), (1, 32768, 1, F16, False, True, False, 0),
    (3, 40, 5, F32, False, False, False, 2), (1, 10240, 2, F16, True, False, False, 0)])
def test_gated_norm(ssdi8, M, D, groups, dtype, z, res, before, cols):
    r = Draw(M + D)
    x, w = r.normal(M, D, dtype=dtype), 1 + 0.1 * r.normal(D)
    zz = r.normal(M, D, dtype=dtype, scale=3.0) if z else None
    rr = r.normal(M, D, dtype=dtype) if res else None
    x[0] = 0      # a row of zeros
    if res:
        rr[0] = 0
    y, e, s = R.norm(x.double(), w.double(), d64(zz), d64(rr), 1e-5, groups, before)
    out = ssdi8.gated_norm(cut(x, cols), dev(w), z=cut(zz, cols), residual=dev(rr), groups=groups,
                           norm_before_gate=before)
    R.assert_within(out["y"], y, R.rounded(dtype, y, e), "y")
    if res:
        R.assert_within(out["residual"], s, R.rounded(dtype, s, R.U * s.abs()), "residual")


def test_gated_norm_in_place(ssdi8):
    r = Draw(1)
    x, rr, w = r.normal(4, 3, 96, dtype=F16), r.normal(4, 3, 96, dtype=F16), torch.ones(96)
    plain = ssdi8.gated_norm(dev(x), dev(w), residual=dev(rr))
    xd, rd = dev(x), dev(rr)
    out = ssdi8.gated_norm(xd, dev(w), residual=rd, residual_out=rd, y=xd)
    assert out["y"] is xd and out["residual"] is rd
    assert torch.equal(xd, plain["y"]) and torch.equal(rd, plain["residual"])


# ------------------------------------------------------------------------------ projections
LINEAR = [  # M, O, K, dtype, bias, act, residual, y fp32, columns before x
    (1, 1, 1, F16, True, None, False, False, 0), (1, 33, 64, BF16, True, "silu", True, False, 0),
    (8, 100, 257, F16, False, "gelu", False, True, 3), (17, 40, 96, "i8", True, None, True, False, 0),
    (33, 70, 1000, BF16, True, "softplus", True, True, 8), (64, 65, 130, "i8", False, "silu", False, True, 1),
    (65, 64, 64, F16, False, None, False, False, 0), (70, 75, 72, F16, True, "silu", True, False, 8),
    (130, 200, 321, BF16, True, None, True, True, 1), (200, 129, 77, "i8", True, "gelu", True, False, 5),
    (1030, 2000, 136, F16, False, None, True, False, 0), (1500, 1800, 208, "i8", False, None, False, False, 16),
    (4100, 4100, 64, F16, True, None, True, False, 0), (4100, 4099, 200, BF16, False, "silu", False, True, 1),
    (4099, 4200, 300, "i8", True, None, True, False, 0)]


@pytest.mark.parametrize("M,O,K,dtype,bias,act,res,y32,before", LINEAR)
def test_linear(ssdi8, M, O, K, dtype, bias, act, res, y32, before):
    r = Draw(M + O + K)
    quantized = dtype == "i8"
    own = F16 if quantized else dtype
    yd = F32 if y32 else own
    if quantized:
        x, w = ((127 * r.uniform(-1, 1, *s)).round().to(torch.int8) for s in ((M, K), (O, K)))
        xs, ws = r.uniform(0.5, 2.0, M) / 64, r.uniform(0.5, 2.0, O) / (64 * K ** 0.5)
        xd = torch.zeros(M, before + K, dtype=torch.int8, device="cuda")
        xd[:, before:] = x.cuda()
        xd = xd[:, before:]
    else:
        x, w = r.normal(M, K, dtype=dtype), r.normal(O, K, dtype=dtype, scale=K ** -0.5)
        xs = ws = None
        xd = cut(x, before)
    b = r.normal(O) if bias else None
    rr = r.normal(M, O, dtype=yd) if res else None
    # the reference on the device: 64-bit products of the larger cases
    y, e = R.linear(x.cuda().double(), w.cuda().double(), dev(b), act, d64(dev(rr)), dev(xs), dev(ws))
    y, e = y.cpu(), e.cpu()
    got = ssdi8.linear(xd, dev(w), bias=dev(b), activation=act, residual=dev(rr), x_scale=dev(xs),
                       w_scale=dev(ws), y_dtype=yd)
    R.assert_within(got, y, R.rounded(yd, y, e), "y")


@pytest.mark.parametrize("M,O", [(4090, 4090), (4090, 3060), (4090, 2040), (2040, 2040), (300, 16500),
                                 (1000, 1000), (640, 1920), (65, 70)])
@pytest.mark.parametrize("K,dtype", [(80, F16), (321, "i8"), (1611, BF16)])
def test_linear_tiles(ssdi8, M, O, K, dtype):
    """A size for each tile of the larger products (256 x 256, 192, 128, 128 x 128, 64 x 64, the last two
    with k split over sets of waves too), whole value by whole value: small integers, whose products and
    sums every type holds exactly."""
    r = Draw(M + O)
    x, w = (r.uniform(-2.5, 2.5, *s).round() for s in ((M, K), (O, K)))
    b, rr = r.uniform(-9, 9, O).round(), r.uniform(-9, 9, M, O).round()
    kind = torch.int8 if dtype == "i8" else dtype
    kw = dict(x_scale=torch.ones(M, device="cuda"), w_scale=torch.ones(O, device="cuda")) if dtype == "i8" else {}
    got = ssdi8.linear(x.to(kind).cuda(), w.to(kind).cuda(), bias=dev(b), residual=dev(rr), y_dtype=F32, **kw)
    want = x.cuda().double() @ w.cuda().double().t() + dev(b) + dev(rr)
    assert torch.equal(got.double(), want)


@pytest.mark.parametrize("M", [3, 80])
def test_linear_writes_its_columns_only(ssdi8, M):
    """y and the residual as columns of wider rows, y over the residual; NaN in a row of x stays there."""
    r = Draw(M)
    x, w = r.normal(2, M, 128, dtype=F16), r.normal(40, 128, dtype=F16)
    x[1, 1] = float("nan")
    wide = r.normal(2 * M, 90, dtype=F16).cuda()
    before = wide.clone()
    ssdi8.linear(dev(x), dev(w), residual=wide[:, 11:51].view(2 * M, 40), y=wide[:, 11:51])
    y, e = R.linear(d64(x).view(-1, 128), d64(w), None, None, d64(before[:, 11:51].cpu()), None, None)
    keep = torch.ones(2 * M, dtype=torch.bool)
    keep[M + 1] = False
    R.assert_within(wide[keep.cuda(), 11:51], y[keep], R.rounded(F16, y, e)[keep], "y")
    assert torch.isnan(wide[M + 1, 11:51]).all()
    assert torch.equal(wide[:, :11], before[:, :11]) and torch.equal(wide[:, 51:], before[:, 51:])


# ------------------------------------------------------------------------------ streams, refusals
def test_other_stream_and_graph(ssdi8):
    """Calls on a stream of their own, captured and replayed, give the bits of the eager call."""
    r = Draw(4)
    i = {k: dev(v) for k, v in scan_inputs(r, 1, 900, 40, 1, 1, 16, False, F16, True, True, True).items()}
    x, w, W = dev(r.normal(1, 900, 40, dtype=F16)), dev(r.normal(40, 4)), dev(r.normal(64, 40, dtype=F16))
    g = torch.ones(40, device="cuda")

    def block(stream=None):
        c = ssdi8.causal_conv(x, w, stream=stream)["y"]
        s = ssdi8.selective_scan(c, i["dt"], i["A"], i["B"], i["C"], D=i["D"], z=i["z"],
                                 init_state=i["state"], stream=stream)
        n = ssdi8.gated_norm(s["y"], g, stream=stream)["y"]
        return ssdi8.linear(n, W, activation="silu", stream=stream), s["final_state"]

    want = [t.clone() for t in block()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = block(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        block()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block()
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        block()


def test_refusals(ssdi8):
    z = lambda *s, dtype=F16: torch.zeros(*s, dtype=dtype, device="cuda")
    f = lambda *s: z(*s, dtype=F32)
    with pytest.raises(ValueError, match="not dense"):
        ssdi8.causal_conv(z(1, 16, 8).transpose(1, 2), f(16, 4))
    with pytest.raises(ValueError, match="split"):
        ssdi8.causal_conv(z(1, 8, 16), f(16, 4), split=(8, 4))
    with pytest.raises(ssdi8.SSDi8Error):
        ssdi8.causal_conv(z(1, 8, 16), f(16, 5))
    with pytest.raises(ValueError, match="state"):
        ssdi8.causal_conv_step(z(2, 16), f(16, 4), z(2, 4, 16))
    with pytest.raises(ValueError, match="dtype"):
        ssdi8.causal_conv(z(1, 8, 16, dtype=torch.float64), f(16, 4))
    with pytest.raises(ValueError, match="device"):
        ssdi8.causal_conv(torch.zeros(1, 8, 16), f(16, 4))
    scan = lambda **k: ssdi8.selective_scan(**{**dict(u=z(1, 8, 16), dt=f(1, 8, 16), A=f(16, 4),
                                                     B=z(1, 8, 1, 4), C=z(1, 8, 1, 4)), **k})
    with pytest.raises(ValueError, match="head"):
        scan(dt=f(1, 8, 5))
    with pytest.raises(ssdi8.SSDi8Error):
        scan(A=f(16, 257), B=z(1, 8, 1, 257), C=z(1, 8, 1, 257))
    with pytest.raises(ValueError, match="A must"):
        scan(A=f(16, 3))
    with pytest.raises(ValueError, match="dt must"):
        scan(dt=z(1, 8, 16, dtype=BF16))
    with pytest.raises(ssdi8.SSDi8Error):
        scan(B=z(1, 8, 3, 4), C=z(1, 8, 3, 4))
    with pytest.raises(ValueError, match="lengths"):
        scan(lengths=z(2, dtype=torch.int32))
    with pytest.raises(ssdi8.SSDi8Error):
        ssdi8.gated_norm(z(2, 16), f(16), groups=3)
    with pytest.raises(ssdi8.SSDi8Error):
        ssdi8.gated_norm(z(2, 16), f(16), eps=-1.0)
    with pytest.raises(ValueError, match="stride"):
        ssdi8.gated_norm(z(2, 5, 16)[:, :3], f(16))
    with pytest.raises(ValueError, match="x_scale"):
        ssdi8.linear(z(2, 16, dtype=torch.int8), z(4, 16, dtype=torch.int8))
    with pytest.raises(ValueError, match="weight"):
        ssdi8.linear(z(2, 16), z(4, 15))
    with pytest.raises(ValueError, match="activation"):
        ssdi8.linear(z(2, 16), z(4, 16), activation="tanh")
    with pytest.raises(ValueError, match="dtype"):
        ssdi8.linear(f(2, 16), f(4, 16))
