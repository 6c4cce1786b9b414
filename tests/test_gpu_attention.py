"""Linear attention with a decay per head against its quadratic form in 64 bits (mixer_ref.py): prompts, tokens,
lengths, strides, shared heads, values that are no numbers, captured calls."""
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


def draw(seed, b, L, Hq, Hk, Hv, K, V, dtype, token=True, init=True, size=1.0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)
    lead = (b,) if L is None else (b, L)
    t = {"q": n(*lead, Hq, K), "k": n(*lead, Hk, K), "v": size * n(*lead, Hv, V)}
    t = {k: x.to(dtype).cuda() for k, x in t.items()}
    t["g"] = -torch.exp(n(*(lead if token else ()), Hv) - 2).cuda()
    t["init"] = n(b, Hv, K, V).cuda() if init else None
    return t


def check(ssdi8, t, lengths=None, scale=None, **kw):
    dtype = t["q"].dtype
    dev = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], scale=scale, init_state=t["init"], lengths=dev, **kw)
    y, e, S, es = R.attention(t["q"].double(), t["k"].double(), t["v"].double(), t["g"], scale, t["init"], dev, dtype)
    R.assert_within(out["y"], y.cpu(), R.rounded(dtype, y, e).cpu(), "y")
    if "final_state" in out:
        R.assert_within(out["final_state"], S.cpu(), R.rounded(F32, S, es).cpu(), "final_state")
    return out


SIZES = [  # b, L, Hq, Hk, Hv, K, V
    (1, 1, 1, 1, 1, 16, 16), (2, 63, 2, 2, 2, 64, 64), (1, 64, 3, 1, 3, 128, 64), (2, 65, 4, 2, 2, 100, 72),
    (1, 130, 1, 1, 4, 128, 128), (1, 200, 2, 2, 2, 256, 128), (1, 97, 2, 1, 1, 33, 1), (1, 31, 1, 1, 1, 1, 130),
    (3, 129, 6, 1, 2, 17, 200), (1, 257, 1, 1, 2, 256, 256), (2, 32, 2, 2, 4, 129, 65),
]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("b,L,Hq,Hk,Hv,K,V", SIZES)
def test_prompts(ssdi8, b, L, Hq, Hk, Hv, K, V, dtype):
    check(ssdi8, draw(L + K, b, L, Hq, Hk, Hv, K, V, dtype, token=K % 2 == 0, init=L % 2 == 1))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_lengths(ssdi8, dtype):
    """Tokens behind a sequence's end are not read, give 0 and leave the state."""
    t = draw(5, 6, 150, 4, 2, 2, 64, 72, dtype)
    lengths = [150, 0, 1, 64, 65, -3]
    for i, n in enumerate(lengths):
        for k in ("q", "k", "v", "g"):
            t[k][i, max(0, n):] = float("nan")
    out = check(ssdi8, t, lengths)
    assert torch.equal(out["final_state"][1], t["init"][1]) and torch.equal(out["final_state"][5], t["init"][5])
    assert (out["y"][1] == 0).all()
    check(ssdi8, draw(6, 2, 70, 1, 1, 1, 32, 16, dtype), [100, 69])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("b,L,Hq,Hk,Hv,K,V", [(9, 130, 30, 30, 30, 64, 128), (3, 101, 90, 30, 30, 100, 72),
                                              (17, 70, 8, 8, 16, 128, 130), (3, 150, 1, 1, 4, 100, 50), (2, 140, 2, 1, 4, 64, 64)])
def test_many_heads_and_pairs(ssdi8, b, L, Hq, Hk, Hv, K, V, dtype):
    """Enough heads for workgroups of 128 columns, and heads that share q and k two by two; lengths inside a chunk; one
    value of v that is no number takes its column from its token on, and no other."""
    t = draw(L + V, b, L, Hq, Hk, Hv, K, V, dtype)
    lengths = [L - 13 * i if i < 7 else 1 for i in range(b)]
    out = check(ssdi8, t, lengths)
    t["v"][0, 67, 1, V - 1] = float("nan")
    bad = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"],
                                 lengths=torch.tensor(lengths, dtype=torch.int32).cuda())
    H, same = max(Hq, Hv), torch.ones_like(out["y"], dtype=torch.bool)
    for h in range(H):
        if h * Hv // H == 1:
            same[0, 67:, h, V - 1] = False
    assert torch.equal(bad["y"][same], out["y"][same]) and torch.isnan(bad["y"][~same]).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("b,L,H,K,V", [(1, 3000, 2, 64, 64), (2, 1025, 1, 128, 128), (1, 2049, 3, 100, 80)])
def test_long_sequences_of_few_heads_are_cut(ssdi8, b, L, H, K, V, dtype):
    d = ssdi8.AttnDims(b, L, H, H, H, K, V)
    assert ssdi8.linear_attention_workspace_size(d, dtype) > 0
    t = draw(L, b, L, H, H, H, K, V, dtype)
    check(ssdi8, t)
    check(ssdi8, t, [L - 700] + [3] * (b - 1))
    t["init"] = None
    a = check(ssdi8, t)
    for final in (True, False):   # with a workspace of the caller's, whatever it holds
        ws = torch.full((ssdi8.linear_attention_workspace_size(d, dtype),), 255, dtype=torch.uint8, device="cuda")
        o = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], workspace=ws, final_state=final)
        assert torch.equal(o["y"], a["y"]) and (not final or torch.equal(o["final_state"], a["final_state"]))


def test_no_tokens(ssdi8):
    t = draw(1, 2, 0, 2, 2, 2, 64, 40, F16)
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    assert out["y"].shape == (2, 0, 2, 40) and torch.equal(out["final_state"], t["init"])
    assert (ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"])["final_state"] == 0).all()
    t = draw(1, 0, 5, 2, 2, 2, 64, 40, F16)
    assert ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"])["y"].shape == (0, 5, 2, 40)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_strides(ssdi8, dtype):
    """q, k, v as columns of one projection's rows (at odd offsets), heads before tokens, one token for all."""
    b, L, H, K, V = 2, 70, 3, 40, 24
    t = draw(3, b, L, H, H, H, K, V, dtype)
    want = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"])
    wide = torch.full((b, L, 5 + H * (2 * K + V) + 3), float("nan"), dtype=dtype, device="cuda")
    at = 5
    cut = {}
    for name, n in (("q", K), ("k", K), ("v", V)):
        cut[name] = wide[..., at:at + H * n].unflatten(-1, (H, n))
        cut[name].copy_(t[name])
        at += H * n
    got = ssdi8.linear_attention(cut["q"], cut["k"], cut["v"], t["g"])
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["final_state"], want["final_state"])
    first = [t[n].transpose(1, 2).contiguous().transpose(1, 2) for n in ("q", "k", "v")]
    gw = torch.full((b, L, 2 * H), float("nan"), device="cuda")
    gw[..., 1:H + 1] = t["g"]
    got = ssdi8.linear_attention(*first, gw[..., 1:H + 1])
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["final_state"], want["final_state"])
    same = [t[n][:1, :1].expand(b, L, -1, -1) for n in ("q", "k", "v")]
    got = ssdi8.linear_attention(*same, t["g"])
    want = ssdi8.linear_attention(*(s.contiguous() for s in same), t["g"])
    assert torch.equal(got["y"], want["y"])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_scale_decays_and_range(ssdi8, dtype):
    t = draw(9, 1, 140, 2, 2, 2, 64, 32, dtype)
    check(ssdi8, t, scale=1.0)
    check(ssdi8, t, scale=-0.25)
    check(ssdi8, {**t, "g": None})
    check(ssdi8, {**t, "g": torch.tensor([0.0, -30.0]).cuda()})
    # values at both ends of what 16 bits hold: p, S and v enter the products in the type's range
    big = {k: x.clone() if x is not None else None for k, x in t.items()}
    big["q"] *= 100
    big["k"] *= 100
    big["v"] *= 1e-3
    check(ssdi8, big)
    small = {**t, "k": (t["k"].float() * 2e-3).to(dtype), "v": (t["v"].float() * 2e-3).to(dtype), "init": None}
    check(ssdi8, small)
    # no decay over a long sequence of alike tokens: a state beyond 65504
    one = draw(2, 1, 1300, 1, 1, 1, 32, 32, dtype, init=False)
    one["k"].fill_(8.0), one["v"].fill_(8.0), one["q"].fill_(0.01)
    check(ssdi8, {**one, "g": None})


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_a_decay_of_zero_starts_anew(ssdi8, dtype):
    t = draw(11, 1, 200, 2, 2, 2, 48, 40, dtype)
    t["g"][:, 77] = float("-inf")
    t["g"][:, 100, 0] = -1e30
    out = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    tail = {k: (x[:, 77:].contiguous() if k != "init" else None) for k, x in t.items()}
    y, e, S, es = R.attention(*(tail[k].double() for k in ("q", "k", "v")), tail["g"].clamp(min=-1e4), dtype=dtype)
    R.assert_within(out["y"][:, 77:], y.cpu(), R.rounded(dtype, y, e).cpu(), "y")
    R.assert_within(out["final_state"], S.cpu(), R.rounded(F32, S, es).cpu(), "state")
    s = t["init"].clone()
    y = ssdi8.linear_attention_step(t["q"][:, 0], t["k"][:, 0], t["v"][:, 0], s, torch.full((2,), -float("inf")).cuda())
    want = t["k"][0, 0].float()[..., None] * t["v"][0, 0].float()[:, None]
    assert torch.equal(s[0], want) and torch.isfinite(y).all()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("what", ["q", "k", "v", "g"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_values_that_are_no_numbers_reach_no_earlier_token(ssdi8, dtype, what, bad):
    if what == "g" and bad > 0:
        pytest.skip("decays are at most 0")
    t = draw(13, 2, 150, 2, 2, 2, 64, 72, dtype)
    want = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    at = 83
    broken = {k: x.clone() for k, x in t.items()}
    if what == "g":
        broken["g"][0, at, 1] = bad
    else:
        broken[what][0, at, 1, 5] = bad
    out = ssdi8.linear_attention(broken["q"], broken["k"], broken["v"], broken["g"], init_state=t["init"])
    same = torch.ones_like(want["y"], dtype=torch.bool)
    if what == "q":
        same[0, at, 1] = False
    elif what == "v":
        same[0, at:, 1, 5] = False
    else:
        same[0, at:, 1] = False
    # the sums over a chunk with such a value may be taken in another order elsewhere: equal all the same here
    assert torch.equal(out["y"][same], want["y"][same])
    assert not torch.isfinite(out["y"][~same]).any()
    fine = torch.isfinite(out["final_state"])
    assert fine[1].all() and fine[0, 0].all()
    if what == "v":
        assert not fine[0, 1, :, 5].any() and fine[0, 1, :, :5].all()
    if what == "q":
        assert fine.all()


STEPS = [(1, 1, 1, 1, 16, 16), (3, 2, 2, 2, 64, 64), (2, 1, 1, 4, 128, 64), (2, 6, 1, 2, 100, 72), (1, 2, 1, 1, 33, 1),
         (2, 1, 1, 1, 256, 130), (1, 4, 4, 4, 1, 67), (2, 3, 3, 3, 65, 3)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("b,Hq,Hk,Hv,K,V", STEPS)
def test_token(ssdi8, b, Hq, Hk, Hv, K, V, dtype):
    t = draw(K + V, b, None, Hq, Hk, Hv, K, V, dtype, token=K % 2 == 0)
    state = t["init"].clone()
    wide = torch.full((b, Hq * K + Hk * K + Hv * V + 7), float("nan"), dtype=dtype, device="cuda")
    q, k, v = (x.unflatten(-1, (-1, n)) for x, n in zip(wide[:, 7:].split((Hq * K, Hk * K, Hv * V), -1), (K, K, V)))
    q.copy_(t["q"]), k.copy_(t["k"]), v.copy_(t["v"])
    y = ssdi8.linear_attention_step(q, k, v, state, t["g"])
    g = t["g"][:, None] if t["g"].dim() == 2 else t["g"]
    Y, e, S, es = R.attention(*(t[n].double()[:, None] for n in ("q", "k", "v")), g, None, t["init"], dtype=F32)
    R.assert_within(y, Y[:, 0].cpu(), R.rounded(dtype, Y[:, 0], e[:, 0]).cpu(), "y")
    R.assert_within(state, S.cpu(), R.rounded(F32, S, es).cpu(), "state")


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompt_in_parts_and_tokens(ssdi8, dtype):
    """A prompt at once, in two parts, and its last tokens one by one leave the same state within the bounds."""
    t = draw(21, 2, 135, 2, 1, 2, 64, 64, dtype, init=False)
    whole = check(ssdi8, t)
    a = ssdi8.linear_attention(*(t[k][:, :70] for k in ("q", "k", "v", "g")))
    state = a["final_state"]
    b = ssdi8.linear_attention(*(t[k][:, 70:132] for k in ("q", "k", "v", "g")), init_state=state)
    y = [a["y"], b["y"]]
    state = b["final_state"]
    for i in range(132, 135):
        y.append(ssdi8.linear_attention_step(*(t[k][:, i] for k in ("q", "k", "v")), state, t["g"][:, i])[:, None])
    Y, e, S, es = R.attention(*(t[k].double() for k in ("q", "k", "v")), t["g"], dtype=dtype)
    R.assert_within(torch.cat(y, 1), Y.cpu(), R.rounded(dtype, Y, 2 * e).cpu(), "y")
    R.assert_within(state, S.cpu(), R.rounded(F32, S, 2 * es).cpu(), "state")
    assert whole["y"].shape == Y.shape


def test_state_in_place_and_streams(ssdi8):
    """final_state over init_state; the general form of the binding (a given stream) gives the same bits."""
    import ctypes
    t = draw(4, 2, 100, 2, 2, 2, 64, 64, F16)
    want = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"], stream=side)
    side.synchronize()
    assert torch.equal(got["y"], want["y"]) and torch.equal(got["final_state"], want["final_state"])
    with torch.cuda.stream(side):
        d, a, y = ssdi8._attention(t["q"], t["k"], t["v"], t["g"], None, None, None)
        state = t["init"].clone()
        a.init_state = a.final_state = state.data_ptr()
        assert ssdi8.lib().ssdi8_linear_attention(ctypes.byref(d), ctypes.byref(a), side.cuda_stream) == 0
    side.synchronize()
    assert torch.equal(y, want["y"]) and torch.equal(state, want["final_state"])


@pytest.mark.parametrize("L,Hq,Hk,Hv", [(2000, 1, 1, 1), (100, 4, 1, 2), (1500, 4, 2, 2), (0, 2, 1, 1)])
def test_state_in_place(ssdi8, L, Hq, Hk, Hv):
    """final_state over init_state where several spans, or several heads of y, begin from it."""
    import ctypes
    t = draw(L, 2, L, Hq, Hk, Hv, 64, 64, F16)
    want = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
    state = t["init"].clone()
    d, a, y = ssdi8._attention(t["q"], t["k"], t["v"], t["g"], None, None, None)
    a.init_state = a.final_state = state.data_ptr()
    need = ssdi8.linear_attention_workspace_size(d, F16)
    assert need >= state.numel() * 4
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), need
    assert ssdi8.lib().ssdi8_linear_attention(ctypes.byref(d), ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(y, want["y"]) and torch.equal(state, want["final_state"])
    assert (ws[need:] == 255).all()


def test_captured(ssdi8):
    """Two graphs with eager calls between their replays; each replay equals the eager result."""
    a, b = draw(7, 1, 1100, 2, 2, 2, 64, 64, F16), draw(8, 1, 1300, 1, 1, 2, 64, 64, BF16)
    states = [t["init"].clone() for t in (a, b)]

    def run(t, s):
        o = ssdi8.linear_attention(t["q"], t["k"], t["v"], t["g"], init_state=t["init"])
        y = ssdi8.linear_attention_step(t["q"][:, 0], t["k"][:, 0], t["v"][:, 0], s, t["g"][:, 0])
        return o["y"], o["final_state"], y

    want = [[x.clone() for x in run(t, s.clone())] for t, s in zip((a, b), states)]
    after = []
    for t, s in zip((a, b), states):
        c = s.clone()
        run(t, c)
        after.append(c)
    graphs, outs = [], []
    torch.cuda.synchronize()
    for t, s in zip((a, b), states):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(t, s))
        graphs.append(g)
    for _ in range(3):
        for i, t in enumerate((a, b)):
            states[i].copy_(t["init"])
            graphs[i].replay()
            run(t, t["init"].clone())
            torch.cuda.synchronize()
            assert all(torch.equal(x, w) for x, w in zip(outs[i], want[i]))
            assert torch.equal(states[i], after[i])


def test_refusals(ssdi8):
    t = draw(1, 2, 10, 2, 2, 2, 64, 64, F16)
    q, k, v, g = (t[n] for n in ("q", "k", "v", "g"))
    for bad in (dict(k=k.float()), dict(k=k[..., :32]), dict(v=v[:, :5]), dict(g=g.half()), dict(g=g[:, :5]),
                dict(q=q.transpose(-1, -2)), dict(q=q.cpu()), dict(v=v.cpu()), dict(q=q[0]), dict(g=g[0, 0, :1])):
        a = {**dict(q=q, k=k, v=v, g=g), **bad}
        with pytest.raises(ValueError):
            ssdi8.linear_attention(a["q"], a["k"], a["v"], a["g"])
    for bad in (dict(init_state=t["init"].half()), dict(init_state=t["init"][:1]), dict(lengths=torch.zeros(2).cuda()),
                dict(y=torch.empty(2, 10, 2, 64, device="cuda")), dict(scale="x")):
        with pytest.raises((ValueError, TypeError)):
            ssdi8.linear_attention(q, k, v, g, **bad)
    with pytest.raises(ssdi8.SSDi8Error):   # three heads of q for two of v
        ssdi8.linear_attention(q[:, :, :1].expand(-1, -1, 3, -1), k, v, g)
    with pytest.raises(ssdi8.SSDi8Error):
        ssdi8.linear_attention(torch.zeros(1, 2, 1, 257, dtype=F16, device="cuda"),
                               torch.zeros(1, 2, 1, 257, dtype=F16, device="cuda"), v[:1, :2, :1])
    with pytest.raises(ValueError):
        ssdi8.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], t["init"].half(), g[:, 0])
