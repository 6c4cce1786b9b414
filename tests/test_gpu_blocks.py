"""The blocks (blocks.py) against themselves and against 64 bits: a prompt in one go, in two pieces and
token by token is one sequence.

Tolerances (relative 2-norm): every fp16 result between the stages adds 2^-11 of its size at most: norm,
projection, convolution, time step, scan, norm, projection; the FP16 SSD layer rounds its operands
too (4 more).  12 x 2^-11 covers a block's branch, and the residual only lowers it.  int8 projections:
an eighth-bit code of values whose largest is about 4 standard deviations is off by 4 / 127 / sqrt(12) =
0.9 % of a standard deviation, the same for weights: sqrt(4) x 0.9 % over both projections' operands, held
to twice that."""
import pytest
import torch

import block_ref as R

pytestmark = pytest.mark.gpu
TOL, TOL8 = 12 * 2.0 ** -11, 0.036


@pytest.fixture(scope="module")
def blocks():
    from paper_2608_21952_amd import blocks as b, ssdi8
    ssdi8.lib()
    return b


def mamba2(seed, d=192, H=3, G=1, W=4):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    di, gn = 64 * H, 128 * G
    w = {"norm": 1 + n(d, scale=0.1), "in_proj": n(2 * di + 2 * gn, d, scale=d ** -0.5).half(),
         "dt_proj": n(H, d, scale=0.3 * d ** -0.5).half(), "dt_bias": n(H, scale=0.3) - 2,
         "conv": n(di + 2 * gn, W, scale=0.4), "conv_bias": n(di + 2 * gn, scale=0.1),
         "A": -torch.exp(2.7 * torch.rand(H, generator=g)), "D": 1 + n(H, scale=0.1),
         "gate_norm": 1 + n(di, scale=0.1), "out_proj": n(d, di, scale=di ** -0.5).half()}
    return w, {"nheads": H, "ngroups": G}


def mamba2_64(w, x, H, G):
    d64 = {k: v.double() for k, v in w.items()}
    B, L, d = x.shape
    di, gn = 64 * H, 128 * G
    norm = lambda v, wt, z=None: R.norm(v.reshape(B * L, -1), wt, None if z is None else z.reshape(B * L, -1),
                                        None, 1e-5, 1, False)[0].view(B, L, -1)
    h = norm(x, d64["norm"])
    zx = h @ d64["in_proj"].t()
    dt = h @ d64["dt_proj"].t() + d64["dt_bias"]
    c, _, conv = R.conv(zx[..., di:], w["conv"], w["conv_bias"], "silu", None, None)
    u, Bt, Ct = c.split((di, gn, gn), -1)
    y, _, state, _ = R.scan(u, dt, d64["A"], Bt.view(B, L, G, 128), Ct.view(B, L, G, 128), d64["D"], None, None,
                            True, None, None)
    return x + norm(y, d64["gate_norm"], zx[..., :di]) @ d64["out_proj"].t(), conv, state


def off(got, want):
    return ((got.double().cpu() - want.double().cpu()).norm() / want.double().cpu().norm()).item()


def cuda(w):
    return {k: v.cuda() for k, v in w.items()}


@pytest.mark.parametrize("L,int8", [(256, False), (300, False), (7, False), (300, True)])
def test_mamba2_block(blocks, L, int8):
    w, sizes = mamba2(L)
    block = blocks.Mamba2Block(cuda(w), int8=int8, **sizes)
    x = torch.randn(2, L + 2, 192, generator=torch.Generator().manual_seed(1)).half()
    want, conv, state = mamba2_64(w, x.double(), sizes["nheads"], sizes["ngroups"])
    tol = TOL8 if int8 else TOL
    y, cache = block.prefill(x[:, :L].cuda())
    assert off(y, want[:, :L]) < tol
    for t in range(L, L + 2):
        y = block.step(x[:, t].cuda(), cache)
        assert off(y, want[:, t]) < tol
    assert off(cache["state"], state) < tol and off(cache["conv"], conv) < tol
    # in two pieces
    k = 256 if L > 256 else L // 2
    _, first = block.prefill(x[:, :k].cuda())
    y, cache = block.prefill(x[:, k:].cuda(), first)
    assert off(y, want[:, k:]) < tol
    assert off(cache["state"], state) < tol


@pytest.mark.parametrize("int8", [False, True])
def test_mamba_block(blocks, int8):
    g = torch.Generator().manual_seed(3)
    n = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    d, di, N, rank, B, L = 160, 320, 16, 10, 3, 130
    w = {"norm": 1 + n(d, scale=0.1), "in_proj": n(2 * di, d, scale=d ** -0.5).half(),
         "conv": n(di, 4, scale=0.4), "conv_bias": n(di, scale=0.1),
         "x_proj": n(rank + 2 * N, di, scale=2 * di ** -0.5).half(),
         "dt_proj": n(di, rank, scale=0.3 * rank ** -0.5).half(), "dt_bias": n(di, scale=0.3) - 2,
         "A": -torch.exp(2.7 * torch.rand(di, N, generator=g)), "D": 1 + n(di, scale=0.1),
         "out_proj": n(d, di, scale=di ** -0.5).half()}
    block = blocks.MambaBlock(cuda(w), int8=int8)
    x = n(B, L + 1, d).half()
    d64 = {k: v.double() for k, v in w.items()}

    def reference(xs):
        b, l = xs.shape[:2]
        h = R.norm(xs.reshape(b * l, d), d64["norm"], None, None, 1e-5, 1, False)[0].view(b, l, d)
        xz = h @ d64["in_proj"].t()
        u, _, _ = R.conv(xz[..., :di], w["conv"], w["conv_bias"], "silu", None, None)
        p = u @ d64["x_proj"].t()
        y, _, s, _ = R.scan(u, p[..., :rank] @ d64["dt_proj"].t(), d64["A"], p[..., None, rank:rank + N],
                            p[..., None, rank + N:], d64["D"], xz[..., di:], d64["dt_bias"], True, None, None)
        return xs + y @ d64["out_proj"].t(), s

    tol = TOL8 if int8 else TOL
    lengths = [L, 41, 1]
    y, cache = block.prefill(x[:, :L].cuda(), lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    nxt = block.step(torch.stack([x[b, k] for b, k in enumerate(lengths)]).cuda(), cache)
    for b, k in enumerate(lengths):
        want, s = reference(x[b:b + 1, :k + 1].double())
        assert off(y[b:b + 1, :k], want[:, :k]) < tol
        assert off(nxt[b:b + 1], want[:, k]) < tol
        assert off(cache["state"][b:b + 1], s) < tol


def mamba(seed, d=96, di=160, N=16, rank=8):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    return {"norm": 1 + n(d, scale=0.1), "in_proj": n(2 * di, d, scale=d ** -0.5).half(),
            "conv": n(di, 4, scale=0.4), "conv_bias": n(di, scale=0.1),
            "x_proj": n(rank + 2 * N, di, scale=2 * di ** -0.5).half(),
            "dt_proj": n(di, rank, scale=0.3 * rank ** -0.5).half(), "dt_bias": n(di, scale=0.3) - 2,
            "A": -torch.exp(2.7 * torch.rand(di, N, generator=g)), "D": 1 + n(di, scale=0.1),
            "out_proj": n(d, di, scale=di ** -0.5).half()}


def no_tokens(blocks, kind, int8):
    """No tokens leave the cache's values, in memory of their own, or zeros; tokens go on from there."""
    if kind == "mamba2":
        w, sizes = mamba2(11)
        block, d = blocks.Mamba2Block(cuda(w), int8=int8, **sizes), 192
    else:
        block, d = blocks.MambaBlock(cuda(mamba(11)), int8=int8), 96
    x = torch.randn(2, 9, d, generator=torch.Generator().manual_seed(3)).half().cuda()
    none = x[:, :0]
    y, fresh = block.prefill(none)
    assert y.shape == none.shape and y.dtype == x.dtype
    assert not fresh["conv"].any() and not fresh["state"].any()
    # the first token on the empty cache is a prompt of one token
    got = block.step(x[:, 0], fresh)
    want, one = block.prefill(x[:, :1])
    assert off(got, want[:, 0]) < TOL and off(fresh["state"], one["state"]) < TOL
    # on a cache: its values, which a step on the new one leaves alone
    _, cache = block.prefill(x[:, :8].contiguous())
    held = {k: v.clone() for k, v in cache.items()}
    y, same = block.prefill(none, cache)
    assert y.shape == none.shape and all(torch.equal(same[k], held[k]) for k in held)
    block.step(x[:, 8], same)
    assert all(torch.equal(cache[k], held[k]) for k in held)


@pytest.mark.parametrize("kind", ["mamba2", "mamba"])
def test_prompt_of_no_tokens(blocks, kind):
    no_tokens(blocks, kind, False)


@pytest.mark.parametrize("kind", ["mamba2", "mamba"])
def test_prompt_of_no_tokens_int8(blocks, kind):
    no_tokens(blocks, kind, True)


@pytest.mark.parametrize("gate_groups", [2, 4])
def test_mamba2_block_with_a_grouped_gate_norm(blocks, gate_groups):
    """The norm behind the scan over groups of channels, as layers with several groups of B and C have it:
    prompt, tokens, and the 64-bit block with the same groups."""
    L, H, G = 260, 4, 2
    w, sizes = mamba2(7, H=H, G=G)
    block = blocks.Mamba2Block(cuda(w), gate_groups=gate_groups, **sizes)
    x = torch.randn(2, L + 1, 192, generator=torch.Generator().manual_seed(2)).half()
    want, _, state = mamba2_64_grouped(w, x.double(), H, G, gate_groups)
    y, cache = block.prefill(x[:, :L].cuda())
    assert off(y, want[:, :L]) < TOL
    assert off(block.step(x[:, L].cuda(), cache), want[:, L]) < TOL
    assert off(cache["state"], state) < TOL
    # without the option the norm is over all channels, as ever
    plain, _, _ = mamba2_64(w, x.double(), H, G)
    assert off(blocks.Mamba2Block(cuda(w), **sizes).prefill(x[:, :L].cuda())[0], plain[:, :L]) < TOL
    assert off(plain, want) > 2 * TOL   # the two are told apart
    with pytest.raises(ValueError, match="gate_groups"):
        blocks.Mamba2Block(cuda(w), gate_groups=3, **sizes)


def mamba2_64_grouped(w, x, H, G, groups):
    d64 = {k: v.double() for k, v in w.items()}
    B, L, _ = x.shape
    di, gn = 64 * H, 128 * G
    rows = lambda v: v.reshape(B * L, -1)
    h = R.norm(rows(x), d64["norm"], None, None, 1e-5, 1, False)[0].view(B, L, -1)
    zx = h @ d64["in_proj"].t()
    c, _, conv = R.conv(zx[..., di:], w["conv"], w["conv_bias"], "silu", None, None)
    u, Bt, Ct = c.split((di, gn, gn), -1)
    y, _, state, _ = R.scan(u, h @ d64["dt_proj"].t() + d64["dt_bias"], d64["A"], Bt.view(B, L, G, 128),
                            Ct.view(B, L, G, 128), d64["D"], None, None, True, None, None)
    y = R.norm(rows(y), d64["gate_norm"], rows(zx[..., :di]), None, 1e-5, groups, False)[0].view(B, L, di)
    return x + y @ d64["out_proj"].t(), conv, state
