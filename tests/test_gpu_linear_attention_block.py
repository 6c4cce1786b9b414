"""LinearAttentionBlock against 64 bits: a prompt in one go, in two pieces, in a padded batch and token by token is one
sequence; captured into a graph.

The reference takes the weights' codes and quantizes its own norms as the format says.  Tolerances (relative 2-norm):
fp16 results between the stages add 2^-11 of their size each: projection, q k products, their products with v, y, norm,
projection, as for the other blocks 12 x 2^-11 in all.  A value in front of the second projection is off by up to e =
6 x 2^-11 then, and goes to the neighbouring code with probability e / s where s is the codes' distance relative to it: off by
sqrt(e s) in the 2-norm.  s of e2m1 is up to 1/2, of e4m3 1/8, of int8 4 / 127 where a row's largest is 4 deviations."""
import pytest
import torch

import mixer_ref as R

pytestmark = pytest.mark.gpu
BASE = 12 * 2.0 ** -11
TOL = {None: BASE, **{f: BASE + (6 * 2.0 ** -11 * s) ** 0.5 for f, s in (("int8", 4 / 127), ("mxfp8", 1 / 8), ("mxfp4", 1 / 2))}}
FORMATS = [None, "int8", "mxfp8", "mxfp4"]


@pytest.fixture(scope="module")
def blocks():
    from paper_2608_21952_amd import blocks as b, ssdi8
    ssdi8.lib()
    return b


def weights(seed, d, heads, key_heads, v_heads, K, V, per_token):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0: scale * torch.randn(*s, generator=g)
    H = max(heads, v_heads)
    w = {"norm": 1 + n(d, scale=0.1),
         "in_proj": n((heads + key_heads) * K + (v_heads + H) * V, d, scale=d ** -0.5).half(),
         "gate_norm": 1 + n(H * V, scale=0.1), "out_proj": n(d, H * V, scale=(H * V) ** -0.5).half()}
    if per_token:
        w |= {"decay_proj": n(v_heads, d, scale=0.3 * d ** -0.5).half(), "decay_bias": n(v_heads, scale=0.3) - 2}
    else:
        w["log_decay"] = -torch.exp(n(v_heads) - 2)
    return {k: v.cuda() for k, v in w.items()}


def matrix(p):
    """A projection's weights in 64 bits."""
    if p.format == "int8":
        return (p.weight.double() * p.scale.double()[:, None]).cpu()
    return p.weight.double().cpu() if p.format is None else R.values(p.weight.codes.cpu(), p.weight.scales.cpu(), "mxfp4")


def coded(y, format):
    """Rows in 64 bits as the projection gets them, filled up to whole blocks."""
    if format is None:
        return y
    if format == "int8":
        step = y.abs().amax(-1, keepdim=True) / 127
        step = torch.where(step == 0, torch.ones_like(step), step)
        return (y / step).round() * step
    return R.values(*R.quantize_mx(y.float().double(), format), format)


def block_64(block, x):
    (Hq, Hk, Hv), K, V, H, w = block.heads, block.K, block.V, block.H, {k: v.double().cpu() for k, v in block.w.items()}
    B, L, d = x.shape
    f = block.in_proj.format
    norm = lambda v, wt, z=None, groups=1: R.norm(v.reshape(B * L, -1), wt, z, None, 1e-5, groups, False)[0]
    n = norm(x, w["norm"])
    p = (coded(n, f) @ matrix(block.in_proj).T).view(B, L, -1)
    q, k, v, z = p.split((Hq * K, Hk * K, Hv * V, H * V), -1)
    g = w["log_decay"].expand(B, L, Hv) if "log_decay" in w else \
        -R.softplus(n @ w["decay_proj"].T + w["decay_bias"]).view(B, L, Hv)
    y, _, S, _ = R.attention(q.reshape(B, L, Hq, K), k.reshape(B, L, Hk, K), v.reshape(B, L, Hv, V), g)
    n = norm(y, w["gate_norm"], z.reshape(B * L, -1), H)
    return x + (coded(n, f) @ matrix(block.out_proj).T).view(B, L, d), S


def off(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


SIZES = [  # d, heads, key_heads, v_heads, K, V, decays per token
    (192, 4, 4, 4, 64, 64, False), (160, 4, 2, 2, 128, 72, True), (200, 2, 2, 6, 33, 48, True), (256, 1, 1, 1, 256, 128, False),
]


@pytest.mark.parametrize("format", FORMATS)
@pytest.mark.parametrize("d,heads,key_heads,v_heads,K,V,per_token", SIZES)
def test_block(blocks, d, heads, key_heads, v_heads, K, V, per_token, format):
    block = blocks.LinearAttentionBlock(weights(d, d, heads, key_heads, v_heads, K, V, per_token), heads=heads, keys=K,
                                        values=V, key_heads=key_heads, v_heads=v_heads, format=format)
    B, L = 3, 150
    x = torch.randn(B, L + 2, d, generator=torch.Generator().manual_seed(1)).half().cuda()
    want, state = block_64(block, x.double().cpu())
    tol = TOL[format]
    y, cache = block.prefill(x[:, :L])
    assert off(y, want[:, :L]) < tol
    for t in (L, L + 1):
        assert off(block.step(x[:, t], cache), want[:, t]) < tol
    assert off(cache["state"], state) < tol
    # in two pieces
    _, first = block.prefill(x[:, :70].contiguous())
    y, cache = block.prefill(x[:, 70:].contiguous(), first)
    assert off(y, want[:, 70:]) < tol and off(cache["state"], state) < tol
    # a padded batch, and a token behind each end
    lengths = [L, 0, 65]
    y, cache = block.prefill(x[:, :L].contiguous(), lengths=torch.tensor(lengths, dtype=torch.int32).cuda())
    nxt = block.step(torch.stack([x[b, k] for b, k in enumerate(lengths)]), cache)
    for b, k in enumerate(lengths):
        if k:
            assert off(y[b, :k], want[b, :k]) < tol
        assert off(nxt[b], want[b, k]) < tol


@pytest.mark.parametrize("format", FORMATS)
def test_no_tokens(blocks, format):
    block = blocks.LinearAttentionBlock(weights(3, 96, 2, 2, 2, 32, 48, True), heads=2, keys=32, values=48, format=format)
    x = torch.randn(2, 9, 96, generator=torch.Generator().manual_seed(3)).half().cuda()
    y, fresh = block.prefill(x[:, :0])
    assert y.shape == (2, 0, 96) and y.dtype == x.dtype and not fresh["state"].any()
    _, cache = block.prefill(x[:, :8].contiguous())
    held = cache["state"].clone()
    _, same = block.prefill(x[:, :0], cache)
    assert torch.equal(same["state"], held)
    block.step(x[:, 8], same)
    assert torch.equal(cache["state"], held) and not torch.equal(same["state"], held)


@pytest.mark.parametrize("format", FORMATS)
def test_captured(blocks, format):
    """A prompt and tokens behind it in one graph, replayed with eager calls between, twice over on one state."""
    block = blocks.LinearAttentionBlock(weights(5, 128, 2, 1, 2, 64, 64, True), heads=2, key_heads=1, keys=64, values=64,
                                        format=format)
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(2, 200, 128, generator=gen).half().cuda()
    token = torch.randn(2, 128, generator=gen).half().cuda()

    def run():
        y, cache = block.prefill(x)
        return y, block.step(token, cache), block.step(token, cache), cache["state"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(3):
        x.copy_(torch.randn(2, 200, 128, generator=gen).half())
        token.copy_(torch.randn(2, 128, generator=gen).half())
        want = [t.clone() for t in run()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_refusals(blocks):
    w = weights(3, 96, 2, 2, 2, 32, 48, False)
    with pytest.raises(ValueError, match="format"):
        blocks.LinearAttentionBlock(w, heads=2, keys=32, values=48, format="fp8")
    with pytest.raises(ValueError, match="in_proj"):
        blocks.LinearAttentionBlock(w, heads=3, keys=32, values=48)
