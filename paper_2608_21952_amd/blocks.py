"""Blocks around the scan, as a program runs them: norm, input projection, causal convolution, scan,
gate, output projection with the residual; over prompts of any length and for single tokens.

    block = Mamba2Block(weights, nheads=24, ngroups=1)
    x, cache = block.prefill(x)            # (B, L, d)
    x = block.step(x_token, cache)         # (B, d); the cache is updated in place

Weights are a dict of device tensors: projections fp16 (outputs, inputs), everything else fp32.
LinearAttentionBlock holds its state by linear attention and takes its projections in few bits from the norms.
"""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from . import ssdi8


class Projection:
    """A projection's weights: fp16, or int8 with a step per output, its input then quantized per
    token."""

    def __init__(self, weight: torch.Tensor, int8: bool = False):
        self.weight, self.scale = weight.contiguous(), None
        if int8:
            amax = weight.float().abs().amax(1)
            self.scale = torch.where(amax > 0, amax / 127, torch.ones_like(amax))
            self.weight = (weight.float() / self.scale[:, None]).round().to(torch.int8)

    def __call__(self, x: torch.Tensor, **kw) -> torch.Tensor:
        if self.scale is None:
            return ssdi8.linear(x, self.weight, **kw)
        codes, steps = self.quantize(x)
        return ssdi8.linear(codes, self.weight, x_scale=steps, w_scale=self.scale, **kw)

    @staticmethod
    def quantize(x: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        rows = x.reshape(-1, 1, 1, x.shape[-1])
        if not rows.numel():   # the quantizer takes no NULL steps, and no rows have none
            return x.to(torch.int8), torch.empty(0, dtype=torch.float32, device=x.device)
        codes, steps = ssdi8.quantize_act(rows, "token")
        return codes.view(x.shape), steps


class Mamba2Block:
    """The SSD layer's block: x | B | C from one convolution, one decay per head, a gated norm behind
    the scan.  Whole chunks of a prompt run through the FP16 SSD layer, the rest through the selective
    scan from the state that they leave; both keep the state in fp32.  Activations are fp16, a batch's
    prompts of one length; int8 is that of the projections.

    weights: norm (d), in_proj (2 di + 2 G N, d) for z, x, B, C, dt_proj (H, d), dt_bias (H),
    conv (di + 2 G N, W), conv_bias, A (H), D (H), gate_norm (di), out_proj (d, di); di = H * 64.
    gate_groups: equal groups of channels that the norm behind the scan takes each by itself; 1, over all
    channels, unless said (models with several groups of B and C often have as many here)."""

    def __init__(self, weights: Dict[str, torch.Tensor], *, nheads: int, ngroups: int,
                 gate_groups: int = 1, int8: bool = False, eps: float = 1e-5):
        self.w, self.H, self.G, self.eps = weights, nheads, ngroups, eps
        if gate_groups < 1 or nheads * ssdi8.P_DIM % gate_groups:
            raise ValueError(f"gate_groups must divide the {nheads * ssdi8.P_DIM} channels, got {gate_groups}")
        self.gate_groups = gate_groups
        self.di, self.gn = nheads * ssdi8.P_DIM, ngroups * ssdi8.N_DIM
        self.in_proj = Projection(weights["in_proj"], int8)
        self.out_proj = Projection(weights["out_proj"], int8)

    def _front(self, x):
        h = ssdi8.gated_norm(x, self.w["norm"], eps=self.eps)["y"]
        zx = self.in_proj(h)
        dt = ssdi8.linear(h, self.w["dt_proj"], bias=self.w["dt_bias"], y_dtype=torch.float32)
        return zx[..., :self.di], zx[..., self.di:], dt

    def _back(self, y, z, x):
        y = ssdi8.gated_norm(y, self.w["gate_norm"], z=z, eps=self.eps,
                             groups=self.gate_groups)["y"]
        return self.out_proj(y, residual=x)

    def _groups(self, t):
        return t.view(*t.shape[:-1], self.G, ssdi8.N_DIM)

    def prefill(self, x: torch.Tensor, cache: Optional[Dict[str, torch.Tensor]] = None
                ) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        cache = cache or {}
        z, xbc, dt = self._front(x)
        c = ssdi8.causal_conv(xbc, self.w["conv"], bias=self.w["conv_bias"],
                              split=(self.di, self.gn, self.gn), init_state=cache.get("conv"))
        u, Bt, Ct = c["y"]
        B, L = x.shape[:2]
        whole = L // ssdi8.CHUNK * ssdi8.CHUNK
        y, state = torch.empty_like(u), cache.get("state")
        if whole:
            part = lambda t: t[:, :whole].contiguous()
            head = ssdi8.ssd_chunk_scan_fp16(
                part(u).view(B, whole, self.H, -1), part(dt), self.w["A"], self._groups(part(Bt)),
                self._groups(part(Ct)), D=self.w["D"],
                init_state=None if state is None else state.view(B, self.H, -1, ssdi8.N_DIM))
            y[:, :whole] = head["y"].view(B, whole, self.di)
            state = head["final_state"].view(B, self.di, ssdi8.N_DIM)
        if whole < L or not L:   # no tokens: the scan copies the cache's state, or gives zeros
            rest = lambda t: t[:, whole:]
            tail = ssdi8.selective_scan(rest(u), rest(dt), self.w["A"], self._groups(rest(Bt)),
                                        self._groups(rest(Ct)), D=self.w["D"], init_state=state)
            y[:, whole:] = tail["y"]
            state = tail["final_state"]
        return self._back(y, z, x), {"conv": c["final_state"], "state": state}

    def step(self, x: torch.Tensor, cache: Dict[str, torch.Tensor]) -> torch.Tensor:
        z, xbc, dt = self._front(x)
        u, Bt, Ct = ssdi8.causal_conv_step(xbc, self.w["conv"], cache["conv"],
                                           bias=self.w["conv_bias"], split=(self.di, self.gn, self.gn))
        y = ssdi8.selective_scan_step(u, dt, self.w["A"], self._groups(Bt), self._groups(Ct),
                                      cache["state"], D=self.w["D"])
        return self._back(y, z, x)


class MambaBlock:
    """The block with a time step and decays per channel and state, the gate inside the scan.

    weights: norm (d), in_proj (2 di, d) for x, z, conv (di, W), conv_bias, x_proj (R + 2 N, di) for the
    low-rank time step, B, C, dt_proj (di, R), dt_bias (di), A (di, N), D (di), out_proj (d, di)."""

    def __init__(self, weights: Dict[str, torch.Tensor], *, int8: bool = False, eps: float = 1e-5):
        self.w, self.eps = weights, eps
        self.di, self.N = weights["A"].shape
        self.R = weights["dt_proj"].shape[1]
        self.in_proj = Projection(weights["in_proj"], int8)
        self.out_proj = Projection(weights["out_proj"], int8)

    def _front(self, x):
        xz = self.in_proj(ssdi8.gated_norm(x, self.w["norm"], eps=self.eps)["y"])
        return xz[..., :self.di], xz[..., self.di:]

    def _selective(self, u):
        p = ssdi8.linear(u, self.w["x_proj"])
        dt = ssdi8.linear(p[..., :self.R], self.w["dt_proj"])
        Bt, Ct = (p[..., self.R + k * self.N:self.R + (k + 1) * self.N].unsqueeze(-2) for k in (0, 1))
        return u, dt, self.w["A"], Bt, Ct

    def prefill(self, x: torch.Tensor, cache: Optional[Dict[str, torch.Tensor]] = None,
                lengths: Optional[torch.Tensor] = None
                ) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """lengths: the sequences' own lengths in a batch padded to one; the cache is that of their
        ends."""
        cache = cache or {}
        u, z = self._front(x)
        c = ssdi8.causal_conv(u, self.w["conv"], bias=self.w["conv_bias"],
                              init_state=cache.get("conv"), lengths=lengths)
        s = ssdi8.selective_scan(*self._selective(c["y"]), D=self.w["D"], z=z,
                                 dt_bias=self.w["dt_bias"], init_state=cache.get("state"),
                                 lengths=lengths)
        return (self.out_proj(s["y"], residual=x),
                {"conv": c["final_state"], "state": s["final_state"]})

    def step(self, x: torch.Tensor, cache: Dict[str, torch.Tensor]) -> torch.Tensor:
        u, z = self._front(x)
        u = ssdi8.causal_conv_step(u, self.w["conv"], cache["conv"], bias=self.w["conv_bias"])
        y = ssdi8.selective_scan_step(*self._selective(u), cache["state"], D=self.w["D"], z=z,
                                      dt_bias=self.w["dt_bias"])
        return self.out_proj(y, residual=x)


class NormedProjection:
    """A projection behind the norm that quantizes its input: int8 with a step per row and per output, or weights in
    mxfp4 and inputs in mxfp8 or mxfp4; without a format all in fp16.

    norm gives the projection's input from a norm's arguments; with with_y also y in x's type."""

    def __init__(self, weight: torch.Tensor, format: Optional[str] = None):
        if format not in (None, "int8", "mxfp8", "mxfp4"):
            raise ValueError(f"format must be None, int8, mxfp8 or mxfp4, got {format!r}")
        self.format = format
        if format in (None, "int8"):
            p = Projection(weight, format == "int8")
            self.weight, self.scale = p.weight, p.scale
        else:
            self.weight, self.scale = ssdi8.quantize_mx(weight), None

    def norm(self, x: torch.Tensor, weight: torch.Tensor, *, with_y: bool = False, **kw) -> Dict[str, torch.Tensor]:
        if self.format is None:
            return ssdi8.gated_norm(x, weight, **kw)
        return ssdi8.norm_quantize(x, weight, format=self.format, with_y=with_y, **kw)

    def __call__(self, n: Dict[str, torch.Tensor], **kw) -> torch.Tensor:
        if self.format is None:
            return ssdi8.linear(n["y"], self.weight, **kw)
        if self.format == "int8":
            return ssdi8.linear(n["codes"], self.weight, x_scale=n["scales"], w_scale=self.scale, **kw)
        return ssdi8.linear_mx(ssdi8.Mx(n["codes"], n["scales"]), self.weight, **kw)


class LinearAttentionBlock:
    """Norm, projection to q, k, v and a gate, linear attention with a decay per head, gated norm per head, output
    projection with the residual.  Activations are fp16, the state (B, v_heads, keys, values) fp32.

    weights: norm (d), in_proj (heads * keys + key_heads * keys + v_heads * values + H * values, d) for q, k, v, the gate, with
    H = max(heads, v_heads), gate_norm (H * values), out_proj (d, H * values), and the decays: log_decay (v_heads), at
    most 0, or, per token, decay_proj (v_heads, d) and decay_bias, of which -softplus is taken.
    key_heads, v_heads: heads unless given.  format: that of the projections (NormedProjection)."""

    def __init__(self, weights: Dict[str, torch.Tensor], *, heads: int, keys: int, values: int,
                 key_heads: Optional[int] = None, v_heads: Optional[int] = None, format: Optional[str] = None,
                 eps: float = 1e-5):
        self.w, self.K, self.V, self.eps = weights, keys, values, eps
        self.heads = (heads, key_heads or heads, v_heads or heads)
        self.H = max(heads, self.heads[2])
        rows = (heads + self.heads[1]) * keys + (self.heads[2] + self.H) * values
        if weights["in_proj"].shape[0] != rows:
            raise ValueError(f"in_proj must have {rows} outputs, got {weights['in_proj'].shape[0]}")
        self.in_proj = NormedProjection(weights["in_proj"], format)
        self.out_proj = NormedProjection(weights["out_proj"], format)

    def _front(self, x):
        per_token = "decay_proj" in self.w
        n = self.in_proj.norm(x, self.w["norm"], eps=self.eps, with_y=per_token)
        p, at, out = self.in_proj(n), 0, []
        for heads, width in zip(self.heads, (self.K, self.K, self.V)):
            out.append(p[..., at:at + heads * width].unflatten(-1, (heads, width)))
            at += heads * width
        decay = self.w.get("log_decay")
        if per_token:
            decay = ssdi8.linear(n["y"], self.w["decay_proj"], bias=self.w["decay_bias"], activation="softplus",
                                 y_dtype=torch.float32).neg_()
        return (*out, decay), p[..., at:]

    def _back(self, y, z, x):
        n = self.out_proj.norm(y.flatten(-2), self.w["gate_norm"], z=z, eps=self.eps, groups=self.H)
        return self.out_proj(n, residual=x)

    def prefill(self, x: torch.Tensor, cache: Optional[Dict[str, torch.Tensor]] = None,
                lengths: Optional[torch.Tensor] = None
                ) -> Tuple[torch.Tensor, Dict[str, torch.Tensor]]:
        """lengths: the sequences' own lengths in a batch padded to one; the cache is that of their ends."""
        x = x.contiguous()
        qkv, z = self._front(x)
        a = ssdi8.linear_attention(*qkv, init_state=(cache or {}).get("state"), lengths=lengths)
        return self._back(a["y"], z, x), {"state": a["final_state"]}

    def step(self, x: torch.Tensor, cache: Dict[str, torch.Tensor]) -> torch.Tensor:
        x = x.contiguous()
        qkv, z = self._front(x)
        return self._back(ssdi8.linear_attention_step(*qkv[:3], cache["state"], qkv[3]), z, x)
