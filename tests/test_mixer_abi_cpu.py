"""The C ABI of linear attention, the quantizing norm and the microscaled products on the CPU: struct layouts, and
every refusal by its status before anything is launched (no pointer given here is ever read)."""
import ctypes

import pytest

from test_block_abi_cpu import A16, changed, refusals, ssdi8, test_structs_match_the_header as check_struct  # noqa: F401


@pytest.mark.parametrize("py,c", [("AttnDims", "ssdi8_attn_dims"), ("AttnArgs", "ssdi8_attn_args"),
                                  ("NormQuantArgs", "ssdi8_norm_quant_args"), ("LinearMxArgs", "ssdi8_linear_mx_args")])
def test_structs_match_the_header(ssdi8, tmp_path, py, c):
    check_struct(ssdi8, tmp_path, py, c)


def test_linear_attention(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    sizes = dict(batch=2, seqlen=10, q_heads=4, k_heads=1, v_heads=2, keys=64, values=48)
    a = s.AttnArgs(dtype=s.F16, scale=1.0, token_decay=1)
    for f in ("q", "k", "v", "log_decay", "init_state", "lengths", "y", "final_state"):
        setattr(a, f, A16)
    call = lambda x, f=L.ssdi8_linear_attention, **n: f(
        ctypes.byref(s.AttnDims(**{**sizes, **n})), ctypes.byref(x), None)
    step = lambda x, **n: call(x, L.ssdi8_linear_attention_step, **n)
    want = [(s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(dtype=-1)), (s.ERR_ARG, dict(scale=float("nan"))),
            (s.ERR_ARG, dict(scale=float("inf"))), (s.ERR_SHAPE, dict(q_batch_stride=-1)),
            (s.ERR_SHAPE, dict(k_head_stride=-1)), (s.ERR_SHAPE, dict(v_head_stride=(1 << 40) + 1)),
            (s.ERR_SHAPE, dict(decay_batch_stride=-1)), (s.ERR_ALIGN, dict(q=A16 + 1)), (s.ERR_ALIGN, dict(y=A16 + 1)),
            (s.ERR_ALIGN, dict(log_decay=A16 + 2)), (s.ERR_ALIGN, dict(final_state=A16 + 2))]
    want += [(s.ERR_NULL, {f: None}) for f in ("q", "k", "v", "y")]
    refusals(call, a, want + [(s.ERR_SHAPE, dict(q_token_stride=-2)), (s.ERR_SHAPE, dict(decay_token_stride=-1)),
                              (s.ERR_ALIGN, dict(lengths=A16 + 1)), (s.ERR_ALIGN, dict(init_state=A16 + 1))])
    refusals(step, a, want + [(s.ERR_NULL, dict(final_state=None))])
    size = lambda **n: L.ssdi8_linear_attention_workspace_size(ctypes.byref(s.AttnDims(**{**sizes, **n})), s.F16)
    bad = [dict(batch=-1), dict(seqlen=-1), dict(q_heads=0), dict(k_heads=0), dict(v_heads=0), dict(keys=0),
           dict(values=0), dict(q_heads=3), dict(v_heads=3), dict(k_heads=4), dict(q_heads=1, v_heads=3, k_heads=2),
           dict(batch=1 << 30, seqlen=1 << 20), dict(values=(1 << 31) - 1, batch=1 << 20), dict(batch=1 << 31)]
    for n in bad:
        assert call(a, **n) == s.ERR_SHAPE, n
        assert size(**n) == 0
        if "seqlen" not in n:
            assert step(a, **n) == s.ERR_SHAPE, n
    assert call(a, keys=257) == step(a, keys=257) == s.ERR_UNSUPPORTED
    # 64 tokens of 2e9 bytes or more; of one token alone no stride is used
    ws = dict(workspace=A16, workspace_bytes=1 << 40)
    for f in ("q_token_stride", "k_token_stride", "v_token_stride"):
        assert call(changed(a, **{f: 15_624_800}, **ws)) == s.ERR_UNSUPPORTED
        assert call(changed(a, **{f: 15_624_800}, **ws), batch=0, seqlen=1) == s.OK
    far = changed(a, v_head_stride=15_624_800 * 32, **ws)   # heads are taken two by two, of one token too
    assert call(far) == call(far, seqlen=1) == s.ERR_UNSUPPORTED
    assert call(far, batch=0, v_heads=1) == s.OK
    assert L.ssdi8_linear_attention(None, ctypes.byref(a), None) == s.ERR_NULL
    assert L.ssdi8_linear_attention(ctypes.byref(s.AttnDims(**sizes)), None, None) == s.ERR_NULL
    assert call(a, batch=0) == step(a, batch=0) == s.OK and size(batch=0) == size(batch=0, seqlen=1 << 20) == 0
    none = changed(a, q=None, k=None, v=None, y=None, final_state=None)
    assert call(none, seqlen=0) == s.OK and size(seqlen=0, q_heads=2) == 0
    # few heads over many tokens need a workspace: a state and a decay for every span but the last, and the states
    # once more; heads of y that share a state these alone
    need, states = size(seqlen=100000), 4 * 2 * 2 * 64 * 48
    assert need > states and (need - states) % (states + 4 * 2 * 2) == 0 and size(seqlen=100000, q_heads=2) > 0
    assert size(seqlen=10) == states and size(seqlen=10, q_heads=2) == 0
    assert call(a, seqlen=100000) == s.ERR_WORKSPACE
    assert call(changed(a, workspace=A16, workspace_bytes=need - 1), seqlen=100000) == s.ERR_WORKSPACE
    assert size(seqlen=1, q_heads=2) == 0
    assert L.ssdi8_linear_attention_workspace_size(ctypes.byref(s.AttnDims(**{**sizes, "seqlen": 100000})), s.I8) == 0
    assert L.ssdi8_linear_attention_workspace_size(None, s.F16) == 0


def test_norm_quantize(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    a = s.NormQuantArgs(dtype=s.BF16, eps=1e-5, format=s.FORMAT["mxfp8"], x=A16, x_row_stride=64, weight=A16, codes=A16,
                        scales=A16)
    call = lambda x, n=(4, 64, 2): L.ssdi8_norm_quantize(*n, ctypes.byref(x), None)
    refusals(call, a, [
        (s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(format=3)), (s.ERR_ARG, dict(format=-1)),
        (s.ERR_ARG, dict(eps=-1e-9)), (s.ERR_ARG, dict(eps=float("nan"))), (s.ERR_ARG, dict(eps=float("inf"))),
        (s.ERR_SHAPE, dict(x_row_stride=-1)), (s.ERR_SHAPE, dict(z_row_stride=-1)), (s.ERR_NULL, dict(x=None)),
        (s.ERR_NULL, dict(weight=None)), (s.ERR_NULL, dict(codes=None)), (s.ERR_NULL, dict(scales=None)),
        (s.ERR_NULL, dict(residual=A16)), (s.ERR_ARG, dict(residual_out=A16)), (s.ERR_ALIGN, dict(x=A16 + 1)),
        (s.ERR_ALIGN, dict(z=A16 + 1)), (s.ERR_ALIGN, dict(y=A16 + 1)), (s.ERR_ALIGN, dict(weight=A16 + 2)),
        (s.ERR_ALIGN, dict(format=0, scales=A16 + 2)), (s.ERR_ALIGN, dict(residual=A16 + 1, residual_out=A16))])
    for n in ((-1, 64, 1), (4, 0, 1), (4, 64, 0), (4, 64, 3), (1 << 31, 64, 1), (1 << 30, 32768, 1)):
        assert call(a, n) == s.ERR_SHAPE, n
    assert call(a, (4, 32776, 1)) == s.ERR_UNSUPPORTED
    assert call(a, (0, 64, 1)) == s.OK and L.ssdi8_norm_quantize(4, 64, 1, None, None) == s.ERR_NULL


def test_quantize_mx(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    good = dict(rows=4, k=40, x=A16, dtype=s.F16, stride=40, format=1, codes=A16, scales=A16)
    call = lambda **k: L.ssdi8_quantize_mx(*{**good, **k}.values(), None)
    for status, k in ((s.ERR_SHAPE, dict(rows=-1)), (s.ERR_SHAPE, dict(k=0)), (s.ERR_SHAPE, dict(rows=1 << 30, k=1 << 20)),
                      (s.ERR_SHAPE, dict(stride=-1)), (s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(format=0)),
                      (s.ERR_ARG, dict(format=3)), (s.ERR_NULL, dict(x=None)), (s.ERR_NULL, dict(codes=None)),
                      (s.ERR_NULL, dict(scales=None)), (s.ERR_ALIGN, dict(x=A16 + 1)), (s.OK, dict(rows=0))):
        assert call(**k) == status, k


def test_linear_mx(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    a = s.LinearMxArgs(x_format=1, x_codes=A16, x_scales=A16, weight_codes=A16, weight_scales=A16, act=1, y=A16,
                       y_row_stride=48, y_dtype=s.BF16)
    call = lambda x, n=(4, 48, 64): L.ssdi8_linear_mx(*n, ctypes.byref(x), None)
    refusals(call, a, [
        (s.ERR_ARG, dict(x_format=0)), (s.ERR_ARG, dict(x_format=3)), (s.ERR_ARG, dict(y_dtype=s.I8)),
        (s.ERR_ARG, dict(act=4)), (s.ERR_ARG, dict(act=-1)), (s.ERR_SHAPE, dict(y_row_stride=47)),
        (s.ERR_SHAPE, dict(residual_row_stride=-1)), (s.ERR_NULL, dict(x_codes=None)), (s.ERR_NULL, dict(x_scales=None)),
        (s.ERR_NULL, dict(weight_codes=None)), (s.ERR_NULL, dict(weight_scales=None)), (s.ERR_NULL, dict(y=None)),
        (s.ERR_ALIGN, dict(x_codes=A16 + 8)), (s.ERR_ALIGN, dict(weight_codes=A16 + 8)), (s.ERR_ALIGN, dict(y=A16 + 1)),
        (s.ERR_ALIGN, dict(bias=A16 + 2)), (s.ERR_ALIGN, dict(residual=A16 + 1))])
    for n in ((-1, 48, 64), (4, 0, 64), (4, 48, 0), (4, 48, 33), (1 << 31, 48, 64), (1 << 30, 48, 1 << 20)):
        assert call(a, n) == s.ERR_SHAPE, n
    assert call(a, (4, 48, 1 << 24)) == s.ERR_UNSUPPORTED
    assert call(a, (0, 48, 64)) == s.OK and L.ssdi8_linear_mx(4, 48, 64, None, None) == s.ERR_NULL


def test_binding_refuses_before_the_library(ssdi8):
    """CPU tensors and other arguments that no call takes."""
    import torch
    h = torch.zeros(2, 3, 2, 16, dtype=torch.float16)
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for bad in (lambda: ssdi8.linear_attention(h, h, h), lambda: ssdi8.linear_attention_step(h[0], h[0], h[0], h),
                lambda: ssdi8.norm_quantize(h, torch.zeros(16)), lambda: ssdi8.norm_quantize(h, torch.zeros(16), format="e4m3"),
                lambda: ssdi8.quantize_mx(h), lambda: ssdi8.quantize_mx(h, "int8"), lambda: ssdi8.linear_attention(None, h, h),
                lambda: ssdi8.linear_mx(ssdi8.Mx(codes, scales), ssdi8.Mx(codes, scales)),
                lambda: ssdi8.linear_mx(h, codes), lambda: ssdi8.linear_mx("x", ssdi8.Mx(codes, scales))):
        with pytest.raises(ValueError):
            bad()
