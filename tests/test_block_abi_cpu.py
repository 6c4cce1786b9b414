"""The C ABI of the operators around the SSD layer on the CPU: struct layouts, and every refusal by its
status before anything is launched (no pointer given here is ever read)."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A16 = 1 << 20      # an aligned stand-in for a device address


@pytest.fixture(scope="module")
def ssdi8():
    from paper_2608_21952_amd import ssdi8 as s
    if not os.path.exists(s.LIB_PATH):
        from paper_2608_21952_amd.build import build
        build()
    s.lib()
    return s


@pytest.mark.parametrize("py,c", [("ConvArgs", "ssdi8_conv_args"), ("SelScanDims", "ssdi8_sel_scan_dims"),
                                  ("SelScanArgs", "ssdi8_sel_scan_args"), ("NormArgs", "ssdi8_norm_args"),
                                  ("LinearArgs", "ssdi8_linear_args")])
def test_structs_match_the_header(ssdi8, tmp_path, py, c):
    cls = getattr(ssdi8, py)
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(
        ['#include <stdio.h>', '#include <stddef.h>', '#include "ssdi8.h"', 'int main(void) {',
         f'printf("%zu\\n", sizeof({c}));']
        + [f'printf("%zu\\n", offsetof({c}, {f}));' for f in fields] + ["return 0; }"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    vals = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True,
                                           check=True).stdout.split()]
    assert vals[0] == ctypes.sizeof(cls)
    assert vals[1:] == [getattr(cls, f).offset for f in fields]


def changed(args, **k):
    new = type(args).from_buffer_copy(args)
    for name, v in k.items():
        if isinstance(v, tuple):
            for i, x in enumerate(v):
                getattr(new, name)[i] = x
        else:
            setattr(new, name, v)
    return new


def refusals(call, args, want):
    for status, k in want:
        assert call(changed(args, **k)) == status, k


def test_conv(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    a = s.ConvArgs(dtype=s.F16, x=A16, x_batch_stride=160, x_token_stride=16, weight=A16, width=4,
                   bias=A16, act=1, final_state=A16)
    a.y[0], a.y_cols[0] = A16, 16
    sizes = [2, 10, 16]
    call = lambda x, n=sizes: L.ssdi8_causal_conv(*n, ctypes.byref(x), None)
    want = [(s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(dtype=-1)), (s.ERR_ARG, dict(act=2)),
            (s.ERR_UNSUPPORTED, dict(width=1)), (s.ERR_UNSUPPORTED, dict(width=5)),
            (s.ERR_SHAPE, dict(x_batch_stride=-1)), (s.ERR_SHAPE, dict(y_cols=(8, 4, 0))),
            (s.ERR_SHAPE, dict(y_cols=(17, -1, 0))), (s.ERR_NULL, dict(y_cols=(8, 8, 0))),
            (s.ERR_NULL, dict(weight=None)), (s.ERR_NULL, dict(x=None)), (s.ERR_NULL, dict(y=(None,))),
            (s.ERR_ALIGN, dict(x=A16 + 1)), (s.ERR_ALIGN, dict(weight=A16 + 2)),
            (s.ERR_ALIGN, dict(lengths=A16 + 2)), (s.ERR_ALIGN, dict(final_state=A16 + 1))]
    refusals(call, a, want + [(s.ERR_SHAPE, dict(x_token_stride=-16))])
    refusals(lambda x: L.ssdi8_causal_conv_step(2, 16, ctypes.byref(x), None), a,
             want + [(s.ERR_NULL, dict(final_state=None))])
    for n in ([-1, 10, 16], [2, -1, 16], [2, 10, 0], [2, 10, (1 << 31) - 8], [1 << 31, 1, 16],
              [1 << 20, 1 << 30, 16]):
        assert call(a, n) == s.ERR_SHAPE, n
    assert L.ssdi8_causal_conv(2, 10, 16, None, None) == s.ERR_NULL
    assert call(a, [0, 10, 16]) == s.OK
    assert call(changed(a, final_state=None), [2, 0, 16]) == s.OK


def test_selective_scan(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    sizes = dict(batch=2, seqlen=10, nheads=16, headdim=4, ngroups=2, dstate=16)
    a = s.SelScanArgs(dtype=s.F16, dt_dtype=s.F32, dt_softplus=1)
    for f in ("u", "dt", "dt_bias", "A", "B", "C", "D", "z", "init_state", "y", "final_state"):
        setattr(a, f, A16)
    call = lambda x, f=L.ssdi8_selective_scan, **n: f(
        ctypes.byref(s.SelScanDims(**{**sizes, **n})), ctypes.byref(x), None)
    step = lambda x, **n: call(x, L.ssdi8_selective_scan_step, **n)
    want = [(s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(dt_dtype=s.BF16)),
            (s.ERR_SHAPE, dict(B_batch_stride=-1)), (s.ERR_ALIGN, dict(u=A16 + 1)),
            (s.ERR_ALIGN, dict(dt=A16 + 2)), (s.ERR_ALIGN, dict(final_state=A16 + 2))]
    want += [(s.ERR_NULL, {f: None}) for f in ("u", "dt", "A", "B", "C", "y")]
    refusals(call, a, want + [(s.ERR_SHAPE, dict(z_token_stride=-2)), (s.ERR_ALIGN, dict(lengths=A16 + 1))])
    refusals(step, a, want + [(s.ERR_ALIGN, dict(final_state=A16 + 8)), (s.ERR_NULL, dict(final_state=None))])
    bad = [dict(batch=-1), dict(seqlen=-1), dict(nheads=0), dict(headdim=0), dict(ngroups=0), dict(dstate=0),
           dict(ngroups=3), dict(nheads=1 << 20, headdim=1 << 12), dict(batch=1 << 30, seqlen=1 << 20)]
    for n in bad:
        assert call(a, **n) == s.ERR_SHAPE, n
        assert L.ssdi8_selective_scan_workspace_size(ctypes.byref(s.SelScanDims(**{**sizes, **n}))) == 0
        if "seqlen" not in n:
            assert step(a, **n) == s.ERR_SHAPE, n
    assert call(a, dstate=257) == step(a, dstate=257) == s.ERR_UNSUPPORTED
    assert L.ssdi8_selective_scan(None, ctypes.byref(a), None) == s.ERR_NULL
    assert call(a, batch=0) == step(a, batch=0) == s.OK
    # few channels over many tokens need a workspace: states and a decay per span and channel
    d = s.SelScanDims(**{**sizes, "seqlen": 100000})
    need = s.selective_scan_workspace_size(d)
    assert need > 0 and need % (4 * 2 * 64 * 17) == 0
    assert call(a, seqlen=100000) == s.ERR_WORKSPACE
    assert call(changed(a, workspace=A16, workspace_bytes=need - 1), seqlen=100000) == s.ERR_WORKSPACE
    assert s.selective_scan_workspace_size(s.SelScanDims(**{**sizes, "seqlen": 1})) == 0


def test_selective_scan_of_no_tokens(ssdi8):
    """The final state of no tokens is a launch like any other, which reads A: refused without it, while
    what belongs to tokens may be missing."""
    s, L = ssdi8, ssdi8.lib()
    for tied in (0, 1):
        d = s.SelScanDims(batch=2, seqlen=0, nheads=16, headdim=4, ngroups=2, dstate=16)
        a = s.SelScanArgs(dtype=s.F16, dt_dtype=s.F32, tied=tied, final_state=A16)
        call = lambda: L.ssdi8_selective_scan(ctypes.byref(d), ctypes.byref(a), None)
        assert call() == s.ERR_NULL
        a.final_state = None
        assert call() == s.OK      # nothing is done
        d.batch, a.final_state = 0, A16
        assert call() == s.OK


def test_gated_norm(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    a = s.NormArgs(dtype=s.F16, x=A16, x_row_stride=16, z=A16, z_row_stride=16, residual=A16, weight=A16,
                   eps=1e-5, y=A16, residual_out=A16)
    call = lambda x, n=(3, 16, 2): L.ssdi8_gated_norm(*n, ctypes.byref(x), None)
    refusals(call, a, [
        (s.ERR_ARG, dict(dtype=s.I8)), (s.ERR_ARG, dict(eps=-1.0)), (s.ERR_ARG, dict(eps=float("nan"))),
        (s.ERR_ARG, dict(eps=float("inf"))), (s.ERR_SHAPE, dict(x_row_stride=-1)),
        (s.ERR_NULL, dict(x=None)), (s.ERR_NULL, dict(weight=None)), (s.ERR_NULL, dict(y=None)),
        (s.ERR_NULL, dict(residual_out=None)), (s.ERR_ARG, dict(residual=None)),
        (s.ERR_ALIGN, dict(z=A16 + 1)), (s.ERR_ALIGN, dict(weight=A16 + 1))])
    for n in ((-1, 16, 2), (3, 0, 1), (3, 16, 3), (3, 16, 0), (1 << 30, 1 << 30, 1)):
        assert call(a, n) == s.ERR_SHAPE, n
    assert call(a, (3, 32769, 1)) == s.ERR_UNSUPPORTED
    assert call(a, (0, 16, 2)) == s.OK


def test_linear(ssdi8):
    s, L = ssdi8, ssdi8.lib()
    a = s.LinearArgs(dtype=s.I8, x=A16, x_row_stride=64, weight=A16, weight_row_stride=64, x_scale=A16,
                     weight_scale=A16, bias=A16, act=1, residual=A16, residual_row_stride=32, y=A16,
                     y_row_stride=32, y_dtype=s.F16)
    call = lambda x, n=(3, 32, 64): L.ssdi8_linear(*n, ctypes.byref(x), None)
    refusals(call, a, [
        (s.ERR_ARG, dict(dtype=s.F32)), (s.ERR_ARG, dict(dtype=4)), (s.ERR_ARG, dict(y_dtype=s.BF16)),
        (s.ERR_ARG, dict(act=4)), (s.ERR_ARG, dict(act=-1)), (s.ERR_ARG, dict(dtype=s.F16)),
        (s.ERR_SHAPE, dict(x_row_stride=-1)), (s.ERR_SHAPE, dict(y_row_stride=31)),
        (s.ERR_NULL, dict(x=None)), (s.ERR_NULL, dict(weight=None)), (s.ERR_NULL, dict(y=None)),
        (s.ERR_NULL, dict(x_scale=None)), (s.ERR_NULL, dict(weight_scale=None)),
        (s.ERR_ALIGN, dict(y=A16 + 1)), (s.ERR_ALIGN, dict(x_scale=A16 + 2))])
    for n in ((-1, 32, 64), (3, 0, 64), (3, 32, 0), (1 << 31, 32, 64), (1 << 30, 1 << 13, 64)):
        assert call(changed(a, y_row_stride=1 << 20), n) == s.ERR_SHAPE, n
    assert call(a, (3, 32, 131073)) == s.ERR_UNSUPPORTED
    assert call(changed(a, x_row_stride=1 << 24)) == s.ERR_UNSUPPORTED
    assert call(changed(a, weight_row_stride=1 << 24)) == s.ERR_UNSUPPORTED
    assert call(a, (0, 32, 64)) == s.OK
