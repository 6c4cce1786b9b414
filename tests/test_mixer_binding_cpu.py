"""The native marshalling of linear attention, the quantizing norm and the microscaled products on the CPU: a second
copy of the module, bound to stand-ins of the library's functions and to CPU tensors.  What reaches the library is what
the tensors say; anything that is not of the plain form comes back as None with no call made."""
import os
import subprocess
import sys

from paper_2608_21952_amd import build as libbuild

PROGRAM = r"""
import ctypes, importlib.machinery, importlib.util, shutil, sys, tempfile
import torch
from paper_2608_21952_amd import ssdi8 as S

path = shutil.copy(sys.argv[1], tempfile.mkdtemp())
loader = importlib.machinery.ExtensionFileLoader("_binding", path)
native = importlib.util.module_from_spec(importlib.util.spec_from_loader("_binding", loader))
loader.exec_module(native)
i64, ptr, i32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
F = ctypes.CFUNCTYPE
nothing = F(i32, ptr)(lambda a: 0)
at = lambda f: ctypes.cast(f, ptr).value
native.bind(*[at(nothing)] * 4, "cpu")
seen = []
def keep(name, cls, sizes, dims=None):
    def call(*a):
        args = cls.from_buffer_copy(ctypes.cast(a[sizes], ctypes.POINTER(cls)).contents)
        n = a[:sizes] if dims is None else [getattr(dims.from_address(a[0]), f[0]) for f in dims._fields_]
        seen.append((name, list(n), args))
        return 0
    return call
size = F(ctypes.c_size_t, ptr, i32)(lambda d, t: 80 + t)
attn = F(i32, ptr, ptr, ptr)(keep("attention", S.AttnArgs, 1, S.AttnDims))
step = F(i32, ptr, ptr, ptr)(keep("step", S.AttnArgs, 1, S.AttnDims))
norm = F(i32, i64, i64, i64, ptr, ptr)(keep("norm", S.NormQuantArgs, 3))
quant = F(i32, i64, i64, ptr, i32, i64, i32, ptr, ptr, ptr)(lambda *a: seen.append(("quant", list(a), None)) or 0)
linear = F(i32, i64, i64, i64, ptr, ptr)(keep("linear", S.LinearMxArgs, 3))
for bad in ([at(attn)] * 5, [at(attn)] * 5 + [0]):
    try:
        native.bind_mixer(*bad)
    except (TypeError, ValueError):
        pass
    else:
        raise AssertionError(bad)
native.bind_mixer(*(at(f) for f in (size, attn, step, norm, quant, linear)))
h = lambda *s: torch.zeros(*s, dtype=torch.float16)
f = lambda *s: torch.zeros(*s)
last = lambda: seen[-1]

wide = h(2, 5, 100)
q, k, v = wide[..., 4:36].unflatten(-1, (4, 8)), wide[..., 36:52].unflatten(-1, (2, 8)), wide[..., 60:72].unflatten(-1, (4, 3))
g = f(2, 5, 9)[..., 2:6]
n32 = torch.zeros(2, dtype=torch.int32)
r = native.attention(q, k, v, g, None, f(2, 4, 8, 3), n32, 1, 0)
name, n, a = last()
assert r[0] == 0 and r[1].shape == (2, 5, 4, 3) and r[1].dtype == torch.float16 and r[2].shape == (2, 4, 8, 3)
assert n == [2, 5, 4, 2, 4, 8, 3] and a.dtype == S.F16 and abs(a.scale - 8 ** -0.5) < 1e-7
assert (a.q_batch_stride, a.q_token_stride, a.q_head_stride) == (500, 100, 8) and a.q == q.data_ptr()
assert (a.v_batch_stride, a.v_token_stride, a.v_head_stride) == (500, 100, 3) and a.k_head_stride == 8
assert (a.token_decay, a.decay_batch_stride, a.decay_token_stride) == (1, 45, 9) and a.log_decay == g.data_ptr()
assert a.workspace_bytes == 80 + S.F16 and a.workspace and a.lengths == n32.data_ptr() and a.final_state == r[2].data_ptr()
r = native.attention(q, k, v[:, :, :2], f(2), 0.5, None, None, 0, 0)
name, n, a = last()
assert r[2] is None and r[1].shape == (2, 5, 4, 3) and n[4] == 2 and a.token_decay == 0 and a.scale == 0.5
st = f(2, 4, 8, 3)
r = native.attention_step(q[:, 1], k[:, 1], v[:, 1], g[:, 1], None, st, 0)
name, n, a = last()
assert name == "step" and r[1].shape == (2, 4, 3) and a.final_state == st.data_ptr() and a.decay_batch_stride == 45
x = wide[..., 10:60]
r = native.norm_quantize(x, f(50), wide[..., :50], h(2, 5, 50), 1e-6, 5, 1, 2, 1, None, 0)
name, n, a = last()
assert n == [10, 50, 5] and (a.x_row_stride, a.z_row_stride, a.format, a.norm_before_gate) == (100, 100, 2, 1)
assert r[1].shape == (2, 5, 32) and r[1].dtype == torch.uint8 and r[2].shape == (2, 5, 2) and r[2].dtype == torch.float8_e8m0fnu
assert r[3].shape == r[4].shape == (2, 5, 50) and a.y == r[3].data_ptr()
r = native.norm_quantize(x, f(50), None, None, 1e-6, 1, 0, 0, 0, None, 0)
assert r[1].shape == (2, 5, 50) and r[1].dtype == torch.int8 and r[2].shape == (2, 5) and r[2].dtype == torch.float32
assert r[3] is None and r[4] is None and not last()[2].y
r = native.quantize_mx(x, 1, 0)
assert last()[1][:2] == [10, 50] and last()[1][4] == 100 and r[1].shape == (2, 5, 64) and r[1].dtype == torch.float8_e4m3fn
w, ws = torch.zeros(7, 32, dtype=torch.uint8), torch.zeros(7, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
res = h(2, 5, 9)[..., :7]
y = native.linear_mx(r[1], r[2], w, ws, f(7), 1, res, S.F16, 0)
name, n, a = last()
assert n == [10, 7, 64] and a.x_format == 1 and (a.residual_row_stride, a.y_row_stride, a.act) == (9, 7, 1)
assert y[1].shape == (2, 5, 7) and a.weight_scales == ws.data_ptr()

count = len(seen)
no = [
    native.attention(q.transpose(-1, -2), k, v, None, None, None, None, 1, 0),
    native.attention(q, k.float(), v, None, None, None, None, 1, 0),
    native.attention(q, k[..., :7], v, None, None, None, None, 1, 0),
    native.attention(q, k[:, :4], v, None, None, None, None, 1, 0),
    native.attention(q, k, v, f(3), None, None, None, 1, 0),
    native.attention(q, k, v, g.half(), None, None, None, 1, 0),
    native.attention(q, k, v, g[:, :4], None, None, None, 1, 0),
    native.attention(q, k, v, g, 1, None, None, 1, 0),
    native.attention(q, k, v, g, None, f(2, 4, 8, 4), None, 1, 0),
    native.attention(q[0], k[0], v[0], None, None, None, None, 1, 0),
    native.attention_step(q[:, 1], k[:, 1], v[:, 1], g[:, 1], None, f(2, 4, 8, 4), 0),
    native.norm_quantize(x, f(50), None, None, 1e-6, 1, 0, 3, 0, None, 0),
    native.norm_quantize(x, f(50), None, None, 1e-6, 1, 0, 1, 0, h(2, 5, 50), 0),
    native.norm_quantize(x, h(50), None, None, 1e-6, 1, 0, 1, 0, None, 0),
    native.norm_quantize(x[:, :0], f(50), None, None, 1e-6, 1, 0, 1, 0, None, 0),
    native.quantize_mx(x, 0, 0),
    native.quantize_mx(x.to(torch.int8), 1, 0),
    native.linear_mx(r[1], r[2], r[1][0], ws, None, 0, None, S.F16, 0),
    native.linear_mx(r[1], ws, w, ws, None, 0, None, S.F16, 0),
    native.linear_mx(r[1], r[2], w, ws[:6], None, 0, None, S.F16, 0),
    native.linear_mx(r[1], r[2], w, ws, None, 0, f(2, 5, 7), S.F16, 0),
    native.linear_mx(r[1], r[2], w, ws, None, 0, None, S.I8, 0),
    native.linear_mx(r[1][..., :63], r[2], w, ws, None, 0, None, S.F16, 0),
    native.linear_mx(r[1], r[2].view(torch.uint8), w, ws, None, 0, None, S.F16, 0),
]
assert no == [None] * len(no), no
assert len(seen) == count
print("done")
"""


def test_native_marshalling():
    if not os.path.exists(libbuild.BINDING):
        libbuild.build()
    r = subprocess.run([sys.executable, "-c", PROGRAM, libbuild.BINDING], capture_output=True, text=True,
                       timeout=300, cwd=libbuild.ROOT)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), \
        (r.returncode, r.stdout[-500:], r.stderr[-2000:])
