// Native argument marshalling of the Python binding (ssdi8.py): checks the tensors, allocates the
// outputs with PyTorch and calls the C ABI, for the calls a program makes per layer or per token.
// A small layer's kernels take 20 to 40 us; the same checks through Python objects and ctypes cost
// 12 us per quantize_act, 22 us per ssd_chunk_scan.
//
// Each entry returns None when an argument is not of the plain form it takes (wrong type, device,
// dtype, shape, layout; a tensor subclass; memory that cannot be allocated), before anything is
// launched: the caller then takes the Python path, which raises the error that belongs to it (or
// accepts what is allowed there).  The GIL is released during the library call.
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ssdi8.h"

namespace {

decltype(&ssdi8_quantize_act) g_quantize = nullptr;
decltype(&ssdi8_ssd_workspace_size) g_workspace_size = nullptr;
decltype(&ssdi8_ssd_chunk_scan) g_scan = nullptr;
decltype(&ssdi8_decode_step) g_decode = nullptr;
decltype(&ssdi8_causal_conv) g_conv = nullptr;
decltype(&ssdi8_causal_conv_step) g_conv_step = nullptr;
decltype(&ssdi8_selective_scan_workspace_size) g_sel_scan_size = nullptr;
decltype(&ssdi8_selective_scan) g_sel_scan = nullptr;
decltype(&ssdi8_selective_scan_step) g_sel_scan_step = nullptr;
decltype(&ssdi8_gated_norm) g_norm = nullptr;
decltype(&ssdi8_linear) g_linear = nullptr;
c10::DeviceType g_device = c10::DeviceType::CUDA;   // where its tensors live

// Thrown (and caught at the entry) for arguments that belong to the Python path.
struct NotPlain {};

struct Shape {
  int64_t v[5];
  int n;
  Shape(std::initializer_list<int64_t> l) : n((int)l.size()) { std::copy(l.begin(), l.end(), v); }
};

const at::Tensor& any_tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) throw NotPlain();
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || t.device().type() != g_device ||
      !t.is_contiguous())
    throw NotPlain();
  return t;
}
const at::Tensor& tensor(PyObject* o, at::ScalarType dtype) {
  const at::Tensor& t = any_tensor(o);
  if (t.scalar_type() != dtype) throw NotPlain();
  return t;
}
bool has_shape(const at::Tensor& t, const Shape& s) {
  return t.dim() == s.n && std::equal(s.v, s.v + s.n, t.sizes().begin());
}
void* shaped(PyObject* o, at::ScalarType dtype, const Shape& s) {
  const at::Tensor& t = tensor(o, dtype);
  if (!has_shape(t, s)) throw NotPlain();
  return t.data_ptr();
}
float* floats(PyObject* o, const Shape& s) {
  return static_cast<float*>(shaped(o, at::kFloat, s));
}
float* floats_or_null(PyObject* o, const Shape& s) { return o == Py_None ? nullptr : floats(o, s); }
int float_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kHalf) return SSDI8_F16;
  if (t.scalar_type() == at::kFloat) return SSDI8_F32;
  throw NotPlain();
}
int64_t integer(PyObject* o) {
  if (!PyLong_Check(o)) throw NotPlain();   // bool is a PyLong
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw NotPlain();
  return v;
}
// No GIL while this lives; it is back also where an exception leaves.
struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};
// An allocation may wait for the device, and the device for a host callback that takes the GIL.
at::Tensor empty(const at::Tensor& like, at::ScalarType dtype, std::initializer_list<int64_t> s) {
  NoGil no_gil;
  return at::empty(s, like.options().dtype(dtype).requires_grad(false));
}
// The library call.  Tensors are looked at before: data_ptr() throws for one without storage (a
// functorch wrapper).
template <typename F> ssdi8_status released(F&& f) {
  NoGil no_gil;
  return f();
}
template <typename F> PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (...) {   // NotPlain, c10 errors (allocation): the Python path decides
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}
void* stream_of(PyObject* o) { return reinterpret_cast<void*>((uintptr_t)integer(o)); }

// bind(quantize, workspace_size, scan, decode, device): the library's addresses and the type of the
// device its tensors live on
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  const char* device = n == 5 ? PyUnicode_AsUTF8(a[4]) : nullptr;
  if (!device) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "bind takes 4 addresses and a device");
    return nullptr;
  }
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  g_quantize = reinterpret_cast<decltype(g_quantize)>(p[0]);
  g_workspace_size = reinterpret_cast<decltype(g_workspace_size)>(p[1]);
  g_scan = reinterpret_cast<decltype(g_scan)>(p[2]);
  g_decode = reinterpret_cast<decltype(g_decode)>(p[3]);
  try {
    g_device = c10::Device(device).type();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
}

// quantize(src, gran, scale or None, out or None, stream) -> (status, out, scale)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !g_quantize) throw NotPlain();
    const at::Tensor& src = any_tensor(a[0]);
    const int code = float_code(src);
    if (src.dim() != 4) throw NotPlain();
    const int64_t b = src.size(0), l = src.size(1), k = src.size(2), m = src.size(3);
    const int gran = (int)integer(a[1]);
    int64_t ns;
    switch (gran) {
      case SSDI8_GRAN_TENSOR: ns = 1; break;
      case SSDI8_GRAN_GROUP: ns = k; break;
      case SSDI8_GRAN_CHANNEL: ns = k * m; break;
      case SSDI8_GRAN_TOKEN: ns = b * l * k; break;
      default: throw NotPlain();
    }
    const bool dynamic = a[2] == Py_None;
    at::Tensor scale = dynamic ? empty(src, at::kFloat, {ns}) : tensor(a[2], at::kFloat);
    if (scale.numel() != ns) throw NotPlain();
    at::Tensor out = a[3] == Py_None ? empty(src, at::kChar, {b, l, k, m}) : tensor(a[3], at::kChar);
    if (!has_shape(out, {b, l, k, m})) throw NotPlain();
    void* st = stream_of(a[4]);
    const void* from = src.data_ptr();
    float* steps = static_cast<float*>(scale.data_ptr());
    int8_t* to = static_cast<int8_t*>(out.data_ptr());
    const ssdi8_status s = released([&] {
      return g_quantize(from, code, b, l, k, m, gran, steps, dynamic ? 1 : 0, to, st);
    });
    return Py_BuildValue("(iNN)", (int)s, THPVariable_Wrap(out), THPVariable_Wrap(scale));
  });
}

// scan(x, dt, A, Bq, Cq, B, C, B_scale, C_scale, xs_scale, state_scale, cb_scale, D, corr, init,
//      y or None, y_dtype (-1: that of x), workspace or None, timeouts or None, dt_softplus,
//      chunk, decay_shift, shift_round, final_state, path, stream)
//   -> (status, y, final_state_q or None, final_state or None)
PyObject* scan(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 26 || !g_scan) throw NotPlain();
    ssdi8_scan_args a = {};
    const at::Tensor& x = any_tensor(o[0]);
    if (x.dim() != 4) throw NotPlain();
    const int64_t B = x.size(0), L = x.size(1), H = x.size(2), P = x.size(3);
    a.x = x.data_ptr();
    a.x_dtype = float_code(x);
    const bool quantized = o[3] != Py_None;
    if (quantized ? (o[4] == Py_None || o[6] != Py_None) : (o[5] == Py_None || o[6] == Py_None))
      throw NotPlain();
    const at::Tensor& b = any_tensor(o[quantized ? 3 : 5]);
    const at::Tensor& c = any_tensor(o[quantized ? 4 : 6]);
    if (b.dim() != 4 || c.scalar_type() != b.scalar_type()) throw NotPlain();
    const int64_t G = b.size(2), N = b.size(3);
    if (!has_shape(b, {B, L, G, N}) || !has_shape(c, {B, L, G, N})) throw NotPlain();
    if (quantized) {
      if (b.scalar_type() != at::kChar) throw NotPlain();
      a.Bq = static_cast<const int8_t*>(b.data_ptr());
      a.Cq = static_cast<const int8_t*>(c.data_ptr());
    } else {
      a.bc_dtype = float_code(b);
      a.B = b.data_ptr();
      a.C = c.data_ptr();
    }
    a.dt = floats(o[1], {B, L, H});
    a.A = floats(o[2], {H});
    a.B_scale = floats(o[7], {G});
    a.c_per_token = tensor(o[8], at::kFloat).dim() == 3;
    a.C_scale = a.c_per_token ? floats(o[8], {B, L, G}) : floats(o[8], {G});
    a.xs_per_head = tensor(o[9], at::kFloat).dim() == 1;
    a.xs_scale = a.xs_per_head ? floats(o[9], {H}) : floats(o[9], {H, P});
    a.state_scale = floats(o[10], {H, P});
    a.cb_scale = floats(o[11], {G});
    a.D = floats_or_null(o[12], {H});
    a.corr = floats_or_null(o[13], {H, P});
    if (o[14] != Py_None)
      a.init_state_q = static_cast<const int8_t*>(shaped(o[14], at::kChar, {B, H, P, N}));
    if (o[18] != Py_None) a.hand_off_timeouts = static_cast<int*>(shaped(o[18], at::kInt, {1}));
    a.dt_softplus = (int)integer(o[19]);
    const ssdi8_dims d = {B, L, H, P, G, N, integer(o[20])};
    a.decay_shift = (int)integer(o[21]);
    a.shift_round = (int)integer(o[22]);
    a.path = (int)integer(o[24]);
    void* st = stream_of(o[25]);
    // allocations last
    const int64_t yd = integer(o[16]);
    a.y_dtype = yd < 0 ? a.x_dtype : (int)yd;
    const at::ScalarType ydt = a.y_dtype == SSDI8_F16 ? at::kHalf : at::kFloat;
    at::Tensor y = o[15] == Py_None ? empty(x, ydt, {B, L, H, P}) : tensor(o[15], ydt);
    if (!has_shape(y, {B, L, H, P})) throw NotPlain();
    a.y = y.data_ptr();
    const int64_t need = (int64_t)g_workspace_size(&d);
    at::Tensor ws = o[17] == Py_None ? empty(x, at::kByte, {need > 1 ? need : 1})
                                     : tensor(o[17], at::kByte);
    a.workspace = ws.data_ptr();
    a.workspace_bytes = (size_t)ws.numel();
    at::Tensor fq, fs;
    if (integer(o[23])) {
      fq = empty(x, at::kChar, {B, H, P, N});
      fs = empty(x, at::kFloat, {B, H, P, N});
      a.final_state_q = static_cast<int8_t*>(fq.data_ptr());
      a.final_state = static_cast<float*>(fs.data_ptr());
    }
    const ssdi8_status s = released([&] { return g_scan(&d, &a, st); });
    auto wrap = [](const at::Tensor& t) {
      if (t.defined()) return THPVariable_Wrap(t);
      Py_INCREF(Py_None);
      return Py_None;
    };
    return Py_BuildValue("(iNNN)", (int)s, wrap(y), wrap(fq), wrap(fs));
  });
}

// decode(x, dt, A, Bq, Cq, B_scale, C_scale, xs_scale, state_scale, cb_scale, state_q, D, corr,
//        dt_softplus, decay_shift, shift_round, y or None, y_dtype (-1: that of x), stream)
//   -> (status, y)
PyObject* decode(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 19 || !g_decode) throw NotPlain();
    ssdi8_decode_args a = {};
    const at::Tensor& x = any_tensor(o[0]);
    if (x.dim() != 3) throw NotPlain();
    const int64_t B = x.size(0), H = x.size(1), P = x.size(2);
    a.x = x.data_ptr();
    a.x_dtype = float_code(x);
    const at::Tensor& b = tensor(o[3], at::kChar);
    if (b.dim() != 3) throw NotPlain();
    const int64_t G = b.size(1), N = b.size(2);
    a.Bq = static_cast<const int8_t*>(shaped(o[3], at::kChar, {B, G, N}));
    a.Cq = static_cast<const int8_t*>(shaped(o[4], at::kChar, {B, G, N}));
    a.dt = floats(o[1], {B, H});
    a.A = floats(o[2], {H});
    a.B_scale = floats(o[5], {G});
    a.c_per_token = tensor(o[6], at::kFloat).dim() == 2;
    a.C_scale = a.c_per_token ? floats(o[6], {B, G}) : floats(o[6], {G});
    a.xs_per_head = tensor(o[7], at::kFloat).dim() == 1;
    a.xs_scale = a.xs_per_head ? floats(o[7], {H}) : floats(o[7], {H, P});
    a.state_scale = floats(o[8], {H, P});
    a.cb_scale = floats(o[9], {G});
    a.state_q = static_cast<int8_t*>(shaped(o[10], at::kChar, {B, H, P, N}));
    a.D = floats_or_null(o[11], {H});
    a.corr = floats_or_null(o[12], {H, P});
    a.dt_softplus = (int)integer(o[13]);
    a.decay_shift = (int)integer(o[14]);
    a.shift_round = (int)integer(o[15]);
    void* st = stream_of(o[18]);
    const int64_t yd = integer(o[17]);
    a.y_dtype = yd < 0 ? a.x_dtype : (int)yd;
    const at::ScalarType ydt = a.y_dtype == SSDI8_F16 ? at::kHalf : at::kFloat;
    at::Tensor y = o[16] == Py_None ? empty(x, ydt, {B, H, P}) : tensor(o[16], ydt);
    if (!has_shape(y, {B, H, P})) throw NotPlain();
    a.y = y.data_ptr();
    const ssdi8_status s = released([&] { return g_decode(B, H, P, G, N, &a, st); });
    return Py_BuildValue("(iN)", (int)s, THPVariable_Wrap(y));
  });
}

// ------------------------------------------------------------------- around the layer in a block
// bind_block(conv, conv_step, sel_scan_workspace_size, sel_scan, sel_scan_step, norm, linear): the
// library's addresses, after bind
PyObject* bind_block(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind_block takes 7 addresses");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
  }
  g_conv = reinterpret_cast<decltype(g_conv)>(p[0]);
  g_conv_step = reinterpret_cast<decltype(g_conv_step)>(p[1]);
  g_sel_scan_size = reinterpret_cast<decltype(g_sel_scan_size)>(p[2]);
  g_sel_scan = reinterpret_cast<decltype(g_sel_scan)>(p[3]);
  g_sel_scan_step = reinterpret_cast<decltype(g_sel_scan_step)>(p[4]);
  g_norm = reinterpret_cast<decltype(g_norm)>(p[5]);
  g_linear = reinterpret_cast<decltype(g_linear)>(p[6]);
  Py_RETURN_NONE;
}

// A tensor whose last `dense` dimensions are dense, the others at any strides.
const at::Tensor& rows(PyObject* o, int dense = 1) {
  if (!THPVariable_CheckExact(o)) throw NotPlain();
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || t.device().type() != g_device || t.dim() < dense ||
      t.numel() == 0)
    throw NotPlain();
  int64_t want = 1;
  for (int k = 1; k <= dense; ++k) {
    if (t.size(-k) != 1 && t.stride(-k) != want) throw NotPlain();
    want *= t.size(-k);
  }
  return t;
}
const at::Tensor& rows(PyObject* o, at::ScalarType dtype, const Shape& s, int dense = 1) {
  const at::Tensor& t = rows(o, dense);
  if (t.scalar_type() != dtype || !has_shape(t, s)) throw NotPlain();
  return t;
}
int type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return SSDI8_F32;
    case at::kHalf: return SSDI8_F16;
    case at::kBFloat16: return SSDI8_BF16;
    case at::kChar: return SSDI8_I8;
    default: throw NotPlain();
  }
}
int activation_code(const at::Tensor& t) {
  const int c = type_code(t.scalar_type());
  if (c == SSDI8_I8) throw NotPlain();
  return c;
}
const int* ints_or_null(PyObject* o, const Shape& s) {
  return o == Py_None ? nullptr : static_cast<int*>(shaped(o, at::kInt, s));
}
PyObject* wrap_or_none(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}

// The arguments that both convolutions share; the outputs into y.
int conv_args(ssdi8_conv_args& a, const at::Tensor& x, PyObject* weight, PyObject* bias, PyObject* act,
              PyObject* split, at::Tensor* y) {
  const int64_t D = x.size(-1), B = x.size(0);
  const at::Tensor& w = tensor(weight, at::kFloat);
  if (w.dim() != 2 || w.size(0) != D) throw NotPlain();
  a.dtype = activation_code(x);
  a.x = x.data_ptr();
  a.x_batch_stride = x.stride(0);
  a.x_token_stride = x.dim() == 3 ? x.stride(1) : 0;
  a.weight = static_cast<float*>(w.data_ptr());
  a.width = (int)w.size(1);
  if (a.width < 2) throw NotPlain();
  a.bias = floats_or_null(bias, {D});
  a.act = (int)integer(act);
  int count = 1;
  if (split == Py_None) {
    a.y_cols[0] = D;
  } else {
    if (!PyTuple_CheckExact(split)) throw NotPlain();
    count = (int)PyTuple_GET_SIZE(split);
    if (count < 1 || count > 3) throw NotPlain();
    int64_t sum = 0;
    for (int i = 0; i < count; ++i) {
      a.y_cols[i] = integer(PyTuple_GET_ITEM(split, i));
      if (a.y_cols[i] < 0) throw NotPlain();
      sum += a.y_cols[i];
    }
    if (sum != D) throw NotPlain();
  }
  for (int i = 0; i < count; ++i) {
    y[i] = x.dim() == 3 ? empty(x, x.scalar_type(), {B, x.size(1), a.y_cols[i]})
                        : empty(x, x.scalar_type(), {B, a.y_cols[i]});
    a.y[i] = y[i].data_ptr();
  }
  return count;
}
PyObject* conv_outputs(PyObject* split, const at::Tensor* y, int count) {
  if (split == Py_None) return THPVariable_Wrap(y[0]);
  PyObject* t = PyTuple_New(count);
  if (!t) throw NotPlain();
  for (int i = 0; i < count; ++i) PyTuple_SET_ITEM(t, i, THPVariable_Wrap(y[i]));
  return t;
}

// conv(x, weight, bias, act, split, init, lengths, final_state, stream)
//   -> (status, y or a tuple, final_state or None)
PyObject* conv(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9 || !g_conv) throw NotPlain();
    ssdi8_conv_args a = {};
    const at::Tensor& x = rows(o[0]);
    if (x.dim() != 3) throw NotPlain();
    const int64_t B = x.size(0), L = x.size(1), D = x.size(2);
    void* st = stream_of(o[8]);
    at::Tensor y[3], last;
    const int count = conv_args(a, x, o[1], o[2], o[3], o[4], y);
    if (o[5] != Py_None) a.init_state = shaped(o[5], x.scalar_type(), {B, a.width - 1, D});
    a.lengths = ints_or_null(o[6], {B});
    if (integer(o[7])) {
      last = empty(x, x.scalar_type(), {B, a.width - 1, D});
      a.final_state = last.data_ptr();
    }
    const ssdi8_status s = released([&] { return g_conv(B, L, D, &a, st); });
    return Py_BuildValue("(iNN)", (int)s, conv_outputs(o[4], y, count), wrap_or_none(last));
  });
}

// conv_step(x, weight, state, bias, act, split, stream) -> (status, y or a tuple)
PyObject* conv_step(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 7 || !g_conv_step) throw NotPlain();
    ssdi8_conv_args a = {};
    const at::Tensor& x = rows(o[0]);
    if (x.dim() != 2) throw NotPlain();
    const int64_t B = x.size(0), D = x.size(1);
    void* st = stream_of(o[6]);
    at::Tensor y[3];
    const int count = conv_args(a, x, o[1], o[3], o[4], o[5], y);
    a.final_state = shaped(o[2], x.scalar_type(), {B, a.width - 1, D});
    const ssdi8_status s = released([&] { return g_conv_step(B, D, &a, st); });
    return Py_BuildValue("(iN)", (int)s, conv_outputs(o[5], y, count));
  });
}

// The arguments that both selective scans share: u, dt, A, B, C, D, z, dt_bias.
void sel_scan_args(ssdi8_sel_scan_dims& d, ssdi8_sel_scan_args& a, const at::Tensor& u, PyObject* const* o) {
  const bool step = u.dim() == 2;
  const at::Tensor& dt = rows(o[1]);
  const at::Tensor& B = rows(o[4], 2);
  if (dt.dim() != u.dim() || B.dim() != u.dim() + 1) throw NotPlain();
  const int64_t b = u.size(0), L = step ? 1 : u.size(1), ch = u.size(-1);
  const int64_t H = dt.size(-1), G = B.size(-2), N = B.size(-1);
  if (ch % H != 0) throw NotPlain();
  d = {b, L, H, ch / H, G, N};
  const at::ScalarType type = u.scalar_type();
  a.dtype = activation_code(u);
  if (dt.scalar_type() != type && dt.scalar_type() != at::kFloat) throw NotPlain();
  a.dt_dtype = type_code(dt.scalar_type());
  auto lead = [&](const at::Tensor& t) {
    if (t.size(0) != b || (!step && t.size(1) != L)) throw NotPlain();
  };
  auto token = [&](const at::Tensor& t) { return step ? (int64_t)0 : t.stride(1); };
  lead(dt);
  lead(B);
  const at::Tensor& C = step ? rows(o[5], type, {b, G, N}, 2) : rows(o[5], type, {b, L, G, N}, 2);
  if (B.scalar_type() != type) throw NotPlain();
  a.u = u.data_ptr(), a.u_batch_stride = u.stride(0), a.u_token_stride = token(u);
  a.dt = dt.data_ptr(), a.dt_batch_stride = dt.stride(0), a.dt_token_stride = token(dt);
  a.B = B.data_ptr(), a.B_batch_stride = B.stride(0), a.B_token_stride = token(B);
  a.C = C.data_ptr(), a.C_batch_stride = C.stride(0), a.C_token_stride = token(C);
  if (o[7] != Py_None) {
    const at::Tensor& z = step ? rows(o[7], type, {b, ch}) : rows(o[7], type, {b, L, ch});
    a.z = z.data_ptr(), a.z_batch_stride = z.stride(0), a.z_token_stride = token(z);
  }
  a.tied = tensor(o[2], at::kFloat).dim() == 1;
  a.A = a.tied ? floats(o[2], {H}) : floats(o[2], {ch, N});
  a.D = floats_or_null(o[6], {H});
  a.dt_bias = floats_or_null(o[8], {H});
  a.dt_softplus = (int)integer(o[9]);
}

// sel_scan(u, dt, A, None, B, C, D, z, dt_bias, dt_softplus, init, lengths, final_state, stream)
//   -> (status, y, final_state or None)
PyObject* sel_scan(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 14 || !g_sel_scan) throw NotPlain();
    const at::Tensor& u = rows(o[0]);
    if (u.dim() != 3) throw NotPlain();
    ssdi8_sel_scan_dims d;
    ssdi8_sel_scan_args a = {};
    sel_scan_args(d, a, u, o);
    const int64_t ch = u.size(2);
    a.init_state = floats_or_null(o[10], {d.batch, ch, d.dstate});
    a.lengths = ints_or_null(o[11], {d.batch});
    void* st = stream_of(o[13]);
    at::Tensor y = empty(u, u.scalar_type(), {d.batch, d.seqlen, ch}), last, ws;
    a.y = y.data_ptr();
    if (integer(o[12])) {
      last = empty(u, at::kFloat, {d.batch, ch, d.dstate});
      a.final_state = static_cast<float*>(last.data_ptr());
    }
    const size_t need = g_sel_scan_size(&d);
    if (need) {
      ws = empty(u, at::kByte, {(int64_t)need});
      a.workspace = ws.data_ptr();
      a.workspace_bytes = need;
    }
    const ssdi8_status s = released([&] { return g_sel_scan(&d, &a, st); });
    return Py_BuildValue("(iNN)", (int)s, THPVariable_Wrap(y), wrap_or_none(last));
  });
}

// sel_scan_step(u, dt, A, state, B, C, D, z, dt_bias, dt_softplus, stream) -> (status, y)
PyObject* sel_scan_step(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 11 || !g_sel_scan_step) throw NotPlain();
    const at::Tensor& u = rows(o[0]);
    if (u.dim() != 2) throw NotPlain();
    ssdi8_sel_scan_dims d;
    ssdi8_sel_scan_args a = {};
    sel_scan_args(d, a, u, o);
    a.final_state = floats(o[3], {d.batch, u.size(1), d.dstate});
    void* st = stream_of(o[10]);
    at::Tensor y = empty(u, u.scalar_type(), {d.batch, u.size(1)});
    a.y = y.data_ptr();
    const ssdi8_status s = released([&] { return g_sel_scan_step(&d, &a, st); });
    return Py_BuildValue("(iN)", (int)s, THPVariable_Wrap(y));
  });
}

// The rows of a tensor: their number, and the stride that they share.
struct Flat {
  int64_t count = 1, stride = 0;
  explicit Flat(const at::Tensor& t) {
    if (t.dim() < 2) throw NotPlain();
    int64_t at = -1;   // what the next outer dimension's stride has to be
    for (int64_t k = t.dim() - 2; k >= 0; --k) {
      if (t.size(k) == 1) continue;
      if (at < 0) stride = t.stride(k);
      else if (t.stride(k) != at) throw NotPlain();
      at = t.stride(k) * t.size(k);
      count *= t.size(k);
    }
  }
};
at::Tensor empty_like_rows(const at::Tensor& t, at::ScalarType dtype, int64_t cols) {
  c10::SmallVector<int64_t, 5> s(t.sizes().begin(), t.sizes().end());
  s.back() = cols;
  NoGil no_gil;
  return at::empty(s, t.options().dtype(dtype).requires_grad(false));
}
bool same_lead(const at::Tensor& a, const at::Tensor& b) {
  return a.dim() == b.dim() && std::equal(a.sizes().begin(), a.sizes().end() - 1, b.sizes().begin());
}

// norm(x, weight, z, residual, eps, groups, norm_before_gate, y, residual_out, stream)
//   -> (status, y, residual_out or None)
PyObject* norm(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !g_norm) throw NotPlain();
    const at::Tensor& x = rows(o[0]);
    const Flat f(x);
    const int64_t D = x.size(-1);
    ssdi8_norm_args a = {};
    a.dtype = activation_code(x);
    a.x = x.data_ptr();
    a.x_row_stride = f.stride;
    a.weight = floats(o[1], {D});
    if (o[2] != Py_None) {
      const at::Tensor& z = rows(o[2]);
      if (z.scalar_type() != x.scalar_type() || !z.sizes().equals(x.sizes())) throw NotPlain();
      a.z = z.data_ptr();
      a.z_row_stride = Flat(z).stride;
    }
    if (!PyFloat_Check(o[4])) throw NotPlain();
    a.eps = (float)PyFloat_AS_DOUBLE(o[4]);
    const int64_t groups = integer(o[5]);
    a.norm_before_gate = (int)integer(o[6]);
    auto dense = [&](PyObject* t) -> const at::Tensor& {
      const at::Tensor& v = tensor(t, x.scalar_type());
      if (!v.sizes().equals(x.sizes())) throw NotPlain();
      return v;
    };
    void* st = stream_of(o[9]);
    at::Tensor sum;
    if (o[3] != Py_None) {
      a.residual = dense(o[3]).data_ptr();
      sum = o[8] == Py_None ? empty_like_rows(x, x.scalar_type(), D) : dense(o[8]);
      a.residual_out = sum.data_ptr();
    } else if (o[8] != Py_None) {
      throw NotPlain();
    }
    at::Tensor y = o[7] == Py_None ? empty_like_rows(x, x.scalar_type(), D) : dense(o[7]);
    a.y = y.data_ptr();
    const ssdi8_status s = released([&] { return g_norm(f.count, D, groups, &a, st); });
    return Py_BuildValue("(iNN)", (int)s, THPVariable_Wrap(y), wrap_or_none(sum));
  });
}

// linear(x, weight, bias, act, residual, x_scale, w_scale, y_dtype (-1: its own), stream) -> (status, y)
PyObject* linear(PyObject*, PyObject* const* o, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 9 || !g_linear) throw NotPlain();
    const at::Tensor& x = rows(o[0]);
    const at::Tensor& w = rows(o[1]);
    const Flat f(x);
    const int64_t K = x.size(-1);
    if (w.dim() != 2 || w.size(1) != K || w.scalar_type() != x.scalar_type()) throw NotPlain();
    const int64_t O = w.size(0);
    ssdi8_linear_args a = {};
    a.dtype = type_code(x.scalar_type());
    if (a.dtype == SSDI8_F32) throw NotPlain();
    const bool quantized = a.dtype == SSDI8_I8;
    if (quantized != (o[5] != Py_None) || quantized != (o[6] != Py_None)) throw NotPlain();
    a.x = x.data_ptr();
    a.x_row_stride = f.stride;
    a.weight = w.data_ptr();
    a.weight_row_stride = w.stride(0);
    if (quantized) {
      const at::Tensor& xs = tensor(o[5], at::kFloat);
      if (xs.numel() != f.count) throw NotPlain();
      a.x_scale = static_cast<float*>(xs.data_ptr());
      a.weight_scale = floats(o[6], {O});
    }
    a.bias = floats_or_null(o[2], {O});
    a.act = (int)integer(o[3]);
    const int64_t yd = integer(o[7]);
    const int own = quantized ? (int)SSDI8_F16 : a.dtype;
    a.y_dtype = yd < 0 ? own : (int)yd;
    if (a.y_dtype != SSDI8_F32 && a.y_dtype != own) throw NotPlain();
    const at::ScalarType ydt = a.y_dtype == SSDI8_F32 ? at::kFloat
                               : a.y_dtype == SSDI8_F16 ? at::kHalf : at::kBFloat16;
    if (o[4] != Py_None) {
      const at::Tensor& r = rows(o[4]);
      if (r.scalar_type() != ydt || r.size(-1) != O || !same_lead(r, x)) throw NotPlain();
      a.residual = r.data_ptr();
      a.residual_row_stride = Flat(r).stride;
    }
    void* st = stream_of(o[8]);
    at::Tensor y = empty_like_rows(x, ydt, O);
    a.y = y.data_ptr();
    a.y_row_stride = O;
    const ssdi8_status s = released([&] { return g_linear(f.count, O, K, &a, st); });
    return Py_BuildValue("(iN)", (int)s, THPVariable_Wrap(y));
  });
}

#define SSDI8_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL
PyMethodDef methods[] = {
    {"bind", SSDI8_FAST(bind), "bind(quantize_act, ssd_workspace_size, ssd_chunk_scan, decode_step, device)"},
    {"quantize", SSDI8_FAST(quantize), "ssdi8_quantize_act"},
    {"scan", SSDI8_FAST(scan), "ssdi8_ssd_chunk_scan"},
    {"decode", SSDI8_FAST(decode), "ssdi8_decode_step"},
    {"bind_block", SSDI8_FAST(bind_block),
     "bind_block(causal_conv, causal_conv_step, selective_scan_workspace_size, selective_scan, "
     "selective_scan_step, gated_norm, linear)"},
    {"conv", SSDI8_FAST(conv), "ssdi8_causal_conv"},
    {"conv_step", SSDI8_FAST(conv_step), "ssdi8_causal_conv_step"},
    {"sel_scan", SSDI8_FAST(sel_scan), "ssdi8_selective_scan"},
    {"sel_scan_step", SSDI8_FAST(sel_scan_step), "ssdi8_selective_scan_step"},
    {"norm", SSDI8_FAST(norm), "ssdi8_gated_norm"},
    {"linear", SSDI8_FAST(linear), "ssdi8_linear"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
