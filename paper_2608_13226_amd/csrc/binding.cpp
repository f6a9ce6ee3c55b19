// The compiled half of the serving operators' Python binding: argument checks,
// outputs and the call into the C-ABI.  A decode step makes a handful of calls
// of a few microseconds of GPU time each, so the host's share of each counts;
// in Python the checks and allocations alone took longer than the kernels.
//
// Host code only.  Every function takes its arguments by position (the Python
// wrappers in serving.py give them names and defaults), returns new references
// and raises: TypeError for types, ValueError for shapes, strides and places,
// CoverPruneError for what the library refuses.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>

#include <cmath>
#include <cstdarg>

#include "../../include/coverprune.h"

namespace {

using at::ScalarType;
using at::Tensor;

PyObject* g_error = nullptr;        // CoverPruneError
PyObject* g_raw_stream = nullptr;   // device index -> current stream's handle
PyObject* g_device = nullptr;       // -> current device's index

constexpr ScalarType kE4m3 = ScalarType::Float8_e4m3fn;

// Thrown with the Python error already set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  PyErr_SetString(type, buf);
  throw Raised();
}

void check(cp_status st) {
  if (st != CP_OK) raise(g_error, "%s: %s", coverprune_status_string(st), coverprune_last_error());
}

// The operators have no backward pass: what they would cut from a graph is refused.
const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a torch.Tensor", name);
  const Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && at::GradMode::is_enabled())
    raise(PyExc_ValueError, "%s requires a gradient, which this operator does not give: detach it, or call under torch.no_grad()", name);
  return t;
}

// A tensor argument that may be None (an undefined tensor then).
Tensor maybe(PyObject* o, const char* name) { return o == Py_None ? Tensor() : tensor(o, name); }

std::string shown(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

void need_type(const Tensor& t, const char* name, ScalarType type) {
  if (t.scalar_type() != type) raise(PyExc_TypeError, "%s must be %s, got %s", name, c10::toString(type), c10::toString(t.scalar_type()));
}

void need_device(const Tensor& t, const char* name, at::Device dev) {
  if (t.device() != dev) raise(PyExc_ValueError, "%s must be on %s, got %s", name, dev.str().c_str(), t.device().str().c_str());
}

void need(const Tensor& t, const char* name, ScalarType type, at::IntArrayRef shape, at::Device dev) {
  need_type(t, name, type);
  if (t.sizes() != shape) raise(PyExc_ValueError, "%s must have shape %s, got %s", name, shown(shape).c_str(), shown(t.sizes()).c_str());
  need_device(t, name, dev);
  if (!t.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous", name);
}

bool half_type(ScalarType t) { return t == ScalarType::BFloat16 || t == ScalarType::Half; }

cp_dtype code(ScalarType t) {
  switch (t) {
    case ScalarType::BFloat16: return CP_BF16;
    case ScalarType::Half: return CP_F16;
    case ScalarType::Float: return CP_F32;
    default: return CP_E4M3;
  }
}

// An output: the caller's, checked, or a new one.
Tensor output(PyObject* o, const char* name, ScalarType type, at::IntArrayRef shape, at::Device dev) {
  if (o == Py_None) return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
  Tensor t = tensor(o, name);
  need(t, name, type, shape, dev);
  return t;
}

// The call has written t (where it is defined): autograd then knows that what it
// has kept of t is gone.
void written(const Tensor& t) {
  if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

template <class T>
T* at_of(const Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

int64_t integer(PyObject* o, const char* name) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    raise(PyExc_TypeError, "%s must be an integer of 64 bits", name);
  }
  return v;
}

double number(PyObject* o, const char* name) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    raise(PyExc_TypeError, "%s must be a number", name);
  }
  return v;
}

bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}

// The current stream of the tensors' GPU, which has to be the current one: that is
// where the library launches.  Everything is checked by then, so a host pointer
// never reaches a kernel.
void* stream_of(at::Device dev) {
  if (!dev.is_cuda()) raise(PyExc_ValueError, "tensors must be on the GPU, got %s", dev.str().c_str());
  PyObject* current = PyObject_CallNoArgs(g_device);
  if (!current) throw Raised();
  const long now = PyLong_AsLong(current);
  Py_DECREF(current);
  if (now == -1 && PyErr_Occurred()) throw Raised();
  if (now != dev.index()) raise(PyExc_ValueError, "tensors must be on the current GPU, %ld, got %s", now, dev.str().c_str());
  PyObject* index = PyLong_FromLong(dev.index());
  if (!index) throw Raised();
  PyObject* s = PyObject_CallOneArg(g_raw_stream, index);
  Py_DECREF(index);
  if (!s) throw Raised();
  void* p = PyLong_AsVoidPtr(s);
  Py_DECREF(s);
  if (!p && PyErr_Occurred()) throw Raised();
  return p;
}

PyObject* wrap(const Tensor& t) {
  if (!t.defined()) Py_RETURN_NONE;
  PyObject* o = THPVariable_Wrap(t);
  if (!o) throw Raised();
  return o;
}

// x, weight, eps, residual, quantize, out, out_scale, residual_out -> (out, scale, residual)
PyObject* rms_norm(PyObject* const* a) {
  const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
  const double eps = number(a[2], "eps");
  const Tensor r = maybe(a[3], "residual");
  const bool quantize = truth(a[4]);
  if (x.dim() != 2) raise(PyExc_ValueError, "x must be [rows, d]");
  const int64_t rows = x.size(0), d = x.size(1);
  const at::Device dev = x.device();
  const ScalarType t = x.scalar_type();
  if (!half_type(t) && t != ScalarType::Float) raise(PyExc_TypeError, "x must be bfloat16, float16 or float32, got %s", c10::toString(t));
  need(x, "x", t, {rows, d}, dev);
  need(w, "weight", t, {d}, dev);
  if (r.defined()) need(r, "residual", t, {rows, d}, dev);
  const ScalarType ot = quantize ? kE4m3 : t;
  const Tensor out = output(a[5], "out", ot, {rows, d}, dev);
  const Tensor scale = quantize ? output(a[6], "out_scale", ScalarType::Float, {rows}, dev) : Tensor();
  const Tensor ro = r.defined() ? output(a[7], "residual_out", t, {rows, d}, dev) : Tensor();
  check(coverprune_rms_norm(x.data_ptr(), code(t), rows, d, at_of<void>(r), w.data_ptr(), float(eps), out.data_ptr(), code(ot),
                            at_of<float>(scale), at_of<void>(ro), stream_of(dev)));
  written(out), written(scale), written(ro);
  PyObject* o = PyTuple_New(3);
  if (!o) throw Raised();
  PyTuple_SET_ITEM(o, 0, wrap(out));
  PyTuple_SET_ITEM(o, 1, wrap(scale));
  PyTuple_SET_ITEM(o, 2, wrap(ro));
  return o;
}

// The type an out_dtype argument (a torch.dtype or None) names.
ScalarType dtype_of(PyObject* o, ScalarType otherwise) {
  if (o == Py_None) return otherwise;
  if (!THPDtype_Check(o)) raise(PyExc_TypeError, "out_dtype must be a torch.dtype");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}

// x, weight, scale, zero, x_scale, out_dtype, out -> out
PyObject* w4_matvec(PyObject* const* a) {
  const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight"), &s = tensor(a[2], "scale");
  const Tensor z = maybe(a[3], "zero"), xs = maybe(a[4], "x_scale");
  if (x.dim() != 2 || w.dim() != 2 || s.dim() != 2) raise(PyExc_ValueError, "x, weight and scale must be matrices");
  const int64_t m = x.size(0), k = x.size(1), n = s.size(0), groups = s.size(1);
  const at::Device dev = x.device();
  const ScalarType t = s.scalar_type(), xt = x.scalar_type();
  if (!half_type(t)) raise(PyExc_TypeError, "scale must be bfloat16 or float16, got %s", c10::toString(t));
  if (xt != t && xt != kE4m3) raise(PyExc_TypeError, "x must be %s or %s, got %s", c10::toString(t), c10::toString(kE4m3), c10::toString(xt));
  if (groups < 1 || k % groups != 0) raise(PyExc_ValueError, "scale has %lld groups for k = %lld", (long long)groups, (long long)k);
  need(x, "x", xt, {m, k}, dev);
  need(w, "weight", ScalarType::Byte, {n, k / 2}, dev);
  need(s, "scale", t, {n, groups}, dev);
  if (z.defined()) need(z, "zero", ScalarType::Byte, {n, groups}, dev);
  if (xs.defined() != (xt == kE4m3)) raise(PyExc_ValueError, "x_scale goes with an 8-bit x, and only with it");
  if (xs.defined()) need(xs, "x_scale", ScalarType::Float, {m}, dev);
  const ScalarType yt = dtype_of(a[5], t);
  if (yt != t && yt != ScalarType::Float) raise(PyExc_TypeError, "out_dtype must be %s or Float, got %s", c10::toString(t), c10::toString(yt));
  const Tensor y = output(a[6], "out", yt, {m, n}, dev);
  check(coverprune_w4_matvec(x.data_ptr(), code(xt), at_of<float>(xs), at_of<uint8_t>(w), s.data_ptr(), at_of<uint8_t>(z), m, n, k,
                             k / groups, code(t), y.data_ptr(), code(yt), stream_of(dev)));
  written(y);
  return wrap(y);
}

// A [tokens, heads, d] view whose heads are contiguous; its head count and token stride.
void heads_of(const Tensor& x, const char* name, ScalarType t, int64_t tokens, int64_t d, at::Device dev, int64_t* heads,
              int64_t* stride) {
  if (x.dim() != 3 || x.size(0) != tokens || x.size(2) != d)
    raise(PyExc_ValueError, "%s must be [%lld, heads, %lld], got %s", name, (long long)tokens, (long long)d, shown(x.sizes()).c_str());
  need_type(x, name, t);
  need_device(x, name, dev);
  *heads = x.size(1);
  if ((x.stride(2) != 1 && d > 1) || (x.stride(1) != d && *heads > 1))
    raise(PyExc_ValueError, "%s: a token's heads must be contiguous", name);
  *stride = tokens < 2 ? *heads * d : x.stride(0);
  if (*stride < *heads * d) raise(PyExc_ValueError, "%s: tokens overlap", name);
}

struct Caches {
  ScalarType type;
  int64_t pages, page;
};
Caches caches_of(const Tensor& kc, const Tensor& vc, ScalarType t, int64_t hk, int64_t d, at::Device dev, const Tensor& ks,
                 const Tensor& vs) {
  if (kc.dim() != 4) raise(PyExc_ValueError, "the caches must be [pages, heads, page_size, d]");
  const Caches c = {kc.scalar_type(), kc.size(0), kc.size(2)};
  if (c.type != t && c.type != kE4m3)
    raise(PyExc_TypeError, "the caches must be %s or %s, got %s", c10::toString(t), c10::toString(kE4m3), c10::toString(c.type));
  need(kc, "k_cache", c.type, {c.pages, hk, c.page, d}, dev);
  need(vc, "v_cache", c.type, {c.pages, hk, c.page, d}, dev);
  if ((ks.defined() || vs.defined()) && c.type != kE4m3) raise(PyExc_ValueError, "k_scale and v_scale go with 8-bit caches");
  if (ks.defined()) need(ks, "k_scale", ScalarType::Float, {hk}, dev);
  if (vs.defined()) need(vs, "v_scale", ScalarType::Float, {hk}, dev);
  return c;
}

// q, k, v, positions, slots, inv_freq, k_cache, v_cache, interleaved, magnitude, k_scale, v_scale, q_out -> q_out
PyObject* kv_append(PyObject* const* a) {
  const Tensor q = maybe(a[0], "q");
  const Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &pos = tensor(a[3], "positions"), &slots = tensor(a[4], "slots");
  const Tensor inv = maybe(a[5], "inv_freq");
  const Tensor &kc = tensor(a[6], "k_cache"), &vc = tensor(a[7], "v_cache");
  const bool inter = truth(a[8]);
  const double magnitude = number(a[9], "magnitude");
  const Tensor ks = maybe(a[10], "k_scale"), vs = maybe(a[11], "v_scale");
  const ScalarType t = k.scalar_type();
  if (!half_type(t)) raise(PyExc_TypeError, "k must be bfloat16 or float16, got %s", c10::toString(t));
  if (k.dim() != 3) raise(PyExc_ValueError, "k must be [tokens, heads, d]");
  const int64_t tokens = k.size(0), d = k.size(2);
  const at::Device dev = k.device();
  int64_t hq = 0, hk, hv, qstride = 0, kstride, vstride;
  heads_of(k, "k", t, tokens, d, dev, &hk, &kstride);
  heads_of(v, "v", t, tokens, d, dev, &hv, &vstride);
  if (hv != hk) raise(PyExc_ValueError, "v has %lld heads, k has %lld", (long long)hv, (long long)hk);
  if (q.defined()) heads_of(q, "q", t, tokens, d, dev, &hq, &qstride);
  need(pos, "positions", ScalarType::Int, {tokens}, dev);
  need(slots, "slots", ScalarType::Long, {tokens}, dev);
  int64_t half = 0;
  if (inv.defined()) {
    half = inv.dim() == 1 ? inv.size(0) : -1;
    need(inv, "inv_freq", ScalarType::Float, {half}, dev);
  }
  const Caches c = caches_of(kc, vc, t, hk, d, dev, ks, vs);
  const Tensor qo = q.defined() ? output(a[12], "q_out", t, {tokens, hq, d}, dev) : Tensor();
  check(coverprune_kv_append(at_of<void>(q), qstride, k.data_ptr(), kstride, v.data_ptr(), vstride, code(t), tokens, hq, hk, d,
                             at_of<int32_t>(pos), at_of<int64_t>(slots), at_of<float>(inv), 2 * half, inter, float(magnitude),
                             at_of<void>(qo), kc.data_ptr(), vc.data_ptr(), code(c.type), c.pages, c.page, at_of<float>(ks),
                             at_of<float>(vs), stream_of(dev)));
  written(qo), written(kc), written(vc);
  return wrap(qo);
}

// q, k_cache, v_cache, table, lengths, max_length, window, scale, k_scale, v_scale, return_lse, out, lse, workspace
//   -> out or (out, lse)
PyObject* paged_attention(PyObject* const* a) {
  const Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &vc = tensor(a[2], "v_cache"), &table = tensor(a[3], "table"),
               &lengths = tensor(a[4], "lengths");
  const Tensor ks = maybe(a[8], "k_scale"), vs = maybe(a[9], "v_scale");
  const bool return_lse = truth(a[10]);
  const ScalarType t = q.scalar_type();
  if (!half_type(t)) raise(PyExc_TypeError, "q must be bfloat16 or float16, got %s", c10::toString(t));
  if (q.dim() != 3 || table.dim() != 2 || kc.dim() != 4)
    raise(PyExc_ValueError, "q must be [batch, heads, d], table [batch, width], the caches [pages, heads, page_size, d]");
  const int64_t batch = q.size(0), hq = q.size(1), d = q.size(2), hk = kc.size(1), width = table.size(1);
  const at::Device dev = q.device();
  need(q, "q", t, {batch, hq, d}, dev);
  const Caches c = caches_of(kc, vc, t, hk, d, dev, ks, vs);
  need(table, "table", ScalarType::Int, {batch, width}, dev);
  need(lengths, "lengths", ScalarType::Int, {batch}, dev);
  const int64_t longest = a[5] == Py_None ? width * c.page : integer(a[5], "max_length");
  const int64_t window = integer(a[6], "window");
  const float scale = a[7] == Py_None ? float(1.0 / std::sqrt(double(d))) : float(number(a[7], "scale"));
  const Tensor out = output(a[11], "out", t, {batch, hq, d}, dev);
  const Tensor lse = return_lse || a[12] != Py_None ? output(a[12], "lse", ScalarType::Float, {batch, hq}, dev) : Tensor();
  void* stream = stream_of(dev);
  Tensor ws = maybe(a[13], "workspace");
  if (ws.defined()) {
    need_device(ws, "workspace", dev);
    if (!ws.is_contiguous()) raise(PyExc_ValueError, "workspace must be contiguous");
  } else if (const size_t bytes = coverprune_paged_attention_workspace(batch, hq, hk, d, longest, window)) {
    ws = at::empty({int64_t(bytes)}, at::TensorOptions().dtype(ScalarType::Byte).device(dev));
  }
  check(coverprune_paged_attention(q.data_ptr(), code(t), batch, hq, hk, d, kc.data_ptr(), vc.data_ptr(), code(c.type), c.pages,
                                   c.page, at_of<float>(ks), at_of<float>(vs), at_of<int32_t>(table), width,
                                   at_of<int32_t>(lengths), longest, window, scale, out.data_ptr(), at_of<float>(lse),
                                   at_of<void>(ws), ws.defined() ? ws.nbytes() : 0, stream));
  written(out), written(lse), written(ws);
  if (!return_lse) return wrap(out);
  PyObject* o = PyTuple_New(2);
  if (!o) throw Raised();
  PyTuple_SET_ITEM(o, 0, wrap(out));
  PyTuple_SET_ITEM(o, 1, wrap(lse));
  return o;
}

// Positional calls only; no C++ exception leaves.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, N);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

// CoverPruneError and the functions that give a device's current stream and the
// current device.
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) {
    PyErr_SetString(PyExc_TypeError, "init(error, raw_stream, device)");
    return nullptr;
  }
  PyObject** const kept[] = {&g_error, &g_raw_stream, &g_device};
  for (int i = 0; i < 3; ++i) {
    Py_INCREF(args[i]);
    Py_XDECREF(*kept[i]);
    *kept[i] = args[i];
  }
  Py_RETURN_NONE;
}

template <class F>
PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef g_methods[] = {
    {"init", fast(&init), METH_FASTCALL, nullptr},
    {"rms_norm", fast(&entry<rms_norm, 8>), METH_FASTCALL, nullptr},
    {"w4_matvec", fast(&entry<w4_matvec, 7>), METH_FASTCALL, nullptr},
    {"kv_append", fast(&entry<kv_append, 13>), METH_FASTCALL, nullptr},
    {"paged_attention", fast(&entry<paged_attention, 14>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", "Compiled half of serving.py.", -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() { return PyModule_Create(&g_module); }
