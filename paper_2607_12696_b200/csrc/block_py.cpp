// Argument checks and marshalling of the operators around the MoE layer for torch tensors: what block.py calls.
//
// The kernels behind a small call take a few microseconds; the same checks in Python and a ctypes call with twenty
// arguments take ten.  Nothing is computed here: every function checks, fills in the arguments of the C entry
// point of include/moev.h and calls it on torch's current stream.  Tensors that do not fit raise MoevError
// (MOEV_EINVAL) before that.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <string>

#include "../../include/moev.h"

namespace {

struct Refused {  // becomes a MoevError
  int status;
  std::string text;
};
[[noreturn]] void bad(const std::string& text) { throw Refused{MOEV_EINVAL, text}; }
void check(moev_status st, const char* text) {
  if (st != MOEV_OK) throw Refused{(int)st, text};
}

const char* type_name(at::ScalarType t) {
  switch (t) {
    case at::kBFloat16: return "bfloat16";
    case at::kFloat: return "float32";
    case at::kHalf: return "float16";
    case at::kDouble: return "float64";
    case at::kByte: return "uint8";
    case at::kInt: return "int32";
    case at::kFloat8_e4m3fn: return "float8_e4m3fn";
    default: return "another type";
  }
}
std::string list(at::IntArrayRef v) {
  std::string s = "[";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + "]";
}
std::string shape(const at::Tensor& t) { return list(t.sizes()) + " " + type_name(t.scalar_type()); }

const at::Tensor* optional(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) bad(std::string(name) + ": expected a tensor or None");
  return &THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, const char* name) {
  const at::Tensor* t = optional(o, name);
  if (!t) bad(std::string(name) + ": expected a tensor");
  return *t;
}

int dev_index(const at::Tensor& t) { return t.is_cuda() ? t.get_device() : -1; }
void* stream_of(const at::Tensor& t) {
  const int dev = dev_index(t);
  if (dev < 0 || dev != c10::cuda::current_device()) bad("tensors must be on the current CUDA device, got " + t.device().str());
  return c10::cuda::getCurrentCUDAStream(dev).stream();
}
void same_device(int dev, std::initializer_list<const at::Tensor*> ts) {
  for (const at::Tensor* t : ts)
    if (t && dev_index(*t) != dev) bad("tensors on different devices: " + t->device().str() + " and another");
}

// Row stride of a tensor whose first dimension is rows and whose others are contiguous (`width` elements).
int64_t rows(const at::Tensor& t, const char* name, int64_t n, int64_t width, at::ScalarType type) {
  if (t.scalar_type() != type || t.dim() < 2 || t.size(0) != n || t.numel() != n * width) {
    bad(std::string(name) + ": expected " + std::to_string(n) + " rows of " + std::to_string(width) + " " + type_name(type) + ", got " + shape(t));
  }
  int64_t step = 1;
  for (int64_t i = t.dim() - 1; i > 0; --i) {
    if (t.size(i) != 1 && t.stride(i) != step) {
      bad(std::string(name) + ": everything behind the first dimension must be contiguous, got strides " + list(t.strides()));
    }
    step *= t.size(i);
  }
  return n > 1 ? t.stride(0) : width;
}
int afmt(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? MOEV_ACT_BF16 : t.scalar_type() == at::kFloat ? MOEV_ACT_FP32 : -1; }
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
bool flat(const at::Tensor& t, at::ScalarType type, std::initializer_list<int64_t> sizes) {
  return t.scalar_type() == type && t.sizes() == at::IntArrayRef(sizes.begin(), sizes.size()) && t.is_contiguous();
}
template <typename P>
P* address(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Refused{-1, ""};
  return static_cast<P*>(p);
}
long integer(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{-1, ""};
  if (v > INT32_MAX || v < INT32_MIN) bad("an integer argument does not fit in 32 bits");
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{-1, ""};
  return v;
}

// x, weight, residual, y, residual_out, codes, scales, eps, act_quant
PyObject* add_rmsnorm(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0], "x");
  const at::Tensor& w = tensor(a[1], "weight");
  const at::Tensor *res = optional(a[2], "residual"), *y = optional(a[3], "y"), *ro = optional(a[4], "out residual"), *codes = optional(a[5], "codes"),
                   *scales = optional(a[6], "scales");
  if (x.dim() != 2 || afmt(x) < 0) bad("x: expected a bfloat16 or float32 matrix, got " + shape(x));
  const int64_t n = x.size(0), H = x.size(1);
  if (n > INT32_MAX || H > INT32_MAX) bad("x: too large");
  same_device(dev_index(x), {&w, res, y, ro, codes, scales});
  if (afmt(w) < 0 || w.dim() != 1 || w.size(0) != H || !w.is_contiguous()) bad("weight: expected " + std::to_string(H) + " contiguous bfloat16 or float32 values");
  moev_norm p{};
  p.n = (int32_t)n;
  p.H = (int32_t)H;
  p.afmt = afmt(x);
  p.wfmt = afmt(w);
  p.eps = (float)number(a[7]);
  p.act_quant = (int32_t)integer(a[8]);
  p.x = ptr(&x);
  p.w = ptr(&w);
  p.x_stride = rows(x, "x", n, H, x.scalar_type());
  if (res) {
    p.residual = ptr(res);
    p.residual_stride = rows(*res, "residual", n, H, x.scalar_type());
  }
  if (y) {
    p.y = ptr(y);
    p.y_stride = rows(*y, "y", n, H, x.scalar_type());
  }
  if (ro) {
    p.residual_out = ptr(ro);
    p.residual_out_stride = rows(*ro, "out residual", n, H, x.scalar_type());
  }
  if (codes) {
    if (codes->scalar_type() != at::kByte && codes->scalar_type() != at::kFloat8_e4m3fn) bad("codes: expected uint8 or float8_e4m3fn, got " + shape(*codes));
    p.codes = static_cast<uint8_t*>(ptr(codes));
    p.codes_stride = rows(*codes, "codes", n, H, codes->scalar_type());
  }
  if (scales) {
    if (!flat(*scales, at::kFloat, {n, (H + 127) / 128}))
      bad("scales: expected contiguous float32 [" + std::to_string(n) + ", " + std::to_string((H + 127) / 128) + "]");
    p.scales = static_cast<float*>(ptr(scales));
  }
  check(moev_add_rmsnorm(&p, stream_of(x)), "moev_add_rmsnorm rejected the call");
  Py_RETURN_NONE;
}

// description, packed weight, bias or 0 (addresses), device, x, y
PyObject* linear_w4(PyObject* const* a) {
  const moev_linear* p = address<moev_linear>(a[0]);
  const int dev = (int)integer(a[3]);
  const at::Tensor& x = tensor(a[4], "x");
  const at::Tensor* y = optional(a[5], "y");
  const int64_t n = x.dim() ? x.size(0) : 0;
  if (n > INT32_MAX) bad("x: too large");
  const int64_t x_stride = rows(x, "x", n, p->K, at::kBFloat16);
  at::Tensor made;
  if (!y) {
    made = at::empty({n, p->N}, x.options());
    y = &made;
  }
  if (afmt(*y) < 0) bad("y: expected bfloat16 or float32, got " + shape(*y));
  const int64_t y_stride = rows(*y, "y", n, p->N, y->scalar_type());
  if (dev_index(x) != dev || dev_index(*y) != dev) bad("x and y must be on the weight's device cuda:" + std::to_string(dev));
  check(moev_linear_w4(p, address<void>(a[1]), address<float>(a[2]), ptr(&x), x_stride, (int32_t)n, ptr(y), y_stride, afmt(*y), stream_of(x)),
        "moev_linear_w4 rejected the call");
  return THPVariable_Wrap(*y);
}

// Heads of D elements in a row; 0 where a row is not made of those.
int64_t heads_of(const at::Tensor& q, int64_t D) {
  int64_t width = 1;
  for (int64_t i = 1; i < q.dim(); ++i) width *= q.size(i);
  return q.dim() > 1 && width % D == 0 ? width / D : 0;
}

moev_draft_batch batch_for(PyObject* o, PyObject* parents, int64_t n_tokens) {
  moev_draft_batch d = *address<moev_draft_batch>(o);
  const long have = integer(parents);
  if (n_tokens > INT32_MAX) bad("too many token rows");
  if (d.parent && have < n_tokens) bad("parent has " + std::to_string(have) + " entries for " + std::to_string(n_tokens) + " token rows");
  d.n_tokens = (int32_t)n_tokens;
  return d;
}

// cache, batch (addresses), parents, device, k, v, rope, q, q_out
PyObject* cache_append(PyObject* const* a) {
  const moev_kv_cache* c = address<moev_kv_cache>(a[0]);
  const int dev = (int)integer(a[3]);
  const at::Tensor &k = tensor(a[4], "k"), &v = tensor(a[5], "v");
  const at::Tensor *rope = optional(a[6], "rope"), *q = optional(a[7], "q"), *o = optional(a[8], "q_out");
  const int64_t T = k.dim() ? k.size(0) : 0, D = c->head_dim, row = D * c->n_kv_heads;
  const moev_draft_batch d = batch_for(a[1], a[2], T);
  const int64_t k_stride = rows(k, "k", T, row, at::kBFloat16), v_stride = rows(v, "v", T, row, at::kBFloat16);
  int64_t heads = 0, q_stride = 0, o_stride = 0;
  if (q) {
    if (!o) o = q;
    heads = heads_of(*q, D);
    q_stride = rows(*q, "q", T, heads * D, at::kBFloat16);
    o_stride = rows(*o, "q_out", T, heads * D, at::kBFloat16);
  } else if (o) {
    bad("q_out without q");
  }
  if (rope && !(rope->dim() == 2 && rope->size(0) <= INT32_MAX && flat(*rope, at::kFloat, {rope->size(0), D})))
    bad("rope: expected contiguous float32 [positions, " + std::to_string(D) + "]");
  same_device(dev, {&k, &v, rope, q, o});
  check(moev_cache_append(c, &d, ptr(&k), k_stride, ptr(&v), v_stride, static_cast<float*>(ptr(rope)), rope ? (int32_t)rope->size(0) : 0, ptr(q),
                          q_stride, (int32_t)heads, ptr(o), o_stride, stream_of(k)),
        "moev_cache_append rejected the call (alignment, strides, head counts or bounds)");
  if (!o) Py_RETURN_NONE;
  return THPVariable_Wrap(*o);
}

// cache, batch (addresses), parents, device, q, out, lse, scale (0: D^-1/2), window, sinks, workspace
PyObject* cache_attend(PyObject* const* a) {
  const moev_kv_cache* c = address<moev_kv_cache>(a[0]);
  const int dev = (int)integer(a[3]);
  const at::Tensor& q = tensor(a[4], "q");
  const at::Tensor *out = optional(a[5], "out"), *lse = optional(a[6], "lse"), *sinks = optional(a[9], "sinks"), *ws = optional(a[10], "workspace");
  const int64_t T = q.dim() ? q.size(0) : 0, D = c->head_dim, heads = heads_of(q, D);
  const moev_draft_batch d = batch_for(a[1], a[2], T);
  const int64_t q_stride = rows(q, "q", T, heads * D, at::kBFloat16);
  at::Tensor made;
  if (!out) {
    made = at::zeros(q.sizes(), q.options());
    out = &made;
  }
  const int64_t o_stride = rows(*out, "out", T, heads * D, at::kBFloat16);
  if (lse && !flat(*lse, at::kFloat, {T, heads})) bad("lse: expected contiguous float32 [" + std::to_string(T) + ", " + std::to_string(heads) + "]");
  if (sinks && !flat(*sinks, at::kFloat, {heads})) bad("sinks: expected contiguous float32 [" + std::to_string(heads) + "]");
  same_device(dev, {&q, out, lse, sinks, ws});
  const int32_t window = (int32_t)integer(a[8]);
  const size_t size = moev_cache_attend_workspace(c, &d, (int32_t)heads, window);
  at::Tensor own;
  if (size && (!ws || !ws->is_contiguous() || ws->nbytes() < size)) {
    own = at::empty({(int64_t)size}, q.options().dtype(at::kByte));
    ws = &own;
  }
  const double scale = number(a[7]);
  check(moev_cache_attend(c, &d, ptr(&q), q_stride, (int32_t)heads, scale == 0.0 ? (float)(1.0 / std::sqrt((double)D)) : (float)scale, window,
                          static_cast<float*>(ptr(sinks)), ptr(out), o_stride, static_cast<float*>(ptr(lse)), size ? ptr(ws) : nullptr, size, stream_of(q)),
        "moev_cache_attend rejected the call (alignment, strides, head counts, scale or bounds)");
  return THPVariable_Wrap(*out);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refused& r) {
    if (r.status == -1) return nullptr;  // Python's own error is set
    PyObject* mod = PyImport_ImportModule("paper_2607_12696_b200.binding");
    PyObject* cls = mod ? PyObject_GetAttrString(mod, "MoevError") : nullptr;
    PyObject* e = cls ? PyObject_CallFunction(cls, "is", r.status, r.text.c_str()) : nullptr;
    if (e) PyErr_SetObject(cls, e);
    Py_XDECREF(e);
    Py_XDECREF(cls);
    Py_XDECREF(mod);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

#define ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(add_rmsnorm, 9), ENTRY(linear_w4, 6), ENTRY(cache_append, 9), ENTRY(cache_attend, 11), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block() { return PyModule_Create(&module_def); }
