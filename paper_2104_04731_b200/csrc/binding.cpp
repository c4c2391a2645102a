// Python side of the 8-bit float operators: checks of torch tensors and the calls into the library.
//
// The calls of single tokens take a few microseconds on the device, and marshalling five tensors in Python cost as much again
// (quantise 5.0 us, product 7.5 us, expert layer 10.9 us of checks and ctypes conversions; here 0.4 to 0.8 us).  The library
// itself is not linked: its entry points are handed over by the package, which has loaded the release or the debug build.
// Every function returns None, or (code, text) for the package to raise.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "b2conv.h"

namespace {

decltype(&b2c_fp8_quantize) p_quantize;
decltype(&b2c_fp8_matmul) p_matmul;
decltype(&b2c_route) p_route;
decltype(&b2c_route_sort_workspace_bytes) p_sort_bytes;
decltype(&b2c_route_sort) p_sort;
decltype(&b2c_route_combine) p_combine;
decltype(&b2c_experts_workspace_bytes) p_experts_bytes;
decltype(&b2c_fp8_experts) p_experts;

// What a call found wrong first.
struct Call {
  const char* name;
  int code = B2C_OK;
  const char* what = "";
  int device = -2;

  bool need(bool ok, const char* text, int c = B2C_E_INVALID_ARG) {
    if (!ok && code == B2C_OK) {
      code = c;
      what = text;
    }
    return code == B2C_OK;
  }
  // The tensor behind `o`, or null (also for None where that is allowed).
  const at::Tensor* tensor(PyObject* o, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    if (!need(THPVariable_Check(o), "a tensor is expected")) return nullptr;
    return &THPVariable_Unpack(o);
  }
  // Every tensor lies on the current device.
  void on_device(const at::Tensor* t) {
    if (t == nullptr || code != B2C_OK) return;
    if (!need(t->is_cuda(), "a tensor is not on the current CUDA device")) return;
    if (device == -2) device = c10::cuda::current_device();
    need(t->get_device() == device, "a tensor is not on the current CUDA device");
  }
  void* stream(PyObject* o) {
    if (o != Py_None) return PyLong_AsVoidPtr(o);
    return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  }
  PyObject* done() {
    if (PyErr_Occurred()) return nullptr;
    if (code == B2C_OK) Py_RETURN_NONE;
    return Py_BuildValue("(is)", code, what);
  }
};

int type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return B2C_F32;
    case at::kHalf: return B2C_F16;
    case at::kBFloat16: return B2C_BF16;
    case at::kFloat8_e4m3fn: return B2C_E4M3;
    case at::kFloat8_e5m2: return B2C_E5M2;
    default: return -1;
  }
}
bool is_f32(const at::Tensor& t) { return t.scalar_type() == at::kFloat; }
bool is_i32(const at::Tensor& t) { return t.scalar_type() == at::kInt; }
bool shaped(const at::Tensor& t, int64_t a) { return t.dim() == 1 && t.size(0) == a; }
bool shaped(const at::Tensor& t, int64_t a, int64_t b) { return t.dim() == 2 && t.size(0) == a && t.size(1) == b; }
bool shaped(const at::Tensor& t, int64_t a, int64_t b, int64_t c) { return t.dim() == 3 && t.size(0) == a && t.size(1) == b && t.size(2) == c; }
bool shaped(const at::Tensor& t, int64_t a, int64_t b, int64_t c, int64_t d) {
  return t.dim() == 4 && t.size(0) == a && t.size(1) == b && t.size(2) == c && t.size(3) == d;
}
int64_t blocks(int64_t n) { return (n + 127) / 128; }
// Distance between the rows of a matrix with contiguous rows; -1 if it has none or they overlap.
int64_t ld(const at::Tensor& t) {
  const int64_t rows = t.size(0), cols = t.size(1);
  if (cols > 1 && t.stride(1) != 1) return -1;
  if (rows <= 1) return cols;
  return t.stride(0) >= cols ? t.stride(0) : -1;
}
size_t bytes_of(const at::Tensor& t) { return (size_t)t.numel() * t.element_size(); }

#define B2C_ARGS(n)                                                                   \
  if (nargs != n) {                                                                   \
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");                    \
    return nullptr;                                                                   \
  }

// quantize(x, q, scale, block_rows, stream)
PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(5)
  Call c{"b2c_fp8_quantize"};
  const at::Tensor *x = c.tensor(args[0]), *q = c.tensor(args[1]), *s = c.tensor(args[2]);
  const long block = PyLong_AsLong(args[3]);
  if (c.code != B2C_OK || PyErr_Occurred()) return c.done();
  if (c.need(x->dim() == 2 && q->dim() == 2 && s->dim() == 2 && (block == 1 || block == 128), "shapes")) {
    const int64_t rows = x->size(0), cols = x->size(1);
    c.need(shaped(*q, rows, cols), "q has not x's shape");
    c.need(shaped(*s, (rows + block - 1) / block, blocks(cols)) && is_f32(*s), "scale");
    c.need(type_of(*x) >= 0 && type_of(*q) >= 0, "types");
    c.need(ld(*x) >= 0 && ld(*q) >= 0 && ld(*s) >= 0, "rows are not contiguous, or overlap");
    c.need(cols <= INT32_MAX, "sizes", B2C_E_UNSUPPORTED);
    for (const at::Tensor* t : {x, q, s}) c.on_device(t);
    if (c.code == B2C_OK)
      c.code = p_quantize(x->data_ptr(), type_of(*x), rows, (int32_t)cols, ld(*x), (int)block, type_of(*q), q->data_ptr(), ld(*q),
                          (float*)s->data_ptr(), ld(*s), c.stream(args[4]));
  }
  return c.done();
}

// matmul(a, a_scale, b, b_scale, y, offsets, stream)
PyObject* matmul(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(7)
  Call c{"b2c_fp8_matmul"};
  const at::Tensor *a = c.tensor(args[0]), *sa = c.tensor(args[1]), *b = c.tensor(args[2]), *sb = c.tensor(args[3]), *y = c.tensor(args[4]),
                   *off = c.tensor(args[5], true);
  if (c.code != B2C_OK) return c.done();
  if (c.need(a->dim() == 2 && sa->dim() == 2 && y->dim() == 2 && (b->dim() == 2 || b->dim() == 3), "shapes") &&
      c.need((b->dim() == 2) == (off == nullptr), "offsets go with a stack of matrices")) {
    const bool stack = b->dim() == 3;
    const int64_t rows = a->size(0), K = a->size(1), N = b->size(-2), groups = stack ? b->size(0) : 1;
    c.need(b->size(-1) == K && shaped(*y, rows, N), "shapes");
    c.need(shaped(*sa, rows, blocks(K)) && is_f32(*sa), "a_scale");
    c.need((stack ? shaped(*sb, groups, blocks(N), blocks(K)) : shaped(*sb, blocks(N), blocks(K))) && is_f32(*sb), "b_scale");
    c.need(b->is_contiguous() && sb->is_contiguous(), "b and b_scale have to be contiguous");
    c.need(off == nullptr || (shaped(*off, groups + 1) && off->is_contiguous() && is_i32(*off)), "offsets");
    c.need(type_of(*a) >= 0 && type_of(*b) >= 0 && type_of(*y) >= 0, "types");
    c.need(ld(*a) >= 0 && ld(*sa) >= 0 && ld(*y) >= 0, "rows are not contiguous, or overlap");
    c.need(N <= INT32_MAX && K <= INT32_MAX && groups <= INT32_MAX, "sizes", B2C_E_UNSUPPORTED);
    for (const at::Tensor* t : {a, sa, b, sb, y, off}) c.on_device(t);
    if (c.code == B2C_OK) {
      const b2c_matmul_desc d = {(int32_t)N, (int32_t)K, (int32_t)groups, type_of(*a), type_of(*b), type_of(*y)};
      c.code = p_matmul(&d, rows, a->data_ptr(), ld(*a), (const float*)sa->data_ptr(), ld(*sa), b->data_ptr(), (const float*)sb->data_ptr(),
                        off ? (const int32_t*)off->data_ptr() : nullptr, y->data_ptr(), ld(*y), c.stream(args[6]));
    }
  }
  return c.done();
}

// route(desc, logits, weights, ids, bias, stream); desc: anything that holds the bytes of a b2c_route_desc
PyObject* route(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(6)
  Call c{"b2c_route"};
  b2c_route_desc d;
  Py_buffer buf;
  if (PyObject_GetBuffer(args[0], &buf, PyBUF_SIMPLE) != 0) return nullptr;
  const bool sized = buf.len == (Py_ssize_t)sizeof(d);
  if (sized) memcpy(&d, buf.buf, sizeof(d));
  PyBuffer_Release(&buf);
  c.need(sized, "desc");
  const at::Tensor *x = c.tensor(args[1]), *w = c.tensor(args[2]), *ids = c.tensor(args[3]), *bias = c.tensor(args[4], true);
  if (c.code != B2C_OK) return c.done();
  if (c.need(x->dim() == 2 && x->size(1) == d.experts, "logits")) {
    const int64_t tokens = x->size(0);
    c.need(shaped(*w, tokens, d.topk) && shaped(*ids, tokens, d.topk) && w->is_contiguous() && ids->is_contiguous(), "outputs");
    c.need(is_f32(*w) && is_i32(*ids), "types of the outputs");
    c.need(bias == nullptr || (shaped(*bias, d.experts) && bias->is_contiguous() && is_f32(*bias)), "bias");
    c.need(type_of(*x) >= 0, "type of the logits");
    c.need(ld(*x) >= 0, "rows are not contiguous, or overlap");
    for (const at::Tensor* t : {x, w, ids, bias}) c.on_device(t);
    if (c.code == B2C_OK) {
      d.logit_type = type_of(*x);
      c.code = p_route(&d, tokens, x->data_ptr(), ld(*x), bias ? (const float*)bias->data_ptr() : nullptr, (float*)w->data_ptr(),
                       (int32_t*)ids->data_ptr(), c.stream(args[5]));
    }
  }
  return c.done();
}

// sort(ids, experts, offsets, rows, order, workspace, stream)
PyObject* sort(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(7)
  Call c{"b2c_route_sort"};
  const long experts = PyLong_AsLong(args[1]);
  const at::Tensor *ids = c.tensor(args[0]), *off = c.tensor(args[2]), *rows = c.tensor(args[3]), *order = c.tensor(args[4], true),
                   *ws = c.tensor(args[5], true);
  if (c.code != B2C_OK || PyErr_Occurred()) return c.done();
  const int64_t n = ids->numel();
  c.need(is_i32(*ids) && is_i32(*off) && is_i32(*rows) && ids->is_contiguous() && off->is_contiguous() && rows->is_contiguous(), "types");
  c.need(experts >= 1 && experts < INT32_MAX && off->numel() == experts + 1 && rows->numel() == n, "shapes");
  c.need(order == nullptr || (is_i32(*order) && order->numel() == n && order->is_contiguous()), "order");
  size_t need = 0;
  if (c.code == B2C_OK) c.code = p_sort_bytes(n, (int32_t)experts, &need);
  c.need(need == 0 || (ws != nullptr && ws->is_contiguous() && bytes_of(*ws) >= need), "workspace", B2C_E_WORKSPACE_TOO_SMALL);
  for (const at::Tensor* t : {ids, off, rows, order, ws}) c.on_device(t);
  if (c.code == B2C_OK)
    c.code = p_sort((const int32_t*)ids->data_ptr(), n, (int32_t)experts, (int32_t*)off->data_ptr(), (int32_t*)rows->data_ptr(),
                    order ? (int32_t*)order->data_ptr() : nullptr, need ? ws->data_ptr() : nullptr, c.stream(args[6]));
  return c.done();
}

// combine(y, rows, weights, out, stream)
PyObject* combine(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(5)
  Call c{"b2c_route_combine"};
  const at::Tensor *y = c.tensor(args[0]), *rows = c.tensor(args[1]), *w = c.tensor(args[2]), *out = c.tensor(args[3]);
  if (c.code != B2C_OK) return c.done();
  if (c.need(y->dim() == 2 && out->dim() == 2 && rows->dim() == 2, "shapes")) {
    const int64_t tokens = rows->size(0), topk = rows->size(1);
    c.need(shaped(*w, tokens, topk) && shaped(*out, tokens, y->size(1)), "shapes");
    c.need(is_i32(*rows) && is_f32(*w) && rows->is_contiguous() && w->is_contiguous(), "rows, weights");
    c.need(type_of(*y) >= 0 && type_of(*out) >= 0, "types");
    c.need(ld(*y) >= 0 && ld(*out) >= 0, "rows are not contiguous, or overlap");
    c.need(topk <= INT32_MAX && y->size(1) <= INT32_MAX, "sizes", B2C_E_UNSUPPORTED);
    for (const at::Tensor* t : {y, rows, w, out}) c.on_device(t);
    if (c.code == B2C_OK)
      c.code = p_combine(y->data_ptr(), type_of(*y), y->size(0), ld(*y), (const int32_t*)rows->data_ptr(), (const float*)w->data_ptr(), tokens,
                         (int32_t)topk, (int32_t)y->size(1), out->data_ptr(), type_of(*out), ld(*out), c.stream(args[4]));
  }
  return c.done();
}

// experts(x, ids, weights, w1, w1_scale, w2, w2_scale, y, workspace, stream)
PyObject* experts(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(10)
  Call c{"b2c_fp8_experts"};
  const at::Tensor* t[9];
  for (int i = 0; i < 9; ++i) t[i] = c.tensor(args[i]);
  if (c.code != B2C_OK) return c.done();
  const at::Tensor &x = *t[0], &ids = *t[1], &w = *t[2], &w1 = *t[3], &s1 = *t[4], &w2 = *t[5], &s2 = *t[6], &y = *t[7], &ws = *t[8];
  if (c.need(x.dim() == 2 && ids.dim() == 2 && w1.dim() == 4 && w2.dim() == 3, "shapes")) {
    const int64_t tokens = x.size(0), hidden = x.size(1), topk = ids.size(1), n = w1.size(0), inter = w1.size(2);
    c.need(shaped(y, tokens, hidden) && y.scalar_type() == x.scalar_type(), "y");
    c.need(shaped(ids, tokens, topk) && shaped(w, tokens, topk) && is_i32(ids) && is_f32(w), "ids, weights");
    c.need(shaped(w1, n, 2, inter, hidden) && shaped(s1, n, 2, blocks(inter), blocks(hidden)), "w1");
    c.need(shaped(w2, n, hidden, inter) && shaped(s2, n, blocks(hidden), blocks(inter)), "w2");
    c.need(type_of(w1) == B2C_E4M3 && type_of(w2) == B2C_E4M3 && is_f32(s1) && is_f32(s2) && type_of(x) >= 0, "types");
    for (int i = 1; i < 7; ++i) c.need(t[i]->is_contiguous(), "ids, weights, matrices and scales have to be contiguous");
    c.need(ws.is_contiguous(), "workspace");
    c.need(ld(x) >= 0 && ld(y) >= 0, "rows are not contiguous, or overlap");
    c.need(hidden <= INT32_MAX && inter <= INT32_MAX && n <= INT32_MAX && topk <= INT32_MAX, "sizes", B2C_E_UNSUPPORTED);
    for (const at::Tensor* v : t) c.on_device(v);
    const b2c_experts_desc d = {(int32_t)hidden, (int32_t)inter, (int32_t)n, (int32_t)topk, type_of(x)};
    size_t need = 0;
    if (c.code == B2C_OK) c.code = p_experts_bytes(&d, tokens, &need);
    c.need(bytes_of(ws) >= need, "workspace", B2C_E_WORKSPACE_TOO_SMALL);
    if (c.code == B2C_OK)
      c.code = p_experts(&d, tokens, x.data_ptr(), ld(x), (const int32_t*)ids.data_ptr(), (const float*)w.data_ptr(), w1.data_ptr(),
                         (const float*)s1.data_ptr(), w2.data_ptr(), (const float*)s2.data_ptr(), y.data_ptr(), ld(y), ws.data_ptr(),
                         c.stream(args[9]));
  }
  return c.done();
}

// bind(addresses of the library's entry points, in the order below)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  B2C_ARGS(8)
  void* p[8];
  for (int i = 0; i < 8; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  p_quantize = (decltype(p_quantize))p[0];
  p_matmul = (decltype(p_matmul))p[1];
  p_route = (decltype(p_route))p[2];
  p_sort_bytes = (decltype(p_sort_bytes))p[3];
  p_sort = (decltype(p_sort))p[4];
  p_combine = (decltype(p_combine))p[5];
  p_experts_bytes = (decltype(p_experts_bytes))p[6];
  p_experts = (decltype(p_experts))p[7];
  Py_RETURN_NONE;
}

// A C++ exception (torch checks its own arguments) becomes a Python one.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t nargs) {
  try {
    return F(self, args, nargs);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define B2C_METHOD(f) {#f, (PyCFunction)(void*)guarded<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {B2C_METHOD(quantize), B2C_METHOD(matmul),  B2C_METHOD(route), B2C_METHOD(sort),
                         B2C_METHOD(combine),  B2C_METHOD(experts), B2C_METHOD(bind),  {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
