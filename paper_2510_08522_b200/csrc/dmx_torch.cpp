// dmx_torch.cpp — what a training step calls (group_norm, linear and their gradients, AdamW's norm and step) for torch callers,
// compiled: argument checks, allocation from torch's caching allocator and the call into the C ABI of include/dmx.h in one
// Python call (through ctypes the calls took 5-28 us on the host, mostly checks and argument marshalling; now 3-14; the kernels of a small
// problem take 4-8 us). train_ops.py wraps these and documents them. A function returns its result, or a negative
// DMX_ERR_* code for arguments it refuses; torch's own errors (out of memory) are raised as Python exceptions.
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dmx.h"

namespace {

// The library's entry points, from the copy that the binding loaded (the checked build is another file).
decltype(&dmx_group_norm_workspace) norm_workspace;
decltype(&dmx_group_norm_forward) norm_forward;
decltype(&dmx_group_norm_backward) norm_backward;
decltype(&dmx_linear_workspace) linear_workspace;
decltype(&dmx_linear_forward) linear_forward;
decltype(&dmx_linear_backward_workspace) linear_backward_workspace;
decltype(&dmx_linear_backward) linear_backward;
decltype(&dmx_adamw_grad_norm) adamw_norm;
decltype(&dmx_adamw_step) adamw_step;

struct Refused {
  int64_t code;
};
[[noreturn]] void refuse(int64_t code = DMX_ERR_ARG) { throw Refused{code}; }
void need(bool ok) {
  if (!ok) refuse();
}

const at::Tensor& tensor(PyObject* o) {
  need(THPVariable_Check(o));
  return THPVariable_Unpack(o);
}
// a tensor or None
const at::Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
long whole(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse();
  }
  return v;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    refuse();
  }
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) {
    PyErr_Clear();
    refuse();
  }
  return v == 1;
}
// An operator whose inputs require a gradient comes back through train_grad.py, which calls it again unrecorded.
constexpr long kRecord = 1;
template <typename... T>
bool recorded(const at::Tensor* given, const T*... inputs) {
  return !given && c10::GradMode::is_enabled() && ((inputs && inputs->requires_grad()) || ...);
}
// what torch's differentiation has kept of t is stale now
void written(const at::Tensor* t) {
  if (t && t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
const void* in(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
void* out(const at::Tensor* t) { return t ? t->mutable_data_ptr() : nullptr; }

struct Call {            // the device and stream of the call's first tensor
  c10::cuda::CUDAGuard guard;
  void* stream;
  explicit Call(const at::Tensor& x) : guard(x.device()), stream(c10::cuda::getCurrentCUDAStream(x.device().index()).stream()) {}
};

at::Tensor workspace(int64_t bytes, const at::Tensor& like) {
  if (bytes < 0) refuse(bytes);
  return bytes ? at::empty({bytes}, like.options().dtype(at::kByte)) : at::Tensor();
}
void* start_of(const at::Tensor& ws) { return ws.defined() ? ws.mutable_data_ptr() : nullptr; }

template <typename F>
PyObject* guarded(F f) {
  HANDLE_TH_ERRORS
  try {
    at::AutoDispatchBelowADInplaceOrView below;
    return f();
  } catch (const Refused& r) {
    return PyLong_FromLongLong(r.code);
  }
  END_HANDLE_TH_ERRORS
}
PyObject* item(const at::Tensor* t) {
  if (!t || !t->defined()) Py_RETURN_NONE;
  return THPVariable_Wrap(*t);
}
PyObject* tuple(const at::Tensor* a, const at::Tensor* b, const at::Tensor* c) {
  PyObject* r = PyTuple_New(c ? 3 : 2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, item(a));
  PyTuple_SET_ITEM(r, 1, item(b));
  if (c) PyTuple_SET_ITEM(r, 2, item(c));
  return r;
}

// ---------------------------------------------------------------------------------------------- group norm

struct Images {          // an (N, ..., C) tensor whose positions lie at one stride and whose channels are dense
  int64_t N, L, C, image, row;
};
Images images(const at::Tensor& x) {
  need(x.dim() >= 3 && x.is_cuda());
  const auto shape = x.sizes(), st = x.strides();
  const int64_t d = x.dim();
  Images r{shape[0], 1, shape[d - 1], st[0], shape[d - 1]};
  need(r.C <= DMX_GN_MAX_CHANNELS);                      // (the C entry takes an int)
  need(r.C <= 1 || st[d - 1] == 1);
  bool first = true;                                     // the innermost dimension of several positions has their stride
  int64_t after = 1;                                     // positions covered by the dimensions behind i
  for (int64_t i = d - 2; i >= 1; --i) {                 // (N, H, W, C): the image's rows have to follow on
    if (shape[i] > 1) {
      if (first) r.row = st[i];
      need(st[i] == r.row * after);
      first = false;
    }
    after *= shape[i];
  }
  r.L = after;
  return r;
}
int type_of(const at::Tensor& x) {
  if (x.scalar_type() == at::kFloat) return DMX_F32;
  need(x.scalar_type() == at::kBFloat16);
  return DMX_BF16;
}
Images same_images(const at::Tensor& t, const at::Tensor& x) {
  need(t.scalar_type() == x.scalar_type() && t.device() == x.device() && t.sizes() == x.sizes());
  return images(t);
}
const float* vector(const at::Tensor* t, const at::Tensor& x, int64_t n) {
  if (!t) return nullptr;
  need(t->scalar_type() == at::kFloat && t->numel() == n && t->device() == x.device() && t->is_contiguous());
  return static_cast<const float*>(t->const_data_ptr());
}

// x, groups, weight, bias, eps, act, out -> (y, mean, rstd)
PyObject* group_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 7);
    const at::Tensor& x = tensor(a[0]);
    const long G = whole(a[1]);
    const at::Tensor *w = maybe(a[2]), *b = maybe(a[3]), *given = maybe(a[6]);
    if (recorded(given, &x, w, b)) return PyLong_FromLong(kRecord);
    const double eps = number(a[4]);
    const int act = (int)whole(a[5]), type = type_of(x);
    const Images X = images(x);
    const float *wp = vector(w, x, X.C), *bp = vector(b, x, X.C);
    need(G >= 1 && G <= X.C);
    const int64_t bytes = norm_workspace(X.N, X.L, (int)X.C, (int)G, type, 0);
    if (bytes < 0) refuse(bytes);
    Call call(x);
    at::Tensor y = given ? *given : at::empty(x.sizes(), x.options());
    const Images Y = given ? same_images(y, x) : images(y);
    at::Tensor mean = at::empty({X.N, G}, x.options().dtype(at::kFloat)), rstd = at::empty({X.N, G}, x.options().dtype(at::kFloat));
    at::Tensor ws = workspace(bytes, x);
    const int rc = norm_forward(X.N, X.L, (int)X.C, (int)G, type, in(&x), X.image, X.row, wp, bp, (float)eps, act, out(&y), Y.image, Y.row,
                                static_cast<float*>(out(&mean)), static_cast<float*>(out(&rstd)), start_of(ws), bytes, call.stream);
    if (rc != DMX_OK) refuse(rc);
    written(given);
    return tuple(&y, &mean, &rstd);
  });
}

// dy, x, mean, rstd, groups, weight, bias, act, out -> (dx, dweight, dbias)
PyObject* group_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 9);
    const at::Tensor &dy = tensor(a[0]), &x = tensor(a[1]), &mean = tensor(a[2]), &rstd = tensor(a[3]);
    const long G = whole(a[4]);
    const at::Tensor *w = maybe(a[5]), *b = maybe(a[6]), *given = maybe(a[8]);
    const int act = (int)whole(a[7]), type = type_of(x);
    const Images X = images(x), D = same_images(dy, x);
    const float *wp = vector(w, x, X.C), *bp = vector(b, x, X.C);
    need(G >= 1 && G <= X.C);
    const float *mp = vector(&mean, x, X.N * G), *rp = vector(&rstd, x, X.N * G);
    const int64_t bytes = norm_workspace(X.N, X.L, (int)X.C, (int)G, type, 1);
    if (bytes < 0) refuse(bytes);
    Call call(x);
    at::Tensor dx = given ? *given : at::empty(x.sizes(), x.options());
    const Images O = given ? same_images(dx, x) : images(dx);
    at::Tensor dw = at::empty({X.C}, x.options().dtype(at::kFloat)), db = at::empty({X.C}, x.options().dtype(at::kFloat));
    at::Tensor ws = workspace(bytes, x);
    const int rc = norm_backward(X.N, X.L, (int)X.C, (int)G, type, in(&dy), D.image, D.row, in(&x), X.image, X.row, mp, rp, wp, bp, act, out(&dx),
                                 O.image, O.row, static_cast<float*>(out(&dw)), static_cast<float*>(out(&db)), start_of(ws), bytes, call.stream);
    if (rc != DMX_OK) refuse(rc);
    written(given);
    return tuple(&dx, &dw, &db);
  });
}

// ---------------------------------------------------------------------------------------------- linear

struct Rows {            // a bf16 matrix with dense rows
  int64_t M, N, ld;
};
Rows rows(const at::Tensor& x) {
  need(x.dim() == 2 && x.is_cuda() && x.scalar_type() == at::kBFloat16);
  const Rows r{x.size(0), x.size(1), x.size(0) > 1 ? x.stride(0) : x.size(1)};
  need(r.N <= 1 || x.stride(1) == 1);
  return r;
}
Rows rows_like(const at::Tensor* t, const at::Tensor& x, int64_t M, int64_t N) {
  if (!t) return Rows{M, N, N};
  const Rows r = rows(*t);
  need(t->device() == x.device() && r.M == M && r.N == N);
  return r;
}
void bf16_vector(const at::Tensor* t, const at::Tensor& x, int64_t n) {
  need(!t || (t->scalar_type() == at::kBFloat16 && t->numel() == n && t->device() == x.device() && t->is_contiguous()));
}

// x, weight, bias, act, residual, save, out -> (y, z)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 7);
    const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
    const at::Tensor *b = maybe(a[2]), *r = maybe(a[4]), *given = maybe(a[6]);
    const int act = (int)whole(a[3]);
    const bool save = truth(a[5]) && act != DMX_ACT_NONE;
    if (recorded(given, &x, &w, b, r)) return PyLong_FromLong(kRecord);
    const Rows X = rows(x), W = rows(w);
    const int64_t M = X.M, N = W.M, K = X.N;
    need(W.N == K && w.device() == x.device());
    bf16_vector(b, x, N);
    const Rows R = rows_like(r, x, M, N);
    Call call(x);
    at::Tensor y = given ? *given : at::empty({M, N}, x.options()), z;
    const Rows Y = rows_like(&y, x, M, N);
    if (save) z = at::empty({M, N}, x.options());
    const int64_t bytes = linear_workspace(M, N, K, in(&x), X.ld, in(&w), W.ld);
    at::Tensor ws = workspace(bytes, x);
    const int rc = linear_forward(M, N, K, in(&x), X.ld, in(&w), W.ld, in(b), act, in(r), R.ld, out(&y), Y.ld, save ? out(&z) : nullptr, N,
                                  start_of(ws), bytes, call.stream);
    if (rc != DMX_OK) refuse(rc);
    written(given);
    return tuple(&y, &z, nullptr);
  });
}

// dy, x, weight, z, act, need (bits), three outputs -> (dx, dweight, dbias)
PyObject* linear_gradient(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 9);
    const at::Tensor &dy = tensor(a[0]), &x = tensor(a[1]), &w = tensor(a[2]);
    const at::Tensor *z = maybe(a[3]), *g0 = maybe(a[6]), *g1 = maybe(a[7]), *g2 = maybe(a[8]);
    const int act = (int)whole(a[4]);
    const long want = whole(a[5]);
    const Rows X = rows(x), W = rows(w);
    const int64_t M = X.M, N = W.M, K = X.N;
    need(W.N == K && w.device() == x.device() && (z || act == DMX_ACT_NONE));
    const Rows G = rows_like(&dy, x, M, N), Z = rows_like(z, x, M, N);
    Call call(x);
    at::Tensor dx, dw, db;
    if (want & 1) dx = g0 ? *g0 : at::empty({M, K}, x.options());
    if (want & 2) dw = g1 ? *g1 : at::empty({N, K}, x.options());
    if (want & 4) db = g2 ? *g2 : at::empty({N}, x.options());
    const Rows DX = rows_like(dx.defined() ? &dx : nullptr, x, M, K), DW = rows_like(dw.defined() ? &dw : nullptr, x, N, K);
    bf16_vector(db.defined() ? &db : nullptr, x, N);
    const int64_t bytes = linear_backward_workspace(M, N, K, in(&dy), G.ld, in(&x), X.ld, in(&w), W.ld, act);
    at::Tensor ws = workspace(bytes, x);
    const int rc = linear_backward(M, N, K, in(&dy), G.ld, in(&x), X.ld, in(&w), W.ld, in(z), Z.ld, act, dx.defined() ? out(&dx) : nullptr, DX.ld,
                                   dw.defined() ? out(&dw) : nullptr, DW.ld, db.defined() ? out(&db) : nullptr, start_of(ws), bytes, call.stream);
    if (rc != DMX_OK) refuse(rc);
    if (want & 1) written(g0);
    if (want & 2) written(g1);
    if (want & 4) written(g2);
    return tuple(&dx, &dw, &db);
  });
}

// ---------------------------------------------------------------------------------------------- AdamW

// One of the optimizer's arrays: n entries of a type, dense, on its device.
void* part(const at::Tensor* t, at::ScalarType type, int64_t n, long device) {
  need(t && t->scalar_type() == type && t->numel() == n && t->is_cuda() && t->device().index() == device && t->is_contiguous());
  return t->mutable_data_ptr();
}
dmx_adamw* handle(PyObject* o) {
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) PyErr_Clear();
  if (!p) refuse(DMX_ERR_HANDLE);
  return static_cast<dmx_adamw*>(p);
}

// handle, device, max_norm, out -> out
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 4);
    const at::Tensor& to = tensor(a[3]);
    void* p = part(&to, at::kFloat, 2, whole(a[1]));
    Call call(to);
    const int rc = adamw_norm(handle(a[0]), (float)number(a[2]), static_cast<float*>(p), call.stream);
    if (rc != DMX_OK) refuse(rc);
    written(&to);
    return item(&to);
  });
}

// handle, device, state bits, blocks, m, v, m_scale, v_scale, grad_scale, lr, beta1, beta2, eps, weight_decay, t, seed, the list of
// parameters and copies that the step writes -> None
PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    need(n == 17 && PyList_CheckExact(a[16]));
    const long device = whole(a[1]), blocks = whole(a[3]);
    const bool codes = whole(a[2]) == 8;
    const at::Tensor &m = tensor(a[4]), &v = tensor(a[5]);
    const at::Tensor *ms = maybe(a[6]), *vs = maybe(a[7]), *gs = maybe(a[8]);
    void *mp = part(&m, codes ? at::kChar : at::kFloat, blocks * 256, device), *vp = part(&v, codes ? at::kByte : at::kFloat, blocks * 256, device);
    void *msp = codes ? part(ms, at::kFloat, blocks, device) : out(ms), *vsp = codes ? part(vs, at::kFloat, blocks, device) : out(vs);
    void* gsp = gs ? part(gs, at::kFloat, 1, device) : nullptr;
    uint32_t seed = 0;
    if (a[15] != Py_None) {
      seed = (uint32_t)PyLong_AsUnsignedLongMask(a[15]);
      if (PyErr_Occurred()) { PyErr_Clear(); refuse(); }
    }
    Call call(m);
    const int rc = adamw_step(handle(a[0]), mp, vp, static_cast<float*>(msp), static_cast<float*>(vsp), static_cast<float*>(gsp), number(a[9]), number(a[10]),
                              number(a[11]), number(a[12]), number(a[13]), whole(a[14]), a[15] != Py_None, seed, call.stream);
    if (rc != DMX_OK) refuse(rc);
    for (const at::Tensor* t : {&m, &v, ms, vs}) written(t);
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[16]); ++i) written(&tensor(PyList_GET_ITEM(a[16], i)));
    Py_RETURN_NONE;
  });
}

// addresses of the nine entry points, in the order of the declarations above
PyObject* connect(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* p[9];
  if (n != 9) return PyErr_SetString(PyExc_TypeError, "nine addresses"), nullptr;
  for (int i = 0; i < 9; ++i)
    if (!(p[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : (PyErr_SetString(PyExc_ValueError, "null address"), nullptr);
  norm_workspace = reinterpret_cast<decltype(norm_workspace)>(p[0]);
  norm_forward = reinterpret_cast<decltype(norm_forward)>(p[1]);
  norm_backward = reinterpret_cast<decltype(norm_backward)>(p[2]);
  linear_workspace = reinterpret_cast<decltype(linear_workspace)>(p[3]);
  linear_forward = reinterpret_cast<decltype(linear_forward)>(p[4]);
  linear_backward_workspace = reinterpret_cast<decltype(linear_backward_workspace)>(p[5]);
  linear_backward = reinterpret_cast<decltype(linear_backward)>(p[6]);
  adamw_norm = reinterpret_cast<decltype(adamw_norm)>(p[7]);
  adamw_step = reinterpret_cast<decltype(adamw_step)>(p[8]);
  Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"connect", FAST(connect)},
                         {"group_norm", FAST(group_norm)},
                         {"group_norm_backward", FAST(group_norm_backward)},
                         {"linear", FAST(linear)},
                         {"linear_backward", FAST(linear_gradient)},
                         {"adamw_grad_norm", FAST(grad_norm)},
                         {"adamw_step", FAST(step)},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_dmx_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dmx_torch() { return PyModule_Create(&module); }
