// Argument marshalling for the operators around the experts: checks torch tensors, fills the descriptors of mcce.h and calls
// the C ABI on the current stream of the tensors' device.  These calls take a few microseconds on the device, so what a
// call costs on the host decides how fast the small ones are: here about 1 us beside the launch, in Python about 6.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "mcce.h"

namespace {

decltype(&mcce_rmsnorm) p_rmsnorm;
decltype(&mcce_rmsnorm_backward_workspace_bytes) p_rmsnorm_backward_workspace_bytes;
decltype(&mcce_rmsnorm_backward) p_rmsnorm_backward;
decltype(&mcce_dispatch_workspace_bytes) p_dispatch_workspace_bytes;
decltype(&mcce_dispatch) p_dispatch;
decltype(&mcce_combine) p_combine;
decltype(&mcce_combine_backward) p_combine_backward;
decltype(&mcce_strerror) p_strerror;
PyObject* error_class = nullptr;

struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
[[noreturn]] void refuse(const std::string& why) { throw Refused(why); }
void need(bool ok, const char* why) {
  if (!ok) refuse(why);
}
void done(int rc) {
  if (rc != MCCE_OK) refuse("mcce error " + std::to_string(rc) + ": " + p_strerror(rc));
}

// A tensor argument; null for None.  The calls record nothing for autograd, so where it is recording a tensor that needs a gradient is
// refused rather than cut off in silence.
const at::Tensor* tensor(PyObject* o, const char* what) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) refuse(std::string(what) + " must be a tensor");
  const at::Tensor* t = &THPVariable_Unpack(o);
  if (at::GradMode::is_enabled() && t->requires_grad())
    refuse(std::string(what) + " requires grad, and this call records no gradient: call it inside a torch.autograd.Function "
           "whose backward makes the gradient call, or under torch.no_grad()");
  return t;
}
const at::Tensor& given(PyObject* o, const char* what) {
  const at::Tensor* t = tensor(o, what);
  if (!t) refuse(std::string(what) + " is missing");
  return *t;
}
int cuda_device(const at::Tensor& t) {
  need(t.is_cuda(), "no CUDA tensor: this library has no CPU path");
  return t.get_device();
}
int code(const at::Tensor& t, const char* what) {
  switch (t.scalar_type()) {
    case at::kFloat: return MCCE_F32;
    case at::kBFloat16: return MCCE_BF16;
    case at::kFloat8_e4m3fn: return MCCE_E4M3;
    default: refuse(std::string(what) + " has dtype " + c10::toString(t.scalar_type()));
  }
}
std::string text(at::IntArrayRef s) {
  std::string r = "[";
  for (int64_t v : s) r += (r.size() > 1 ? ", " : "") + std::to_string(v);
  return r + "]";
}
void placed(const at::Tensor& t, at::IntArrayRef shape, int dev, const char* what) {
  if (!t.is_cuda() || t.get_device() != dev || t.sizes() != shape)
    refuse(std::string(what) + " is " + text(t.sizes()) + " on " + t.device().str() + ", expected " + text(shape) + " on cuda:" +
           std::to_string(dev));
}
// Row stride of a tensor of this shape whose rows are evenly spaced (the stride may exceed the width).
int64_t ld(const at::Tensor* p, at::IntArrayRef shape, int dev, const char* what) {
  if (!p) return 0;
  const at::Tensor& t = *p;
  placed(t, shape, dev, what);
  const int64_t d = shape.back(), n = t.dim();
  if (t.is_contiguous()) return d;
  if (t.stride(n - 1) != 1 && d != 1) refuse(std::string(what) + ": the columns of a row must be contiguous");
  int64_t step = -1, next = 0;   // stride of the rows; what a step in the dimension before must be
  for (int64_t i = n - 2; i >= 0; --i) {
    if (t.size(i) == 1) continue;
    if (step < 0) step = t.stride(i), next = step * t.size(i);
    else if (t.stride(i) != next) refuse(std::string(what) + ": rows must be evenly spaced");
    else next *= t.size(i);
  }
  if (step < 0) return d;   // a single row
  if (step < d) refuse(std::string(what) + ": rows overlap");
  return step;
}
void dense(const at::Tensor* p, at::IntArrayRef shape, at::ScalarType type, int dev, const char* what) {
  if (!p) return;
  placed(*p, shape, dev, what);
  if (p->scalar_type() != type || !p->is_contiguous())
    refuse(std::string(what) + ": expected contiguous " + c10::toString(type));
}
void* at_(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int32_t i32(int64_t v, const char* what) {
  if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(what) + " is too large");
  return (int32_t)v;
}

struct Where {
  c10::cuda::CUDAGuard guard;
  void* stream;
  explicit Where(int dev) : guard((c10::DeviceIndex)dev), stream(c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream()) {}
};
at::Tensor workspace(size_t bytes, const at::Tensor& like) {
  return at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
}

// A call writes its results behind torch's back: count them as changed, so that a backward pass that saved one of them says so.
void changed(std::initializer_list<const at::Tensor*> results) {
  for (const at::Tensor* t : results)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// rmsnorm(x, weight, eps, add, quant_group, out, sum, q, scales)
void run_rmsnorm(PyObject* const* a) {
  const at::Tensor &x = given(a[0], "x"), &w = given(a[1], "weight");
  const at::Tensor *add = tensor(a[3], "add"), *out = tensor(a[5], "out"), *sum = tensor(a[6], "sum"), *q = tensor(a[7], "q"),
                   *scales = tensor(a[8], "scales");
  const int dev = cuda_device(x);
  need(x.dim() >= 1 && x.size(-1) >= 1, "x must have columns");
  const at::IntArrayRef shape = x.sizes();
  const int64_t d = shape.back();
  mcce_norm n{};
  n.rows = x.numel() / d, n.d = i32(d, "the width"), n.dtype = code(x, "x");
  n.add_dtype = add ? code(*add, "add") : n.dtype, n.weight_dtype = code(w, "weight");
  n.eps = (float)PyFloat_AsDouble(a[2]);
  if (PyErr_Occurred()) throw python_error();
  need(!out || out->scalar_type() == x.scalar_type(), "out must have the type of x");
  need(!sum || sum->scalar_type() == x.scalar_type(), "sum must have the type of x");
  if (q) {
    need(a[4] != Py_None && scales, "8-bit rows need quant_group and scales");
    n.quant_group = i32(PyLong_AsLong(a[4]), "quant_group");
    if (PyErr_Occurred()) throw python_error();
    need(n.quant_group >= 0, "quant_group is negative");
    need(q->scalar_type() == at::kFloat8_e4m3fn, "q must be float8_e4m3fn");
    auto s = shape.vec();
    s.back() = n.quant_group ? ceil_div(d, n.quant_group) : 1;
    dense(scales, s, at::kFloat, dev, "scales");
    n.ld_q = ld(q, shape, dev, "q");
  } else {
    need(a[4] == Py_None && !scales, "quant_group without 8-bit rows");
  }
  dense(&w, {d}, w.scalar_type(), dev, "weight");
  n.ld_x = ld(&x, shape, dev, "x"), n.ld_add = ld(add, shape, dev, "add");
  n.ld_sum = ld(sum, shape, dev, "sum"), n.ld_out = ld(out, shape, dev, "out");
  Where on(dev);
  done(p_rmsnorm(&n, x.data_ptr(), at_(add), w.data_ptr(), at_(sum), at_(out), at_(q), (float*)at_(scales), on.stream));
  changed({sum, out, q, scales});
}

// rmsnorm_backward(dout, h, weight, eps, dsum, dx, dweight)
void run_rmsnorm_backward(PyObject* const* a) {
  const at::Tensor &g = given(a[0], "dout"), &h = given(a[1], "h"), &w = given(a[2], "weight"), &dx = given(a[5], "dx");
  const at::Tensor *ds = tensor(a[4], "dsum"), *dw = tensor(a[6], "dweight");
  const int dev = cuda_device(h);
  need(h.dim() >= 1 && h.size(-1) >= 1, "h must have columns");
  const at::IntArrayRef shape = h.sizes();
  const int64_t d = shape.back();
  mcce_norm n{};
  n.rows = h.numel() / d, n.d = i32(d, "the width"), n.dtype = n.add_dtype = code(h, "h"), n.weight_dtype = code(w, "weight");
  n.eps = (float)PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) throw python_error();
  need(g.scalar_type() == h.scalar_type(), "dout must have the type of h");
  need(!ds || ds->scalar_type() == h.scalar_type(), "dsum must have the type of h");
  need(dx.scalar_type() == h.scalar_type(), "dx must have the type of h");
  dense(&w, {d}, w.scalar_type(), dev, "weight");
  dense(dw, {d}, at::kFloat, dev, "dweight");
  n.ld_x = ld(&h, shape, dev, "h"), n.ld_add = ld(ds, shape, dev, "dsum");
  n.ld_sum = ld(&dx, shape, dev, "dx"), n.ld_out = ld(&g, shape, dev, "dout");
  Where on(dev);
  at::Tensor ws;
  const size_t bytes = dw ? p_rmsnorm_backward_workspace_bytes(&n) : 0;
  if (bytes) ws = workspace(bytes, h);
  done(p_rmsnorm_backward(&n, g.data_ptr(), h.data_ptr(), at_(ds), w.data_ptr(), dx.data_ptr(), (float*)at_(dw),
                          bytes ? ws.data_ptr() : nullptr, bytes, on.stream));
  changed({&dx, dw});
}

// Leading sizes of [(L,)T,K]
struct Lead {
  int64_t L, T, K;
  bool layers;
  Lead(const at::Tensor& t, const char* what) {
    if (t.dim() != 2 && t.dim() != 3) refuse(std::string(what) + " must be [T,K] or [L,T,K]");
    layers = t.dim() == 3, L = layers ? t.size(0) : 1, T = t.size(-2), K = t.size(-1);
  }
  c10::SmallVector<int64_t, 3> shape(int64_t rows, int64_t cols) const {
    if (layers) return {L, rows, cols};
    return {rows, cols};
  }
  c10::SmallVector<int64_t, 2> flat(int64_t n) const {
    if (layers) return {L, n};
    return {n};
  }
};

// dispatch(sel_idx, n_experts, x, scales, offsets, perm, inv, rows, row_scales)
void run_dispatch(PyObject* const* a) {
  const at::Tensor &sel = given(a[0], "sel_idx"), &off = given(a[4], "offsets"), &inv = given(a[6], "inv");
  const at::Tensor *x = tensor(a[2], "x"), *sc = tensor(a[3], "scales"), *perm = tensor(a[5], "perm"), *rows = tensor(a[7], "rows"),
                   *osc = tensor(a[8], "scales of the rows");
  const int dev = cuda_device(sel);
  const Lead n(sel, "sel_idx");
  const long E = PyLong_AsLong(a[1]);
  if (PyErr_Occurred()) throw python_error();
  mcce_rows r{};
  r.n_layers = i32(n.L, "L"), r.n_tokens = i32(n.T, "T"), r.top_k = i32(n.K, "K"), r.n_experts = i32(E, "n_experts"), r.d = 1;
  r.dtype = r.token_dtype = MCCE_BF16;
  need(n.T * n.K <= INT32_MAX, "too many pairs");
  dense(&sel, sel.sizes(), at::kInt, dev, "sel_idx");
  dense(&off, n.flat(E + 1), at::kInt, dev, "offsets");
  dense(&inv, sel.sizes(), at::kInt, dev, "inv");
  dense(perm, n.flat(n.T * n.K), at::kInt, dev, "perm");
  need((x == nullptr) == (rows == nullptr) && (sc == nullptr) == (osc == nullptr),
       "rows and scales are wanted exactly where x and scales are given");
  if (x) {
    need(x->dim() == sel.dim(), "x must have the leading sizes of sel_idx");
    r.d = i32(x->size(-1), "the width"), r.dtype = r.token_dtype = code(*x, "x");
    need(rows->scalar_type() == x->scalar_type(), "rows must have the type of x");
    r.ld_token = ld(x, n.shape(n.T, r.d), dev, "x"), r.ld_rows = ld(rows, n.shape(n.T * n.K, r.d), dev, "rows");
  }
  if (sc) {
    need(sc->dim() == sel.dim(), "scales must have the leading sizes of sel_idx");
    r.scale_cols = i32(sc->size(-1), "scales");
    dense(sc, n.shape(n.T, r.scale_cols), at::kFloat, dev, "scales");
    dense(osc, n.shape(n.T * n.K, r.scale_cols), at::kFloat, dev, "scales of the rows");
  }
  Where on(dev);
  at::Tensor ws;
  const size_t bytes = p_dispatch_workspace_bytes(&r);
  if (bytes) ws = workspace(bytes, sel);
  const bool move_scales = sc && r.scale_cols > 0;
  done(p_dispatch(&r, (const int32_t*)sel.data_ptr(), at_(x), move_scales ? (const float*)sc->data_ptr() : nullptr,
                  (int32_t*)off.data_ptr(), (int32_t*)at_(perm), (int32_t*)inv.data_ptr(), at_(rows),
                  move_scales ? (float*)osc->data_ptr() : nullptr, bytes ? ws.data_ptr() : nullptr, bytes, on.stream));
  changed({&off, perm, &inv, rows, osc});
}

mcce_rows pairs(const Lead& n, const at::Tensor& rows, const at::Tensor& token) {
  mcce_rows r{};
  r.n_layers = i32(n.L, "L"), r.n_tokens = i32(n.T, "T"), r.top_k = i32(n.K, "K"), r.n_experts = 1;
  r.d = i32(rows.size(-1), "the width"), r.dtype = code(rows, "rows"), r.token_dtype = code(token, "the token rows");
  need(n.T * n.K <= INT32_MAX, "too many pairs");
  return r;
}

// combine(rows, inv, sel_w, add, out)
void run_combine(PyObject* const* a) {
  const at::Tensor &rows = given(a[0], "rows"), &inv = given(a[1], "inv"), &y = given(a[4], "out");
  const at::Tensor *w = tensor(a[2], "sel_w"), *add = tensor(a[3], "add");
  const int dev = cuda_device(rows);
  const Lead n(inv, "inv");
  need(rows.dim() == inv.dim(), "rows must be [T*K,d] or [L,T*K,d] like inv");
  mcce_rows r = pairs(n, rows, y);
  dense(&inv, inv.sizes(), at::kInt, dev, "inv");
  dense(w, inv.sizes(), at::kFloat, dev, "sel_w");
  r.ld_rows = ld(&rows, n.shape(n.T * n.K, r.d), dev, "rows"), r.ld_token = ld(&y, n.shape(n.T, r.d), dev, "out");
  need(!add || (add->scalar_type() == y.scalar_type() && ld(add, n.shape(n.T, r.d), dev, "add") == r.ld_token),
       "add must have the type and the row stride of out");
  Where on(dev);
  done(p_combine(&r, rows.data_ptr(), (const int32_t*)inv.data_ptr(), (const float*)at_(w), at_(add), y.data_ptr(), on.stream));
  changed({&y});
}

// combine_backward(dy, rows, inv, sel_w, drows, dw)
void run_combine_backward(PyObject* const* a) {
  const at::Tensor &dy = given(a[0], "dy"), &rows = given(a[1], "rows"), &inv = given(a[2], "inv"), &dr = given(a[4], "drows");
  const at::Tensor *w = tensor(a[3], "sel_w"), *dw = tensor(a[5], "dw");
  const int dev = cuda_device(rows);
  const Lead n(inv, "inv");
  need(rows.dim() == inv.dim(), "rows must be [T*K,d] or [L,T*K,d] like inv");
  mcce_rows r = pairs(n, rows, dy);
  dense(&inv, inv.sizes(), at::kInt, dev, "inv");
  dense(w, inv.sizes(), at::kFloat, dev, "sel_w");
  dense(dw, inv.sizes(), at::kFloat, dev, "dw");
  r.ld_rows = ld(&rows, n.shape(n.T * n.K, r.d), dev, "rows"), r.ld_token = ld(&dy, n.shape(n.T, r.d), dev, "dy");
  need(dr.scalar_type() == rows.scalar_type() && ld(&dr, n.shape(n.T * n.K, r.d), dev, "drows") == r.ld_rows,
       "drows must have the type and the row stride of rows");
  Where on(dev);
  done(p_combine_backward(&r, dy.data_ptr(), rows.data_ptr(), (const int32_t*)inv.data_ptr(), (const float*)at_(w), dr.data_ptr(),
                          (float*)at_(dw), on.stream));
  changed({&dr, dw});
}

template <void (*RUN)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N || !error_class) {
    PyErr_SetString(PyExc_TypeError, error_class ? "wrong number of arguments" : "not connected to the library");
    return nullptr;
  }
  try {
    RUN(args);
  } catch (const Refused& e) {
    PyErr_SetString(error_class, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// connect(error class, addresses of the eight functions above in their order)
PyObject* connect(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void** const to[8] = {(void**)&p_rmsnorm, (void**)&p_rmsnorm_backward_workspace_bytes, (void**)&p_rmsnorm_backward,
                        (void**)&p_dispatch_workspace_bytes, (void**)&p_dispatch, (void**)&p_combine, (void**)&p_combine_backward,
                        (void**)&p_strerror};
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  for (int i = 0; i < 8; ++i) {
    *to[i] = PyLong_AsVoidPtr(args[1 + i]);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(args[0]);
  error_class = args[0];
  Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))(f), METH_FASTCALL
PyMethodDef methods[] = {
    {"connect", FAST(connect), "connect(error class, addresses)"},
    {"rmsnorm", FAST((entry<run_rmsnorm, 9>)), "rmsnorm(x, weight, eps, add, quant_group, out, sum, q, scales)"},
    {"rmsnorm_backward", FAST((entry<run_rmsnorm_backward, 7>)), "rmsnorm_backward(dout, h, weight, eps, dsum, dx, dweight)"},
    {"dispatch", FAST((entry<run_dispatch, 9>)), "dispatch(sel_idx, n_experts, x, scales, offsets, perm, inv, rows, row_scales)"},
    {"combine", FAST((entry<run_combine, 5>)), "combine(rows, inv, sel_w, add, out)"},
    {"combine_backward", FAST((entry<run_combine_backward, 6>)), "combine_backward(dy, rows, inv, sel_w, drows, dw)"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Marshalling of torch tensors to the C ABI of mcce.h", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python that this file was compiled against, for the binding to compare
PyMODINIT_FUNC PyInit__marshal(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", MCCE_BUILT_FOR) < 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
