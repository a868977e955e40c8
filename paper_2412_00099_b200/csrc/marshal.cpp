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
#include <tuple>
#include <utility>

#include "mcce.h"

namespace {

decltype(&mcce_rmsnorm) p_rmsnorm;
decltype(&mcce_rmsnorm_backward_workspace_bytes) p_rmsnorm_backward_workspace_bytes;
decltype(&mcce_rmsnorm_backward) p_rmsnorm_backward;
decltype(&mcce_dispatch_workspace_bytes) p_dispatch_workspace_bytes;
decltype(&mcce_dispatch) p_dispatch;
decltype(&mcce_combine) p_combine;
decltype(&mcce_combine_backward) p_combine_backward;
decltype(&mcce_expert_linear_workspace_bytes) p_expert_linear_workspace_bytes;
decltype(&mcce_expert_linear) p_expert_linear;
decltype(&mcce_expert_linear_backward_workspace_bytes) p_expert_linear_backward_workspace_bytes;
decltype(&mcce_expert_linear_backward) p_expert_linear_backward;
decltype(&mcce_expert_linear_dweight_workspace_bytes) p_expert_linear_dweight_workspace_bytes;
decltype(&mcce_expert_linear_dweight) p_expert_linear_dweight;
decltype(&mcce_checkpoint_pack) p_checkpoint_pack;
decltype(&mcce_checkpoint_unpack) p_checkpoint_unpack;
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

// Sizes of the experts' products: weights [(L,)E,n,k] with evenly spaced matrices and rows
struct Experts {
  int64_t L, E, R, n, k;
  bool layers;
  int dev;
  Experts(const at::Tensor& w, const at::Tensor& rows, const at::Tensor& offsets, const char* what) : dev(cuda_device(w)) {
    if (w.dim() != 3 && w.dim() != 4) refuse(std::string(what) + " must be [E,n,k] or [L,E,n,k]");
    layers = w.dim() == 4, L = layers ? w.size(0) : 1, E = w.size(-3), n = w.size(-2), k = w.size(-1);
    need(L >= 1 && E >= 1 && n >= 1 && k >= 1, "weights without elements");
    if (rows.dim() != w.dim() - 1) refuse(std::string("rows must be [R,columns], or [L,R,columns] where ") + what + " has layers");
    R = rows.size(-2);
    dense(&offsets, layers ? at::IntArrayRef{L, E + 1} : at::IntArrayRef{E + 1}, at::kInt, dev, "offsets");
  }
  c10::SmallVector<int64_t, 3> rows(int64_t cols) const {
    if (layers) return {L, R, cols};
    return {R, cols};
  }
  c10::SmallVector<int64_t, 4> weights() const {
    if (layers) return {L, E, n, k};
    return {E, n, k};
  }
  c10::SmallVector<int64_t, 3> biases() const {
    if (layers) return {L, E, n};
    return {E, n};
  }
  mcce_linear describe(int32_t type) const {
    mcce_linear p{};
    p.n_layers = i32(L, "L"), p.n_experts = i32(E, "E"), p.rows = R, p.n = i32(n, "n"), p.k = i32(k, "k");
    p.dtype = p.out_dtype = p.bias_dtype = p.saved_dtype = type;
    return p;
  }
  // strides of a row and of a matrix
  std::pair<int64_t, int64_t> strides(const at::Tensor& t, const char* what) const {
    placed(t, weights(), dev, what);
    const int64_t d = t.dim();
    if (k > 1 && t.stride(d - 1) != 1) refuse(std::string(what) + ": the columns of a row must be contiguous");
    const int64_t ld = n > 1 ? t.stride(d - 2) : k;
    const int64_t step = E > 1 ? t.stride(d - 3) : L > 1 ? t.stride(0) : n * ld;
    if (L > 1 && E > 1 && t.stride(0) != E * step) refuse(std::string(what) + ": matrices must be evenly spaced");
    if (ld < k || step < (n - 1) * ld + k) refuse(std::string(what) + ": rows or matrices overlap");
    return {ld, step};
  }
  void alike(const at::Tensor* t, const at::Tensor& first, const char* what) const {
    if (!t) return;
    if (t->scalar_type() != first.scalar_type() || strides(*t, what) != strides(first, what))
      refuse(std::string(what) + ": both matrices of a layer, and what is added to gradients, must have the same type and strides");
  }
};
int64_t blocks(int64_t cols) { return ceil_div(cols, 32); }
// What is kept for the backward pass and, where it holds 8 bits, its scales; `halves` of `cols` columns
int32_t saved_type(const at::Tensor& saved, const at::Tensor* scales, const at::Tensor& like, const Experts& s, int64_t halves, int64_t cols,
                   const char* what) {
  if (saved.scalar_type() == at::kFloat8_e4m3fn) {
    if (!scales) refuse(std::string(what) + " in 8 bits needs scales");
    dense(scales, s.rows(halves * blocks(cols)), at::kFloat8_e8m0fnu, s.dev, "scales");
    return MCCE_E4M3;
  }
  if (scales || saved.scalar_type() != like.scalar_type())
    refuse(std::string(what) + " must have the type of the rows, or be float8_e4m3fn with scales");
  return code(saved, what);
}
int32_t number(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (PyErr_Occurred()) throw python_error();
  return i32(v, "act");
}

// expert_linear(x, offsets, w, w_up, bias, bias_up, act, add, out, saved, scales)
void run_expert_linear(PyObject* const* a) {
  const at::Tensor &x = given(a[0], "x"), &off = given(a[1], "offsets"), &w = given(a[2], "w"), &out = given(a[8], "out");
  const at::Tensor *wu = tensor(a[3], "w_up"), *b = tensor(a[4], "bias"), *bu = tensor(a[5], "bias_up"), *add = tensor(a[7], "add");
  const at::Tensor *saved = tensor(a[9], "saved"), *scales = tensor(a[10], "scales");
  const Experts s(w, x, off, "w");
  mcce_linear p = s.describe(code(x, "x"));
  p.gated = wu != nullptr, p.act = number(a[6]);
  need(w.scalar_type() == x.scalar_type(), "w must have the type of x");
  s.alike(wu, w, "w_up");
  std::tie(p.ld_w, p.step_w) = s.strides(w, "w");
  p.ld_x = ld(&x, s.rows(s.k), s.dev, "x"), p.ld_y = ld(&out, s.rows(s.n), s.dev, "out");
  p.out_dtype = code(out, "out");
  if (b) {
    p.bias_dtype = code(*b, "bias");
    dense(b, s.biases(), b->scalar_type(), s.dev, "bias");
    dense(bu, s.biases(), b->scalar_type(), s.dev, "bias_up");
  } else {
    need(!bu, "bias_up without bias");
  }
  if (add) {
    need(add->scalar_type() == out.scalar_type(), "add must have the type of out");
    p.ld_add = ld(add, s.rows(s.n), s.dev, "add");
  }
  if (saved) {
    p.saved_dtype = saved_type(*saved, scales, x, s, 1 + p.gated, s.n, "saved");
    p.ld_saved = ld(saved, s.rows((1 + p.gated) * s.n), s.dev, "saved");
  } else {
    need(!scales, "scales without saved");
  }
  Where on(s.dev);
  at::Tensor ws;
  const size_t bytes = p_expert_linear_workspace_bytes(&p, x.data_ptr(), w.data_ptr(), at_(wu));
  if (bytes) ws = workspace(bytes, x);
  done(p_expert_linear(&p, x.data_ptr(), (const int32_t*)off.data_ptr(), w.data_ptr(), at_(wu), at_(b), at_(bu), at_(add), out.data_ptr(),
                       at_(saved), at_(scales), bytes ? ws.data_ptr() : nullptr, bytes, on.stream));
  changed({&out, saved, scales});
}

// expert_linear_backward(dout, offsets, w, w_up, act, add, saved, scales, dx, h)
void run_expert_linear_backward(PyObject* const* a) {
  const at::Tensor &g = given(a[0], "dout"), &off = given(a[1], "offsets"), &w = given(a[2], "w"), &dx = given(a[8], "dx");
  const at::Tensor *wu = tensor(a[3], "w_up"), *add = tensor(a[5], "add"), *saved = tensor(a[6], "saved"), *scales = tensor(a[7], "scales"),
                   *h = tensor(a[9], "h");
  const Experts s(w, g, off, "w");
  mcce_linear p = s.describe(code(g, "dout"));
  p.gated = wu != nullptr, p.act = number(a[4]);
  need(w.scalar_type() == g.scalar_type() && dx.scalar_type() == g.scalar_type() && (!add || add->scalar_type() == g.scalar_type()) &&
           (!h || h->scalar_type() == g.scalar_type()),
       "w, add, dx and h must have the type of dout");
  s.alike(wu, w, "w_up");
  std::tie(p.ld_w, p.step_w) = s.strides(w, "w");
  p.ld_y = ld(&g, s.rows((1 + p.gated) * s.n), s.dev, "dout");
  if (saved) {
    need(saved->dim() >= 1 && (saved->size(-1) == s.k || saved->size(-1) == 2 * s.k), "saved must have the columns of the input, or twice as many");
    p.below = (int32_t)(saved->size(-1) / s.k);
    p.saved_dtype = saved_type(*saved, scales, g, s, p.below, s.k, "saved");
    p.ld_saved = ld(saved, s.rows(p.below * s.k), s.dev, "saved");
  } else {
    need(!scales, "scales without saved");
  }
  p.ld_add = ld(add, s.rows(s.k), s.dev, "add"), p.ld_h = ld(h, s.rows(s.k), s.dev, "h");
  p.ld_x = ld(&dx, s.rows(p.below == 2 ? 2 * s.k : s.k), s.dev, "dx");
  Where on(s.dev);
  at::Tensor ws;
  const size_t bytes = p_expert_linear_backward_workspace_bytes(&p, g.data_ptr(), w.data_ptr(), at_(wu));
  if (bytes) ws = workspace(bytes, g);
  done(p_expert_linear_backward(&p, g.data_ptr(), (const int32_t*)off.data_ptr(), w.data_ptr(), at_(wu), at_(add), at_(saved), at_(scales),
                                dx.data_ptr(), at_(h), bytes ? ws.data_ptr() : nullptr, bytes, on.stream));
  changed({&dx, h});
}

// expert_linear_dweight(dout, x, scales, offsets, add_dw, add_dw_up, add_db, add_db_up, dw, dw_up, db, db_up)
void run_expert_linear_dweight(PyObject* const* a) {
  const at::Tensor &g = given(a[0], "dout"), &x = given(a[1], "x"), &off = given(a[3], "offsets"), &dw = given(a[8], "dw");
  const at::Tensor *scales = tensor(a[2], "scales"), *adw = tensor(a[4], "add.dw"), *adwu = tensor(a[5], "add.dw_up"),
                   *adb = tensor(a[6], "add.db"), *adbu = tensor(a[7], "add.db_up"), *dwu = tensor(a[9], "dw_up"), *db = tensor(a[10], "db"),
                   *dbu = tensor(a[11], "db_up");
  const Experts s(dw, g, off, "dw");
  mcce_linear p = s.describe(code(g, "dout"));
  p.gated = dwu != nullptr, p.out_dtype = code(dw, "dw");
  s.alike(dwu, dw, "dw_up"), s.alike(adw, dw, "add.dw"), s.alike(adwu, dw, "add.dw_up");
  std::tie(p.ld_w, p.step_w) = s.strides(dw, "dw");
  for (const at::Tensor* t : {db, dbu, adb, adbu}) dense(t, s.biases(), dw.scalar_type(), s.dev, "db");
  p.ld_y = ld(&g, s.rows((1 + p.gated) * s.n), s.dev, "dout"), p.ld_x = ld(&x, s.rows(s.k), s.dev, "x");
  p.saved_dtype = saved_type(x, scales, g, s, 1, s.k, "x");
  Where on(s.dev);
  at::Tensor ws;
  const size_t bytes = p_expert_linear_dweight_workspace_bytes(&p, g.data_ptr(), x.data_ptr());
  if (bytes) ws = workspace(bytes, g);
  done(p_expert_linear_dweight(&p, g.data_ptr(), x.data_ptr(), s.R ? at_(scales) : nullptr, (const int32_t*)off.data_ptr(), at_(adw), at_(adwu),
                               at_(adb), at_(adbu), dw.data_ptr(), at_(dwu), at_(db), at_(dbu), bytes ? ws.data_ptr() : nullptr, bytes,
                               on.stream));
  changed({&dw, dwu, db, dbu});
}

struct Flat {
  int64_t rows, d, ld_x, ld_q;
  int dev;
  int32_t type;
  Flat(const at::Tensor& x, const at::Tensor& q, const at::Tensor& scales) : dev(cuda_device(x)), type(code(x, "x")) {
    need(x.dim() >= 1 && x.size(-1) >= 1, "x must have columns");
    d = x.size(-1), rows = x.numel() / d;
    need(q.scalar_type() == at::kFloat8_e4m3fn, "q must be float8_e4m3fn");
    auto shape = x.sizes().vec();
    ld_x = ld(&x, x.sizes(), dev, "x"), ld_q = ld(&q, x.sizes(), dev, "q");
    shape.back() = blocks(d);
    dense(&scales, shape, at::kFloat8_e8m0fnu, dev, "scales");
  }
};
// checkpoint_pack(x, q, scales)
void run_checkpoint_pack(PyObject* const* a) {
  const at::Tensor &x = given(a[0], "x"), &q = given(a[1], "q"), &scales = given(a[2], "scales");
  const Flat f(x, q, scales);
  Where on(f.dev);
  done(p_checkpoint_pack(x.data_ptr(), f.type, f.rows, i32(f.d, "the width"), f.ld_x, f.ld_q, q.data_ptr(), scales.data_ptr(), on.stream));
  changed({&q, &scales});
}
// checkpoint_unpack(q, scales, x)
void run_checkpoint_unpack(PyObject* const* a) {
  const at::Tensor &q = given(a[0], "q"), &scales = given(a[1], "scales"), &x = given(a[2], "x");
  const Flat f(x, q, scales);
  Where on(f.dev);
  done(p_checkpoint_unpack(q.data_ptr(), scales.data_ptr(), f.type, f.rows, i32(f.d, "the width"), f.ld_x, f.ld_q, x.data_ptr(), on.stream));
  changed({&x});
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

// connect(error class, addresses of the functions above in their order)
PyObject* connect(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void** const to[] = {(void**)&p_rmsnorm, (void**)&p_rmsnorm_backward_workspace_bytes, (void**)&p_rmsnorm_backward,
                       (void**)&p_dispatch_workspace_bytes, (void**)&p_dispatch, (void**)&p_combine, (void**)&p_combine_backward,
                       (void**)&p_expert_linear_workspace_bytes, (void**)&p_expert_linear, (void**)&p_expert_linear_backward_workspace_bytes,
                       (void**)&p_expert_linear_backward, (void**)&p_expert_linear_dweight_workspace_bytes,
                       (void**)&p_expert_linear_dweight, (void**)&p_checkpoint_pack, (void**)&p_checkpoint_unpack, (void**)&p_strerror};
  constexpr int kFunctions = sizeof(to) / sizeof(to[0]);
  if (n != 1 + kFunctions) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  for (int i = 0; i < kFunctions; ++i) {
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
    {"expert_linear", FAST((entry<run_expert_linear, 11>)), "expert_linear(x, offsets, w, w_up, bias, bias_up, act, add, out, saved, scales)"},
    {"expert_linear_backward", FAST((entry<run_expert_linear_backward, 10>)),
     "expert_linear_backward(dout, offsets, w, w_up, act, add, saved, scales, dx, h)"},
    {"expert_linear_dweight", FAST((entry<run_expert_linear_dweight, 12>)),
     "expert_linear_dweight(dout, x, scales, offsets, add_dw, add_dw_up, add_db, add_db_up, dw, dw_up, db, db_up)"},
    {"checkpoint_pack", FAST((entry<run_checkpoint_pack, 3>)), "checkpoint_pack(x, q, scales)"},
    {"checkpoint_unpack", FAST((entry<run_checkpoint_unpack, 3>)), "checkpoint_unpack(q, scales, x)"},
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
