// Host side of the 8-bit linear layer's Python binding: the checks of plain calls, the
// outputs' allocation and the call into libprm, natively.  In Python they cost 15 to 25 us a
// call, several times the GPU's for one token.
//
// Every function returns what the operator does (with the gradients' node, where one is
// to be recorded), a negative PRM_E* code that libprm gave (the caller raises it), or None:
// not a plain call (a tensor subclass, another device than the current one, a layout
// that needs a copy, a type or shape that is wrong, a tracer or a forward-mode tangent), and
// the Python binding then takes or refuses it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include <cstdint>

#include "../../include/prm.h"

extern "C" uint64_t prm_internal_int8_linear_backward_workspace(int64_t m, int64_t n, int64_t k, int32_t dx, int32_t dw, int32_t db);

namespace {

PyObject* g_parameter = nullptr;  // torch.nn.Parameter
constexpr int64_t kMaxLayer = 1 << 20;  // tokens and outputs of prm_int8_linear

// A strided device tensor whose metadata and pointer are its own: no subclass (those
// answer for themselves in Python), no functional transform's wrapper, no tangent; and no tracer,
// which would record the outputs' allocation alone.
const at::Tensor* plain(PyObject* o) {
  if (torch::jit::tracer::isTracing() || c10::impl::TorchDispatchModeTLS::get_mode(c10::impl::TorchDispatchModeKey::PROXY)) return nullptr;
  if (!THPVariable_CheckExact(o) && (PyObject*)Py_TYPE(o) != g_parameter) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || !t.has_storage() || t.layout() != at::kStrided) return nullptr;
  if (t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                               c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                               c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
                                               c10::DispatchKey::ZeroTensor})) ||
      t._fw_grad(0).defined())
    return nullptr;
  return &t;
}

int code_of(at::ScalarType t) {
  return t == at::kFloat ? PRM_F32 : t == at::kBFloat16 ? PRM_BF16 : t == at::kHalf ? PRM_F16 : -1;
}
at::ScalarType type_of(long code) {
  return code == PRM_F32 ? at::kFloat : code == PRM_BF16 ? at::kBFloat16 : code == PRM_F16 ? at::kHalf : at::ScalarType::Undefined;
}

// The last dimension's rows as a matrix without a copy: contiguous rows, evenly spaced
// over all leading dimensions.
struct Rows {
  int64_t rows = 0, cols = 0, ld = 0;
};
bool rows_of(const at::Tensor& t, Rows* r) {
  const int64_t d = t.dim();
  if (d < 1) return false;
  r->cols = t.size(d - 1);
  if (r->cols < 1 || t.numel() == 0) return false;
  r->rows = t.numel() / r->cols;
  if (r->cols > 1 && t.stride(d - 1) != 1) return false;
  int64_t rows = 1, step = 0;  // rows of the inner dimensions, and how far apart
  for (int64_t i = d - 2; i >= 0; --i) {
    if (t.size(i) == 1) continue;
    if (rows == 1) step = t.stride(i);
    else if (t.stride(i) != rows * step) return false;
    rows *= t.size(i);
  }
  if (rows > 1 && step < r->cols) return false;
  r->ld = rows > 1 ? step : r->cols;
  return true;
}
bool vector_of(const at::Tensor& t, const at::Tensor& like, at::ScalarType type, int64_t n) {
  return t.dim() == 1 && t.size(0) == n && t.scalar_type() == type && t.device() == like.device() && (n <= 1 || t.stride(0) == 1);
}
bool here(const at::Tensor& t) { return t.get_device() == c10::hip::current_device(); }
void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }
bool records(const at::Tensor* t) { return t && t->requires_grad() && at::GradMode::is_enabled(); }

// int8 rows that start on 16-byte boundaries, with the leading dimensions of `lead`
at::Tensor eight_bits(c10::IntArrayRef lead, int64_t cols, const at::Tensor& like, int64_t* ld) {
  c10::SmallVector<int64_t, 6> size(lead.begin(), lead.end());
  *ld = (cols + 15) / 16 * 16;
  size.push_back(*ld);
  at::Tensor q = at::empty(size, like.options().dtype(at::kChar).requires_grad(false));
  return *ld == cols ? q : q.narrow(-1, 0, cols);
}
at::Tensor empty(c10::IntArrayRef size, at::ScalarType type, const at::Tensor& like) {
  return at::empty(size, like.options().dtype(type).requires_grad(false).memory_format(c10::nullopt));
}
PyObject* wrap(at::Tensor t) { return t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None); }
// optional argument: false where it is there and not plain
bool optional(PyObject* o, const at::Tensor** t) {
  *t = nullptr;
  if (o == Py_None) return true;
  return (*t = plain(o)) != nullptr;
}
const void* data(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }

// A call that libprm refused.
struct Refused : std::runtime_error {
  int code;
  explicit Refused(int rc) : std::runtime_error("libprm error " + std::to_string(rc) + ": " + prm_last_error()), code(rc) {}
};
void check(int rc) {
  if (rc < 0) throw Refused(rc);
}
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const Refused& e) {
    return PyLong_FromLong(e.code);
  } catch (...) {  // out of memory above all, or what a hook raised: as torch's own calls raise it
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

at::Tensor bytes(uint64_t n, const at::Tensor& like) { return n ? empty({(int64_t)n}, at::kByte, like) : at::Tensor(); }
void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
c10::IntArrayRef lead_of(const at::Tensor& t) { return t.sizes().slice(0, t.dim() - 1); }
at::Tensor with_last(c10::IntArrayRef lead, int64_t n, const at::Tensor& like, at::ScalarType type) {
  c10::SmallVector<int64_t, 6> size(lead.begin(), lead.end());
  size.push_back(n);
  return empty(size, type, like);
}

// quantize_rows(x)
PyObject* quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 1) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor* x = plain(args[0]);
    Rows r;
    if (!x || code_of(x->scalar_type()) < 0 || !here(*x) || !rows_of(*x, &r)) Py_RETURN_NONE;
    int64_t ldq;
    at::Tensor q = eight_bits(lead_of(*x), r.cols, *x, &ldq), s = empty(lead_of(*x), at::kFloat, *x);
    check(prm_quantize_rows(x->const_data_ptr(), code_of(x->scalar_type()), r.rows, r.cols, r.ld, (int8_t*)q.data_ptr(), ldq,
                            (float*)s.data_ptr(), stream()));
    return Py_BuildValue("(NN)", wrap(std::move(q)), wrap(std::move(s)));
  });
}

// quantize_cols(x)
PyObject* quantize_cols(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 1) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor* x = plain(args[0]);
    Rows r;
    if (!x || x->dim() != 2 || code_of(x->scalar_type()) < 0 || !here(*x) || !rows_of(*x, &r)) Py_RETURN_NONE;
    int64_t ldq;
    at::Tensor q = eight_bits({r.cols}, r.rows, *x, &ldq), s = empty({r.cols}, at::kFloat, *x);
    const uint64_t need = prm_quantize_cols_workspace(r.rows, r.cols);
    at::Tensor ws = bytes(need, *x);
    check(prm_quantize_cols(x->const_data_ptr(), code_of(x->scalar_type()), r.rows, r.cols, r.ld, (int8_t*)q.data_ptr(), ldq,
                            (float*)s.data_ptr(), nullptr, at_of(ws), need, stream()));
    return Py_BuildValue("(NN)", wrap(std::move(q)), wrap(std::move(s)));
  });
}

// int8_matmul(a, a_scale, b, b_scale, bias, type code)
PyObject* int8_matmul(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *a = plain(args[0]), *sa = plain(args[1]), *b = plain(args[2]), *sb = plain(args[3]), *bias;
    const long code = PyLong_AsLong(args[5]);
    if (!a || !sa || !b || !sb || !optional(args[4], &bias) || type_of(code) == at::ScalarType::Undefined) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    Rows ra, rb;
    if (a->scalar_type() != at::kChar || b->scalar_type() != at::kChar || !here(*a) || b->device() != a->device() || b->dim() != 2 ||
        !rows_of(*a, &ra) || !rows_of(*b, &rb) || ra.cols != rb.cols)
      Py_RETURN_NONE;
    if (sa->scalar_type() != at::kFloat || sa->sizes() != lead_of(*a) || !sa->is_contiguous() || sa->device() != a->device() ||
        !vector_of(*sb, *a, at::kFloat, rb.rows) || (bias && !vector_of(*bias, *a, type_of(code), rb.rows)))
      Py_RETURN_NONE;
    at::Tensor out = with_last(lead_of(*a), rb.rows, *a, type_of(code));
    const uint64_t need = prm_int8_matmul_workspace((const int8_t*)a->const_data_ptr(), ra.ld, (const int8_t*)b->const_data_ptr(), rb.ld,
                                                    ra.rows, rb.rows, ra.cols);
    at::Tensor ws = bytes(need, *a);
    check(prm_int8_matmul((const int8_t*)a->const_data_ptr(), ra.ld, (const float*)sa->const_data_ptr(), (const int8_t*)b->const_data_ptr(),
                          rb.ld, (const float*)sb->const_data_ptr(), data(bias), (int32_t)code, out.data_ptr(), rb.rows, ra.rows, rb.rows,
                          ra.cols, at_of(ws), need, stream()));
    return wrap(std::move(out));
  });
}

// ---- gradients -----------------------------------------------------------------------
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// An absent argument: a Function takes no undefined tensor, and counts only those that are
// there when it says whose gradients are needed.
using Maybe = std::optional<at::Tensor>;
Maybe maybe(const at::Tensor* t) { return t ? Maybe(*t) : Maybe(); }
at::Tensor or_none(const Maybe& t) { return t ? *t : at::Tensor(); }

// The gradients of gradients are refused, where they are asked for and not before.
variable_list once(variable_list grads, bool recording) {
  if (!recording) return grads;
  for (at::Tensor& g : grads)
    if (g.defined()) g = g.detach().set_requires_grad(true);
  auto refuse = std::make_shared<torch::autograd::DelayedError>("these gradients are not differentiable", (int64_t)grads.size());
  return (*refuse)(std::move(grads));
}
// memory that holds the values, in rows (a gradient may be a view that stands for the negative)
at::Tensor with_rows(const at::Tensor& t, Rows* r) {
  if (!t.is_neg() && rows_of(t, r)) return t;
  at::Tensor c = t.resolve_neg().contiguous();
  rows_of(c, r);
  return c;
}

// What a saved tensor's hooks gave back is what was saved.
void as_saved(const at::Tensor& t, const at::Tensor& like, bool ok) {
  if (!t.is_cuda() || t.device() != like.device() || t.scalar_type() != like.scalar_type() || !ok)
    throw std::runtime_error("a saved tensor came back with another type, device or shape");
}

at::Tensor linear(const at::Tensor& x, const at::Tensor& w, const at::Tensor& bias) {
  Rows rx, rw;
  rows_of(x, &rx);
  rows_of(w, &rw);
  at::Tensor y = with_last(lead_of(x), rw.rows, x, x.scalar_type());
  const uint64_t need = prm_int8_linear_workspace(rx.rows, rw.rows, rx.cols);
  at::Tensor ws = bytes(need, x);
  check(prm_int8_linear(x.const_data_ptr(), rx.ld, w.const_data_ptr(), rw.ld, bias.defined() ? bias.const_data_ptr() : nullptr,
                        code_of(x.scalar_type()), y.data_ptr(), rw.rows, rx.rows, rw.rows, rx.cols, at_of(ws), need, stream()));
  return y;
}

struct Linear : torch::autograd::Function<Linear> {
  static at::Tensor forward(AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, const Maybe& bias) {
    // each serves the other's gradient alone
    ctx->save_for_backward({w.requires_grad() ? x : at::Tensor(), x.requires_grad() ? w : at::Tensor()});
    ctx->saved_data["x"] = x.sizes();
    ctx->saved_data["bias"] = bias.has_value();
    return linear(x, w, or_none(bias));
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool recording = at::GradMode::is_enabled();
    variable_list out(3);
    {
      at::AutoGradMode off(false);
      const variable_list saved = ctx->get_saved_variables();
      const std::vector<int64_t> sizes = ctx->saved_data["x"].toIntVector();
      Rows rg, rx, rw;
      const at::Tensor gy = with_rows(grads[0], &rg);
      const int64_t m = rg.rows, n = rg.cols, k = sizes.back();
      at::Tensor x, w;
      if (ctx->needs_input_grad(0)) {
        w = with_rows(saved[1], &rw);
        as_saved(w, gy, rw.rows == n && rw.cols == k);
        out[0] = empty(sizes, gy.scalar_type(), gy);
      }
      if (ctx->needs_input_grad(1)) {
        x = with_rows(saved[0], &rx);
        as_saved(x, gy, rx.rows == m && rx.cols == k);
        out[1] = empty({n, k}, gy.scalar_type(), gy);
      }
      if (ctx->saved_data["bias"].toBool() && ctx->needs_input_grad(2)) out[2] = empty({n}, gy.scalar_type(), gy);
      const uint64_t need = prm_internal_int8_linear_backward_workspace(m, n, k, out[0].defined(), out[1].defined(), out[2].defined());
      at::Tensor ws = bytes(need, gy);
      check(prm_int8_linear_backward(gy.const_data_ptr(), rg.ld, x.defined() ? x.const_data_ptr() : nullptr, rx.ld,
                                     w.defined() ? w.const_data_ptr() : nullptr, rw.ld, code_of(gy.scalar_type()), at_of(out[0]), k,
                                     at_of(out[1]), k, at_of(out[2]), m, n, k, at_of(ws), need, stream()));
    }
    return once(std::move(out), recording);
  }
};

// int8_linear(x, weight, bias)
PyObject* int8_linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *x = plain(args[0]), *w = plain(args[1]), *bias;
    Rows rx, rw;
    if (!x || !w || !optional(args[2], &bias) || code_of(x->scalar_type()) < 0 || !here(*x) || w->dim() != 2 ||
        w->scalar_type() != x->scalar_type() || w->device() != x->device() || !rows_of(*x, &rx) || !rows_of(*w, &rw) || rx.cols != rw.cols ||
        (bias && !vector_of(*bias, *x, x->scalar_type(), rw.rows)))
      Py_RETURN_NONE;
    // more than prm_int8_linear takes in one call (its gradients' sums among them): from its parts
    if (rx.rows > kMaxLayer || rw.rows > kMaxLayer) Py_RETURN_NONE;
    const Maybe b = maybe(bias);
    return wrap(records(x) || records(w) || records(bias) ? Linear::apply(*x, *w, b) : linear(*x, *w, or_none(b)));
  });
}

// (y, h or nothing), or (q, scale, h or nothing)
variable_list norm(const at::Tensor& x, const at::Tensor& w, const at::Tensor& res, float eps, bool quantize) {
  Rows r, rr;
  rows_of(x, &r);
  if (res.defined()) rows_of(res, &rr);
  at::Tensor h, y, q, s;
  int64_t ldq = 0;
  if (res.defined()) h = empty(x.sizes(), x.scalar_type(), x);
  if (quantize) {
    q = eight_bits(lead_of(x), r.cols, x, &ldq);
    s = empty(lead_of(x), at::kFloat, x);
  } else {
    y = empty(x.sizes(), x.scalar_type(), x);
  }
  check(prm_rms_norm(x.const_data_ptr(), r.ld, res.defined() ? res.const_data_ptr() : nullptr, rr.ld,
                     w.defined() ? w.const_data_ptr() : nullptr, code_of(x.scalar_type()), r.rows, r.cols, eps, at_of(h), r.cols, at_of(y),
                     r.cols, (int8_t*)at_of(q), ldq, (float*)at_of(s), stream()));
  variable_list out = quantize ? variable_list{q, s} : variable_list{y};
  if (h.defined()) out.push_back(h);
  return out;
}

struct Norm : torch::autograd::Function<Norm> {
  static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const Maybe& w, const Maybe& res, double eps) {
    variable_list out = norm(x, or_none(w), or_none(res), (float)eps, false);
    ctx->save_for_backward({res ? out[1] : x, or_none(w)});
    ctx->saved_data["res"] = res.has_value();
    ctx->saved_data["eps"] = eps;
    ctx->set_materialize_grads(false);
    return out;
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const bool recording = at::GradMode::is_enabled();
    variable_list out(4);
    {
      at::AutoGradMode off(false);
      const variable_list saved = ctx->get_saved_variables();
      const at::Tensor w = saved[1].defined() ? saved[1].resolve_neg() : saved[1];
      const bool need_dw = w.defined() && ctx->needs_input_grad(1), kept = grads.size() > 1 && grads[1].defined();
      at::Tensor dx;
      if (!grads[0].defined()) {  // only the kept sum has a gradient
        dx = kept ? grads[1] : at::Tensor();
      } else {
        Rows rg, rs, rh;
        const at::Tensor gy = with_rows(grads[0], &rg), gh = kept ? with_rows(grads[1], &rs) : at::Tensor(), h = with_rows(saved[0], &rh);
        as_saved(h, gy, h.sizes() == gy.sizes());
        if (w.defined()) as_saved(w, gy, vector_of(w, gy, gy.scalar_type(), rg.cols));
        dx = empty(h.sizes(), h.scalar_type(), h);
        at::Tensor ws;
        uint64_t need = 0;
        if (need_dw) {
          out[1] = empty({rh.cols}, h.scalar_type(), h);
          need = prm_rms_norm_backward_workspace(rh.rows, rh.cols);
          ws = bytes(need, h);
        }
        check(prm_rms_norm_backward(gy.const_data_ptr(), rg.ld, kept ? gh.const_data_ptr() : nullptr, rs.ld, h.const_data_ptr(), rh.ld,
                                    w.defined() ? w.const_data_ptr() : nullptr, code_of(h.scalar_type()), rh.rows, rh.cols,
                                    (float)ctx->saved_data["eps"].toDouble(), dx.data_ptr(), rh.cols, at_of(out[1]), at_of(ws), need,
                                    stream()));
      }
      if (ctx->needs_input_grad(0)) out[0] = dx;
      if (ctx->saved_data["res"].toBool() && ctx->needs_input_grad(w.defined() ? 2 : 1)) out[2] = dx;
    }
    return once(std::move(out), recording);
  }
};

// rms_norm(x, weight, residual, eps, quantize): y, (y, h), (q, scale) or (q, scale, h)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 5) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *x = plain(args[0]), *w, *res;
    if (!x || !optional(args[1], &w) || !optional(args[2], &res) || !PyFloat_CheckExact(args[3])) Py_RETURN_NONE;
    const double eps = PyFloat_AS_DOUBLE(args[3]);
    const bool quantize = args[4] == Py_True, record = records(x) || records(w) || records(res);
    Rows r;
    if ((quantize ? record : args[4] != Py_False) || code_of(x->scalar_type()) < 0 || !here(*x) || !rows_of(*x, &r) ||
        (w && !vector_of(*w, *x, x->scalar_type(), r.cols)))
      Py_RETURN_NONE;
    if (res && (res->scalar_type() != x->scalar_type() || res->sizes() != x->sizes() || res->device() != x->device() || !rows_of(*res, &r)))
      Py_RETURN_NONE;
    const Maybe wt = maybe(w), rt = maybe(res);
    variable_list out = record ? Norm::apply(*x, wt, rt, eps) : norm(*x, or_none(wt), or_none(rt), (float)eps, quantize);
    if (out.size() == 1) return wrap(std::move(out[0]));
    if (out.size() == 2) return Py_BuildValue("(NN)", wrap(std::move(out[0])), wrap(std::move(out[1])));
    return Py_BuildValue("(NNN)", wrap(std::move(out[0])), wrap(std::move(out[1])), wrap(std::move(out[2])));
  });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(quantize_rows), METHOD(quantize_cols), METHOD(int8_matmul), METHOD(int8_linear), METHOD(rms_norm),
                          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_operators", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__operators() {
  PyObject* nn = PyImport_ImportModule("torch.nn");
  if (!nn) return nullptr;
  g_parameter = PyObject_GetAttrString(nn, "Parameter");
  Py_DECREF(nn);
  if (!g_parameter) return nullptr;
  return PyModule_Create(&kModule);
}
