// Host side of the 8-bit linear layer's Python binding: the checks of plain calls, the
// outputs' allocation and the call into libprm, natively.  In Python they cost 15 to 25 us a
// call, several times the GPU's for one token.
//
// Every function returns what the operator does, a negative PRM_E* code that libprm gave
// (the caller raises it), or None: not a plain call (a tensor subclass, another device
// than the current one, a layout that needs a copy, a type or shape that is wrong, a
// gradient to record), and the Python binding then takes or refuses it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/prm.h"

namespace {

PyObject* g_parameter = nullptr;  // torch.nn.Parameter

// A strided device tensor whose metadata and pointer are its own: no subclass (those
// answer for themselves in Python), no functional transform's wrapper.
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o) && (PyObject*)Py_TYPE(o) != g_parameter) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || !t.is_cuda() || !t.has_storage() || t.layout() != at::kStrided) return nullptr;
  if (t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                               c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                               c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
                                               c10::DispatchKey::ZeroTensor})))
    return nullptr;
  return &t;
}

int code_of(at::ScalarType t) {
  return t == at::kFloat ? PRM_F32 : t == at::kBFloat16 ? PRM_BF16 : t == at::kHalf ? PRM_F16 : -1;
}
at::ScalarType type_of(long code) {
  return code == PRM_F32 ? at::kFloat : code == PRM_BF16 ? at::kBFloat16 : code == PRM_F16 ? at::kHalf : at::ScalarType::Undefined;
}

// The last dimension's rows as a matrix without a copy: 2-D with contiguous rows, or
// contiguous as a whole.
struct Rows {
  int64_t rows = 0, cols = 0, ld = 0;
};
bool rows_of(const at::Tensor& t, Rows* r) {
  const int64_t d = t.dim();
  if (d < 1) return false;
  r->cols = t.size(d - 1);
  if (r->cols < 1 || t.numel() == 0) return false;
  r->rows = t.numel() / r->cols;
  if (d == 2 && (t.stride(1) == 1 || r->cols == 1) && (t.stride(0) >= r->cols || r->rows == 1)) {
    r->ld = r->rows == 1 ? r->cols : t.stride(0);
    return true;
  }
  r->ld = r->cols;
  return t.is_contiguous();
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

template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {  // out of memory above all
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// ---- the operators on checked tensors; a negative code where libprm refuses ------------
struct Eight {
  at::Tensor q, scale, sum;
  Rows r;  // of q
  int rc = 0;
};
Eight rows_in_eight(const at::Tensor& x, const Rows& r) {
  Eight e;
  const c10::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
  e.q = eight_bits(lead, r.cols, x, &e.r.ld);
  e.r.rows = r.rows;
  e.r.cols = r.cols;
  e.scale = empty(lead, at::kFloat, x);
  e.rc = prm_quantize_rows(x.const_data_ptr(), code_of(x.scalar_type()), r.rows, r.cols, r.ld, (int8_t*)e.q.data_ptr(), e.r.ld,
                           (float*)e.scale.data_ptr(), stream());
  return e;
}
Eight cols_in_eight(const at::Tensor& x, const Rows& r, bool with_sum) {
  Eight e;
  e.q = eight_bits({r.cols}, r.rows, x, &e.r.ld);
  e.r.rows = r.cols;
  e.r.cols = r.rows;
  e.scale = empty({r.cols}, at::kFloat, x);
  if (with_sum) e.sum = empty({r.cols}, x.scalar_type(), x);
  const uint64_t need = prm_quantize_cols_workspace(r.rows, r.cols);
  at::Tensor ws = empty({(int64_t)need}, at::kByte, x);
  e.rc = prm_quantize_cols(x.const_data_ptr(), code_of(x.scalar_type()), r.rows, r.cols, r.ld, (int8_t*)e.q.data_ptr(), e.r.ld,
                           (float*)e.scale.data_ptr(), with_sum ? e.sum.data_ptr() : nullptr, ws.data_ptr(), need, stream());
  return e;
}
int product(const at::Tensor& a, const Rows& ra, const at::Tensor& sa, const at::Tensor& b, const Rows& rb, const at::Tensor& sb,
            const at::Tensor* bias, c10::IntArrayRef lead, int code, at::Tensor* out) {
  c10::SmallVector<int64_t, 6> size(lead.begin(), lead.end());
  size.push_back(rb.rows);
  *out = empty(size, type_of(code), a);
  const uint64_t need = prm_int8_matmul_workspace(ra.rows, rb.rows, ra.cols);
  at::Tensor ws;
  if (need) ws = empty({(int64_t)need}, at::kByte, a);
  return prm_int8_matmul((const int8_t*)a.const_data_ptr(), ra.ld, (const float*)sa.const_data_ptr(), (const int8_t*)b.const_data_ptr(),
                         rb.ld, (const float*)sb.const_data_ptr(), data(bias), code, out->data_ptr(), rb.rows, ra.rows, rb.rows, ra.cols,
                         need ? ws.data_ptr() : nullptr, need, stream());
}

// quantize_rows(x)
PyObject* quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 1) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor* x = plain(args[0]);
    Rows r;
    if (!x || code_of(x->scalar_type()) < 0 || !here(*x) || !rows_of(*x, &r)) Py_RETURN_NONE;
    Eight e = rows_in_eight(*x, r);
    if (e.rc < 0) return PyLong_FromLong(e.rc);
    return Py_BuildValue("(NN)", wrap(std::move(e.q)), wrap(std::move(e.scale)));
  });
}

// quantize_cols(x, with_sum)
PyObject* quantize_cols(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor* x = plain(args[0]);
    Rows r;
    if (!x || x->dim() != 2 || code_of(x->scalar_type()) < 0 || !here(*x) || !rows_of(*x, &r)) Py_RETURN_NONE;
    Eight e = cols_in_eight(*x, r, args[1] == Py_True);
    if (e.rc < 0) return PyLong_FromLong(e.rc);
    return Py_BuildValue("(NNN)", wrap(std::move(e.q)), wrap(std::move(e.scale)), wrap(std::move(e.sum)));
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
    const c10::IntArrayRef lead = a->sizes().slice(0, a->dim() - 1);
    if (sa->scalar_type() != at::kFloat || sa->sizes() != lead || !sa->is_contiguous() || sa->device() != a->device() ||
        !vector_of(*sb, *a, at::kFloat, rb.rows) || (bias && !vector_of(*bias, *a, type_of(code), rb.rows)))
      Py_RETURN_NONE;
    at::Tensor out;
    const int rc = product(*a, ra, *sa, *b, rb, *sb, bias, lead, (int)code, &out);
    if (rc < 0) return PyLong_FromLong(rc);
    return wrap(std::move(out));
  });
}

// linear_forward(x, weight, bias): the layer's output
PyObject* linear_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *x = plain(args[0]), *w = plain(args[1]), *bias;
    Rows rx, rw;
    if (!x || !w || !optional(args[2], &bias) || code_of(x->scalar_type()) < 0 || !here(*x) || w->dim() != 2 ||
        w->scalar_type() != x->scalar_type() || w->device() != x->device() || !rows_of(*x, &rx) || !rows_of(*w, &rw) || rx.cols != rw.cols ||
        (bias && !vector_of(*bias, *x, x->scalar_type(), rw.rows)))
      Py_RETURN_NONE;
    Eight ex = rows_in_eight(*x, rx);
    if (ex.rc < 0) return PyLong_FromLong(ex.rc);
    Eight ew = rows_in_eight(*w, rw);
    if (ew.rc < 0) return PyLong_FromLong(ew.rc);
    at::Tensor out;
    const int rc = product(ex.q, ex.r, ex.scale, ew.q, ew.r, ew.scale, bias, x->sizes().slice(0, x->dim() - 1), code_of(x->scalar_type()), &out);
    if (rc < 0) return PyLong_FromLong(rc);
    return wrap(std::move(out));
  });
}

// linear_backward(gy, x, weight, need_x, need_w, need_b): (dx, dw, db)
PyObject* linear_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *gy = plain(args[0]), *x = plain(args[1]), *w = plain(args[2]);
    Rows rg, rx, rw;
    if (!gy || !x || !w || code_of(x->scalar_type()) < 0 || !here(*x) || gy->scalar_type() != x->scalar_type() || gy->device() != x->device() ||
        w->scalar_type() != x->scalar_type() || w->device() != x->device() || !rows_of(*gy, &rg) || !rows_of(*x, &rx) || !rows_of(*w, &rw) ||
        rg.rows != rx.rows || rg.cols != rw.rows || rx.cols != rw.cols)
      Py_RETURN_NONE;
    const bool need_x = args[3] == Py_True, need_w = args[4] == Py_True, need_b = args[5] == Py_True;
    const int code = code_of(x->scalar_type());
    at::Tensor dx, dw, db;
    if (need_x) {
      Eight g = rows_in_eight(*gy, rg);
      if (g.rc < 0) return PyLong_FromLong(g.rc);
      Eight ew = cols_in_eight(*w, rw, false);
      if (ew.rc < 0) return PyLong_FromLong(ew.rc);
      const int rc = product(g.q, g.r, g.scale, ew.q, ew.r, ew.scale, nullptr, x->sizes().slice(0, x->dim() - 1), code, &dx);
      if (rc < 0) return PyLong_FromLong(rc);
    }
    if (need_w || need_b) {
      Eight g = cols_in_eight(*gy, rg, need_b);
      if (g.rc < 0) return PyLong_FromLong(g.rc);
      db = g.sum;
      if (need_w) {
        Eight ex = cols_in_eight(*x, rx, false);
        if (ex.rc < 0) return PyLong_FromLong(ex.rc);
        const int64_t rows[1] = {rg.cols};
        const int rc = product(g.q, g.r, g.scale, ex.q, ex.r, ex.scale, nullptr, rows, code, &dw);
        if (rc < 0) return PyLong_FromLong(rc);
      }
    }
    return Py_BuildValue("(NNN)", wrap(std::move(dx)), wrap(std::move(dw)), wrap(std::move(db)));
  });
}

// rms_norm(x, weight, residual, eps, quantize, record): y, (y, h), (q, scale) or (q, scale, h);
// None where a gradient is to be recorded, unless `record` says that the caller does that
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *x = plain(args[0]), *w, *res;
    if (!x || !optional(args[1], &w) || !optional(args[2], &res) || !PyFloat_CheckExact(args[3])) Py_RETURN_NONE;
    const float eps = (float)PyFloat_AS_DOUBLE(args[3]);
    const bool quantize = args[4] == Py_True;
    if (args[5] != Py_True && (records(x) || records(w) || records(res))) Py_RETURN_NONE;
    Rows r, rr;
    const int code = code_of(x->scalar_type());
    if (code < 0 || !here(*x) || !rows_of(*x, &r) || (w && !vector_of(*w, *x, x->scalar_type(), r.cols))) Py_RETURN_NONE;
    if (res && (res->scalar_type() != x->scalar_type() || res->sizes() != x->sizes() || res->device() != x->device() || !rows_of(*res, &rr)))
      Py_RETURN_NONE;
    at::Tensor h, y, q, s;
    int64_t ldq = 0;
    if (res) h = empty(x->sizes(), x->scalar_type(), *x);
    if (quantize) {
      const c10::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
      q = eight_bits(lead, r.cols, *x, &ldq);
      s = empty(lead, at::kFloat, *x);
    } else {
      y = empty(x->sizes(), x->scalar_type(), *x);
    }
    const int rc = prm_rms_norm(x->const_data_ptr(), r.ld, data(res), rr.ld, data(w), code, r.rows, r.cols, eps, res ? h.data_ptr() : nullptr,
                                r.cols, quantize ? nullptr : y.data_ptr(), r.cols, quantize ? (int8_t*)q.data_ptr() : nullptr, ldq,
                                quantize ? (float*)s.data_ptr() : nullptr, stream());
    if (rc < 0) return PyLong_FromLong(rc);
    if (quantize)
      return res ? Py_BuildValue("(NNN)", wrap(std::move(q)), wrap(std::move(s)), wrap(std::move(h)))
                 : Py_BuildValue("(NN)", wrap(std::move(q)), wrap(std::move(s)));
    return res ? Py_BuildValue("(NN)", wrap(std::move(y)), wrap(std::move(h))) : wrap(std::move(y));
  });
}

// rms_norm_backward(gy, gh, h, weight, eps, need_dw): (dx, dw)
PyObject* rms_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const at::Tensor *gy = plain(args[0]), *gh, *h = plain(args[2]), *w;
    if (!gy || !optional(args[1], &gh) || !h || !optional(args[3], &w) || !PyFloat_CheckExact(args[4])) Py_RETURN_NONE;
    const bool need_dw = args[5] == Py_True;
    Rows rg, rs, rh;
    const int code = code_of(h->scalar_type());
    if (code < 0 || !here(*h) || !rows_of(*h, &rh) || !rows_of(*gy, &rg) || (gh && !rows_of(*gh, &rs)) ||
        (w && !vector_of(*w, *h, h->scalar_type(), rh.cols)))
      Py_RETURN_NONE;
    for (const at::Tensor* t : {gy, gh})
      if (t && (t->scalar_type() != h->scalar_type() || t->sizes() != h->sizes() || t->device() != h->device())) Py_RETURN_NONE;
    at::Tensor dx = empty(h->sizes(), h->scalar_type(), *h), dw, ws;
    uint64_t need = 0;
    if (need_dw) {
      dw = empty({rh.cols}, h->scalar_type(), *h);
      need = prm_rms_norm_backward_workspace(rh.rows, rh.cols);
      ws = empty({(int64_t)need}, at::kByte, *h);
    }
    const int rc = prm_rms_norm_backward(gy->const_data_ptr(), rg.ld, data(gh), rs.ld, h->const_data_ptr(), rh.ld, data(w), code, rh.rows,
                                         rh.cols, (float)PyFloat_AS_DOUBLE(args[4]), dx.data_ptr(), rh.cols, need_dw ? dw.data_ptr() : nullptr,
                                         need_dw ? ws.data_ptr() : nullptr, need, stream());
    if (rc < 0) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", wrap(std::move(dx)), wrap(std::move(dw)));
  });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {METHOD(quantize_rows), METHOD(quantize_cols),     METHOD(int8_matmul),
                          METHOD(linear_forward), METHOD(linear_backward),  METHOD(rms_norm),
                          METHOD(rms_norm_backward), {nullptr, nullptr, 0, nullptr}};

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
