// CPython module behind paper_2511_05814_amd.attention: checks of tensors,
// allocation of results and the calls of the C ABI (include/moe_offload.h).
//
// A decode step makes a dozen of these calls a layer, and a kernel launch takes
// the host some 3 us; through ctypes the checks and the marshalling took more
// than that.  Every function takes its positional arguments in attention.py's
// order and the stream as an integer last.  ValueError: tensors that do not fit
// together; the classes given to set_errors: what the library refuses, and no
// memory for a result or a workspace.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include "moe_offload.h"

namespace {

PyObject *g_error = nullptr;     // binding.MoeError
PyObject *g_memory = nullptr;    // torch.OutOfMemoryError

// Thrown with the Python error set.
struct Raised {};

[[noreturn]] void value_error(const std::string &what) {
  PyErr_SetString(PyExc_ValueError, what.c_str());
  throw Raised();
}

void check_rc(int rc, const char *where) {
  if (rc == MOE_OK) return;
  PyObject *e = g_error ? PyObject_CallFunction(g_error, "iss", rc, where, moe_last_error()) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_Format(PyExc_RuntimeError, "%s failed with %d: %s", where, rc, moe_last_error());
  }
  throw Raised();
}

const at::Tensor &tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) value_error(std::string(name) + " must be a tensor");
  const at::Tensor &t = THPVariable_Unpack(o);
  // the result would come back detached
  if (t.requires_grad() && c10::GradMode::is_enabled())
    value_error(std::string(name) + " requires grad, and these operators have no gradient: detach it or use torch.no_grad()");
  return t;
}
bool given(PyObject *o) { return o != Py_None; }

int64_t integer(PyObject *o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
// An int of the C ABI; out-of-range values go on as one that it refuses.
int small(int64_t v) { return v > INT32_MAX || v < INT32_MIN ? INT32_MIN : (int)v; }
double real(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}
void *stream_of(PyObject *o) {
  void *p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised();
  return p;
}

std::string text(const at::Tensor &t) {
  std::ostringstream s;
  s << t.scalar_type() << " " << t.sizes() << " of strides " << t.strides() << " on " << t.device();
  return s.str();
}
[[noreturn]] void bad(const char *name, const at::Tensor &t, at::ScalarType type, at::IntArrayRef shape, int device) {
  std::ostringstream s;
  s << name << " must be " << type << " " << shape << " with contiguous rows on GPU " << device << ", not " << text(t);
  value_error(s.str());
}

int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return MOE_DTYPE_F32;
  if (t == at::kBFloat16) return MOE_DTYPE_BF16;
  std::ostringstream s;
  s << "tensors must be float32 or bfloat16, not " << t;
  value_error(s.str());
}

struct Where {
  int device;
  at::ScalarType type;
  int code;
};
Where where(const at::Tensor &t, at::ScalarType type) {
  if (!t.is_cuda()) value_error("tensors must be on the GPU, not on " + t.device().str());
  return Where{t.get_device(), type, dtype_code(type)};
}

// Elements between the rows of t, which must be of this type, device and shape
// (2 or 3 dimensions), everything but the first contiguous.
int64_t rows(const char *name, const at::Tensor &t, int device, at::ScalarType type, at::IntArrayRef shape) {
  if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.sizes() != shape) bad(name, t, type, shape, device);
  int64_t inner = 1;
  for (size_t d = shape.size() - 1; d > 0; --d) {
    if (shape[d] > 1 && t.stride(d) != inner) bad(name, t, type, shape, device);
    inner *= shape[d];
  }
  return shape[0] > 1 ? t.stride(0) : inner;
}

void *vector(const char *name, const at::Tensor &t, int device, at::ScalarType type, int64_t n) {
  if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
    bad(name, t, type, {n}, device);
  return t.data_ptr();
}

void dims(const char *name, const at::Tensor &t, int64_t n, const char *what) {
  if (t.dim() != n) value_error(std::string(name) + " must be " + what);
}

moe_kv4_batch batch_of(int device, const at::Tensor &pool, const at::Tensor &table, const at::Tensor &start,
                       const at::Tensor &length, int64_t tokens, int64_t head_dim) {
  if (pool.dim() != 3 || pool.scalar_type() != at::kByte || !pool.is_contiguous() || !pool.is_cuda() || pool.get_device() != device)
    value_error("pool must be a contiguous uint8 [pages, kv heads, record] on the call's GPU, not " + text(pool));
  const int64_t record = pool.size(2), page = head_dim > 0 ? record * 8 / (9 * head_dim) : 0;
  if (head_dim <= 0 || page * head_dim * 9 != record * 8)
    value_error("records of " + std::to_string(record) + " bytes are not whole tokens of " + std::to_string(head_dim) + " dimensions");
  dims("page_table", table, 2, "[sequences, columns]");
  const int64_t seqs = table.size(0), cols = table.size(1);
  moe_kv4_batch b;
  b.table_stride = rows("page_table", table, device, at::kInt, {seqs, cols});
  b.pool = pool.data_ptr();
  b.page_table = static_cast<const int32_t *>(table.data_ptr());
  b.q_start = static_cast<const int32_t *>(vector("q_start", start, device, at::kInt, seqs + 1));
  b.kv_len = static_cast<const int32_t *>(vector("kv_len", length, device, at::kInt, seqs));
  b.pages = small(pool.size(0));
  b.page_size = small(page);
  b.kv_heads = small(pool.size(1));
  b.head_dim = small(head_dim);
  b.table_cols = small(cols);
  b.seqs = small(seqs);
  b.tokens = small(tokens);
  return b;
}

// Takes n arguments and runs f, which returns a new reference.
template <typename F>
PyObject *call(Py_ssize_t got, Py_ssize_t n, F f) {
  if (got != n) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", n, got);
    return nullptr;
  }
  try {
    return f();
  } catch (const Raised &) {
  } catch (const c10::OutOfMemoryError &e) {
    PyErr_SetString(g_memory ? g_memory : PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject *q4_matmul(PyObject *, PyObject *const *a, Py_ssize_t got) {
  return call(got, 5, [&] {
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w");
    const int64_t n = integer(a[2]);
    dims("x", x, 2, "[rows, k]");
    const int64_t t = x.size(0), k = x.size(1);
    const Where at_ = where(x, x.scalar_type());
    const size_t bytes = n > 0 && k > 0 ? moe_q4_matrix_bytes((size_t)n, (size_t)k) : 0;
    if (!bytes) value_error("a 4-bit matrix [" + std::to_string(n) + " x " + std::to_string(k) + "]: columns must be a multiple of 64");
    const void *weights = vector("w", w, at_.device, at::kByte, (int64_t)bytes);
    const int64_t x_stride = rows("x", x, at_.device, at_.type, {t, k});
    at::Tensor y = given(a[3]) ? tensor(a[3], "out") : at::empty({t, n}, x.options());
    const int64_t y_stride = given(a[3]) ? rows("out", y, at_.device, at_.type, {t, n}) : n;
    check_rc(moe_q4_matmul(x.data_ptr(), x_stride, weights, y.data_ptr(), y_stride, small(t), small(n), small(k), at_.code,
                           stream_of(a[4])), "moe_q4_matmul");
    return THPVariable_Wrap(std::move(y));
  });
}

PyObject *kv4_append(PyObject *, PyObject *const *a, Py_ssize_t got) {
  return call(got, 11, [&] {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &cos = tensor(a[3], "cos"), &sin = tensor(a[4], "sin");
    dims("q", q, 3, "[tokens, heads, head_dim]");
    dims("cos", cos, 2, "[positions, rot_dim / 2]");
    const int64_t t = q.size(0), heads = q.size(1), d = q.size(2), positions = cos.size(0), half = cos.size(1);
    const Where at_ = where(q, q.scalar_type());
    const moe_kv4_batch b = batch_of(at_.device, tensor(a[5], "pool"), tensor(a[6], "page_table"), tensor(a[7], "q_start"), tensor(a[8], "kv_len"), t, d);
    rows("cos", cos, at_.device, at::kFloat, {positions, half});
    rows("sin", sin, at_.device, at::kFloat, {positions, half});
    if (!cos.is_contiguous() || !sin.is_contiguous()) value_error("cos and sin must be contiguous");
    const int64_t qs = rows("q", q, at_.device, at_.type, {t, heads, d});
    const int64_t ks = rows("k", k, at_.device, at_.type, {t, (int64_t)b.kv_heads, d});
    const int64_t vs = rows("v", v, at_.device, at_.type, {t, (int64_t)b.kv_heads, d});
    at::Tensor o = given(a[9]) ? tensor(a[9], "out") : at::empty({t, heads, d}, q.options());
    const int64_t os = given(a[9]) ? rows("out", o, at_.device, at_.type, {t, heads, d}) : heads * d;
    check_rc(moe_kv4_append(&b, q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, static_cast<const float *>(cos.data_ptr()),
                            static_cast<const float *>(sin.data_ptr()), small(positions), small(2 * half), o.data_ptr(), os, small(heads),
                            at_.code, stream_of(a[10])), "moe_kv4_append");
    return THPVariable_Wrap(std::move(o));
  });
}

PyObject *kv4_read(PyObject *, PyObject *const *a, Py_ssize_t got) {
  return call(got, 8, [&] {
    const at::Tensor &pool = tensor(a[0], "pool");
    const int64_t t = integer(a[4]), d = integer(a[5]);
    const Where at_ = where(pool, integer(a[6]) == MOE_DTYPE_F32 ? at::kFloat : at::kBFloat16);
    if (t < 0) value_error("tokens must not be negative");
    const moe_kv4_batch b = batch_of(at_.device, pool, tensor(a[1], "page_table"), tensor(a[2], "q_start"), tensor(a[3], "kv_len"), t, d);
    at::Tensor k = at::empty({t, b.kv_heads, d}, pool.options().dtype(at_.type)), v = at::empty({t, b.kv_heads, d}, k.options());
    check_rc(moe_kv4_read(&b, k.data_ptr(), v.data_ptr(), at_.code, stream_of(a[7])), "moe_kv4_read");
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
  });
}

PyObject *kv4_attention(PyObject *, PyObject *const *a, Py_ssize_t got) {
  return call(got, 11, [&] {
    const at::Tensor &q = tensor(a[0], "q");
    dims("q", q, 3, "[tokens, heads, head_dim]");
    const int64_t t = q.size(0), heads = q.size(1), d = q.size(2);
    const Where at_ = where(q, q.scalar_type());
    const moe_kv4_batch b = batch_of(at_.device, tensor(a[1], "pool"), tensor(a[2], "page_table"), tensor(a[3], "q_start"), tensor(a[4], "kv_len"), t, d);
    const int64_t seqs = std::max<int64_t>(1, b.seqs);
    const int max_new = given(a[6]) ? small(integer(a[6])) : (int)std::max<int64_t>(1, (t + seqs - 1) / seqs);
    const int max_len = given(a[7]) ? small(integer(a[7])) : small(std::max<int64_t>(1, (int64_t)b.table_cols * b.page_size));
    const int64_t qs = rows("q", q, at_.device, at_.type, {t, heads, d});
    at::Tensor o = given(a[8]) ? tensor(a[8], "out") : at::empty({t, heads, d}, q.options());
    const int64_t os = given(a[8]) ? rows("out", o, at_.device, at_.type, {t, heads, d}) : heads * d;
    at::Tensor workspace;
    size_t bytes = 0;
    if (given(a[9])) {
      workspace = tensor(a[9], "workspace");
      bytes = (size_t)workspace.numel();
      vector("workspace", workspace, at_.device, at::kByte, (int64_t)bytes);
    } else {
      bytes = moe_kv4_attention_workspace_bytes(&b, small(heads), max_new, max_len);
      if (bytes) workspace = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
    }
    check_rc(moe_kv4_attention(&b, q.data_ptr(), qs, o.data_ptr(), os, small(heads), (float)real(a[5]), at_.code, max_new, max_len,
                               bytes ? workspace.data_ptr() : nullptr, bytes, stream_of(a[10])), "moe_kv4_attention");
    return THPVariable_Wrap(std::move(o));
  });
}

PyObject *norm_residual(PyObject *, PyObject *const *a, Py_ssize_t got) {
  return call(got, 12, [&] {
    const at::Tensor &h = tensor(a[0], "h");
    dims("h", h, 2, "[rows, d]");
    const int64_t n = h.size(0), d = h.size(1), code = integer(a[7]);  // code: of x without y, or -1
    const at::ScalarType type = given(a[1]) ? tensor(a[1], "y").scalar_type() : code == MOE_DTYPE_BF16 ? at::kBFloat16 : at::kFloat;
    const Where at_ = where(h, type);
    if (given(a[1]) && code >= 0 && code != at_.code) value_error("y is of another type than dtype");
    const int64_t hs = rows("h", h, at_.device, at::kFloat, {n, d});
    const void *y = nullptr;
    int64_t ys = d, gs = 0, ho_s = d;
    if (given(a[1])) {
      ys = rows("y", tensor(a[1], "y"), at_.device, type, {n, d});
      y = tensor(a[1], "y").data_ptr();
    }
    const float *vec[3] = {nullptr, nullptr, nullptr};  // gate, post, pre
    if (given(a[2])) {
      const at::Tensor &gate = tensor(a[2], "gate");
      if (gate.dim() == 1) {
        vec[0] = static_cast<const float *>(vector("gate", gate, at_.device, at::kFloat, d));
      } else {
        gs = rows("gate", gate, at_.device, at::kFloat, {n, d});
        vec[0] = static_cast<const float *>(gate.data_ptr());
      }
    }
    if (given(a[3])) vec[1] = static_cast<const float *>(vector("post", tensor(a[3], "post"), at_.device, at::kFloat, d));
    if (given(a[4])) vec[2] = static_cast<const float *>(vector("pre", tensor(a[4], "pre"), at_.device, at::kFloat, d));
    at::Tensor h_out, x;
    if (given(a[8])) {
      h_out = tensor(a[8], "h_out");
      ho_s = rows("h_out", h_out, at_.device, at::kFloat, {n, d});
    } else if (PyObject_IsTrue(a[9])) {
      h_out = at::empty({n, d}, h.options());
    }
    if (PyObject_IsTrue(a[10])) x = at::empty({n, d}, h.options().dtype(type));
    check_rc(moe_norm_residual(static_cast<const float *>(h.data_ptr()), hs, y, ys, vec[0], gs, vec[1], vec[2], (float)real(a[5]),
                               (float)real(a[6]), h_out.defined() ? static_cast<float *>(h_out.data_ptr()) : nullptr, ho_s,
                               x.defined() ? x.data_ptr() : nullptr, d, small(n), small(d), at_.code, stream_of(a[11])),
             "moe_norm_residual");
    PyObject *first;
    if (given(a[8])) {
      Py_INCREF(a[8]);
      first = a[8];
    } else if (h_out.defined()) {
      first = THPVariable_Wrap(std::move(h_out));
    } else {
      Py_INCREF(Py_None);
      first = Py_None;
    }
    if (x.defined()) return Py_BuildValue("(NN)", first, THPVariable_Wrap(std::move(x)));
    return Py_BuildValue("(NO)", first, Py_None);
  });
}

void set_class(PyObject **to, PyObject *cls) {
  Py_INCREF(cls);
  Py_XDECREF(*to);
  *to = cls;
}
PyObject *set_errors(PyObject *, PyObject *args) {
  PyObject *error, *memory;
  if (!PyArg_ParseTuple(args, "OO", &error, &memory)) return nullptr;
  set_class(&g_error, error);
  set_class(&g_memory, memory);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(q4_matmul), FAST(kv4_append), FAST(kv4_read), FAST(kv4_attention), FAST(norm_residual),
                         {"set_errors", set_errors, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_attention_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attention_ops() { return PyModule_Create(&module_def); }
