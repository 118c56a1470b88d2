// Module descriptors of a projection call, and the rows of a token loss, gathered
// from the Python objects.
//
// A call over a model's modules passes four tensors each: checking them and
// reading their pointers, shapes and strides attribute by attribute from Python
// took 250 us for 48 modules, several times what the kernels of a short batch
// take (here: 15 us).  modules() makes the binding's checks on exact torch
// tensors and returns None as soon as one does not hold or anything is of
// another kind (a subclass, a wrapper without storage, a CPU tensor): the
// binding's own Python checks then run, and raise or accept.  token_call() makes the
// checks of a token loss on its rows and vectors, and the library's call too (the
// checks in Python take 7 us, where a small call's kernel takes 4); rows_call() does the same
// for embedding and layer norm over token rows.  written() tells autograd
// of tensors that a call wrote through their pointers (168 weights: under 2 us, 8 us in
// Python): a backward pass that saved their earlier values then raises, as after any change
// in place.
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <vector>

#include "attr.h"

namespace {

struct Names {
  PyObject *a, *g, *R, *S, *out_col, *v_out, *v_in;
  PyObject *logits, *target, *weight, *n_examples, *T, *row_offset, *length, *logit_scale;
} names;

// a new reference, or NULL
struct Ref {
  PyObject* p;
  explicit Ref(PyObject* o) : p(o) {}
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  ~Ref() { Py_XDECREF(p); }
};

const at::Tensor* tensor_of(PyObject* o) {
  return o && THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr;
}

// rows, width and row stride of a tensor whose last dimension is contiguous
// and whose leading dimensions are packed
bool rows_of(const at::Tensor& t, int64_t& rows, int64_t& width, int64_t& ld) {
  const int64_t n = t.dim();
  if (n < 2 || t.stride(n - 1) != 1) return false;
  rows = 1;
  for (int64_t d = 0; d < n - 1; ++d) rows *= t.size(d);
  for (int64_t d = 0; d < n - 2; ++d)
    if (t.stride(d) != t.stride(d + 1) * t.size(d + 1)) return false;
  width = t.size(n - 1);
  ld = t.stride(n - 2);
  return true;
}

bool on(const at::Tensor& t, const at::Device& dev) { return t.is_cuda() && t.device() == dev; }

// None, or a contiguous vector of `type` on dev with at least n elements
bool vector_ok(PyObject* o, at::ScalarType type, int64_t n, const at::Device& dev) {
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o);
  return t && t->scalar_type() == type && t->is_contiguous() && t->numel() >= n && on(*t, dev);
}

bool matrix_ok(const at::Tensor* t, at::ScalarType type, int64_t r, int64_t c, const at::Device& dev) {
  return t && t->scalar_type() == type && t->dim() == 2 && t->size(0) == r && t->size(1) == c &&
         t->is_contiguous() && on(*t, dev);
}

// an optional fp32 factor of n elements; sets *p (NULL for None)
bool factor_ok(PyObject* o, int64_t n, const at::Device& dev, const float** p) {
  *p = nullptr;
  if (!o) return false;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o);
  if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() != n || !on(*t, dev))
    return false;
  *p = static_cast<const float*>(t->mutable_data_ptr());
  return true;
}

bool gather(PyObject* mods, PyObject* module_type, int64_t k, int64_t n_ex, int64_t T, PyObject* row_offset,
            PyObject* length, PyObject* out_o, int64_t rows_needed, std::vector<attr_module>& cm, int& dtype) {
  if (!PyList_CheckExact(mods) && !PyTuple_CheckExact(mods)) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(mods);
  const at::Tensor* out = tensor_of(out_o);
  if (n < 1 || !out || !out->is_cuda() || out->scalar_type() != at::kFloat || out->dim() != 2 ||
      out->stride(1) != 1 || out->size(0) < rows_needed || n_ex < 0 || T < 1)
    return false;
  const at::Device dev = out->device();
  if (!vector_ok(row_offset, at::kLong, n_ex, dev) || !vector_ok(length, at::kInt, n_ex, dev)) return false;
  at::ScalarType type = at::kFloat;
  cm.resize((size_t)n);
  for (Py_ssize_t j = 0; j < n; ++j) {
    PyObject* m = PySequence_Fast_GET_ITEM(mods, j);
    if ((PyObject*)Py_TYPE(m) != module_type) return false;
    const Ref a(PyObject_GetAttr(m, names.a)), g(PyObject_GetAttr(m, names.g)), R(PyObject_GetAttr(m, names.R)),
        S(PyObject_GetAttr(m, names.S)), col(PyObject_GetAttr(m, names.out_col)),
        vo(PyObject_GetAttr(m, names.v_out)), vi(PyObject_GetAttr(m, names.v_in));
    const at::Tensor *ta = tensor_of(a.p), *tg = tensor_of(g.p);
    if (!ta || !tg || !col.p || !PyLong_CheckExact(col.p)) return false;
    if (j == 0) {
      type = ta->scalar_type();
      if (type != at::kFloat && type != at::kBFloat16) return false;
    }
    attr_module& c = cm[(size_t)j];
    int64_t na, ng, d_in, d_out, lda, ldg;
    if (ta->scalar_type() != type || tg->scalar_type() != type || !on(*ta, dev) || !on(*tg, dev) ||
        !rows_of(*ta, na, d_in, lda) || !rows_of(*tg, ng, d_out, ldg))
      return false;
    if (row_offset == Py_None && (na < n_ex * T || ng < n_ex * T)) return false;
    const at::Tensor *tR = tensor_of(R.p), *tS = tensor_of(S.p);
    if (!matrix_ok(tR, type, d_out, k, dev) || !matrix_ok(tS, type, d_in, k, dev)) return false;
    if (!factor_ok(vo.p, d_out, dev, &c.v_out) || !factor_ok(vi.p, d_in, dev, &c.v_in)) return false;
    c.out_col = PyLong_AsLongLong(col.p);
    if (PyErr_Occurred() || c.out_col < 0 || c.out_col > out->size(1) - k * k) return false;
    c.a = ta->mutable_data_ptr();
    c.g = tg->mutable_data_ptr();
    c.R = tR->mutable_data_ptr();
    c.S = tS->mutable_data_ptr();
    c.lda = lda;
    c.ldg = ldg;
    c.d_in = d_in;
    c.d_out = d_out;
  }
  dtype = type == at::kFloat ? ATTR_F32 : ATTR_BF16;
  return true;
}

// modules(mods, Module, k, n_examples, T, row_offset, length, out, rows_needed)
// -> (dtype code, bytearray of attr_module) or None
PyObject* py_modules(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 9) {
    PyErr_SetString(PyExc_TypeError, "modules() takes 9 arguments");
    return nullptr;
  }
  int64_t v[4];
  const int at_arg[4] = {2, 3, 4, 8};
  bool ok = true;
  for (int i = 0; ok && i < 4; ++i) {
    ok = PyLong_CheckExact(args[at_arg[i]]);
    if (ok) v[i] = PyLong_AsLongLong(args[at_arg[i]]);
    // sizes whose products stay inside 64 bits
    ok = ok && !PyErr_Occurred() && v[i] >= 0 && v[i] <= ((int64_t)1 << 31);
  }
  std::vector<attr_module> cm;
  int dtype = 0;
  try {
    ok = ok && gather(args[0], args[1], v[0], v[1], v[2], args[5], args[6], args[7], v[3], cm, dtype);
  } catch (...) {  // a tensor without storage, for one
    ok = false;
  }
  if (!ok) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  PyObject* buf = PyByteArray_FromStringAndSize(reinterpret_cast<const char*>(cm.data()),
                                                (Py_ssize_t)(cm.size() * sizeof(attr_module)));
  return buf ? Py_BuildValue("iN", dtype, buf) : nullptr;
}

// a size that products of two stay inside 64 bits with
bool size_of(PyObject* o, int64_t& v) {
  if (!o || !PyLong_CheckExact(o)) return false;
  v = PyLong_AsLongLong(o);
  return !PyErr_Occurred() && v >= 0 && v <= ((int64_t)1 << 31);
}

// None or a tuple of fp32 vectors (or None) of at least n elements on dev
bool vectors_ok(PyObject* o, int64_t n, const at::Device& dev) {
  if (!PyTuple_CheckExact(o)) return false;
  for (Py_ssize_t j = 0; j < PyTuple_GET_SIZE(o); ++j)
    if (!vector_ok(PyTuple_GET_ITEM(o, j), at::kFloat, n, dev)) return false;
  return true;
}

bool gather_rows(PyObject* rows, PyObject* rows_type, PyObject* const* vecs, PyObject* dlogits, attr_token_rows& c,
                 int64_t& ldd) {
  if ((PyObject*)Py_TYPE(rows) != rows_type) return false;
  const Ref logits(PyObject_GetAttr(rows, names.logits)), target(PyObject_GetAttr(rows, names.target)),
      weight(PyObject_GetAttr(rows, names.weight)), n_ex(PyObject_GetAttr(rows, names.n_examples)),
      T(PyObject_GetAttr(rows, names.T)), off(PyObject_GetAttr(rows, names.row_offset)),
      len(PyObject_GetAttr(rows, names.length)), scale(PyObject_GetAttr(rows, names.logit_scale));
  const at::Tensor *z = tensor_of(logits.p), *y = tensor_of(target.p);
  if (!z || !y || !weight.p || !off.p || !len.p || !scale.p || !PyFloat_CheckExact(scale.p) || !z->is_cuda() ||
      !size_of(n_ex.p, c.n_examples) || !size_of(T.p, c.T) || c.T < 1)
    return false;
  const at::Device dev = z->device();
  const at::ScalarType type = z->scalar_type();
  if (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf) return false;
  if (!rows_of(*z, c.n_rows, c.V, c.ldl) || (off.p == Py_None && c.n_rows < c.n_examples * c.T)) return false;
  if (target.p == Py_None || !vector_ok(target.p, at::kLong, c.n_rows, dev) ||
      !vector_ok(weight.p, at::kFloat, c.n_rows, dev) || !vector_ok(off.p, at::kLong, c.n_examples, dev) ||
      !vector_ok(len.p, at::kInt, c.n_examples, dev) || !vectors_ok(vecs[0], c.n_rows, dev) ||
      !vectors_ok(vecs[1], c.n_examples, dev) || !vectors_ok(vecs[2], c.n_examples / 2, dev))
    return false;
  ldd = 0;
  if (dlogits != Py_None) {
    const at::Tensor* d = tensor_of(dlogits);
    int64_t n, V;
    if (!d || !on(*d, dev) || d->scalar_type() != type || !rows_of(*d, n, V, ldd) || n != c.n_rows || V != c.V)
      return false;
  }
  auto ptr = [](PyObject* o) -> void* { return o == Py_None ? nullptr : THPVariable_Unpack(o).mutable_data_ptr(); };
  c.logits = z->mutable_data_ptr();
  c.dtype = type == at::kFloat ? ATTR_F32 : type == at::kBFloat16 ? ATTR_BF16 : ATTR_F16;
  c.logit_scale = (float)PyFloat_AS_DOUBLE(scale.p);
  c.target = static_cast<const int64_t*>(y->mutable_data_ptr());
  c.weight = static_cast<const float*>(ptr(weight.p));
  c.row_offset = static_cast<const int64_t*>(ptr(off.p));
  c.length = static_cast<const int32_t*>(ptr(len.p));
  return true;
}

float* floats(PyObject* tuple, Py_ssize_t j) {
  PyObject* o = PyTuple_GET_ITEM(tuple, j);
  return o == Py_None ? nullptr : static_cast<float*>(THPVariable_Unpack(o).mutable_data_ptr());
}

void bump(PyObject* o) {
  if (!o || !THPVariable_Check(o)) return;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();  // inference tensors count no versions
}

// written(list or tuple of tensors) -> True, or None where it is neither
PyObject* py_written(PyObject*, PyObject* seq) {
  if (!PyList_CheckExact(seq) && !PyTuple_CheckExact(seq)) Py_RETURN_NONE;
  try {
    for (Py_ssize_t j = 0; j < PySequence_Fast_GET_SIZE(seq); ++j) bump(PySequence_Fast_GET_ITEM(seq, j));
  } catch (...) {
    Py_RETURN_NONE;
  }
  Py_RETURN_TRUE;
}

// The library's entry points, by the numbers that token_call() takes.
typedef attr_status (*LogpFn)(const attr_token_rows*, float*, void*, size_t, void*);
typedef attr_status (*PolicyFn)(const attr_token_rows*, const float*, int32_t, const float*, const float*, float, float,
                                float, float*, float*, void*, int64_t, void*, size_t, void*);
typedef attr_status (*PreferenceFn)(const attr_token_rows*, const float*, const float*, float, float, float, float*,
                                    float*, float*, void*, int64_t, void*, size_t, void*);
constexpr int kLogp = 0, kPolicy = 1, kPolicyPerToken = 2, kPreference = 3;

// token_call(op, address, rows, TokenRows, per_row, per_example, per_pair, dlogits,
//            scalars, workspace, workspace_bytes, stream) -> status, or None
// The three tuples hold the call's fp32 vectors by the number of their elements:
//   attr_token_logp       (logp), (), ()
//   attr_policy_loss      (logp, logp_old, logp_ref), (loss, advantage), ()
//    with per_token       (logp, logp_old, logp_ref, advantage), (loss), ()
//   attr_preference_loss  (logp, logp_ref), (log_ratio), (loss, pair_weight)
// scalars: three numbers (clip_low, clip_high, beta; beta, margin, label_smoothing).
PyObject* py_token_call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 12) {
    PyErr_SetString(PyExc_TypeError, "token_call() takes 12 arguments");
    return nullptr;
  }
  attr_token_rows c;
  std::memset(&c, 0, sizeof(c));
  int64_t ldd = 0;
  bool ok = false;
  double x[3] = {0, 0, 0};
  void* d = nullptr;
  const long op = PyLong_AsLong(args[0]);
  void* fn = PyLong_AsVoidPtr(args[1]);
  void* ws = PyLong_AsVoidPtr(args[9]);
  const size_t ws_bytes = PyLong_AsSize_t(args[10]);
  void* stream = PyLong_AsVoidPtr(args[11]);
  PyObject* const* v = args + 4;
  try {
    ok = !PyErr_Occurred() && fn && gather_rows(args[2], args[3], v, args[7], c, ldd) && PyTuple_CheckExact(args[8]) &&
         PyTuple_GET_SIZE(args[8]) == (op == kLogp ? 0 : 3);
    if (ok && args[7] != Py_None) d = THPVariable_Unpack(args[7]).mutable_data_ptr();
  } catch (...) {  // a tensor without storage, for one
    ok = false;
  }
  for (int k = 0; ok && op != kLogp && k < 3; ++k) x[k] = PyFloat_AsDouble(PyTuple_GET_ITEM(args[8], k));
  const int sizes[4][3] = {{1, 0, 0}, {3, 2, 0}, {4, 1, 0}, {2, 1, 2}};
  ok = ok && !PyErr_Occurred() && op >= 0 && op <= 3;
  for (int k = 0; ok && k < 3; ++k) ok = PyTuple_GET_SIZE(v[k]) == sizes[op][k];
  if (!ok) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  attr_status st;
  try {
    float *r0 = floats(v[0], 0), *r1 = op == kLogp ? nullptr : floats(v[0], 1),
          *r2 = op == kPolicy || op == kPolicyPerToken ? floats(v[0], 2) : nullptr,
          *e0 = op == kLogp ? nullptr : floats(v[1], 0);
    float *a = op == kPolicy ? floats(v[1], 1) : op == kPolicyPerToken ? floats(v[0], 3) : nullptr,
          *p0 = op == kPreference ? floats(v[2], 0) : nullptr, *p1 = op == kPreference ? floats(v[2], 1) : nullptr;
    Py_BEGIN_ALLOW_THREADS;
    if (op == kLogp)
      st = reinterpret_cast<LogpFn>(fn)(&c, r0, ws, ws_bytes, stream);
    else if (op == kPreference)
      st = reinterpret_cast<PreferenceFn>(fn)(&c, r1, p1, (float)x[0], (float)x[1], (float)x[2], p0, e0, r0, d, ldd, ws,
                                              ws_bytes, stream);
    else
      st = reinterpret_cast<PolicyFn>(fn)(&c, a, op == kPolicyPerToken, r1, r2, (float)x[0], (float)x[1], (float)x[2], e0,
                                          r0, d, ldd, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS;
    if (st == ATTR_OK) {
      bump(args[7]);
      bump(PyTuple_GET_ITEM(v[0], 0));
      if (op != kLogp) bump(PyTuple_GET_ITEM(v[1], 0));
      if (op == kPreference) bump(PyTuple_GET_ITEM(v[2], 0));
    }
  } catch (...) {
    Py_RETURN_NONE;
  }
  return PyLong_FromLong((long)st);
}

// ----------------------------------------------------------------------------
// embedding and layer norm over token rows
// ----------------------------------------------------------------------------
typedef attr_status (*EmbedFn)(const attr_rows*, const int64_t*, const void*, attr_dtype, int64_t, int64_t, int64_t, float,
                               void*, attr_dtype, int64_t, void*);
typedef attr_status (*EmbedBackFn)(const attr_rows*, const int64_t*, const void*, attr_dtype, int64_t, int64_t, int64_t,
                                   float, void*, attr_dtype, int64_t, int32_t, void*, size_t, void*);
typedef attr_status (*NormFn)(const attr_rows*, const void*, attr_dtype, int64_t, int64_t, const void*, const void*,
                              attr_dtype, float, void*, attr_dtype, int64_t, float*, float*, void*);
typedef attr_status (*NormBackFn)(const attr_rows*, const void*, attr_dtype, int64_t, const void*, attr_dtype, int64_t,
                                  int64_t, const float*, const float*, const void*, attr_dtype, void*, int64_t, float*,
                                  int64_t, float*, int64_t, int32_t, int32_t, void*, size_t, void*);
constexpr int kEmbed = 0, kEmbedBack = 1, kNorm = 2, kNormBack = 3;

// A matrix of a call: its rows, type and stride, as the binding's _matrix() has them.
struct Mat {
  void* p = nullptr;
  int64_t n = 0, w = 0, ld = 0;
  attr_dtype type = ATTR_F32;
  // `o` on dev (or, first of a call, on any GPU) with w columns (0: any number) and n rows (-1: any)
  bool take(PyObject* o, const at::Device* dev, int64_t rows, int64_t width) {
    const at::Tensor* t = tensor_of(o);
    if (!t || !t->is_cuda() || (dev && t->device() != *dev) || !rows_of(*t, n, w, ld)) return false;
    if ((rows >= 0 && n != rows) || (width > 0 && w != width)) return false;
    const at::ScalarType k = t->scalar_type();
    if (k != at::kFloat && k != at::kBFloat16 && k != at::kHalf) return false;
    type = k == at::kFloat ? ATTR_F32 : k == at::kBFloat16 ? ATTR_BF16 : ATTR_F16;
    if (n <= 1 && ld < w) ld = w;
    p = t->mutable_data_ptr();
    return true;
  }
};
// None, or a contiguous vector of exactly d elements of a norm's weights' one type
bool weight_ok(PyObject* o, int64_t d, const at::Device& dev, bool& any, attr_dtype& type, void** p) {
  *p = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor_of(o);
  if (!t || !on(*t, dev) || t->dim() != 1 || t->numel() != d || !t->is_contiguous()) return false;
  const at::ScalarType k = t->scalar_type();
  if (k != at::kFloat && k != at::kBFloat16 && k != at::kHalf) return false;
  const attr_dtype mine = k == at::kFloat ? ATTR_F32 : k == at::kBFloat16 ? ATTR_BF16 : ATTR_F16;
  if (any && type != mine) return false;
  any = true;
  type = mine;
  *p = t->mutable_data_ptr();
  return true;
}
void* data_of(PyObject* o) { return o == Py_None ? nullptr : THPVariable_Unpack(o).mutable_data_ptr(); }

// The call's rows: None (every row is a token of one example) or an ExampleRows.
bool batch_ok(PyObject* rows, PyObject* rows_type, int64_t n_rows, const at::Device& dev, attr_rows& c) {
  c.n_rows = n_rows;
  c.row_offset = nullptr;
  c.length = nullptr;
  if (rows == Py_None) {
    c.n_examples = n_rows ? 1 : 0;
    c.T = n_rows ? n_rows : 1;
    return true;
  }
  if ((PyObject*)Py_TYPE(rows) != rows_type) return false;
  const Ref n_ex(PyObject_GetAttr(rows, names.n_examples)), T(PyObject_GetAttr(rows, names.T)),
      off(PyObject_GetAttr(rows, names.row_offset)), len(PyObject_GetAttr(rows, names.length));
  if (!off.p || !len.p || !size_of(n_ex.p, c.n_examples) || !size_of(T.p, c.T) || c.T < 1) return false;
  if (off.p == Py_None && n_rows < c.n_examples * c.T) return false;
  if (!vector_ok(off.p, at::kLong, c.n_examples, dev) || !vector_ok(len.p, at::kInt, c.n_examples, dev)) return false;
  c.row_offset = static_cast<const int64_t*>(data_of(off.p));
  c.length = static_cast<const int32_t*>(data_of(len.p));
  return true;
}

// What a call's tensors and numbers are, once checked; run() makes it.
struct RowsCall {
  attr_rows rows;
  Mat a, b, c;
  attr_dtype w_type = ATTR_F32;
  void *v[4] = {nullptr, nullptr, nullptr, nullptr};
  int64_t ldw = 0, ldb = 0;
  double x = 0;
  int flag[2] = {0, 0};

  bool gather(int op, PyObject* where, PyObject* rows_type, PyObject* const* t, PyObject* const* num) {
    const auto truth = [](PyObject* o, int& f) { return (f = PyObject_IsTrue(o)) >= 0; };
    if (op == kEmbed || op == kEmbedBack) {  // (table or dtable, token, out or dout), (scale[, accumulate])
      if (!b.take(t[2], nullptr, -1, 0)) return false;
      const at::Device dev = THPVariable_Unpack(t[2]).device();
      const at::Tensor* table = tensor_of(t[0]);
      if (!table || table->dim() < 1 || !a.take(t[0], &dev, table->size(0), b.w)) return false;
      if (t[1] == Py_None || !vector_ok(t[1], at::kLong, b.n, dev) || !batch_ok(where, rows_type, b.n, dev, rows)) return false;
      v[0] = data_of(t[1]);
      x = PyFloat_AsDouble(num[0]);
      return !PyErr_Occurred() && (op == kEmbed || truth(num[1], flag[0]));
    }
    // (x, y or dy, weight, bias or dx, mean, rstd[, dweight, dbias]), (eps) or (per_example, accumulate)
    if (!a.take(t[0], nullptr, -1, 0)) return false;
    const at::Device dev = THPVariable_Unpack(t[0]).device();
    bool any = false;
    if (!b.take(t[1], &dev, a.n, a.w) || !weight_ok(t[2], a.w, dev, any, w_type, &v[0]) ||
        !vector_ok(t[4], at::kFloat, a.n, dev) || !vector_ok(t[5], at::kFloat, a.n, dev) ||
        !batch_ok(where, rows_type, a.n, dev, rows))
      return false;
    v[2] = data_of(t[4]);
    v[3] = data_of(t[5]);
    if (op == kNorm) {
      x = PyFloat_AsDouble(num[0]);
      return !PyErr_Occurred() && weight_ok(t[3], a.w, dev, any, w_type, &v[1]);
    }
    if (t[4] == Py_None || t[5] == Py_None || !truth(num[0], flag[0]) || !truth(num[1], flag[1])) return false;
    if (t[3] != Py_None && (!c.take(t[3], &dev, a.n, a.w) || c.type != a.type)) return false;
    int64_t* const lds[2] = {&ldw, &ldb};
    for (int k = 0; k < 2; ++k) {
      *lds[k] = a.w;
      PyObject* o = t[6 + k];
      if (o == Py_None) continue;
      Mat m;
      const at::Tensor* g = tensor_of(o);
      if (!g || g->scalar_type() != at::kFloat || !on(*g, dev)) return false;
      if (flag[0] ? !m.take(o, &dev, rows.n_examples, a.w) : g->dim() != 1 || g->numel() != a.w || !g->is_contiguous()) return false;
      if (flag[0]) *lds[k] = m.ld;
    }
    return true;
  }
  attr_status run(int op, void* fn, float* dweight, float* dbias, void* ws, size_t ws_bytes, void* stream) {
    const int64_t* token = static_cast<const int64_t*>(v[0]);
    switch (op) {
      case kEmbed:
        return reinterpret_cast<EmbedFn>(fn)(&rows, token, a.p, a.type, a.n, a.w, a.ld, (float)x, b.p, b.type, b.ld, stream);
      case kEmbedBack:
        return reinterpret_cast<EmbedBackFn>(fn)(&rows, token, b.p, b.type, b.ld, a.n, a.w, (float)x, a.p, a.type, a.ld,
                                                 flag[0], ws, ws_bytes, stream);
      case kNorm:
        return reinterpret_cast<NormFn>(fn)(&rows, a.p, a.type, a.w, a.ld, v[0], v[1], w_type, (float)x, b.p, b.type, b.ld,
                                            static_cast<float*>(v[2]), static_cast<float*>(v[3]), stream);
      default:
        return reinterpret_cast<NormBackFn>(fn)(&rows, b.p, b.type, b.ld, a.p, a.type, a.w, a.ld,
                                                static_cast<float*>(v[2]), static_cast<float*>(v[3]), v[0], w_type, c.p, c.ld,
                                                dweight, ldw, dbias, ldb, flag[0], flag[1], ws, ws_bytes, stream);
    }
  }
};

// rows_call(op, address, rows, ExampleRows, tensors, numbers, workspace, workspace_bytes, stream)
// -> status, or None
PyObject* py_rows_call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 9) {
    PyErr_SetString(PyExc_TypeError, "rows_call() takes 9 arguments");
    return nullptr;
  }
  const long op = PyLong_AsLong(args[0]);
  void* fn = PyLong_AsVoidPtr(args[1]);
  void* ws = PyLong_AsVoidPtr(args[6]);
  const size_t ws_bytes = PyLong_AsSize_t(args[7]);
  void* stream = PyLong_AsVoidPtr(args[8]);
  const Py_ssize_t sizes[4] = {3, 3, 6, 8}, numbers[4] = {1, 2, 1, 2};
  RowsCall c;
  float *dweight = nullptr, *dbias = nullptr;
  bool ok = false;
  try {
    ok = !PyErr_Occurred() && fn && op >= 0 && op <= 3 && PyTuple_CheckExact(args[4]) && PyTuple_CheckExact(args[5]) &&
         PyTuple_GET_SIZE(args[4]) == sizes[op] && PyTuple_GET_SIZE(args[5]) == numbers[op] &&
         c.gather((int)op, args[2], args[3], reinterpret_cast<PyTupleObject*>(args[4])->ob_item, reinterpret_cast<PyTupleObject*>(args[5])->ob_item);
    if (ok && op == kNormBack) {
      dweight = static_cast<float*>(data_of(PyTuple_GET_ITEM(args[4], 6)));
      dbias = static_cast<float*>(data_of(PyTuple_GET_ITEM(args[4], 7)));
    }
  } catch (...) {  // a tensor without storage, for one
    ok = false;
  }
  if (!ok || PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  attr_status st;
  Py_BEGIN_ALLOW_THREADS;
  st = c.run((int)op, fn, dweight, dbias, ws, ws_bytes, stream);
  Py_END_ALLOW_THREADS;
  if (st == ATTR_OK) {  // what it wrote
    const int written[4][4] = {{2, -1, -1, -1}, {0, -1, -1, -1}, {1, 4, 5, -1}, {3, 6, 7, -1}};
    try {
      for (int k = 0; k < 4; ++k)
        if (written[op][k] >= 0) bump(PyTuple_GET_ITEM(args[4], written[op][k]));
    } catch (...) {  // the call is made: None would make it again
    }
  }
  return PyLong_FromLong((long)st);
}

PyMethodDef methods[] = {{"modules", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_modules)),
                          METH_FASTCALL, "module descriptors of a projection call, or None"},
                         {"token_call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_token_call)),
                          METH_FASTCALL, "status of a token loss's call, or None"},
                         {"rows_call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_rows_call)),
                          METH_FASTCALL, "status of an embedding's or a layer norm's call, or None"},
                         {"written", py_written, METH_O, "counts a change in place of every tensor"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
  struct {
    PyObject** at;
    const char* name;
  } const all[] = {{&names.a, "a"}, {&names.g, "g"}, {&names.R, "R"}, {&names.S, "S"}, {&names.out_col, "out_col"},
                   {&names.v_out, "v_out"}, {&names.v_in, "v_in"}, {&names.logits, "logits"},
                   {&names.target, "target"}, {&names.weight, "weight"}, {&names.n_examples, "n_examples"},
                   {&names.T, "T"}, {&names.row_offset, "row_offset"}, {&names.length, "length"},
                   {&names.logit_scale, "logit_scale"}};
  for (const auto& n : all)
    if (!(*n.at = PyUnicode_InternFromString(n.name))) return nullptr;
  return PyModule_Create(&module_def);
}
