// Native marshalling of the calls a program makes once per layer and step (binding.py): reads the
// descriptor, checks the tensors, allocates the output and calls the C entry point with the
// interpreter lock released.  Through ctypes a call of one linear spent more time in Python than its
// kernel on the GPU.  Every function takes its arguments by position, in the order
// binding.py passes them, and keeps nothing from one call for the next.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <optional>
#include <vector>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "peqa.h"

namespace {

PyObject* g_error = nullptr;                       // binding.PeqaError
PyObject *s_bits, *s_N, *s_K, *s_group, *s_qweight, *s_zeros, *s_scales;
PyObject *s_k, *s_v_cache, *s_page_table, *s_k_scales, *s_v_scales;
PyObject *s_w, *s_X, *s_dY, *s_Y, *s_dX, *s_dS, *s_m, *s_v, *s_workspace;

// A Python error is set; unwinds to the function's END_HANDLE_TH_ERRORS.
[[noreturn]] void fail() { throw python_error(); }

struct Ref {                                       // owned reference
  PyObject* p;
  explicit Ref(PyObject* o) : p(o) {
    if (!p) fail();
  }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
  ~Ref() { Py_DECREF(p); }
};

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_AttributeError, "%s: expected a tensor, got %.200s", name, Py_TYPE(o)->tp_name);
    fail();
  }
  return THPVariable_Unpack(o);
}

// A contiguous CUDA tensor of this type.
const at::Tensor& dev(PyObject* o, at::ScalarType dtype, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda() || t.scalar_type() != dtype || !t.is_contiguous()) {
    const char* type = dtype == at::kBFloat16 ? "bfloat16" : dtype == at::kFloat ? "float32" : "int32";
    PyErr_Format(PyExc_ValueError, "%s: expected a contiguous CUDA tensor of torch.%s", name, type);
    fail();
  }
  return t;
}

void* ptr_or_null(PyObject* o, const char* name) { return o == Py_None ? nullptr : tensor(o, name).data_ptr(); }

// Whole numbers as ctypes takes them: whatever has __index__, modulo the width.
long long as_long(PyObject* o) {
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
  if (v == ~0ull && PyErr_Occurred()) fail();
  return (long long)v;
}
int as_int(PyObject* o) { return (int)as_long(o); }
float as_float(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) fail();
  return (float)v;
}
int attr_int(PyObject* o, PyObject* name) { return as_int(Ref(PyObject_GetAttr(o, name)).p); }
void* attr_ptr(PyObject* o, PyObject* name) {
  Ref t(PyObject_GetAttr(o, name));
  return tensor(t.p, PyUnicode_AsUTF8(name)).data_ptr();
}

peqa_qweight_t weight(PyObject* o) {
  peqa_qweight_t w;
  w.bits = attr_int(o, s_bits);
  w.out_features = attr_int(o, s_N);
  w.in_features = attr_int(o, s_K);
  w.group_size = attr_int(o, s_group);
  w.qweight = static_cast<const uint32_t*>(attr_ptr(o, s_qweight));
  w.zeros = static_cast<const uint8_t*>(attr_ptr(o, s_zeros));
  w.scales = static_cast<const float*>(attr_ptr(o, s_scales));
  return w;
}

struct Workspace {
  void* p = nullptr;
  size_t bytes = 0;
  explicit Workspace(PyObject* o) {
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o, "workspace");
    p = t.data_ptr();
    bytes = (size_t)t.numel() * t.element_size();
  }
};

void* stream() { return static_cast<void*>(c10::cuda::getCurrentCUDAStream().stream()); }

void check(int status, const char* where) {
  if (status == PEQA_OK) return;
  if (!g_error) {
    PyErr_Format(PyExc_RuntimeError, "%s: status %d", where, status);
    fail();
  }
  Ref e(PyObject_CallFunction(g_error, "is", status, where));
  PyErr_SetObject(reinterpret_cast<PyObject*>(Py_TYPE(e.p)), e.p);
  fail();
}

void arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return;
  PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
  fail();
}

// The output: the caller's, or a new tensor beside `like` (of its class, if that is not torch's own).
PyObject* output(PyObject* given, PyObject* like, int64_t rows, int64_t cols, void** data) {
  if (given != Py_None) {
    *data = tensor(given, "Y").data_ptr();
    Py_INCREF(given);
    return given;
  }
  if (!THPVariable_CheckExact(like)) {
    PyObject* made = PyObject_CallMethod(like, "new_empty", "((LL))", (long long)rows, (long long)cols);
    if (!made) fail();
    if (!THPVariable_Check(made)) {
      Py_DECREF(made);
      PyErr_SetString(PyExc_TypeError, "new_empty did not return a tensor");
      fail();
    }
    *data = THPVariable_Unpack(made).data_ptr();
    return made;
  }
  at::Tensor t = THPVariable_Unpack(like).new_empty({rows, cols});
  *data = t.data_ptr();
  return THPVariable_Wrap(std::move(t));
}

template <typename F>
int unlocked(F&& call) {
  PyThreadState* save = PyEval_SaveThread();
  const int rc = call();
  PyEval_RestoreThread(save);
  return rc;
}

PyObject* bind_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

// (w, X, Y, workspace) -> Y
PyObject* qlinear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 4);
  const at::Tensor& X = dev(a[1], at::kBFloat16, "X");
  const int64_t T = X.size(0);
  const peqa_qweight_t w = weight(a[0]);
  void* y;
  Ref Y(output(a[2], a[1], T, w.out_features, &y));
  const Workspace ws(a[3]);
  void *x = X.data_ptr(), *st = stream();
  check(unlocked([&] { return peqa_qlinear_fwd(&w, x, (int)T, y, ws.p, ws.bytes, st); }), "peqa_qlinear_fwd");
  Py_INCREF(Y.p);
  return Y.p;
  END_HANDLE_TH_ERRORS
}

// (w, zeros_f, X, Y) -> Y
PyObject* qlinear_fwd_zf(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 4);
  const float* zf = static_cast<const float*>(dev(a[1], at::kFloat, "zeros_f").data_ptr());
  const at::Tensor& X = dev(a[2], at::kBFloat16, "X");
  const int64_t T = X.size(0);
  const peqa_qweight_t w = weight(a[0]);
  void* y;
  Ref Y(output(a[3], a[2], T, w.out_features, &y));
  void *x = X.data_ptr(), *st = stream();
  check(unlocked([&] { return peqa_qlinear_fwd_zf(&w, zf, x, (int)T, y, st); }), "peqa_qlinear_fwd_zf");
  Py_INCREF(Y.p);
  return Y.p;
  END_HANDLE_TH_ERRORS
}

// (w, X, Y, workspace) -> Y
PyObject* qlinear_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 4);
  const at::Tensor& X = dev(a[1], at::kBFloat16, "X");
  const int64_t M = X.size(0);
  const peqa_qweight_t w = weight(a[0]);
  void* y;
  Ref Y(output(a[2], a[1], M, w.out_features, &y));
  void *x = X.data_ptr(), *st = stream();
  const Workspace given(a[3]);
  at::Tensor own;
  void* wp = given.p;
  size_t wb = given.bytes;
  if (a[3] == Py_None) {
    wb = peqa_workspace_bytes(PEQA_OP_DECODE, (int)M, &w);
    if (wb > 0) {
      own = at::empty({(int64_t)wb}, X.options().dtype(at::kByte));
      wp = own.data_ptr();
    }
  }
  check(unlocked([&] { return peqa_qlinear_decode(&w, x, (int)M, y, wp, wb, st); }), "peqa_qlinear_decode");
  Py_INCREF(Y.p);
  return Y.p;
  END_HANDLE_TH_ERRORS
}

// (w, prepared, X, Y, scale_table, task_ids) -> Y
PyObject* qlinear_decode_prepared(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 6);
  const uint32_t* prepared = static_cast<const uint32_t*>(dev(a[1], at::kInt, "prepared").data_ptr());
  const at::Tensor& X = dev(a[2], at::kBFloat16, "X");
  const int64_t M = X.size(0);
  const peqa_qweight_t w = weight(a[0]);
  void* y;
  Ref Y(output(a[3], a[2], M, w.out_features, &y));
  const float* table = nullptr;
  const int32_t* ids = nullptr;
  int n_tasks = 0;
  if (a[5] != Py_None) {
    const at::Tensor& t = dev(a[4], at::kFloat, "scale_table");
    table = static_cast<const float*>(t.data_ptr());
    ids = static_cast<const int32_t*>(dev(a[5], at::kInt, "task_ids").data_ptr());
    n_tasks = (int)t.size(0);
  } else {
    table = static_cast<const float*>(ptr_or_null(a[4], "scale_table"));
  }
  void *x = X.data_ptr(), *st = stream();
  check(unlocked([&] {
          return peqa_qlinear_decode_prepared(&w, prepared, x, (int)M, y, table, n_tasks, ids, st);
        }),
        "peqa_qlinear_decode_prepared");
  Py_INCREF(Y.p);
  return Y.p;
  END_HANDLE_TH_ERRORS
}

// (values, gradient, m, v, lr, beta1, beta2, eps, weight_decay, step), for the scales or the zero-points
template <typename F>
PyObject* adamw(PyObject* const* a, Py_ssize_t n, const char* values, const char* grad, F entry, const char* where) {
  arity(n, 10);
  const at::Tensor& t = dev(a[0], at::kFloat, values);
  float* s = static_cast<float*>(t.data_ptr());
  const int64_t count = t.numel();
  const float* g = static_cast<const float*>(dev(a[1], at::kFloat, grad).data_ptr());
  float* m = static_cast<float*>(dev(a[2], at::kFloat, "m").data_ptr());
  float* v = static_cast<float*>(dev(a[3], at::kFloat, "v").data_ptr());
  float c[5];
  for (int i = 0; i < 5; ++i) c[i] = as_float(a[4 + i]);
  const long long step = as_long(a[9]);
  void* st = stream();
  check(unlocked([&] { return entry(s, g, m, v, count, c[0], c[1], c[2], c[3], c[4], (int64_t)step, st); }), where);
  Py_RETURN_NONE;
}
PyObject* scale_adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return adamw(a, n, "scales", "dS", peqa_scale_adamw, "peqa_scale_adamw");
  END_HANDLE_TH_ERRORS
}
PyObject* zero_adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return adamw(a, n, "zeros_f", "dZ", peqa_zero_adamw, "peqa_zero_adamw");
  END_HANDLE_TH_ERRORS
}

// (linears, apply_adamw, lr, beta1, beta2, eps, weight_decay, step)
PyObject* layer_train_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 8);
  if (!PySequence_Check(a[0])) {                   // (an iterator would be used up by one look at it)
    PyErr_SetString(PyExc_TypeError, "linears: expected a sequence of LayerLinear");
    fail();
  }
  Ref seq(PySequence_Fast(a[0], "linears: expected a sequence of LayerLinear"));
  const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq.p);
  if (count == 0) {
    PyErr_SetString(PyExc_IndexError, "linears: at least one linear is needed");
    fail();
  }
  std::vector<peqa_layer_linear_t> L((size_t)count);
  int64_t T = 0;
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyObject* o = PySequence_Fast_GET_ITEM(seq.p, i);
    const Ref X(PyObject_GetAttr(o, s_X)), dY(PyObject_GetAttr(o, s_dY)), Y(PyObject_GetAttr(o, s_Y)),
        dX(PyObject_GetAttr(o, s_dX)), dS(PyObject_GetAttr(o, s_dS)), m(PyObject_GetAttr(o, s_m)),
        v(PyObject_GetAttr(o, s_v)), ws(PyObject_GetAttr(o, s_workspace)), w(PyObject_GetAttr(o, s_w));
    const at::Tensor& tx = dev(X.p, at::kBFloat16, "X");
    const at::Tensor& ty = dev(dY.p, at::kBFloat16, "dY");
    peqa_layer_linear_t& l = L[(size_t)i];
    l.X_bf16 = tx.data_ptr();
    l.dY_bf16 = ty.data_ptr();
    l.Y_bf16 = dev(Y.p, at::kBFloat16, "Y").data_ptr();
    l.dX_bf16 = dev(dX.p, at::kBFloat16, "dX").data_ptr();
    l.dS = static_cast<float*>(dev(dS.p, at::kFloat, "dS").data_ptr());
    if (i == 0) T = ty.size(0);
    if (ty.size(0) != T || tx.size(0) != T) {
      PyErr_SetString(PyExc_ValueError, "all linears of a layer step take the same number of tokens");
      fail();
    }
    l.w = weight(w.p);
    l.m = static_cast<float*>(ptr_or_null(m.p, "m"));
    l.v = static_cast<float*>(ptr_or_null(v.p, "v"));
    const Workspace space(ws.p);
    l.workspace = space.p;
    l.workspace_bytes = space.bytes;
  }
  const int apply = PyObject_IsTrue(a[1]);
  if (apply < 0) fail();
  float c[5];
  for (int i = 0; i < 5; ++i) c[i] = as_float(a[2 + i]);
  const long long step = as_long(a[7]);
  void* st = stream();
  check(unlocked([&] {
          return peqa_layer_train_step(L.data(), (int)count, (int)T, apply, c[0], c[1], c[2], c[3], c[4], (int64_t)step, st);
        }),
        "peqa_layer_train_step");
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// ---- the paged key-value cache

[[noreturn]] void refuse(const char* what, const char* wanted) {
  PyErr_Format(PyExc_ValueError, "%s: expected %s", what, wanted);
  fail();
}

// Memory of the current device, in use by the current stream.
void here(const at::Tensor& t, const char* name) {
  if (!t.is_cuda() || t.get_device() != c10::cuda::current_device()) refuse(name, "a tensor on the current CUDA device");
}

// A contiguous tensor of this type and of n values in all, on the current device.
const at::Tensor& values(PyObject* o, at::ScalarType dtype, int64_t n, const char* name) {
  const at::Tensor& t = dev(o, dtype, name);
  here(t, name);
  if (t.numel() != n) {
    PyErr_Format(PyExc_ValueError, "%s: expected %lld values, got %lld", name, (long long)n, (long long)t.numel());
    fail();
  }
  return t;
}

int whole(PyObject* o, const char* name) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) fail();
  if (v < INT32_MIN || v > INT32_MAX) refuse(name, "a whole number of 32 bits");
  return (int)v;
}
int size32(const at::Tensor& t, int dim, const char* name) {
  const int64_t n = t.size(dim);
  if (n > INT32_MAX) refuse(name, "sizes of 31 bits");
  return (int)n;
}

// bf16 [rows, heads, head_dim], channels dense.
struct HeadRows {
  peqa_rows_t r;
  int rows, heads;
  int64_t dim;
  const at::Tensor& t;
  const char* name;
  HeadRows(PyObject* o, const char* what) : t(tensor(o, what)), name(what) {
    if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || t.stride(2) != 1) refuse();
    r.data = t.data_ptr();
    r.row_stride = t.stride(0);
    r.head_stride = t.stride(1);
    rows = size32(t, 0, name);
    heads = size32(t, 1, name);
    dim = t.size(2);
  }
  void belong_to(const peqa_kv_cache_t& c) const {
    here(t, name);
    if (dim != c.head_dim) refuse();
  }
  [[noreturn]] void refuse() const { ::refuse(name, "a torch.bfloat16 tensor [rows, heads, head_dim] with dense channels"); }
};

// The places of HeadRows as an arithmetic of elements: n steps of a stride, one where the stride says nothing.
struct Steps {
  int64_t n, stride;
  Steps(int64_t count, int64_t by) : n(by == 0 ? 1 : count), stride(n > 1 ? by : 0) {}
  int64_t span() const { return (n - 1) * stride; }
};

int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }          // b > 0

bool same_places(const HeadRows& a, const HeadRows& b) {
  const Steps ra(a.rows, a.r.row_stride), rb(b.rows, b.r.row_stride), ha(a.heads, a.r.head_stride), hb(b.heads, b.r.head_stride);
  return a.r.data == b.r.data && ra.n == rb.n && ra.stride == rb.stride && ha.n == hb.n && ha.stride == hb.stride;
}

// Whether heads of a and heads of b have an element in common, b's rows being as long as a's.  Exact where the rows of both follow in one
// stride (as parts of the rows of one matrix do) or their extents lie apart; what else lies within one extent counts as common.
bool meet(const HeadRows& a, const HeadRows& b) {
  if (a.t.numel() == 0 || b.t.numel() == 0) return false;
  const int64_t size = 2, dim = a.dim * size;                                    // from here on in bytes
  const Steps ra(a.rows, a.r.row_stride * size), rb(b.rows, b.r.row_stride * size), ha(a.heads, a.r.head_stride * size),
      hb(b.heads, b.r.head_stride * size);
  const intptr_t at = reinterpret_cast<intptr_t>(b.r.data) - reinterpret_cast<intptr_t>(a.r.data);
  if (at >= ra.span() + ha.span() + dim || -at >= rb.span() + hb.span() + dim) return false;
  if (ra.n > 1 && rb.n > 1 && ra.stride != rb.stride) return true;
  const int64_t row = ra.n > 1 ? ra.stride : rb.stride;
  if (row > 0) {                                                                 // b's heads beside a's in every row
    const int64_t from = at - floor_div(at, row) * row;
    if (ha.span() + dim <= from && from + hb.span() + dim <= row) return false;
  }
  // heads j of a and l of b, i rows behind: j ha - l hb + i row - at is where the one begins in the other
  const bool one_stride = ha.n == 1 || hb.n == 1 || ha.stride == hb.stride;      // then j ha - l hb is a multiple of it
  const int64_t head = ha.n > 1 ? ha.stride : hb.stride;
  if (!one_stride && ha.n * hb.n > (1 << 20)) return true;
  auto common = [&](int64_t apart) {
    apart -= at;
    if (row == 0) return -dim < apart && apart < dim;
    const int64_t first = std::max(-(rb.n - 1), floor_div(-dim - apart, row) + 1);   // least i with i row + apart > -dim
    return first <= ra.n - 1 && first * row + apart < dim;
  };
  if (one_stride) {
    for (int64_t d = -(hb.n - 1); d < ha.n; ++d)
      if (common(d * head)) return true;
    return false;
  }
  for (int64_t j = 0; j < ha.n; ++j)
    for (int64_t l = 0; l < hb.n; ++l)
      if (common(j * ha.stride - l * hb.stride)) return true;
  return false;
}

struct Cache {
  peqa_kv_cache_t c = {};
  static void check_scales(PyObject* o, const at::Tensor& k, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (t.dim() != 3 || t.size(0) != k.size(0) || t.size(1) != k.size(2) || t.size(2) != k.size(1))
      refuse(name, "[n_pages, n_kv_heads, page_size]");
  }
  explicit Cache(PyObject* o) {
    const Ref pk(PyObject_GetAttr(o, s_k)), pv(PyObject_GetAttr(o, s_v_cache)), pt(PyObject_GetAttr(o, s_page_table)),
        pks(PyObject_GetAttr(o, s_k_scales)), pvs(PyObject_GetAttr(o, s_v_scales));
    const at::Tensor &k = tensor(pk.p, "k"), &v = tensor(pv.p, "v");
    const bool codes = k.scalar_type() == at::kChar;
    if ((!codes && k.scalar_type() != at::kBFloat16) || k.dim() != 4 || k.stride(3) != 1)
      refuse("cache.k", "a torch.bfloat16 or torch.int8 tensor [n_pages, page_size, n_kv_heads, head_dim] with dense channels");
    if (v.scalar_type() != k.scalar_type() || v.sizes() != k.sizes()) refuse("cache.v", "a tensor of cache.k's type and shape");
    for (int d = 0; d < 4; ++d)
      if (k.size(d) != 1 && k.stride(d) != v.stride(d)) refuse("cache.v", "cache.k's strides");
    if (codes) {                           // as many values in another order would be taken for other tokens' scales
      check_scales(pks.p, k, "cache.k_scales");
      check_scales(pvs.p, k, "cache.v_scales");
    }
    here(k, "cache.k");
    here(v, "cache.v");
    c.type = codes ? PEQA_KV_INT8 : PEQA_KV_BF16;
    c.n_pages = size32(k, 0, "cache.k");
    c.page_size = size32(k, 1, "cache.k");
    c.n_kv_heads = size32(k, 2, "cache.k");
    c.head_dim = size32(k, 3, "cache.k");
    c.page_stride = k.stride(0);
    c.token_stride = k.stride(1);
    c.head_stride = k.stride(2);
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    if (codes) {
      const int64_t n = k.size(0) * k.size(1) * k.size(2);
      c.k_scales = static_cast<float*>(values(pks.p, at::kFloat, n, "cache.k_scales").data_ptr());
      c.v_scales = static_cast<float*>(values(pvs.p, at::kFloat, n, "cache.v_scales").data_ptr());
    }
    const at::Tensor& t = dev(pt.p, at::kInt, "cache.page_table");
    here(t, "cache.page_table");
    if (t.dim() != 2) refuse("cache.page_table", "[n_seqs, max_pages]");
    c.n_seqs = size32(t, 0, "cache.page_table");
    c.max_pages = size32(t, 1, "cache.page_table");
    c.page_table = static_cast<const int32_t*>(t.data_ptr());
  }
};

// (cache, q, k, v, cos_sin, seq_lens, starts, q_out, interleaved) -> q_out
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 9);
  const HeadRows k(a[2], "k"), v(a[3], "v");
  if (v.heads != k.heads || v.rows != k.rows || v.dim != k.dim) refuse("v", "k's shape");
  std::optional<HeadRows> q, to;
  if (a[1] != Py_None) {
    q.emplace(a[1], "q");
    if (q->rows != k.rows || q->dim != k.dim) refuse("q", "k's rows");
  }
  if (a[7] != Py_None) {
    if (!q) refuse("q_out", "q beside it");
    to.emplace(a[7], "q_out");
    if (to->rows != q->rows || to->heads != q->heads || to->dim != q->dim) refuse("q_out", "q's shape");
    // a CTA reads rows that others write
    if (!same_places(*to, *q) && meet(*to, *q)) refuse("q_out", "q itself or memory apart from q");
    if (meet(*to, k) || meet(*to, v)) refuse("q_out", "memory apart from k and v");
  }
  const Cache cache(a[0]);
  k.belong_to(cache.c);
  v.belong_to(cache.c);
  if (k.heads != cache.c.n_kv_heads) refuse("k", "the cache's heads");
  const at::Tensor& table = dev(a[4], at::kFloat, "cos_sin");
  here(table, "cos_sin");
  if (table.dim() != 2) refuse("cos_sin", "[n_positions, rotary_dim]");
  const int positions = size32(table, 0, "cos_sin"), rotary = size32(table, 1, "cos_sin");
  const int32_t* lens = static_cast<const int32_t*>(values(a[5], at::kInt, cache.c.n_seqs, "seq_lens").data_ptr());
  const int32_t* starts = nullptr;
  if (a[6] != Py_None)
    starts = static_cast<const int32_t*>(values(a[6], at::kInt, (int64_t)cache.c.n_seqs + 1, "starts").data_ptr());
  else if (k.rows != cache.c.n_seqs)
    refuse("k", "one row per sequence, or starts");
  const int interleaved = PyObject_IsTrue(a[8]);
  if (interleaved < 0) fail();
  void* st = stream();
  const float* angles = static_cast<const float*>(table.data_ptr());
  if (!q) {
    check(unlocked([&] {
            return peqa_kv_append(&cache.c, nullptr, 0, &k.r, &v.r, k.rows, angles, positions, rotary, interleaved, lens, starts,
                                  nullptr, st);
          }),
          "peqa_kv_append");
    Py_RETURN_NONE;
  }
  q->belong_to(cache.c);
  PyObject* made = a[7];
  if (!to) {
    // rows that are left out keep what their memory had: a new tensor has zeros there
    made = THPVariable_Wrap(at::zeros({q->rows, q->heads, cache.c.head_dim}, q->t.options()));
    if (!made) fail();
  } else {
    to->belong_to(cache.c);
    Py_INCREF(made);
  }
  Ref out(made);
  if (!to) to.emplace(out.p, "q_out");
  check(unlocked([&] {
          return peqa_kv_append(&cache.c, &q->r, q->heads, &k.r, &v.r, k.rows, angles, positions, rotary, interleaved, lens, starts,
                                &to->r, st);
        }),
        "peqa_kv_append");
  Py_INCREF(out.p);
  return out.p;
  END_HANDLE_TH_ERRORS
}

// (cache, q, seq_lens, scale, window, out, workspace, return_lse) -> out, or (out, lse)
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  arity(n, 8);
  const Cache cache(a[0]);
  const HeadRows q(a[1], "q");
  q.belong_to(cache.c);
  if (q.rows != cache.c.n_seqs) refuse("q", "one row per sequence");
  const int32_t* lens = static_cast<const int32_t*>(values(a[2], at::kInt, cache.c.n_seqs, "seq_lens").data_ptr());
  const float scale = a[3] == Py_None ? (float)(1.0 / std::sqrt((double)cache.c.head_dim)) : as_float(a[3]);
  const int window = whole(a[4], "window");
  const at::Tensor& like = tensor(a[1], "q");
  at::Tensor out, lse, own;
  if (a[5] == Py_None) {
    out = at::empty({q.rows, q.heads, cache.c.head_dim}, like.options());
  } else {
    out = values(a[5], at::kBFloat16, (int64_t)q.rows * q.heads * cache.c.head_dim, "out");
    if (out.dim() != 3 || out.size(0) != q.rows || out.size(1) != q.heads) refuse("out", "q's shape");
    const char *o = static_cast<const char*>(out.data_ptr()), *first = static_cast<const char*>(q.r.data);
    const int64_t last = q.rows > 0 && q.heads > 0 ? (q.rows - 1) * q.r.row_stride + (q.heads - 1) * q.r.head_stride + cache.c.head_dim : 0;
    if (o < first + 2 * last && first < o + out.nbytes()) refuse("out", "memory apart from q");
  }
  const int with_lse = PyObject_IsTrue(a[7]);
  if (with_lse < 0) fail();
  if (with_lse) lse = at::empty({q.rows, q.heads}, like.options().dtype(at::kFloat));
  void* wp = nullptr;
  size_t wb = 0;
  if (a[6] == Py_None) {
    wb = peqa_attn_workspace_bytes(&cache.c, q.heads);
    if (wb > 0) {
      own = at::empty({(int64_t)wb}, like.options().dtype(at::kByte));
      wp = own.data_ptr();
    }
  } else {
    const at::Tensor& t = tensor(a[6], "workspace");
    here(t, "workspace");
    if (!t.is_contiguous()) refuse("workspace", "a contiguous tensor");
    const Workspace given(a[6]);
    wp = given.p;
    wb = given.bytes;
  }
  void *o = out.data_ptr(), *st = stream();
  float* l = with_lse ? static_cast<float*>(lse.data_ptr()) : nullptr;
  check(unlocked([&] { return peqa_attn_decode(&cache.c, &q.r, q.heads, lens, scale, window, o, l, wp, wb, st); }),
        "peqa_attn_decode");
  Ref first(a[5] == Py_None ? THPVariable_Wrap(std::move(out)) : (Py_INCREF(a[5]), a[5]));
  if (!with_lse) {
    Py_INCREF(first.p);
    return first.p;
  }
  Ref second(THPVariable_Wrap(std::move(lse)));
  return PyTuple_Pack(2, first.p, second.p);
  END_HANDLE_TH_ERRORS
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FAST(qlinear_fwd),       FAST(qlinear_fwd_zf), FAST(qlinear_decode), FAST(qlinear_decode_prepared),
                          FAST(scale_adamw),       FAST(zero_adamw),     FAST(layer_train_step),
                          FAST(kv_append),         FAST(attn_decode),
                          {"bind_error", bind_error, METH_O, nullptr},   {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
  const struct {
    PyObject** to;
    const char* text;
  } names[] = {{&s_bits, "bits"}, {&s_N, "N"}, {&s_K, "K"}, {&s_group, "group_size"}, {&s_qweight, "qweight"},
               {&s_zeros, "zeros"}, {&s_scales, "scales"}, {&s_w, "w"}, {&s_X, "X"}, {&s_dY, "dY"}, {&s_Y, "Y"},
               {&s_dX, "dX"}, {&s_dS, "dS"}, {&s_m, "m"}, {&s_v, "v"}, {&s_workspace, "workspace"},
               {&s_k, "k"}, {&s_v_cache, "v"}, {&s_page_table, "page_table"}, {&s_k_scales, "k_scales"},
               {&s_v_scales, "v_scales"}};
  for (const auto& e : names)
    if (!(*e.to = PyUnicode_InternFromString(e.text))) return nullptr;
  return PyModule_Create(&kModule);
}
