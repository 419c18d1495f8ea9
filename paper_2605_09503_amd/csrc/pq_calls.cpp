// The calls of the Python binding that a forward pass or a calibration hook makes once a layer, as a CPython module:
// their arguments go from the interpreter's objects to the C entry points without ctypes.  A call of these launches one or two
// kernels that may take 3 us, and the host has to keep up: issuing a launch takes 2.7 us by itself, a wrapper in Python, its
// tensors' methods and ctypes took 2 more.  NVFP4 256 x 512 x 512, quantizer and product, one pair after another: 10.4 us before, 6.8
// then, where the kernels alone took 6.5 (in a graph, 5.5 now); INT4 g128 77 x 1000 x 1152 from the stored layout 13.9 -> 10.2 (7.6 with
// one launch less).
//
// Marshalling only: pointers, sizes and strides of the tensors, the current stream, the result code.  pq.py holds the
// declarations that users read, the exception type and the helpers that allocate (handed over by bind()).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <new>

#include "../../include/permuquant.h"

namespace {

PyObject* g_raise = nullptr;        // raise(rc): raises the error of the last call
PyObject* g_operand = nullptr;      // operand(fmt, group, rows, K, like) -> tensor
PyObject* g_workspace = nullptr;    // workspace(op, fmt, group, M, N, K, n_batches, like) -> tensor or None
PyObject* g_refuse = nullptr;       // refuse(message): raises the error of arguments that do not fit
PyObject* g_attn_workspace = nullptr;   // attn_workspace(cache, seqs, q_heads, max_len, window) -> tensor
PyObject* g_route_workspace = nullptr;  // route_workspace(tokens, experts, k, like) -> tensor
PyObject* g_route = nullptr;            // route(tokens, experts, k, like) -> Route

// thrown when a Python error is set
struct PyFailed {};

[[noreturn]] void fail(PyObject* type, const char* what) {
  PyErr_SetString(type, what);
  throw PyFailed{};
}

struct Ref {
  PyObject* p;
  explicit Ref(PyObject* o) : p(o) {
    if (!o) throw PyFailed{};
  }
  ~Ref() { Py_XDECREF(p); }
  Ref(const Ref&) = delete;
  Ref& operator=(const Ref&) = delete;
};

// integers and what stands for one (__index__: numpy's integers, a tensor of one)
int64_t as_int(PyObject* o) {
  if (!PyLong_Check(o)) {
    if (!PyIndex_Check(o)) fail(PyExc_TypeError, "an integer is required");
    Ref n(PyNumber_Index(o));
    return as_int(n.p);
  }
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyFailed{};
  return v;
}

// what int(o) gives
int64_t to_int(PyObject* o) {
  Ref n(PyNumber_Long(o));
  return as_int(n.p);
}

bool given(PyObject* o) { return o && o != Py_None; }

// a torch tensor itself; other objects, subclasses that override methods among them, are asked through their methods
const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

void* pointer(PyObject* o) {
  if (!given(o)) return nullptr;
  if (const at::Tensor* t = tensor(o)) return t->data_ptr();
  Ref r(PyObject_CallMethod(o, "data_ptr", nullptr));
  void* p = PyLong_AsVoidPtr(r.p);
  if (!p && PyErr_Occurred()) throw PyFailed{};
  return p;
}
int64_t size(PyObject* o, int64_t dim) {
  if (const at::Tensor* t = tensor(o)) {
    if (dim >= t->dim()) fail(PyExc_IndexError, "tuple index out of range");
    return t->size(dim);
  }
  Ref shape(PyObject_GetAttrString(o, "shape"));
  Ref n(PySequence_GetItem(shape.p, dim));
  return as_int(n.p);
}
int64_t row_stride(PyObject* o) {
  if (const at::Tensor* t = tensor(o)) return t->stride(0);
  Ref r(PyObject_CallMethod(o, "stride", "i", 0));
  return as_int(r.p);
}
size_t numel(PyObject* o) {
  if (const at::Tensor* t = tensor(o)) return (size_t)t->numel();
  Ref r(PyObject_CallMethod(o, "numel", nullptr));
  return (size_t)as_int(r.p);
}
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

int64_t or_size(PyObject* o, PyObject* t, int64_t dim) { return given(o) ? as_int(o) : size(t, dim); }
int64_t or_stride(PyObject* o, PyObject* t) { return given(o) ? as_int(o) : row_stride(t); }

// Arguments by position or name into slots, nullptr where absent; the first `required` must be there.
struct Spec {
  const char* name;
  int n, required;
  const char* const* args;
};
void take(const Spec& s, PyObject* const* args, Py_ssize_t nargs, PyObject* names, PyObject** slot) {
  for (int i = 0; i < s.n; ++i) slot[i] = nullptr;
  if (nargs > s.n) {
    PyErr_Format(PyExc_TypeError, "%s() takes at most %d arguments (%zd given)", s.name, s.n, nargs);
    throw PyFailed{};
  }
  for (Py_ssize_t i = 0; i < nargs; ++i) slot[i] = args[i];
  const Py_ssize_t n_names = names ? PyTuple_GET_SIZE(names) : 0;
  for (Py_ssize_t k = 0; k < n_names; ++k) {
    PyObject* name = PyTuple_GET_ITEM(names, k);
    int at = 0;
    while (at < s.n && PyUnicode_CompareWithASCIIString(name, s.args[at]) != 0) ++at;
    if (at == s.n) {
      PyErr_Format(PyExc_TypeError, "%s() got an unexpected keyword argument '%U'", s.name, name);
      throw PyFailed{};
    }
    if (slot[at]) {
      PyErr_Format(PyExc_TypeError, "%s() got multiple values for argument '%U'", s.name, name);
      throw PyFailed{};
    }
    slot[at] = args[nargs + k];
  }
  for (int i = 0; i < s.required; ++i) {
    if (!slot[i]) {
      PyErr_Format(PyExc_TypeError, "%s() missing required argument: '%s'", s.name, s.args[i]);
      throw PyFailed{};
    }
  }
}

// the entry point without the interpreter's lock, as ctypes calls it
template <class F>
void call(F&& f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  if (rc != PQ_OK) {
    Ref unused(PyObject_CallFunction(g_raise, "i", rc));
    fail(PyExc_RuntimeError, "the library reported an error");       // not reached: raise() raises
  }
}

// torch.OutOfMemoryError, as torch's own allocations raise it
void set_out_of_memory(const char* what) {
  PyObject* torch = PyImport_ImportModule("torch");
  PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
  if (type) PyErr_SetString(type, what);
  Py_XDECREF(type);
  Py_XDECREF(torch);
}

// runs a call's body; errors of the interpreter and C++ exceptions of torch become Python exceptions
template <class F>
PyObject* guarded(F&& f) {
  try {
    return f();
  } catch (const PyFailed&) {
    return nullptr;
  } catch (const c10::IndexError& e) {
    PyErr_SetString(PyExc_IndexError, e.what_without_backtrace());
  } catch (const c10::OutOfMemoryError& e) {
    set_out_of_memory(e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::bad_alloc&) {
    PyErr_NoMemory();
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* none() { Py_RETURN_NONE; }

// the operand buffer that was passed, or a new one: a new reference
PyObject* operand_of(PyObject* o, int64_t fmt, int64_t group, int64_t rows, int64_t K, PyObject* like) {
  if (given(o)) {
    Py_INCREF(o);
    return o;
  }
  return PyObject_CallFunction(g_operand, "LLLLO", (long long)fmt, (long long)group, (long long)rows, (long long)K, like);
}

#define PQ_CALL(fn) static PyObject* fn(PyObject*, PyObject* const* args, Py_ssize_t nargs, PyObject* names)
#define PQ_TAKE(fn, required, ...)                                                    \
  static const char* const arg_names[] = {__VA_ARGS__};                               \
  constexpr int n_args = sizeof(arg_names) / sizeof(arg_names[0]);                    \
  static const Spec spec = {#fn, n_args, required, arg_names};                        \
  PyObject* a[n_args];                                                                \
  take(spec, args, nargs, names, a)

PQ_CALL(quantize_act) {
  return guarded([&] {
    PQ_TAKE(pq_quantize_act, 7, "fmt", "group", "x", "perm", "tensor_scale", "codes", "scales", "M", "K", "ld");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const int64_t M = or_size(a[7], a[2], 0), K = or_size(a[8], a[2], 1), ld = or_stride(a[9], a[2]);
    void *x = pointer(a[2]), *perm = pointer(a[3]), *ts = pointer(a[4]), *codes = pointer(a[5]), *scales = pointer(a[6]), *st = stream();
    call([&] {
      return pq_quantize_act((pq_format)fmt, group, x, M, K, ld, (const int32_t*)perm, (const float*)ts, (uint8_t*)codes, scales, st);
    });
    return none();
  });
}

PQ_CALL(quantize_act_packed) {
  return guarded([&] {
    PQ_TAKE(pq_quantize_act_packed, 4, "fmt", "group", "x", "tensor_scale", "operand", "codes", "scales", "K");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const int64_t M = size(a[2], 0), K = or_size(a[7], a[2], 1);
    Ref out(operand_of(a[4], fmt, group, M, K, a[2]));
    void *x = pointer(a[2]), *ts = pointer(a[3]), *op = pointer(out.p), *codes = pointer(a[5]), *scales = pointer(a[6]), *st = stream();
    const int64_t ld = row_stride(a[2]);
    const size_t bytes = numel(out.p);
    call([&] {
      return pq_quantize_act_packed((pq_format)fmt, group, x, M, K, ld, (const float*)ts, op, bytes, (uint8_t*)codes, scales, st);
    });
    Py_INCREF(out.p);
    return out.p;
  });
}

PQ_CALL(norm_quantize_act_packed) {
  return guarded([&] {
    PQ_TAKE(pq_norm_quantize_act_packed, 6, "kind", "fmt", "group", "x", "eps", "tensor_scale", "perm", "gamma", "mod_scale",
            "mod_shift", "rows_per_mod", "operand", "y", "K");
    const int fmt = (int)as_int(a[1]), group = (int)as_int(a[2]);
    const int64_t M = size(a[3], 0), K = or_size(a[13], a[3], 1);
    Ref out(operand_of(a[11], fmt, group, M, K, a[3]));
    pq_norm_params p;
    p.kind = (decltype(p.kind))to_int(a[0]);
    p.perm = (decltype(p.perm))pointer(a[6]);
    p.gamma = pointer(a[7]);
    p.mod_scale = pointer(a[8]);
    p.mod_shift = pointer(a[9]);
    p.rows_per_mod = a[10] ? to_int(a[10]) : 0;
    p.eps = (float)PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) throw PyFailed{};
    void *x = pointer(a[3]), *ts = pointer(a[5]), *op = pointer(out.p), *y = pointer(a[12]), *st = stream();
    const int64_t ld = row_stride(a[3]), ldy = given(a[12]) ? row_stride(a[12]) : 0;
    const size_t bytes = numel(out.p);
    call([&] {
      return pq_norm_quantize_act_packed(&p, (pq_format)fmt, group, x, M, K, ld, (const float*)ts, op, bytes, y, ldy, st);
    });
    Py_INCREF(out.p);
    return out.p;
  });
}

PQ_CALL(hadamard_quantize_act_packed) {
  return guarded([&] {
    PQ_TAKE(pq_hadamard_quantize_act_packed, 4, "fmt", "group", "x", "tensor_scale", "perm", "operand", "y", "K");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const int64_t M = size(a[2], 0), K = or_size(a[7], a[2], 1);
    Ref out(operand_of(a[5], fmt, group, M, K, a[2]));
    void *x = pointer(a[2]), *ts = pointer(a[3]), *perm = pointer(a[4]), *op = pointer(out.p), *y = pointer(a[6]), *st = stream();
    const int64_t ld = row_stride(a[2]), ldy = given(a[6]) ? row_stride(a[6]) : 0;
    const size_t bytes = numel(out.p);
    call([&] {
      return pq_hadamard_quantize_act_packed((const int32_t*)perm, (pq_format)fmt, group, x, M, K, ld, (const float*)ts, op, bytes, y,
                                             ldy, st);
    });
    Py_INCREF(out.p);
    return out.p;
  });
}

template <class F>
PyObject* product_packed(PyObject* const* a, PyObject* y, PyObject* m, PyObject* n, PyObject* k, PyObject* ldy, F&& entry) {
  const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
  void *ao = pointer(a[2]), *ats = pointer(a[3]), *wo = pointer(a[4]), *wts = pointer(a[5]), *yp = pointer(y), *st = stream();
  const int64_t M = as_int(m), N = as_int(n), K = as_int(k), ld = or_stride(ldy, y);
  call([&] { return entry((pq_format)fmt, group, ao, (const float*)ats, wo, (const float*)wts, M, N, K, yp, ld, st); });
  return none();
}

PQ_CALL(qgemm_packed) {
  return guarded([&] {
    PQ_TAKE(pq_qgemm_packed, 10, "fmt", "group", "a_operand", "a_tensor_scale", "w_operand", "w_tensor_scale", "y", "M", "N", "K", "ldy");
    return product_packed(a, a[6], a[7], a[8], a[9], a[10], pq_qgemm_packed);
  });
}
PQ_CALL(qgemm_packed_f32) {
  return guarded([&] {
    PQ_TAKE(pq_qgemm_packed_f32, 10, "fmt", "group", "a_operand", "a_tensor_scale", "w_operand", "w_tensor_scale", "y", "M", "N", "K",
            "ldy");
    return product_packed(a, a[6], a[7], a[8], a[9], a[10],
                          [](pq_format fmt, int group, const void* ao, const float* ats, const void* wo, const float* wts, int64_t M,
                             int64_t N, int64_t K, void* y, int64_t ldy, void* st) {
                            return pq_qgemm_packed_f32(fmt, group, ao, ats, wo, wts, M, N, K, (float*)y, ldy, st);
                          });
  });
}
PQ_CALL(qgemm_packed_bias) {
  return guarded([&] {
    PQ_TAKE(pq_qgemm_packed_bias, 11, "fmt", "group", "a_operand", "a_tensor_scale", "w_operand", "w_tensor_scale", "bias", "y", "M",
            "N", "K", "ldy");
    void* bias = pointer(a[6]);
    return product_packed(a, a[7], a[8], a[9], a[10], a[11],
                          [&](pq_format fmt, int group, const void* ao, const float* ats, const void* wo, const float* wts, int64_t M,
                              int64_t N, int64_t K, void* y, int64_t ldy, void* st) {
                            return pq_qgemm_packed_bias(fmt, group, ao, ats, wo, wts, M, N, K, bias, y, ldy, st);
                          });
  });
}

// a workspace that was passed, or a new one (None where none is needed): a new reference
PyObject* workspace_of(PyObject* o, int op, int fmt, int group, int64_t M, int64_t N, int64_t K, int n_batches, PyObject* like) {
  if (given(o)) {
    Py_INCREF(o);
    return o;
  }
  return PyObject_CallFunction(g_workspace, "iiiLLLiO", op, fmt, group, (long long)M, (long long)N, (long long)K, n_batches, like);
}

PQ_CALL(qgemm) {
  return guarded([&] {
    PQ_TAKE(pq_qgemm, 9, "fmt", "group", "a_codes", "a_scales", "a_tensor_scale", "w_codes", "w_scales", "w_tensor_scale", "y",
            "workspace", "M", "N", "K", "ldy");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const int64_t M = or_size(a[10], a[2], 0), K = given(a[12]) ? as_int(a[12]) : 2 * size(a[2], 1), N = or_size(a[11], a[5], 0);
    const int64_t ldy = or_stride(a[13], a[8]);
    Ref ws(workspace_of(a[9], PQ_OP_QGEMM, fmt, group, M, N, K, 0, a[2]));
    void *ac = pointer(a[2]), *as = pointer(a[3]), *ats = pointer(a[4]), *wc = pointer(a[5]), *wsc = pointer(a[6]),
         *wts = pointer(a[7]), *y = pointer(a[8]), *wp = pointer(ws.p), *st = stream();
    const size_t bytes = given(ws.p) ? numel(ws.p) : 0;
    call([&] {
      return pq_qgemm((pq_format)fmt, group, (const uint8_t*)ac, as, (const float*)ats, (const uint8_t*)wc, wsc, (const float*)wts, M, N,
                      K, y, ldy, wp, bytes, st);
    });
    return none();
  });
}

PQ_CALL(calib_moments) {
  return guarded([&] {
    PQ_TAKE(pq_calib_moments, 2, "x", "sumsq", "absmax", "workspace", "rows", "K", "ld");
    const int64_t rows = or_size(a[4], a[0], 0), K = or_size(a[5], a[0], 1), ld = or_stride(a[6], a[0]);
    Ref ws(workspace_of(a[3], PQ_OP_CALIB_MOMENTS, 0, 0, rows, 0, K, 1, a[0]));
    void *x = pointer(a[0]), *sumsq = pointer(a[1]), *absmax = pointer(a[2]), *wp = pointer(ws.p), *st = stream();
    const size_t bytes = given(ws.p) ? numel(ws.p) : 0;
    call([&] { return pq_calib_moments(x, rows, K, ld, (double*)sumsq, (float*)absmax, wp, bytes, st); });
    return none();
  });
}

// ---- key-value cache: tensors are checked as pq.py's functions check them (a wrong type or size would be read past its end)
template <class... A>
[[noreturn]] void refuse(const char* format, A... a) {
  Ref text(PyUnicode_FromFormat(format, a...));
  Ref unused(PyObject_CallFunctionObjArgs(g_refuse, text.p, nullptr));
  fail(PyExc_RuntimeError, "arguments do not fit");                     // not reached: refuse() raises
}

struct Cache {
  const pq_kv_cache* c;
  c10::Device device;
};
Cache cache_of(PyObject* o) {
  Ref address(PyObject_GetAttrString(o, "_address")), data(PyObject_GetAttrString(o, "data"));
  const at::Tensor* t = tensor(data.p);
  if (!t) fail(PyExc_TypeError, "the cache's data must be a tensor");
  const auto* c = (const pq_kv_cache*)PyLong_AsVoidPtr(address.p);
  if (PyErr_Occurred()) throw PyFailed{};
  if (!c) fail(PyExc_TypeError, "a key-value cache is required");
  return Cache{c, t->device()};
}
const at::Tensor& as_tensor(PyObject* o, const char* name) {
  const at::Tensor* t = THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr;
  if (!t) PyErr_Format(PyExc_TypeError, "%s must be a tensor", name), throw PyFailed{};
  return *t;
}

// bf16 [rows, heads, head_dim]; strides of one row or head do not matter
struct HeadRows {
  void* p;
  int64_t ld, head;
};
HeadRows head_rows(const Cache& c, const char* name, const at::Tensor& t, int64_t rows, int64_t heads) {
  if (t.scalar_type() != at::kBFloat16 || t.dim() != 3 || t.size(0) != rows || t.size(1) != heads || t.size(2) != c.c->head_dim ||
      t.stride(2) != 1 || t.device() != c.device)
    refuse("%s must be bfloat16 [%lld, %lld, %d] with adjacent channels, on the cache's device", name, (long long)rows, (long long)heads,
           c.c->head_dim);
  return HeadRows{t.data_ptr(), rows > 1 ? t.stride(0) : 0, heads > 1 ? t.stride(1) : 0};
}
void* indices(const Cache& c, const char* name, const at::Tensor& t, at::ScalarType type, const char* type_name, int64_t dims) {
  if (t.scalar_type() != type || t.dim() != dims || (t.numel() > 1 && t.stride(dims - 1) != 1) || t.device() != c.device)
    refuse("%s must be %s with %lld dimension%s, the last one contiguous, on the cache's device", name, type_name, (long long)dims,
           dims > 1 ? "s" : "");
  return t.data_ptr();
}
void* stream_of(const Cache& c) {
  if (!c.device.is_cuda()) refuse("the cache must lie in GPU memory");
  return stream();
}
at::Tensor new_rows(const Cache& c, int64_t rows, int64_t heads) {
  return at::empty({rows, heads, c.c->head_dim}, at::TensorOptions().dtype(at::kBFloat16).device(c.device));
}

PQ_CALL(kv_write) {
  return guarded([&] {
    PQ_TAKE(pq_kv_write, 4, "cache", "k", "v", "slots");
    const Cache c = cache_of(a[0]);
    const at::Tensor &slots = as_tensor(a[3], "slots"), &k = as_tensor(a[1], "k"), &v = as_tensor(a[2], "v");
    const int64_t* s = (const int64_t*)indices(c, "slots", slots, at::kLong, "torch.int64", 1);
    const int64_t n = slots.size(0);
    const HeadRows kr = head_rows(c, "k", k, n, c.c->kv_heads), vr = head_rows(c, "v", v, n, c.c->kv_heads);
    void* st = stream_of(c);
    call([&] { return pq_kv_write(c.c, kr.p, kr.ld, kr.head, vr.p, vr.ld, vr.head, s, n, st); });
    return none();
  });
}

PQ_CALL(kv_read) {
  return guarded([&] {
    PQ_TAKE(pq_kv_read, 2, "cache", "slots", "k", "v");
    const Cache c = cache_of(a[0]);
    const at::Tensor& slots = as_tensor(a[1], "slots");
    const int64_t* s = (const int64_t*)indices(c, "slots", slots, at::kLong, "torch.int64", 1);
    const int64_t n = slots.size(0);
    const at::Tensor k = given(a[2]) ? as_tensor(a[2], "k") : new_rows(c, n, c.c->kv_heads);
    const at::Tensor v = given(a[3]) ? as_tensor(a[3], "v") : new_rows(c, n, c.c->kv_heads);
    const HeadRows kr = head_rows(c, "k", k, n, c.c->kv_heads), vr = head_rows(c, "v", v, n, c.c->kv_heads);
    void* st = stream_of(c);
    call([&] { return pq_kv_read(c.c, s, n, kr.p, kr.ld, kr.head, vr.p, vr.ld, vr.head, st); });
    Ref ko(THPVariable_Wrap(k)), vo(THPVariable_Wrap(v));
    return PyTuple_Pack(2, ko.p, vo.p);
  });
}

PQ_CALL(attn_decode) {
  return guarded([&] {
    PQ_TAKE(pq_attn_decode, 6, "cache", "q", "table", "lengths", "max_len", "scale", "out", "lse", "window", "workspace");
    const Cache c = cache_of(a[0]);
    const at::Tensor &q = as_tensor(a[1], "q"), &table = as_tensor(a[2], "table"), &lengths = as_tensor(a[3], "lengths");
    if (q.dim() != 3) refuse("q must be bfloat16 [seqs, q_heads, head_dim]");
    const int64_t seqs = q.size(0), q_heads = q.size(1), max_len = as_int(a[4]), window = given(a[8]) ? as_int(a[8]) : 0;
    const float scale = (float)PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) throw PyFailed{};
    const HeadRows qr = head_rows(c, "q", q, seqs, q_heads);
    const int32_t* tab = (const int32_t*)indices(c, "table", table, at::kInt, "torch.int32", 2);
    const int32_t* len = (const int32_t*)indices(c, "lengths", lengths, at::kInt, "torch.int32", 1);
    if (table.size(0) != seqs || lengths.size(0) != seqs || table.size(1) * c.c->page < max_len)
      refuse("table and lengths must have a row for each of %lld sequences, and table the pages of %lld tokens", (long long)seqs,
             (long long)max_len);
    float* lse = nullptr;
    if (given(a[7])) {
      const at::Tensor& t = as_tensor(a[7], "lse");
      if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != seqs || t.size(1) != q_heads || !t.is_contiguous() ||
          t.device() != c.device)
        refuse("lse must be contiguous float32 [%lld, %lld] on the cache's device", (long long)seqs, (long long)q_heads);
      lse = (float*)t.data_ptr();
    }
    const at::Tensor out = given(a[6]) ? as_tensor(a[6], "out") : new_rows(c, seqs, q_heads);
    const HeadRows outr = head_rows(c, "out", out, seqs, q_heads);
    PyObject* w = nullptr;
    if (given(a[9])) {
      w = a[9];
      Py_INCREF(w);
    } else {
      w = PyObject_CallFunction(g_attn_workspace, "OLLLL", a[0], (long long)seqs, (long long)q_heads, (long long)max_len, (long long)window);
    }
    Ref ws(w);
    const at::Tensor& wt = as_tensor(ws.p, "workspace");
    if (!wt.is_contiguous() || wt.device() != c.device) refuse("workspace must be contiguous, on the cache's device");
    void *wp = wt.data_ptr(), *st = stream_of(c);
    const size_t bytes = wt.numel() * wt.element_size();
    const int64_t table_ld = seqs > 1 ? table.stride(0) : table.size(1);
    call([&] {
      return pq_attn_decode(c.c, qr.p, qr.ld, qr.head, tab, table_ld, len, seqs, (int)q_heads, max_len, window, scale, outr.p, outr.ld,
                            outr.head, lse, wp, bytes, st);
    });
    return THPVariable_Wrap(out);
  });
}

// ---- reading back, products by expert, routing: tensors are checked as pq.py's functions check them
at::Tensor bf16_rows(int64_t rows, int64_t width, c10::Device device) {
  return at::empty({rows, width}, at::TensorOptions().dtype(at::kBFloat16).device(device));
}
void on_current_device(const char* name, const at::Tensor& t, const at::Tensor* like) {
  if (!t.is_cuda() || (like ? t.device() != like->device() : t.device().index() != c10::hip::current_device()))
    refuse("%s must lie in the memory of the current GPU, with the call's other tensors", name);
}
// contiguous, of these sizes (a second size of -1: one dimension)
void* array(const char* name, const at::Tensor& t, at::ScalarType type, const char* type_name, int64_t n0, int64_t n1, const at::Tensor& like) {
  const bool two = n1 >= 0;
  if (t.scalar_type() != type || t.dim() != (two ? 2 : 1) || t.size(0) != n0 || (two && t.size(1) != n1) || !t.is_contiguous()) {
    if (two) refuse("%s must be contiguous %s [%lld, %lld]", name, type_name, (long long)n0, (long long)n1);
    refuse("%s must be contiguous %s [%lld]", name, type_name, (long long)n0);
  }
  on_current_device(name, t, &like);
  return t.data_ptr();
}
// bf16 [rows, width] with adjacent columns; the stride of a single row does not matter
struct Rows2 {
  void* p;
  int64_t ld;
};
Rows2 rows2(const char* name, const at::Tensor& t, int64_t rows, int64_t width, const at::Tensor* like) {
  if (t.scalar_type() != at::kBFloat16 || t.dim() != 2 || t.size(0) != rows || t.size(1) != width || (width > 1 && t.stride(1) != 1))
    refuse("%s must be bfloat16 [%lld, %lld] with adjacent columns", name, (long long)rows, (long long)width);
  on_current_device(name, t, like);
  return Rows2{t.data_ptr(), rows > 1 ? t.stride(0) : (width + 7) / 8 * 8};
}

PQ_CALL(dequantize) {
  return guarded([&] {
    PQ_TAKE(pq_dequantize, 4, "fmt", "group", "codes", "scales", "tensor_scale", "y");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const at::Tensor &codes = as_tensor(a[2], "codes"), &scales = as_tensor(a[3], "scales");
    if (codes.dim() != 2 || codes.scalar_type() != at::kByte || !codes.is_contiguous()) refuse("codes must be contiguous uint8 [rows, K/2]");
    const int64_t rows = codes.size(0), K = codes.size(1) * 2;
    on_current_device("codes", codes, nullptr);
    const auto type = fmt == PQ_FMT_NVFP4 || fmt == PQ_FMT_MXFP4 ? at::kByte : at::kFloat;
    if (scales.scalar_type() != type || !scales.is_contiguous() || scales.numel() * group != rows * K)
      refuse("scales must be contiguous, one for every %d channels", group);
    on_current_device("scales", scales, &codes);
    const void* ts = nullptr;
    if (given(a[4])) {
      const at::Tensor& t = as_tensor(a[4], "tensor_scale");
      if (t.scalar_type() != at::kFloat || t.numel() < 1) refuse("tensor_scale must be float32");
      on_current_device("tensor_scale", t, &codes);
      ts = t.data_ptr();
    }
    const at::Tensor y = given(a[5]) ? as_tensor(a[5], "y") : bf16_rows(rows, K, codes.device());
    const Rows2 yr = rows2("y", y, rows, K, &codes);
    void *c = codes.data_ptr(), *sp = scales.data_ptr(), *st = stream();
    call([&] { return pq_dequantize((pq_format)fmt, group, (const uint8_t*)c, sp, (const float*)ts, rows, K, yr.p, yr.ld, st); });
    return THPVariable_Wrap(y);
  });
}

PQ_CALL(qgemm_grouped) {
  return guarded([&] {
    PQ_TAKE(pq_qgemm_grouped, 9, "fmt", "group", "a_operand", "a_rows", "w_operands", "offsets", "y", "N", "K", "rows", "bias");
    const int fmt = (int)as_int(a[0]), group = (int)as_int(a[1]);
    const int64_t a_rows = as_int(a[3]), N = as_int(a[7]), K = as_int(a[8]);
    const at::Tensor &ao = as_tensor(a[2], "a_operand"), &w = as_tensor(a[4], "w_operands"), &off = as_tensor(a[5], "offsets"), &y = as_tensor(a[6], "y");
    if (w.dim() != 2 || w.scalar_type() != at::kByte || !w.is_contiguous()) refuse("w_operands must be contiguous uint8 [experts, bytes of an operand]");
    if (y.dim() != 2) refuse("y must be bfloat16 [M, %lld] with adjacent columns", (long long)N);
    const int64_t experts = w.size(0), M = y.size(0);
    const size_t need = pq_operand_bytes((pq_format)fmt, group, N, K);
    if (need && (size_t)w.size(1) != need) refuse("w_operands must hold %zu bytes an expert", need);
    const Rows2 yr = rows2("y", y, M, N, nullptr);
    on_current_device("w_operands", w, &y);
    on_current_device("a_operand", ao, &y);
    if (ao.scalar_type() != at::kByte || !ao.is_contiguous() || (size_t)ao.numel() < pq_operand_bytes((pq_format)fmt, group, a_rows, K))
      refuse("a_operand must be contiguous uint8 and hold an operand of %lld rows", (long long)a_rows);
    if (experts > INT32_MAX) refuse("w_operands has too many experts");
    const void* op = array("offsets", off, at::kInt, "torch.int32", experts + 1, -1, y);
    const void* rp = given(a[9]) ? array("rows", as_tensor(a[9], "rows"), at::kInt, "torch.int32", M, -1, y) : nullptr;
    const void* bp = given(a[10]) ? array("bias", as_tensor(a[10], "bias"), at::kBFloat16, "torch.bfloat16", experts, N, y) : nullptr;
    void *ap = ao.data_ptr(), *wp = w.data_ptr(), *st = stream();
    call([&] {
      return pq_qgemm_grouped((pq_format)fmt, group, ap, a_rows, wp, (int)experts, (const int32_t*)op, (const int32_t*)rp, M, N, K, bp, yr.p, yr.ld, st);
    });
    return none();
  });
}

PQ_CALL(moe_route) {
  return guarded([&] {
    PQ_TAKE(pq_moe_route, 2, "logits", "k", "renormalize", "out", "workspace");
    const at::Tensor& x = as_tensor(a[0], "logits");
    if (x.dim() != 2 || (x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16) || (x.size(1) > 1 && x.stride(1) != 1))
      refuse("logits must be float32 or bfloat16 [tokens, experts] with adjacent experts");
    const int64_t tokens = x.size(0), experts = x.size(1), k = as_int(a[1]);
    const int renormalize = given(a[2]) ? PyObject_IsTrue(a[2]) : 1;
    if (renormalize < 0) throw PyFailed{};
    if (k > INT32_MAX || k < INT32_MIN || experts > INT32_MAX) refuse("k=%lld or experts=%lld out of range", (long long)k, (long long)experts);
    on_current_device("logits", x, nullptr);
    PyObject* w = nullptr;
    if (given(a[4])) {
      w = a[4];
      Py_INCREF(w);
    } else {
      w = PyObject_CallFunction(g_route_workspace, "LLLO", (long long)tokens, (long long)experts, (long long)k, a[0]);
    }
    Ref ws(w);
    const at::Tensor& wt = as_tensor(ws.p, "workspace");
    if (!wt.is_contiguous()) refuse("workspace must be contiguous");
    on_current_device("workspace", wt, &x);
    PyObject* o = nullptr;
    if (given(a[3])) {
      o = a[3];
      Py_INCREF(o);
    } else {
      o = PyObject_CallFunction(g_route, "LLLO", (long long)tokens, (long long)experts, (long long)k, a[0]);
    }
    Ref out(o);
    if (!PyTuple_Check(out.p) || PyTuple_GET_SIZE(out.p) != 5) fail(PyExc_TypeError, "out must be a Route");
    const auto part = [&](int i, const char* name) -> const at::Tensor& { return as_tensor(PyTuple_GET_ITEM(out.p, i), name); };
    void* ids = array("ids", part(0, "ids"), at::kInt, "torch.int32", tokens, k, x);
    void* weights = array("weights", part(1, "weights"), at::kFloat, "torch.float32", tokens, k, x);
    void* offsets = array("offsets", part(2, "offsets"), at::kInt, "torch.int32", experts + 1, -1, x);
    void* rows = array("rows", part(3, "rows"), at::kInt, "torch.int32", tokens * k, -1, x);
    void* positions = array("positions", part(4, "positions"), at::kInt, "torch.int32", tokens, k, x);
    const pq_logits type = x.scalar_type() == at::kBFloat16 ? PQ_LOGITS_BF16 : PQ_LOGITS_F32;
    void *xp = x.data_ptr(), *wp = wt.data_ptr(), *st = stream();
    const int64_t ld = tokens > 1 ? x.stride(0) : experts;
    const size_t bytes = wt.numel() * wt.element_size();
    call([&] {
      return pq_moe_route(type, xp, tokens, (int)experts, ld, (int)k, renormalize, (int32_t*)ids, (float*)weights, (int32_t*)offsets, (int32_t*)rows,
                          (int32_t*)positions, wp, bytes, st);
    });
    Py_INCREF(out.p);
    return out.p;
  });
}

PQ_CALL(moe_combine) {
  return guarded([&] {
    PQ_TAKE(pq_moe_combine, 3, "y", "positions", "weights", "addend", "out");
    const at::Tensor &y = as_tensor(a[0], "y"), &pos = as_tensor(a[1], "positions"), &weights = as_tensor(a[2], "weights");
    if (y.dim() != 2 || pos.dim() != 2) refuse("y must be bfloat16 [rows, N], positions int32 [tokens, k]");
    const int64_t rows = y.size(0), N = y.size(1), tokens = pos.size(0), k = pos.size(1);
    const Rows2 yr = rows2("y", y, rows, N, nullptr);
    const void* pp = array("positions", pos, at::kInt, "torch.int32", tokens, k, y);
    const void* wp = array("weights", weights, at::kFloat, "torch.float32", tokens, k, y);
    const Rows2 ar = given(a[3]) ? rows2("addend", as_tensor(a[3], "addend"), tokens, N, &y) : Rows2{nullptr, 0};
    const at::Tensor out = given(a[4])    ? as_tensor(a[4], "out")
                           : N % 8 == 0 ? bf16_rows(tokens, N, y.device())
                                        : bf16_rows(tokens, (N + 7) / 8 * 8, y.device()).narrow(1, 0, N);
    const Rows2 outr = rows2("out", out, tokens, N, &y);
    if (k > INT32_MAX) refuse("k=%lld out of range", (long long)k);
    void* st = stream();
    call([&] {
      return pq_moe_combine(yr.p, rows, yr.ld, (const int32_t*)pp, (const float*)wp, tokens, (int)k, N, ar.p, ar.ld, outr.p, outr.ld, st);
    });
    return THPVariable_Wrap(out);
  });
}

PyObject* bind(PyObject*, PyObject* args) {
  constexpr int n = 7;
  PyObject* given_by[n] = {};
  if (!PyArg_ParseTuple(args, "OOOOO|OO", &given_by[0], &given_by[1], &given_by[2], &given_by[3], &given_by[4], &given_by[5], &given_by[6])) return nullptr;
  PyObject** const slots[n] = {&g_raise, &g_operand, &g_workspace, &g_refuse, &g_attn_workspace, &g_route_workspace, &g_route};
  for (int i = 0; i < n; ++i) {
    if (!given_by[i]) continue;                // what stands stays
    Py_INCREF(given_by[i]);
    Py_XSETREF(*slots[i], given_by[i]);
  }
  Py_RETURN_NONE;
}

#define PQ_METHOD(fn, signature, text) \
  {"pq_" #fn, (PyCFunction)(void (*)(void))fn, METH_FASTCALL | METH_KEYWORDS, "pq_" #fn signature "\n--\n\n" text}
PyMethodDef methods[] = {
    PQ_METHOD(quantize_act, "(fmt, group, x, perm, tensor_scale, codes, scales, M=None, K=None, ld=None)",
              "Dynamic activation quantization into the stored layout."),
    PQ_METHOD(quantize_act_packed, "(fmt, group, x, tensor_scale, operand=None, codes=None, scales=None, K=None)",
              "Dynamic activation quantization straight into the GEMM's panel layout."),
    PQ_METHOD(norm_quantize_act_packed,
              "(kind, fmt, group, x, eps, tensor_scale, perm=None, gamma=None, mod_scale=None, mod_shift=None, rows_per_mod=0, "
              "operand=None, y=None, K=None)",
              "pq_norm_reorder feeding the activation quantizer directly: returns the GEMM operand."),
    PQ_METHOD(hadamard_quantize_act_packed, "(fmt, group, x, tensor_scale, perm=None, operand=None, y=None, K=None)",
              "The rotation feeding the activation quantizer directly: returns the GEMM operand."),
    PQ_METHOD(qgemm_packed, "(fmt, group, a_operand, a_tensor_scale, w_operand, w_tensor_scale, y, M, N, K, ldy=None)",
              "y[M, N] (bf16) = the product of two packed operands."),
    PQ_METHOD(qgemm_packed_f32, "(fmt, group, a_operand, a_tensor_scale, w_operand, w_tensor_scale, y, M, N, K, ldy=None)",
              "The packed product in fp32, before the rounding to bf16."),
    PQ_METHOD(qgemm_packed_bias, "(fmt, group, a_operand, a_tensor_scale, w_operand, w_tensor_scale, bias, y, M, N, K, ldy=None)",
              "The packed product plus the layer's bias (bf16 [N]), added before the rounding to bf16."),
    PQ_METHOD(qgemm,
              "(fmt, group, a_codes, a_scales, a_tensor_scale, w_codes, w_scales, w_tensor_scale, y, workspace=None, M=None, N=None, "
              "K=None, ldy=None)",
              "y[M, N] (bf16) = dequant(A) @ dequant(W)^T."),
    PQ_METHOD(calib_moments, "(x, sumsq, absmax=None, workspace=None, rows=None, K=None, ld=None)",
              "sumsq[K] (float64, in/out) += column sums of squares of bf16 x[rows, ld]."),
    PQ_METHOD(kv_write, "(cache, k, v, slots)",
              "Quantizes keys and values, bf16 [n, kv_heads, head_dim] (slices of a fused projection's rows are), into the slots (int64 [n])."),
    PQ_METHOD(kv_read, "(cache, slots, k=None, v=None)", "(k, v) of the slots as bf16 [n, kv_heads, head_dim] (allocated unless given)."),
    PQ_METHOD(attn_decode, "(cache, q, table, lengths, max_len, scale, out=None, lse=None, window=0, workspace=None)",
              "Attention of one new token a sequence, q bf16 [seqs, q_heads, head_dim], over the lengths[b] (int32) tokens whose pages\n"
              "table[b] (int32) names; out like q (allocated unless given), lse float32 [seqs, q_heads].  max_len: no sequence is longer."),
    PQ_METHOD(dequantize, "(fmt, group, codes, scales, tensor_scale=None, y=None)",
              "The values that stored codes [rows, K/2] and scales stand for, bf16 [rows, K] (allocated unless given)."),
    PQ_METHOD(qgemm_grouped, "(fmt, group, a_operand, a_rows, w_operands, offsets, y, N, K, rows=None, bias=None)",
              "y[i] (bf16 [M, N]) = row rows[i] (int32 [M], or i) of A times the weights of the expert whose rows offsets (int32 [experts + 1])\n"
              "places i in, plus bias[expert] (bf16 [experts, N]).  w_operands: uint8 [experts, pq_operand_bytes(fmt, group, N, K)]."),
    PQ_METHOD(moe_route, "(logits, k, renormalize=True, out=None, workspace=None)",
              "The k largest of every row of logits (float32 or bf16 [tokens, experts]), their softmax weights, and the order of the rows by\n"
              "expert (allocated unless given)."),
    PQ_METHOD(moe_combine, "(y, positions, weights, addend=None, out=None)",
              "out[t] = addend[t] + sum_j weights[t, j] * y[positions[t, j]], bf16 [tokens, N] (allocated unless given); y bf16 [rows, N],\n"
              "positions int32 and weights float32 [tokens, k]."),
    {"bind", bind, METH_VARARGS, "bind(raise_, operand, workspace, refuse, attn_workspace, route_workspace, route): the helpers of pq.py"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pq_calls", "Hot calls of the binding (see pq.py).", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pq_calls() { return PyModule_Create(&module); }
