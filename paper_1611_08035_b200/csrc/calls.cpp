// The calls of the 8-bit operators from Python without ctypes: on a few tokens the GPU needs two or three microseconds, and
// marshalling seventeen arguments in Python took as long again.
//
// Each function takes what its namesake in binding.py takes.  It handles positional arguments of the right types; whatever
// else it is given it hands to that namesake, which says what is wrong or sorts out the keywords.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "b2gemm.h"

namespace {

struct Entry {
  void* fn = nullptr;          // the library's function
  PyObject* full = nullptr;    // its namesake in binding.py
};
Entry g_norm, g_norm_bwd, g_quant, g_gemm, g_wgrad, g_gemm_act, g_act_bwd, g_adamw;
PyObject* g_error = nullptr;   // binding.B2Error

// Reads arguments one after the other; ok turns false at the first that is not what was asked for.
struct Args {
  PyObject* const* a;
  Py_ssize_t n, i = 0;
  bool ok = true;
  int64_t integer() {
    if (!ok || i >= n || !PyLong_Check(a[i])) return ok = false, 0;
    const long long v = PyLong_AsLongLong(a[i++]);
    if (v == -1 && PyErr_Occurred()) PyErr_Clear(), ok = false;
    return v;
  }
  double number() {
    if (!ok || i >= n || !(PyFloat_Check(a[i]) || PyLong_Check(a[i]))) return ok = false, 0.0;
    const double v = PyFloat_AsDouble(a[i++]);
    if (v == -1.0 && PyErr_Occurred()) PyErr_Clear(), ok = false;
    return v;
  }
  char letter() {
    Py_ssize_t len = 0;
    const char* s = ok && i < n && PyUnicode_Check(a[i]) ? PyUnicode_AsUTF8AndSize(a[i++], &len) : nullptr;
    if (!s || len != 1) return ok = false, PyErr_Clear(), '\0';
    return s[0];
  }
  // a CUDA tensor, or nullptr for None where that is allowed
  const at::Tensor* tensor(bool none = false) {
    if (!ok || i >= n) return ok = false, nullptr;
    if (none && a[i] == Py_None) return ++i, nullptr;
    if (!THPVariable_Check(a[i])) return ok = false, nullptr;
    const at::Tensor* t = &THPVariable_Unpack(a[i++]);
    if (!t->is_cuda()) ok = false;
    return t;
  }
  void* typed(at::ScalarType type, bool none = false) {
    const at::Tensor* t = tensor(none);
    if (!t) return nullptr;
    if (t->scalar_type() != type) ok = false;
    return t->data_ptr();
  }
  bool all_read() {  // and the optional `check` at the end was left out or is True
    return ok && (i == n || (i + 1 == n && a[i] == Py_True));
  }
};

int type_code(const at::Tensor* t) {
  return !t ? 0 : t->scalar_type() == at::kBFloat16 ? B2_TYPE_BF16 : t->scalar_type() == at::kFloat ? B2_TYPE_F32 : 0;
}
int scale_code(const at::Tensor* t) {
  return !t ? -1 : t->scalar_type() == at::kFloat8_e8m0fnu ? B2_SCALE_E8M0 : t->scalar_type() == at::kFloat ? B2_SCALE_F32 : -1;
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

PyObject* hand_over(const Entry& e, PyObject* const* a, Py_ssize_t n, PyObject* names) { return PyObject_Vectorcall(e.full, a, (size_t)n, names); }

// Calls the library and turns its answer into Python's.  Other threads run meanwhile: a launch waits when the stream is full, and what would
// make room may be one of theirs (a callback on the host).
template <typename Call>
PyObject* result(const char* name, const Call& call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = call();
  Py_END_ALLOW_THREADS
  if (rc == 0) return PyLong_FromLong(0);
  PyObject* err = PyObject_CallFunction(g_error, "si", name, rc);
  if (err) {
    PyErr_SetObject(g_error, err);
    Py_DECREF(err);
  }
  return nullptr;
}

PyObject* norm(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const int64_t d = p.integer(), t = p.integer();
  const at::Tensor* x = p.tensor();
  const int code = type_code(x);
  const auto type = x ? x->scalar_type() : at::kFloat;
  const int64_t ldx = p.integer();
  void* r = p.typed(type, true);
  const int64_t ldr = p.integer();
  void* w = p.typed(type);
  const double eps = p.number();
  void* h = p.typed(type, true);
  const int64_t ldh = p.integer();
  void* q = p.typed(at::kFloat8_e4m3fn);
  const int64_t ldq = p.integer();
  void* s = p.typed(at::kFloat8_e8m0fnu);
  const int64_t lds = p.integer();
  void* rstd = p.typed(at::kFloat, true);
  if (names || !code || !p.all_read()) return hand_over(g_norm, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_rmsnorm_f8)>(g_norm.fn);
  void *X = x->data_ptr(), *st = stream();
  return result("b2_rmsnorm_f8", [&] { return fn(d, t, code, X, ldx, r, ldr, w, (float)eps, h, ldh, q, ldq, s, lds, static_cast<float*>(rstd), st); });
}

PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const int64_t d = p.integer(), t = p.integer();
  const at::Tensor* dy = p.tensor();
  const int code = type_code(dy);
  const auto type = dy ? dy->scalar_type() : at::kFloat;
  const int64_t lddy = p.integer();
  void* h = p.typed(type);
  const int64_t ldh = p.integer();
  void* rstd = p.typed(at::kFloat);
  void* w = p.typed(type);
  void* dh = p.typed(type, true);
  const int64_t lddh = p.integer();
  void* dx = p.typed(type);
  const int64_t lddx = p.integer();
  void* dw = p.typed(at::kFloat);
  const at::Tensor* ws = p.tensor(true);
  if (names || !code || !p.all_read()) return hand_over(g_norm_bwd, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_rmsnorm_backward)>(g_norm_bwd.fn);
  void *DY = dy->data_ptr(), *W = ws ? ws->data_ptr() : nullptr, *st = stream();
  const size_t bytes = ws ? ws->nbytes() : 0;
  return result("b2_rmsnorm_backward", [&] {
    return fn(d, t, code, DY, lddy, h, ldh, static_cast<float*>(rstd), w, dh, lddh, dx, lddx, static_cast<float*>(dw), W, bytes, st);
  });
}

PyObject* quant(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const int64_t d = p.integer(), t = p.integer(), block = p.integer();
  const at::Tensor* x = p.tensor();
  const int code = type_code(x);
  const int64_t ldx = p.integer();
  void* q = p.typed(at::kFloat8_e4m3fn);
  const int64_t ldq = p.integer();
  void* s = p.typed(at::kFloat8_e8m0fnu);
  const int64_t lds = p.integer();
  if (names || !code || block != (int)block || !p.all_read()) return hand_over(g_quant, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_quant_f8)>(g_quant.fn);
  void *X = x->data_ptr(), *st = stream();
  return result("b2_quant_f8", [&] { return fn(d, t, (int)block, code, X, ldx, q, ldq, s, lds, st); });
}

PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const char ta = p.letter(), tb = p.letter();
  const int64_t m = p.integer(), nn = p.integer(), k = p.integer();
  const double alpha = p.number();
  void* A = p.typed(at::kFloat8_e4m3fn);
  const int64_t lda = p.integer();
  const at::Tensor* SA = p.tensor();
  const int64_t ldsa = p.integer(), block_a = p.integer();
  void* B = p.typed(at::kFloat8_e4m3fn);
  const int64_t ldb = p.integer();
  const at::Tensor* SB = p.tensor();
  const int64_t ldsb = p.integer(), block_b = p.integer();
  const double beta = p.number();
  const at::Tensor* C = p.tensor();
  const int64_t ldc = p.integer();
  const at::Tensor* ws = p.i < p.n ? p.tensor(true) : nullptr;
  const int code = type_code(C), ca = scale_code(SA), cb = scale_code(SB);
  if (names || !code || ca < 0 || cb < 0 || block_a != (int)block_a || block_b != (int)block_b || !p.all_read()) return hand_over(g_gemm, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_gemm_f8)>(g_gemm.fn);
  void *sa = SA->data_ptr(), *sb = SB->data_ptr(), *c = C->data_ptr(), *W = ws ? ws->data_ptr() : nullptr, *st = stream();
  const size_t bytes = ws ? ws->nbytes() : 0;
  return result("b2_gemm_f8", [&] {
    return fn(ta, tb, m, nn, k, (float)alpha, A, lda, sa, ldsa, (int)block_a, ca, B, ldb, sb, ldsb, (int)block_b, cb, (float)beta, c, ldc, code, W, bytes, st);
  });
}

PyObject* wgrad(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const int64_t m = p.integer(), nn = p.integer(), k = p.integer();
  const double alpha = p.number();
  void* Q = p.typed(at::kFloat8_e4m3fn);
  const int64_t ldq = p.integer();
  void* S = p.typed(at::kFloat8_e8m0fnu);
  const int64_t lds = p.integer();
  void* Y = p.typed(at::kBFloat16);
  const int64_t ldy = p.integer();
  const double beta = p.number();
  const at::Tensor* C = p.tensor();
  const int64_t ldc = p.integer();
  const at::Tensor* ws = p.i < p.n ? p.tensor(true) : nullptr;
  const int code = type_code(C);
  if (names || !code || !p.all_read()) return hand_over(g_wgrad, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_wgrad_f8)>(g_wgrad.fn);
  void *c = C->data_ptr(), *W = ws ? ws->data_ptr() : nullptr, *st = stream();
  const size_t bytes = ws ? ws->nbytes() : 0;
  return result("b2_wgrad_f8", [&] { return fn(m, nn, k, (float)alpha, Q, ldq, S, lds, Y, ldy, (float)beta, c, ldc, code, W, bytes, st); });
}

// the type that the tensors share which are there; 0 where two differ, fp32 where there is none
int shared_type(std::initializer_list<const at::Tensor*> tensors) {
  const at::Tensor* first = nullptr;
  for (const at::Tensor* t : tensors) {
    if (t && first && t->scalar_type() != first->scalar_type()) return 0;
    first = first ? first : t;
  }
  return first ? type_code(first) : B2_TYPE_F32;
}
void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

PyObject* gemm_act(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const char ta = p.letter(), tb = p.letter();
  const int64_t m = p.integer(), nn = p.integer(), k = p.integer();
  const double alpha = p.number();
  void* A = p.typed(at::kFloat8_e4m3fn);
  const int64_t lda = p.integer();
  const at::Tensor* SA = p.tensor();
  const int64_t ldsa = p.integer(), block_a = p.integer();
  void* B = p.typed(at::kFloat8_e4m3fn);
  const int64_t ldb = p.integer();
  const at::Tensor* SB = p.tensor();
  const int64_t ldsb = p.integer(), block_b = p.integer(), act = p.integer();
  void* bias = p.typed(at::kFloat, true);
  const at::Tensor* Z = p.tensor(true);
  const int64_t ldz = p.integer();
  const at::Tensor* R = p.tensor(true);
  const int64_t ldr = p.integer();
  const at::Tensor* C = p.tensor(true);
  const int64_t ldc = p.integer();
  void* q = p.typed(at::kFloat8_e4m3fn, true);
  const int64_t ldq = p.integer();
  void* s = p.typed(at::kFloat8_e8m0fnu, true);
  const int64_t lds = p.integer();
  const at::Tensor* ws = p.i < p.n ? p.tensor(true) : nullptr;
  const int code = p.ok ? shared_type({C, Z, R}) : 0, ca = scale_code(SA), cb = scale_code(SB);
  if (names || !code || ca < 0 || cb < 0 || block_a != (int)block_a || block_b != (int)block_b || act != (int)act || !p.all_read()) return hand_over(g_gemm_act, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_gemm_f8_act)>(g_gemm_act.fn);
  void *sa = SA->data_ptr(), *sb = SB->data_ptr(), *z = address(Z), *r = address(R), *c = address(C), *W = address(ws), *st = stream();
  const size_t bytes = ws ? ws->nbytes() : 0;
  return result("b2_gemm_f8_act", [&] {
    return fn(ta, tb, m, nn, k, (float)alpha, A, lda, sa, ldsa, (int)block_a, ca, B, ldb, sb, ldsb, (int)block_b, cb, (int)act, static_cast<float*>(bias), z, ldz, r, ldr, c, ldc, code, q,
              ldq, s, lds, W, bytes, st);
  });
}

PyObject* act_bwd(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  Args p{a, n};
  const int64_t d = p.integer(), t = p.integer(), act = p.integer();
  const at::Tensor* dy = p.tensor();
  const int64_t lddy = p.integer();
  const at::Tensor* Z = p.tensor(true);
  const int64_t ldz = p.integer();
  const at::Tensor* DZ = p.tensor(true);
  const int64_t lddz = p.integer();
  void* q = p.typed(at::kFloat8_e4m3fn, true);
  const int64_t ldq = p.integer();
  void* s = p.typed(at::kFloat8_e8m0fnu, true);
  const int64_t lds = p.integer();
  void* db = p.typed(at::kFloat, true);
  const at::Tensor* ws = p.i < p.n ? p.tensor(true) : nullptr;
  const int code = p.ok ? shared_type({dy, Z, DZ}) : 0;
  if (names || !code || act != (int)act || !p.all_read()) return hand_over(g_act_bwd, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_act_backward)>(g_act_bwd.fn);
  void *y = dy->data_ptr(), *z = address(Z), *dz = address(DZ), *W = address(ws), *st = stream();
  const size_t bytes = ws ? ws->nbytes() : 0;
  return result("b2_act_backward", [&] { return fn(d, t, code, (int)act, y, lddy, z, ldz, dz, lddz, q, ldq, s, lds, static_cast<float*>(db), W, bytes, st); });
}

// Entry i of a list or tuple, a contiguous CUDA tensor; nullptr if it is anything else.
const at::Tensor* entry(PyObject* list, Py_ssize_t i) {
  PyObject* o = PyList_Check(list) ? PyList_GET_ITEM(list, i) : PyTuple_GET_ITEM(list, i);
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor* t = &THPVariable_Unpack(o);
  return t->is_cuda() && t->is_contiguous() ? t : nullptr;
}
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  auto length = [](PyObject* o) { return PyList_Check(o) ? PyList_GET_SIZE(o) : PyTuple_Check(o) ? PyTuple_GET_SIZE(o) : (Py_ssize_t)-1; };
  if (names || n < 12) return hand_over(g_adamw, a, n, names);
  const Py_ssize_t count = length(a[0]);
  const bool scales = a[4] != Py_None;
  bool ok = count >= 0 && count == (int)count;
  for (int i = 1; i < 6 && ok; ++i) ok = (i >= 4 && !scales) ? a[i] == Py_None : length(a[i]) == count;
  if (!ok) return hand_over(g_adamw, a, n, names);
  std::vector<b2_adamw_tensor> table(count);
  int device = -1;  // of all tensors
  auto here = [&](const at::Tensor* t) { return (device = device < 0 ? t->get_device() : device) == t->get_device(); };
  for (Py_ssize_t i = 0; i < count && ok; ++i) {
    const at::Tensor* t[6] = {};
    for (int j = 0; j < 4 && ok; ++j) {
      t[j] = entry(a[j], i);
      ok = t[j] && t[j]->numel() == t[0]->numel() && here(t[j]);
    }
    if (!ok) break;
    const int64_t size = t[0]->numel();
    const bool eight = t[2]->scalar_type() == at::kFloat8_e4m3fn;
    const auto state = eight ? at::kFloat8_e4m3fn : at::kFloat;
    ok = type_code(t[0]) && type_code(t[1]) && t[2]->scalar_type() == state && t[3]->scalar_type() == state && (!eight || scales);
    for (int j = 4; j < 6 && eight && ok; ++j) {
      t[j] = entry(a[j], i);
      ok = t[j] && t[j]->scalar_type() == at::kFloat8_e8m0fnu && t[j]->numel() == (size + 127) / 128 && here(t[j]);
    }
    if (ok) table[i] = {t[0]->data_ptr(), t[1]->data_ptr(), t[2]->data_ptr(), t[3]->data_ptr(), address(t[4]), address(t[5]), size, type_code(t[0]), type_code(t[1]), eight ? 8 : 32, 0};
  }
  Args p{a, n};
  p.i = 6;
  // a number, or where that is given one number on the device
  auto either = [&](at::ScalarType type) -> void* {
    if (!p.ok || p.i >= p.n || !THPVariable_Check(a[p.i])) return nullptr;
    const at::Tensor* t = p.tensor();
    if (t && (t->scalar_type() != type || t->numel() != 1 || !here(t))) p.ok = false;
    return p.ok ? t->data_ptr() : nullptr;
  };
  void* lr_device = either(at::kFloat);
  const double lr = lr_device ? 0.0 : p.number(), beta1 = p.number(), beta2 = p.number(), eps = p.number(), decay = p.number();
  void* step_device = either(at::kLong);
  const int64_t step = step_device ? 1 : p.integer(), seed = p.i < p.n ? p.integer() : 0;
  const at::Tensor* scale = p.i < p.n ? p.tensor(true) : nullptr;
  if (!ok || (scale && (scale->scalar_type() != at::kFloat || scale->numel() != 1 || !here(scale))) || !p.all_read()) return hand_over(g_adamw, a, n, names);
  const auto fn = reinterpret_cast<decltype(&b2_adamw)>(g_adamw.fn);
  void *gs = address(scale), *st = stream();
  return result("b2_adamw", [&] {
    return fn(table.data(), (int)count, lr, beta1, beta2, eps, decay, step, (uint64_t)seed, static_cast<float*>(gs), static_cast<float*>(lr_device), static_cast<int64_t*>(step_device), st);
  });
}

// connect(error class, {name: (address in the library, function in binding.py)})
PyObject* connect(PyObject*, PyObject* args) {
  PyObject *error, *table;
  if (!PyArg_ParseTuple(args, "OO!", &error, &PyDict_Type, &table)) return nullptr;
  const struct {
    const char* name;
    Entry* e;
  } entries[] = {{"b2_rmsnorm_f8", &g_norm}, {"b2_rmsnorm_backward", &g_norm_bwd}, {"b2_quant_f8", &g_quant}, {"b2_gemm_f8", &g_gemm}, {"b2_wgrad_f8", &g_wgrad},
                {"b2_gemm_f8_act", &g_gemm_act}, {"b2_act_backward", &g_act_bwd}, {"b2_adamw", &g_adamw}};
  for (const auto& it : entries) {
    PyObject* pair = PyDict_GetItemString(table, it.name);
    PyObject* full;
    unsigned long long address;
    if (!pair || !PyArg_ParseTuple(pair, "KO", &address, &full)) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, it.name);
      return nullptr;
    }
    Py_INCREF(full);
    Py_XDECREF(it.e->full);
    it.e->fn = reinterpret_cast<void*>(address), it.e->full = full;
  }
  Py_INCREF(error);
  Py_XDECREF(g_error);
  g_error = error;
  Py_RETURN_NONE;
}

// No C++ exception leaves a function that Python calls (a tensor without storage throws when it is asked for its address).
template <PyObject* (*FN)(PyObject*, PyObject* const*, Py_ssize_t, PyObject*)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n, PyObject* names) {
  try {
    return FN(self, a, n, names);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

#define B2_CALL(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<fn>)), METH_FASTCALL | METH_KEYWORDS, "The function of the same name in binding.py, called without ctypes."}
PyMethodDef g_methods[] = {B2_CALL("b2_rmsnorm_f8", norm),   B2_CALL("b2_rmsnorm_backward", norm_bwd), B2_CALL("b2_quant_f8", quant),
                           B2_CALL("b2_gemm_f8", gemm),      B2_CALL("b2_wgrad_f8", wgrad),
                           B2_CALL("b2_gemm_f8_act", gemm_act), B2_CALL("b2_act_backward", act_bwd), B2_CALL("b2_adamw", adamw), {"connect", connect, METH_VARARGS, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_b2calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__b2calls() { return PyModule_Create(&g_module); }
