// The serving calls' short way from Python to the library: the checks, the allocations and the call of the Python
// functions of the same names, for arguments that are as they should be and lie on the current device. For anything
// else a function here answers NotImplemented, having done nothing, and the Python function goes its own way, which
// says what is wrong. A decode step's calls take less time on the GPU than their checks take in Python: host time
// of a call of 16 rows (us, Python alone and with this file) rope 8.5, 4.4; plan 10.2, 5.1; store and load 16.5, 8.9;
// packed prompts 9.0, 4.7; attention over the cache 10.5, 5.4; a launch is 2.4 of it, an allocation 0.6.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/qgemm.h"

namespace {

// Entry points of the library as the Python side has loaded it, and torch's current raw stream of a device.
struct {
  decltype(&qgemm_kv_plan) kv_plan;
  decltype(&qgemm_rope) rope;
  decltype(&qgemm_kv4_store) store;
  decltype(&qgemm_kv4_load) load;
  decltype(&qgemm_attention_packed) packed;
  decltype(&qgemm_attention_kv4) kv4;
  decltype(&qgemm_attention_kv4_workspace) kv4_workspace;
  PyObject* raw_stream;
} lib = {};

PyObject* not_here() {
  PyErr_Clear();
  Py_RETURN_NOTIMPLEMENTED;
}

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

bool dense(const at::Tensor* t, at::ScalarType type, int64_t dims) {
  return t && t->is_cuda() && t->scalar_type() == type && t->dim() == dims && t->is_contiguous();
}

// [T][heads][D] with the heads of a row end to end; the elements between rows
bool rows(const at::Tensor* t, int64_t* stride) {
  if (!t || !t->is_cuda() || t->dim() != 3) return false;
  const int64_t T = t->size(0), h = t->size(1), D = t->size(2);
  if ((D > 1 && t->stride(2) != 1) || (h > 1 && t->stride(1) != D)) return false;
  *stride = T > 1 ? t->stride(0) : h * D;
  return true;
}

// Whether the tensors lie on the current device; its stream.
bool stream_of(std::initializer_list<const at::Tensor*> ts, hipStream_t* s) {
  static const c10::impl::VirtualGuardImpl guard(c10::DeviceType::CUDA);
  const c10::DeviceIndex dev = guard.getDevice().index();
  for (const at::Tensor* t : ts)
    if (t && t->get_device() != dev) return false;
  PyObject* d = PyLong_FromLong(dev);
  PyObject* r = d ? PyObject_CallOneArg(lib.raw_stream, d) : nullptr;
  Py_XDECREF(d);
  if (!r) return false;
  *s = static_cast<hipStream_t>(PyLong_AsVoidPtr(r));
  Py_DECREF(r);
  return !PyErr_Occurred();
}

bool to_int(PyObject* o, int* v) {
  const long x = PyLong_Check(o) ? PyLong_AsLong(o) : -1;
  *v = (int)x;
  return PyLong_Check(o) && !PyErr_Occurred() && x >= INT32_MIN && x <= INT32_MAX;
}

bool to_float(PyObject* o, float* v) {
  *v = (float)PyFloat_AsDouble(o);
  return !PyErr_Occurred();
}

// None gives the usual 1 / sqrt(D)
bool to_scale(PyObject* o, int64_t D, float* v) {
  if (o != Py_None) return to_float(o, v);
  *v = (float)std::pow((double)D, -0.5);
  return D > 0;
}

bool small(std::initializer_list<int64_t> sizes) {
  for (int64_t n : sizes)
    if (n > INT32_MAX) return false;
  return true;
}

bool cache_sizes(const at::Tensor* c, int64_t D, int* pages, int* Hkv, int* page) {
  if (!dense(c, at::kByte, 3) || D < 16 || !small({c->size(0), c->size(1), c->size(2), D})) return false;
  const int64_t record = c->size(2);
  if (record * 16 % (17 * D) != 0) return false;
  *pages = (int)c->size(0);
  *Hkv = (int)c->size(1);
  *page = (int)(record * 16 / (17 * D));
  return true;
}

// A tensor's memory, null for none; throws for a tensor that has no memory (one inside torch.vmap, say), so it is
// read before the interpreter's lock is let go.
template <typename T = void>
T* memory(const at::Tensor* t) {
  return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

// Calls f without the interpreter's lock (a launch may wait for room in the queue), which is held again however f ends.
template <typename F>
int call(F&& f) {
  struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  } unlocked;
  return f();
}

// n elements of a dense tensor from `at` on, as a tensor of their own (five of them 0.7 us less than as views)
at::Tensor piece(const at::Tensor& t, int64_t at, int64_t n) {
  at::Tensor p = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(t.storage()), t.key_set(), t.dtype());
  p.unsafeGetTensorImpl()->set_storage_offset(at);
  p.unsafeGetTensorImpl()->set_sizes_contiguous({n});
  return p;
}

// (kv_len, q_len, block_table, free_pages, page, tokens) -> (cu_q, kv_len, used, positions, slots)
PyObject* kv_plan_(PyObject* const* a) {
  const at::Tensor *kv = tensor(a[0]), *ql = tensor(a[1]), *tab = tensor(a[2]), *fr = tensor(a[3]);
  int page, T;
  hipStream_t s;
  if (!dense(kv, at::kInt, 1) || !dense(ql, at::kInt, 1) || !dense(tab, at::kInt, 2) || !dense(fr, at::kInt, 1) || !to_int(a[4], &page) ||
      !to_int(a[5], &T) || T < 0)
    return not_here();
  const int64_t R = kv->size(0), W = tab->size(1), F = fr->size(0);
  if (ql->size(0) != R || tab->size(0) != R || !small({R, W, F}) || !stream_of({kv, ql, tab, fr}, &s)) return not_here();
  const at::Tensor buf = at::empty({2 * R + 2 + 2 * (int64_t)T}, kv->options());
  int32_t *p = memory<int32_t>(&buf), *kvp = memory<int32_t>(kv), *qp = memory<int32_t>(ql), *tp = memory<int32_t>(tab),
          *fp = memory<int32_t>(fr);
  if (call([&] {
        return lib.kv_plan(kvp, qp, tp, fp, p, p + 2 * R + 2, p + 2 * R + 2 + T, p + R + 1, p + 2 * R + 1, (int)R, (int)W, (int)F, page,
                           T, s);
      }) != 0)
    return not_here();
  const at::Tensor out[5] = {piece(buf, 0, R + 1), piece(buf, R + 1, R), piece(buf, 2 * R + 1, 1), piece(buf, 2 * R + 2, T),
                             piece(buf, 2 * R + 2 + T, T)};
  PyObject* r = PyTuple_New(5);
  for (int i = 0; r && i < 5; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(out[i]));
  return r;
}

// (x, positions, inv_freq, rot_heads, interleaved, gain, out)
PyObject* rope_(PyObject* const* a) {
  const at::Tensor *x = tensor(a[0]), *pos = tensor(a[1]), *f = tensor(a[2]), *o = a[6] == Py_None ? nullptr : tensor(a[6]);
  int64_t xs, ys;
  int rot_heads;
  float gain;
  hipStream_t s;
  if (!rows(x, &xs) || (x->scalar_type() != at::kFloat && x->scalar_type() != at::kBFloat16) || !dense(pos, at::kInt, 1) ||
      !dense(f, at::kDouble, 1) || !to_int(a[3], &rot_heads) || !PyBool_Check(a[4]) || !to_float(a[5], &gain) || (a[6] != Py_None && !o))
    return not_here();
  const int64_t T = x->size(0), heads = x->size(1), D = x->size(2);
  if (pos->size(0) != T || !small({T, heads, D, 2 * f->size(0)}) || !stream_of({x, pos, f, o}, &s)) return not_here();
  at::Tensor made;
  if (!o) {
    made = at::empty({T, heads, D}, x->options().dtype(at::kBFloat16));
    ys = heads * D;
  } else if (!rows(o, &ys) || o->scalar_type() != at::kBFloat16 || o->sizes() != x->sizes()) {
    return not_here();
  }
  void *y = memory(o ? o : &made), *xp = memory(x);
  const int32_t* pp = memory<int32_t>(pos);
  const double* fp = memory<double>(f);
  const int type = x->scalar_type() == at::kBFloat16 ? QGEMM_BF16 : QGEMM_F32, rot = (int)(2 * f->size(0)), inter = a[4] == Py_True;
  if (call([&] { return lib.rope(xp, type, pp, fp, y, (int)T, (int)heads, rot_heads, (int)D, rot, xs, ys, inter, gain, s); }) != 0)
    return not_here();
  return o ? Py_NewRef(a[6]) : THPVariable_Wrap(made);
}

// (k, v, slots, cache)
PyObject* kv4_store_(PyObject* const* a) {
  const at::Tensor *k = tensor(a[0]), *v = tensor(a[1]), *sl = tensor(a[2]), *c = tensor(a[3]);
  int64_t ks, vs;
  int pages, Hkv, page;
  hipStream_t s;
  if (!rows(k, &ks) || !rows(v, &vs) || k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16 || !dense(sl, at::kInt, 1) ||
      v->sizes() != k->sizes() || !cache_sizes(c, k->size(2), &pages, &Hkv, &page) || Hkv != k->size(1) || sl->size(0) != k->size(0) ||
      !small({k->size(0)}) || !stream_of({k, v, sl, c}, &s))
    return not_here();
  void *kp = memory(k), *vp = memory(v), *cp = memory(c);
  const int32_t* sp = memory<int32_t>(sl);
  const int T = (int)k->size(0), D = (int)k->size(2);
  if (call([&] { return lib.store(kp, vp, sp, cp, T, Hkv, D, ks, vs, pages, page, s); }) != 0)
    return not_here();
  Py_RETURN_NONE;
}

// (cache, slots, D) -> (k, v)
PyObject* kv4_load_(PyObject* const* a) {
  const at::Tensor *c = tensor(a[0]), *sl = tensor(a[1]);
  int D, pages, Hkv, page;
  hipStream_t s;
  if (!to_int(a[2], &D) || !dense(sl, at::kInt, 1) || !cache_sizes(c, D, &pages, &Hkv, &page) || !small({sl->size(0)}) ||
      !stream_of({c, sl}, &s))
    return not_here();
  const int64_t T = sl->size(0);
  const auto opt = c->options().dtype(at::kBFloat16);
  const at::Tensor k = at::empty({T, Hkv, D}, opt), v = at::empty({T, Hkv, D}, opt);
  void *kp = memory(&k), *vp = memory(&v), *cp = memory(c);
  const int32_t* sp = memory<int32_t>(sl);
  if (call([&] { return lib.load(cp, sp, kp, vp, (int)T, Hkv, D, pages, page, s); }) != 0)
    return not_here();
  PyObject* r = PyTuple_New(2);
  if (r) {
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(k));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(v));
  }
  return r;
}

// (q, k, v, cu, scale, out)
PyObject* attention_packed_(PyObject* const* a) {
  const at::Tensor *q = tensor(a[0]), *k = tensor(a[1]), *v = tensor(a[2]), *cu = tensor(a[3]), *o = a[5] == Py_None ? nullptr : tensor(a[5]);
  int64_t qs, ks, vs, ys;
  float scale;
  hipStream_t s;
  if (!rows(q, &qs) || !rows(k, &ks) || !rows(v, &vs) || q->scalar_type() != at::kBFloat16 || k->scalar_type() != at::kBFloat16 ||
      v->scalar_type() != at::kBFloat16 || !dense(cu, at::kInt, 1) || (a[5] != Py_None && !o))
    return not_here();
  const int64_t T = q->size(0), H = q->size(1), D = q->size(2), R = cu->size(0) - 1;
  if (k->sizes() != v->sizes() || k->size(0) != T || k->size(2) != D || R < 0 || !small({T, H, D, R, k->size(1)}) || !to_scale(a[4], D, &scale) ||
      !stream_of({q, k, v, cu, o}, &s))
    return not_here();
  at::Tensor made;
  if (!o) {
    made = at::empty({T, H, D}, q->options());
    ys = H * D;
  } else if (!rows(o, &ys) || o->scalar_type() != at::kBFloat16 || o->sizes() != q->sizes()) {
    return not_here();
  }
  void *y = memory(o ? o : &made), *qp = memory(q), *kp = memory(k), *vp = memory(v);
  const int32_t* cp = memory<int32_t>(cu);
  const int Hkv = (int)k->size(1);
  if (call([&] { return lib.packed(qp, kp, vp, cp, y, (int)T, (int)R, (int)H, Hkv, (int)D, qs, ks, vs, ys, scale, s); }) != 0)
    return not_here();
  return o ? Py_NewRef(a[5]) : THPVariable_Wrap(made);
}

// (q, cache, block_table, kv_len, cu_q, scale, out)
PyObject* attention_kv4_(PyObject* const* a) {
  const at::Tensor *q = tensor(a[0]), *c = tensor(a[1]), *tab = tensor(a[2]), *kv = tensor(a[3]);
  const at::Tensor *cu = a[4] == Py_None ? nullptr : tensor(a[4]), *o = a[6] == Py_None ? nullptr : tensor(a[6]);
  int64_t qs;
  int pages, Hkv, page;
  float scale;
  hipStream_t s;
  if (!rows(q, &qs) || q->scalar_type() != at::kBFloat16 || !dense(tab, at::kInt, 2) || !dense(kv, at::kInt, 1) || (a[4] != Py_None && !cu) ||
      (a[6] != Py_None && !o))
    return not_here();
  const int64_t T = q->size(0), H = q->size(1), D = q->size(2), R = tab->size(0), W = tab->size(1);
  if (!cache_sizes(c, D, &pages, &Hkv, &page) || kv->size(0) != R || (cu ? !dense(cu, at::kInt, 1) || cu->size(0) != R + 1 : T != R) ||
      !small({T, H, R, W}) || !to_scale(a[5], D, &scale) || !stream_of({q, c, tab, kv, cu, o}, &s))
    return not_here();
  if (o && (!dense(o, at::kBFloat16, 3) || o->sizes() != q->sizes())) return not_here();
  int64_t need = 0;
  if (lib.kv4_workspace((int)T, (int)R, (int)H, Hkv, (int)D, (int)W, page, &need) != 0) return not_here();
  at::Tensor made;
  if (!o) made = at::empty({T, H, D}, q->options());
  // of the call's own: torch's allocator keeps it from other streams, and inside a capture it is the graph's
  const at::Tensor ws = at::empty({need}, q->options().dtype(at::kByte));
  void *y = memory(o ? o : &made), *qp = memory(q), *cp = memory(c), *wp = memory(&ws);
  const int32_t *tp = memory<int32_t>(tab), *kp = memory<int32_t>(kv), *up = memory<int32_t>(cu);
  if (call([&] {
        return lib.kv4(qp, cp, tp, kp, up, y, wp, need, (int)T, (int)R, (int)H, Hkv, (int)D, (int)W, pages, page, qs, scale, s);
      }) != 0)
    return not_here();
  return o ? Py_NewRef(a[6]) : THPVariable_Wrap(made);
}

// C++ exceptions (an allocation that fails, a tensor without memory) end here: Python's way meets and reports them.
template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N || !lib.raw_stream) return not_here();
  try {
    return F(args);
  } catch (...) {
    return not_here();
  }
}

// (raw_stream, kv_plan, rope, store, load, packed, kv4, kv4_workspace): a callable and addresses
PyObject* bind(PyObject*, PyObject* args) {
  PyObject* stream;
  unsigned long long p[7];
  if (!PyArg_ParseTuple(args, "OKKKKKKK", &stream, p, p + 1, p + 2, p + 3, p + 4, p + 5, p + 6)) return nullptr;
  auto at = [&](int i, auto*& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>((uintptr_t)p[i]); };
  at(0, lib.kv_plan);
  at(1, lib.rope);
  at(2, lib.store);
  at(3, lib.load);
  at(4, lib.packed);
  at(5, lib.kv4);
  at(6, lib.kv4_workspace);
  Py_INCREF(stream);
  Py_XSETREF(lib.raw_stream, stream);
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), Py_ssize_t N>
constexpr PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F, N>));
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"kv_plan", fast<kv_plan_, 6>(), METH_FASTCALL, nullptr},
    {"rope", fast<rope_, 7>(), METH_FASTCALL, nullptr},
    {"kv4_store", fast<kv4_store_, 4>(), METH_FASTCALL, nullptr},
    {"kv4_load", fast<kv4_load_, 3>(), METH_FASTCALL, nullptr},
    {"attention_packed", fast<attention_packed_, 6>(), METH_FASTCALL, nullptr},
    {"attention_kv4", fast<attention_kv4_, 7>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// What this was built from and against: the library's header and torch. The Python side compares both.
#ifndef QGEMM_HEADER
#define QGEMM_HEADER ""
#endif
#ifndef QGEMM_TORCH
#define QGEMM_TORCH ""
#endif

PyMODINIT_FUNC PyInit__binding(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && (PyModule_AddStringConstant(m, "header", QGEMM_HEADER) < 0 || PyModule_AddStringConstant(m, "torch", QGEMM_TORCH) < 0)) Py_CLEAR(m);
  return m;
}
