// The per-layer calls of the binding, marshalled natively: a decode step makes one call per layer, and in
// Python the checks and pointers of its tensors cost 2 us and more of it (both sides in binding.py).
//
// What a call does is what binding.py does for it - tensor type, device, contiguity and dtype checked, then the
// C entry point - for plain torch.Tensor arguments that pass and structures of binding.py's own classes; anything
// else returns None, and binding.py's own path takes the call and raises what it always raised.  Nothing is kept
// between calls but the entry points' addresses and the two classes, which bind() hands over once.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <c10/core/impl/VirtualGuardImpl.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/vidkv.h"

namespace {

decltype(&vidkv_decode_attention) g_decode;
decltype(&vidkv_decode_attention_noalloc) g_decode_noalloc;
decltype(&vidkv_flush_residual) g_flush;
decltype(&vidkv_rotary_apply) g_rotary;
decltype(&vidkv_cache8_write) g_write8;
decltype(&vidkv_cache8_read) g_read8;
decltype(&vidkv_cache8_attention) g_attend8;
PyTypeObject* g_params_type;         // binding.VidkvParams
PyTypeObject* g_side_type;           // binding.VidkvSideStream
PyTypeObject* g_rotary_type;         // binding.VidkvRotary
PyTypeObject* g_cache8_type;         // binding.VidkvCache8

// Memory of a ctypes structure of class `type` and exactly `size` bytes (ctypes refuses other objects, whatever
// buffer they have).
class Struct {
 public:
  Struct(PyObject* o, PyTypeObject* type, size_t size) {
    if (!PyObject_TypeCheck(o, type)) return;
    if (PyObject_GetBuffer(o, &view_, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return; }
    held_ = true;
    if ((size_t)view_.len == size) ptr_ = view_.buf;
  }
  ~Struct() { if (held_) PyBuffer_Release(&view_); }
  Struct(const Struct&) = delete;
  const void* get() const { return ptr_; }

 private:
  Py_buffer view_;
  bool held_ = false;
  const void* ptr_ = nullptr;
};

// Data pointer (and size) of a contiguous device tensor of type t; None gives NULL where that is allowed.
bool tensor(PyObject* o, c10::ScalarType t, bool none_ok, void** ptr, size_t* bytes = nullptr) {
  *ptr = nullptr;
  if (o == Py_None) return none_ok;
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (!x.defined() || !x.has_storage() || !x.is_cuda() || x.scalar_type() != t || !x.is_contiguous()) return false;
  *ptr = x.data_ptr();
  if (bytes) *bytes = x.nbytes();
  return true;
}

bool integer(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &over);
  if (over || x < INT32_MIN || x > INT32_MAX) return false;
  *v = (int32_t)x;
  return true;
}

bool handle(PyObject* o, void** v) {
  if (!PyLong_CheckExact(o)) return false;
  *v = PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}

// The stream's handle, asked for when the other arguments have passed: fn(stream).  -1: a Python error is set.
int stream_handle(PyObject* fn, PyObject* stream, void** v) {
  PyObject* h = PyObject_CallFunctionObjArgs(fn, stream, nullptr);
  if (!h) return -1;
  const bool ok = handle(h, v);
  Py_DECREF(h);
  return ok;
}

// f() may throw (a tensor without data): then the Python path takes the call
template <class F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (params, layer, q, packed_K, packed_V, K_tail, V_tail, tail_capacity, tail_len, out, workspace, stream function, stream, side or None)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 14 || !g_decode) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    int32_t layer, cap;
    void *q, *pk, *pv, *kt, *vt, *tl, *out, *ws, *stream;
    size_t wsb = 0;
    if (!integer(a[1], &layer) || !tensor(a[2], at::kHalf, true, &q) || !tensor(a[3], at::kByte, true, &pk) ||
        !tensor(a[4], at::kByte, true, &pv) || !tensor(a[5], at::kHalf, true, &kt) || !tensor(a[6], at::kHalf, true, &vt) ||
        !integer(a[7], &cap) || !tensor(a[8], at::kInt, true, &tl) || !tensor(a[9], at::kHalf, true, &out) ||
        !tensor(a[10], at::kByte, false, &ws, &wsb))
      Py_RETURN_NONE;
    const Struct p(a[0], g_params_type, sizeof(vidkv_params));
    if (!p.get()) Py_RETURN_NONE;
    vidkv_side_stream side;
    const bool has_side = a[13] != Py_None;
    if (has_side) {
      const Struct s(a[13], g_side_type, sizeof(side));
      if (!s.get()) Py_RETURN_NONE;
      side = *static_cast<const vidkv_side_stream*>(s.get());
    }
    const int got = stream_handle(a[11], a[12], &stream);
    if (got < 0) return nullptr;
    if (!got) Py_RETURN_NONE;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = g_decode(static_cast<const vidkv_params*>(p.get()), layer, q, pk, pv, kt, vt, cap, static_cast<const int32_t*>(tl),
                  out, ws, wsb, stream, has_side ? &side : nullptr);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  });
}

// (params, layer, q, packed_K, packed_V, K_tail, V_tail, tail_capacity, tail_len, out, stream function, stream)
PyObject* decode_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 12 || !g_decode_noalloc) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    int32_t layer, cap;
    void *q, *pk, *pv, *kt, *vt, *tl, *out, *stream;
    if (!integer(a[1], &layer) || !tensor(a[2], at::kHalf, true, &q) || !tensor(a[3], at::kByte, true, &pk) ||
        !tensor(a[4], at::kByte, true, &pv) || !tensor(a[5], at::kHalf, true, &kt) || !tensor(a[6], at::kHalf, true, &vt) ||
        !integer(a[7], &cap) || !tensor(a[8], at::kInt, true, &tl) || !tensor(a[9], at::kHalf, true, &out))
      Py_RETURN_NONE;
    const Struct p(a[0], g_params_type, sizeof(vidkv_params));
    if (!p.get()) Py_RETURN_NONE;
    const int got = stream_handle(a[10], a[11], &stream);
    if (got < 0) return nullptr;
    if (!got) Py_RETURN_NONE;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = g_decode_noalloc(static_cast<const vidkv_params*>(p.get()), layer, q, pk, pv, kt, vt, cap,
                          static_cast<const int32_t*>(tl), out, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  });
}

// (params, layer, K_tail, V_tail, tail_capacity, n_flush, packed_K, packed_V, stream function, stream)
PyObject* flush(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 10 || !g_flush) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    int32_t layer, cap, nf;
    void *kt, *vt, *pk, *pv, *stream;
    size_t kb = 0, vb = 0;
    if (!integer(a[1], &layer) || !tensor(a[2], at::kHalf, true, &kt) || !tensor(a[3], at::kHalf, true, &vt) ||
        !integer(a[4], &cap) || !integer(a[5], &nf) || !tensor(a[6], at::kByte, false, &pk, &kb) ||
        !tensor(a[7], at::kByte, false, &pv, &vb))
      Py_RETURN_NONE;
    const Struct p(a[0], g_params_type, sizeof(vidkv_params));
    if (!p.get()) Py_RETURN_NONE;
    const int got = stream_handle(a[8], a[9], &stream);
    if (got < 0) return nullptr;
    if (!got) Py_RETURN_NONE;
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = g_flush(static_cast<const vidkv_params*>(p.get()), layer, kt, vt, cap, nf, pk, kb, pv, vb, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  });
}

// (addresses of vidkv_decode_attention, vidkv_decode_attention_noalloc, vidkv_flush_residual; the classes of
// vidkv_params and vidkv_side_stream)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[3];
  if (n != 5 || !handle(a[0], &f[0]) || !handle(a[1], &f[1]) || !handle(a[2], &f[2]) || !PyType_Check(a[3]) ||
      !PyType_Check(a[4])) {
    PyErr_SetString(PyExc_TypeError, "bind: three addresses and two classes");
    return nullptr;
  }
  Py_INCREF(a[3]);                                     // (kept, with the module, for as long as the process)
  Py_INCREF(a[4]);
  g_params_type = reinterpret_cast<PyTypeObject*>(a[3]);
  g_side_type = reinterpret_cast<PyTypeObject*>(a[4]);
  g_decode = reinterpret_cast<decltype(g_decode)>(f[0]);
  g_decode_noalloc = reinterpret_cast<decltype(g_decode_noalloc)>(f[1]);
  g_flush = reinterpret_cast<decltype(g_flush)>(f[2]);
  Py_RETURN_NONE;
}

// ---- rotary positions and the 8-bit cache ----
bool boolean(PyObject* o, int32_t* v) {
  if (!PyBool_Check(o)) return false;
  *v = o == Py_True;
  return true;
}

// A plain device tensor on the current device `dev`.
const at::Tensor* here(PyObject* o, int dev) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& x = THPVariable_Unpack(o);
  return x.defined() && x.has_storage() && x.is_cuda() && x.device().index() == dev ? &x : nullptr;
}

// Data pointer (and size) of a contiguous one of type t and, if given, a shape; None gives NULL where that is allowed.
bool tensor_here(PyObject* o, int dev, c10::ScalarType t, std::initializer_list<int64_t> shape, bool none_ok, void** ptr,
                 size_t* bytes = nullptr) {
  *ptr = nullptr;
  if (o == Py_None) return none_ok;
  const at::Tensor* x = here(o, dev);
  if (!x || x->scalar_type() != t || !x->is_contiguous()) return false;
  if (shape.size() && !x->sizes().equals(at::IntArrayRef(shape))) return false;
  *ptr = x->data_ptr();
  if (bytes) *bytes = x->nbytes();
  return true;
}

// binding.py's _view: [B, heads, n, channels] of any strides, channels next to each other; what is written to must not
// overlap itself.
bool view(PyObject* o, int dev, int64_t B, int64_t h, int64_t n, int64_t d, bool written, vidkv_view* v) {
  const at::Tensor* x = here(o, dev);
  if (!x || x->dim() != 4) return false;
  const auto size = x->sizes(), stride = x->strides();
  if (size[0] != B || size[1] != h || size[2] != n || size[3] != d || stride[3] != 1) return false;
  switch (x->scalar_type()) {
    case at::kHalf: v->dtype = VIDKV_F16; break;
    case at::kBFloat16: v->dtype = VIDKV_BF16; break;
    case at::kFloat: v->dtype = VIDKV_F32; break;
    default: return false;
  }
  int64_t st[3], order[3] = {0, 1, 2};
  for (int i = 0; i < 3; ++i) st[i] = size[i] > 1 ? stride[i] : 0;
  if (written) {
    std::sort(order, order + 3, [&](int64_t a, int64_t b) { return st[a] < st[b]; });
    int64_t extent = d;
    for (int64_t i : order) {
      if (size[i] <= 1) continue;
      if (st[i] < extent) return false;
      extent += st[i] * (size[i] - 1);
    }
  }
  v->data = x->data_ptr();
  v->stride_batch = st[0]; v->stride_head = st[1]; v->stride_token = st[2];
  return true;
}

// Heads and tokens of a 4-dimensional tensor, or false.
bool dims(PyObject* o, int64_t* B, int64_t* h, int64_t* n) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (!x.defined() || x.dim() != 4) return false;
  *B = x.size(0); *h = x.size(1); *n = x.size(2);
  return *B > 0 && *h > 0 && *n > 0 && *B <= INT32_MAX && *h <= INT32_MAX && *n <= INT32_MAX;
}

int current_device() { return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index(); }

// What is left of a call when its arguments have passed: the stream, and f(stream) without the interpreter.
template <class F>
PyObject* enqueue(PyObject* fn, PyObject* stream, F f) {
  void* s;
  const int got = stream_handle(fn, stream, &s);
  if (got < 0) return nullptr;
  if (!got) Py_RETURN_NONE;
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = f(s);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(st);
}

// (rotary, positions, q, q_out, k, k_out, inverse, stream function, stream)
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9 || !g_rotary) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const Struct r(a[0], g_rotary_type, sizeof(vidkv_rotary));
    const auto* rot = static_cast<const vidkv_rotary*>(r.get());
    const bool q = a[2] != Py_None, k = a[4] != Py_None;
    int64_t B = 0, t = 0, hq = 0, hk = 0, Bk = 0, tk = 0;
    int32_t inverse;
    void* pos;
    vidkv_view v[4];
    if (!rot || (!q && !k) || !boolean(a[6], &inverse)) Py_RETURN_NONE;
    if ((q && !dims(a[2], &B, &hq, &t)) || (k && !dims(a[4], &Bk, &hk, &tk))) Py_RETURN_NONE;
    if (!q) { B = Bk; t = tk; }
    const int dev = current_device();
    const int64_t d = rot->head_dim;
    if ((q && (!view(a[2], dev, B, hq, t, d, false, &v[0]) || !view(a[3], dev, B, hq, t, d, true, &v[1]))) ||
        (k && (!view(a[4], dev, B, hk, t, d, false, &v[2]) || !view(a[5], dev, B, hk, t, d, true, &v[3]))) ||
        !tensor_here(a[1], dev, at::kInt, {rot->n_axes, B, t}, false, &pos))
      Py_RETURN_NONE;
    return enqueue(a[7], a[8], [&](void* s) {
      return g_rotary(rot, inverse, (int32_t)B, (int32_t)t, static_cast<const int32_t*>(pos), (int32_t)hq, q ? &v[0] : nullptr,
                      q ? &v[1] : nullptr, (int32_t)hk, k ? &v[2] : nullptr, k ? &v[3] : nullptr, s);
    });
  });
}

// (cache8, layer, cache, K, V, start, count, rotary, positions, stream function, stream)
PyObject* write8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_write8) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const Struct ps(a[0], g_cache8_type, sizeof(vidkv_cache8));
    const auto* p = static_cast<const vidkv_cache8*>(ps.get());
    int32_t layer;
    int64_t B, h, t;
    void *cache, *start, *count, *pos;
    size_t bytes = 0;
    vidkv_view K, V;
    if (!p || !integer(a[1], &layer) || !dims(a[3], &B, &h, &t)) Py_RETURN_NONE;
    const bool turn = a[7] != Py_None;
    const Struct rs(turn ? a[7] : a[0], turn ? g_rotary_type : g_cache8_type, turn ? sizeof(vidkv_rotary) : sizeof(vidkv_cache8));
    const auto* rot = turn ? static_cast<const vidkv_rotary*>(rs.get()) : nullptr;
    if (turn != (a[8] != Py_None) || (turn && !rot)) Py_RETURN_NONE;
    const int dev = current_device();
    if (!view(a[3], dev, p->batch, p->n_kv_heads, t, 128, false, &K) ||
        !view(a[4], dev, p->batch, p->n_kv_heads, t, 128, false, &V) ||
        !tensor_here(a[5], dev, at::kInt, {p->batch}, false, &start) || !tensor_here(a[6], dev, at::kInt, {p->batch}, true, &count) ||
        !tensor_here(a[8], dev, at::kInt, {turn ? rot->n_axes : 0, p->batch, t}, !turn, &pos) ||
        !tensor_here(a[2], dev, at::kByte, {}, false, &cache, &bytes))
      Py_RETURN_NONE;
    return enqueue(a[9], a[10], [&](void* s) {
      return g_write8(p, layer, (int32_t)t, &K, &V, static_cast<const int32_t*>(start), static_cast<const int32_t*>(count), rot,
                      static_cast<const int32_t*>(pos), cache, bytes, s);
    });
  });
}

// (cache8, layer, cache, start, K, V, stream function, stream)
PyObject* read8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !g_read8) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const Struct ps(a[0], g_cache8_type, sizeof(vidkv_cache8));
    const auto* p = static_cast<const vidkv_cache8*>(ps.get());
    const bool k = a[4] != Py_None, v = a[5] != Py_None;
    int32_t layer;
    int64_t B, h, t;
    void *cache, *start;
    size_t bytes = 0;
    vidkv_view K, V;
    if (!p || (!k && !v) || !integer(a[1], &layer) || !dims(k ? a[4] : a[5], &B, &h, &t)) Py_RETURN_NONE;
    const int dev = current_device();
    if ((k && !view(a[4], dev, p->batch, p->n_kv_heads, t, 128, true, &K)) ||
        (v && !view(a[5], dev, p->batch, p->n_kv_heads, t, 128, true, &V)) ||
        !tensor_here(a[3], dev, at::kInt, {p->batch}, false, &start) || !tensor_here(a[2], dev, at::kByte, {}, false, &cache, &bytes))
      Py_RETURN_NONE;
    return enqueue(a[6], a[7], [&](void* s) {
      return g_read8(p, layer, (int32_t)t, static_cast<const int32_t*>(start), cache, bytes, k ? &K : nullptr, v ? &V : nullptr, s);
    });
  });
}

// (cache8, layer, cache, q, out, length, workspace, q_count, causal, stream function, stream)
PyObject* attend8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !g_attend8) Py_RETURN_NONE;
  return guarded([&]() -> PyObject* {
    const Struct ps(a[0], g_cache8_type, sizeof(vidkv_cache8));
    const auto* p = static_cast<const vidkv_cache8*>(ps.get());
    int32_t layer, causal;
    int64_t B, h, t;
    void *cache, *length, *count, *ws;
    size_t bytes = 0, wsb = 0;
    vidkv_view q, out;
    if (!p || !integer(a[1], &layer) || !boolean(a[8], &causal) || !dims(a[3], &B, &h, &t)) Py_RETURN_NONE;
    const int dev = current_device();
    if (!view(a[3], dev, p->batch, p->n_q_heads, t, 128, false, &q) || !view(a[4], dev, p->batch, p->n_q_heads, t, 128, true, &out) ||
        !tensor_here(a[2], dev, at::kByte, {}, false, &cache, &bytes) ||
        !tensor_here(a[5], dev, at::kInt, {p->batch}, false, &length) || !tensor_here(a[7], dev, at::kInt, {p->batch}, true, &count) ||
        !tensor_here(a[6], dev, at::kByte, {}, false, &ws, &wsb))
      Py_RETURN_NONE;
    return enqueue(a[9], a[10], [&](void* s) {
      return g_attend8(p, layer, (int32_t)t, causal, &q, cache, bytes, static_cast<const int32_t*>(length),
                       static_cast<const int32_t*>(count), &out, ws, wsb, s);
    });
  });
}

// (addresses of vidkv_rotary_apply, vidkv_cache8_write, _read, _attention; the classes of vidkv_rotary and vidkv_cache8)
PyObject* bind8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[4];
  if (n != 6 || !handle(a[0], &f[0]) || !handle(a[1], &f[1]) || !handle(a[2], &f[2]) || !handle(a[3], &f[3]) ||
      !PyType_Check(a[4]) || !PyType_Check(a[5])) {
    PyErr_SetString(PyExc_TypeError, "bind8: four addresses and two classes");
    return nullptr;
  }
  Py_INCREF(a[4]);
  Py_INCREF(a[5]);
  g_rotary_type = reinterpret_cast<PyTypeObject*>(a[4]);
  g_cache8_type = reinterpret_cast<PyTypeObject*>(a[5]);
  g_rotary = reinterpret_cast<decltype(g_rotary)>(f[0]);
  g_write8 = reinterpret_cast<decltype(g_write8)>(f[1]);
  g_read8 = reinterpret_cast<decltype(g_read8)>(f[2]);
  g_attend8 = reinterpret_cast<decltype(g_attend8)>(f[3]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"decode_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode)), METH_FASTCALL, nullptr},
    {"decode_attention_noalloc", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode_noalloc)), METH_FASTCALL, nullptr},
    {"flush_residual", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(flush)), METH_FASTCALL, nullptr},
    {"rotary", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rotary)), METH_FASTCALL, nullptr},
    {"cache8_write", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(write8)), METH_FASTCALL, nullptr},
    {"cache8_read", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(read8)), METH_FASTCALL, nullptr},
    {"cache8_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attend8)), METH_FASTCALL, nullptr},
    {"bind8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind8)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "vidkv_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and the torch that this was compiled against (binding.py uses it with no other)
PyMODINIT_FUNC PyInit_vidkv_marshal(void) {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", VIDKV_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
