// Argument marshalling of the decode step as native code.  A step of few sequences takes the GPU less time than the same checks
// took in Python: the smallest step 8.1 us a call, 4.5 from here, of which the launch itself is 2.6; with a workspace from
// torch.empty 9.8, from the allocator here 5 (one sequence, 4 KV heads, W = 512, where the kernel is the bound: 9.8 -> 9.15).
//
// decode_step(q, k_new, v_new, pos, k_ring, v_ring, state, gamma_swa, gamma_rla, softmax_scale, rms_eps, out, feature_map)
// returns the output; None when the arguments are not plainly what the step takes (the caller's Python path then converts
// or raises as it always did), and a status as an int when the library refuses the call.  The calls over packed rings and trees of
// drafted tokens are handed over in the same way (ring_pack and the others below): the smallest of them 8.3 us a call from Python.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <ATen/ATen.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <string.h>

#include "rattn.h"

namespace {

typedef rattn_status (*step_fn)(const rattn_decode_params*, const void*, const void*, const void*, const int32_t*, void*, void*,
                                float*, const float*, const float*, void*, void*, size_t, void*);
typedef rattn_status (*bytes_fn)(const rattn_decode_params*, size_t*);
step_fn g_step = nullptr;
bytes_fn g_bytes = nullptr;

// bind(address of rattn_decode_step_ws, address of rattn_decode_workspace_bytes) of the loaded library
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) return PyErr_Format(PyExc_TypeError, "bind takes two addresses");
  g_step = (step_fn)PyLong_AsVoidPtr(args[0]);
  g_bytes = (bytes_fn)PyLong_AsVoidPtr(args[1]);
  if (PyErr_Occurred()) return nullptr;
  Py_RETURN_NONE;
}

// a plain tensor on device `dev`, contiguous, of type `dt` and `nd` dimensions
bool plain(const at::Tensor& t, int dev, at::ScalarType dt, int nd) {
  return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.get_device() == dev && t.scalar_type() == dt && t.dim() == nd &&
         t.is_contiguous() && t.has_storage();
}
bool shaped(const at::Tensor& t, int64_t a, int64_t b, int64_t c) { return t.size(0) == a && t.size(1) == b && t.size(2) == c; }

// The interpreter lock is free while one of these lives, as in a ctypes call
struct NoGil {
  PyThreadState* state = PyEval_SaveThread();
  ~NoGil() { PyEval_RestoreThread(state); }
};

PyObject* step(PyObject* const* args) {
  const at::Tensor* t[7];
  for (int i = 0; i < 7; ++i) {
    if (!THPVariable_CheckExact(args[i])) Py_RETURN_NONE;
    t[i] = &THPVariable_Unpack(args[i]);
  }
  const at::Tensor &q = *t[0], &kn = *t[1], &vn = *t[2], &pos = *t[3], &kr = *t[4], &vr = *t[5], &state = *t[6];
  const at::ScalarType dt = q.scalar_type();
  const int dev = q.is_cuda() ? q.get_device() : -1;
  if ((dt != at::kFloat && dt != at::kBFloat16) || dev < 0 || dev != c10::hip::current_device()) Py_RETURN_NONE;
  if (!plain(q, dev, dt, 3) || !plain(kn, dev, dt, 3) || !plain(vn, dev, dt, 3) || !plain(pos, dev, at::kInt, 1) ||
      !plain(kr, dev, dt, 4) || !plain(vr, dev, dt, 4) || !plain(state, dev, at::kFloat, 4))
    Py_RETURN_NONE;
  const int64_t N = q.size(0), Hq = q.size(1), D = q.size(2), Hkv = kr.size(1), W = kr.size(2);
  if (!shaped(kn, N, Hkv, D) || !shaped(vn, N, Hkv, D) || pos.size(0) != N || !shaped(kr, N, Hkv, W) || kr.size(3) != D ||
      !shaped(vr, N, Hkv, W) || vr.size(3) != D || !shaped(state, N, Hkv, D) || state.size(3) != D)
    Py_RETURN_NONE;
  if (N > INT32_MAX || Hq > INT32_MAX || Hkv > INT32_MAX || D > INT32_MAX || W > INT32_MAX) Py_RETURN_NONE;
  const float* gain[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i) {
    PyObject* a = args[7 + i];
    if (a == Py_None) continue;
    if (!THPVariable_CheckExact(a)) Py_RETURN_NONE;
    const at::Tensor& g = THPVariable_Unpack(a);
    if (!plain(g, dev, at::kFloat, 2) || g.size(0) != Hq || g.size(1) != D) Py_RETURN_NONE;
    gain[i] = (const float*)g.data_ptr();
  }
  if (!PyFloat_CheckExact(args[9]) || !PyFloat_CheckExact(args[10]) || !PyUnicode_CheckExact(args[12])) Py_RETURN_NONE;
  rattn_decode_params p;
  p.N = (int32_t)N; p.Hq = (int32_t)Hq; p.Hkv = (int32_t)Hkv; p.D = (int32_t)D; p.window = (int32_t)W;
  p.dtype = dt == at::kFloat ? RATTN_F32 : RATTN_BF16;
  p.softmax_scale = (float)PyFloat_AS_DOUBLE(args[9]);
  p.rms_eps = (float)PyFloat_AS_DOUBLE(args[10]);
  if (PyUnicode_CompareWithASCIIString(args[12], "softmax") == 0) p.feature_map = RATTN_PHI_SOFTMAX;
  else if (PyUnicode_CompareWithASCIIString(args[12], "relu") == 0) p.feature_map = RATTN_PHI_RELU;
  else if (PyUnicode_CompareWithASCIIString(args[12], "identity") == 0) p.feature_map = RATTN_PHI_IDENTITY;
  else Py_RETURN_NONE;
  // The result as an object ahead of the step: behind it nothing may fail, since a caller that is told so would step again and
  // fold the evicted token into the state twice
  THPObjectPtr result;
  void* o;
  if (args[11] == Py_None) {
    at::Tensor fresh = at::empty_like(q);
    o = fresh.data_ptr();
    result = THPVariable_Wrap(std::move(fresh));
    if (!result) return nullptr;
  } else {
    if (!THPVariable_CheckExact(args[11])) Py_RETURN_NONE;
    const at::Tensor& out = THPVariable_Unpack(args[11]);   // the step writes N Hq D elements of it, whatever its shape
    if (!plain(out, dev, dt, out.dim()) || out.numel() < q.numel()) Py_RETURN_NONE;
    o = out.data_ptr();
    Py_INCREF(args[11]);
    result = args[11];
  }
  const void *qp = q.data_ptr(), *knp = kn.data_ptr(), *vnp = vn.data_ptr();
  void *posp = pos.data_ptr(), *krp = kr.data_ptr(), *vrp = vr.data_ptr(), *sp = state.data_ptr();
  rattn_status s;
  {
    NoGil others_run;   // the allocator may wait for the device, a launch for room in the stream's queue
    size_t bytes = 0;
    s = g_bytes(&p, &bytes);
    if (s == RATTN_OK) {
      c10::DataPtr ws;   // from the caching allocator, on the current stream: back in its pool when the step is enqueued
      if (bytes > 0) ws = c10::hip::HIPCachingAllocator::get()->allocate(bytes);
      void* stream = (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)dev).stream();
      s = g_step(&p, qp, knp, vnp, (const int32_t*)posp, krp, vrp, (float*)sp, gain[0], gain[1], o, ws.get(), bytes, stream);
    }
  }
  return s == RATTN_OK ? result.release() : PyLong_FromLong(s);
}

PyObject* decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 13 || !g_step) return PyErr_Format(PyExc_TypeError, "decode_step takes 13 arguments, after bind");
  try {
    return step(args);
  } catch (const std::exception&) {   // (an allocation that failed, a tensor without memory: as the Python path says it)
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
}

// ---- packed rings and trees of drafted tokens
struct CacheFns {
  rattn_status (*pack)(const rattn_decode_params*, const void*, const void*, void*, void*, void*, void*, void*);
  rattn_status (*unpack)(const rattn_decode_params*, const void*, const void*, const void*, const void*, void*, void*, void*);
  bytes_fn packed_bytes;
  rattn_status (*packed_step)(const rattn_decode_params*, const void*, const void*, const void*, const int32_t*, void*, void*, void*, void*,
                              float*, const float*, const float*, void*, void*, size_t, void*);
  rattn_status (*tree_bytes)(const rattn_tree_params*, int32_t, size_t*);
  rattn_status (*tree_step)(const rattn_tree_params*, const void*, const void*, const void*, const int32_t*, const int32_t*, const int32_t*,
                            const void*, const void*, const void*, const void*, const float*, const float*, const float*, void*, void*,
                            size_t, void*);
  rattn_status (*tree_commit)(const rattn_tree_params*, const void*, const void*, const int32_t*, const int32_t*, const int32_t*, void*,
                              void*, void*, void*, float*, void*);
};
CacheFns g_cache = {};

// bind_cache(addresses of the loaded library's functions, in the order of CacheFns)
PyObject* bind_cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* f[7];
  if (n != 7) return PyErr_Format(PyExc_TypeError, "bind_cache takes seven addresses");
  for (int i = 0; i < 7; ++i) f[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  static_assert(sizeof(f) == sizeof(g_cache), "seven functions");
  memcpy(&g_cache, f, sizeof(f));
  Py_RETURN_NONE;
}

constexpr at::ScalarType CODES = at::ScalarType::Float8_e4m3fn, SCALES = at::ScalarType::Float8_e8m0fnu;
const at::Tensor* tensor(PyObject* a) { return THPVariable_CheckExact(a) ? &THPVariable_Unpack(a) : nullptr; }
bool plain4(const at::Tensor* t, int dev, at::ScalarType dt, int64_t a, int64_t b, int64_t c, int64_t d) {
  return t && plain(*t, dev, dt, 4) && shaped(*t, a, b, c) && t->size(3) == d;
}
bool ints(const at::Tensor* t, int dev, int64_t n) { return t && plain(*t, dev, at::kInt, 1) && t->size(0) == n; }
// a contiguous tensor of `dt` on the current device; -1 otherwise
int device_of(const at::Tensor* t, at::ScalarType& dt) {
  if (!t || !t->defined() || !t->is_cuda()) return -1;
  dt = t->scalar_type();
  const int dev = t->get_device();
  return (dt == at::kFloat || dt == at::kBFloat16) && dev == c10::hip::current_device() ? dev : -1;
}
bool small(std::initializer_list<int64_t> sizes) {
  for (int64_t x : sizes)
    if (x > INT32_MAX) return false;
  return true;
}
int type_of(at::ScalarType dt) { return dt == at::kFloat ? RATTN_F32 : RATTN_BF16; }
bool map_of(PyObject* a, int32_t& phi) {
  if (!PyUnicode_CheckExact(a)) return false;
  const char* names[] = {"softmax", "relu", "identity"};
  for (phi = 0; phi < 3; ++phi)
    if (PyUnicode_CompareWithASCIIString(a, names[phi]) == 0) return true;
  return false;
}
bool gain_of(PyObject* a, int dev, int64_t Hq, int64_t D, const float*& p) {
  p = nullptr;
  if (a == Py_None) return true;
  const at::Tensor* g = tensor(a);
  if (!g || !plain(*g, dev, at::kFloat, 2) || g->size(0) != Hq || g->size(1) != D) return false;
  p = (const float*)g->data_ptr();
  return true;
}
// the output: the caller's, of q's type, shape and place, or a new one
bool output(PyObject* a, const at::Tensor& q, int dev, bool zero, THPObjectPtr& result, void*& o) {
  if (a == Py_None) {
    at::Tensor fresh = zero ? at::zeros_like(q) : at::empty_like(q);
    o = fresh.data_ptr();
    result = THPVariable_Wrap(std::move(fresh));
    return (bool)result;
  }
  const at::Tensor* t = tensor(a);
  if (!t || !plain(*t, dev, q.scalar_type(), (int)q.dim()) || t->sizes() != q.sizes()) return false;
  o = t->data_ptr();
  Py_INCREF(a);
  result = a;
  return true;
}
void* stream_of(int dev) { return (void*)c10::hip::getCurrentHIPStream((c10::DeviceIndex)dev).stream(); }

// ring_pack(k_ring, v_ring, out): the four packed tensors, `out` itself where it is given
PyObject* do_pack(PyObject* const* args) {
  at::ScalarType dt;
  const at::Tensor *k = tensor(args[0]), *v = tensor(args[1]);
  const int dev = device_of(k, dt);
  if (dev < 0 || k->dim() != 4) Py_RETURN_NONE;
  const int64_t N = k->size(0), H = k->size(1), W = k->size(2), D = k->size(3);
  if (!plain4(k, dev, dt, N, H, W, D) || !plain4(v, dev, dt, N, H, W, D) || !small({N, H, W, D})) Py_RETURN_NONE;
  THPObjectPtr result;
  if (args[2] == Py_None) {
    result = PyTuple_New(4);
    if (!result) return nullptr;
    for (int i = 0; i < 4; ++i) {
      PyObject* t = THPVariable_Wrap(at::empty({N, H, W, i & 1 ? D / 32 : D}, k->options().dtype(i & 1 ? SCALES : CODES)));
      if (!t) return nullptr;
      PyTuple_SET_ITEM(result.get(), i, t);
    }
  } else {
    if (!PyTuple_CheckExact(args[2]) || PyTuple_GET_SIZE(args[2]) != 4) Py_RETURN_NONE;
    Py_INCREF(args[2]);
    result = args[2];
  }
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    const at::Tensor* t = tensor(PyTuple_GET_ITEM(result.get(), i));
    if (!plain4(t, dev, i & 1 ? SCALES : CODES, N, H, W, i & 1 ? D / 32 : D)) Py_RETURN_NONE;
    p[i] = t->data_ptr();
  }
  const rattn_decode_params par = {(int32_t)N, (int32_t)H, (int32_t)H, (int32_t)D, (int32_t)W, type_of(dt), 1.f, 1e-6f, 0};
  const void *kp = k->data_ptr(), *vp = v->data_ptr();
  rattn_status s;
  { NoGil others_run; s = g_cache.pack(&par, kp, vp, p[0], p[1], p[2], p[3], stream_of(dev)); }
  return s == RATTN_OK ? result.release() : PyLong_FromLong(s);
}

// ring_unpack(k_codes, k_scale, v_codes, v_scale, out): `out`, a tuple of two rings
PyObject* do_unpack(PyObject* const* args) {
  at::ScalarType dt;
  if (!PyTuple_CheckExact(args[4]) || PyTuple_GET_SIZE(args[4]) != 2) Py_RETURN_NONE;
  const at::Tensor *k = tensor(PyTuple_GET_ITEM(args[4], 0)), *v = tensor(PyTuple_GET_ITEM(args[4], 1));
  const int dev = device_of(k, dt);
  if (dev < 0 || k->dim() != 4) Py_RETURN_NONE;
  const int64_t N = k->size(0), H = k->size(1), W = k->size(2), D = k->size(3);
  if (!plain4(k, dev, dt, N, H, W, D) || !plain4(v, dev, dt, N, H, W, D) || !small({N, H, W, D})) Py_RETURN_NONE;
  const void* p[4];
  for (int i = 0; i < 4; ++i) {
    const at::Tensor* t = tensor(args[i]);
    if (!plain4(t, dev, i & 1 ? SCALES : CODES, N, H, W, i & 1 ? D / 32 : D)) Py_RETURN_NONE;
    p[i] = t->data_ptr();
  }
  const rattn_decode_params par = {(int32_t)N, (int32_t)H, (int32_t)H, (int32_t)D, (int32_t)W, type_of(dt), 1.f, 1e-6f, 0};
  void *kp = k->data_ptr(), *vp = v->data_ptr();
  rattn_status s;
  { NoGil others_run; s = g_cache.unpack(&par, p[0], p[1], p[2], p[3], kp, vp, stream_of(dev)); }
  if (s != RATTN_OK) return PyLong_FromLong(s);
  Py_INCREF(args[4]);
  return args[4];
}

// decode_step_packed(q, k_new, v_new, pos, k_codes, k_scale, v_codes, v_scale, state, gamma_swa, gamma_rla, softmax_scale, rms_eps,
// out, feature_map)
PyObject* do_packed_step(PyObject* const* args) {
  const at::Tensor* t[9];
  for (int i = 0; i < 9; ++i)
    if (!(t[i] = tensor(args[i]))) Py_RETURN_NONE;
  at::ScalarType dt;
  const int dev = device_of(t[0], dt);
  if (dev < 0 || t[0]->dim() != 3 || t[4]->dim() != 4) Py_RETURN_NONE;
  const int64_t N = t[0]->size(0), Hq = t[0]->size(1), D = t[0]->size(2), H = t[4]->size(1), W = t[4]->size(2);
  if (!plain(*t[0], dev, dt, 3) || !plain(*t[1], dev, dt, 3) || !plain(*t[2], dev, dt, 3) || !shaped(*t[1], N, H, D) || !shaped(*t[2], N, H, D) ||
      !ints(t[3], dev, N) || !plain4(t[8], dev, at::kFloat, N, H, D, D) || !small({N, Hq, H, D, W}))
    Py_RETURN_NONE;
  for (int i = 0; i < 4; ++i)
    if (!plain4(t[4 + i], dev, i & 1 ? SCALES : CODES, N, H, W, i & 1 ? D / 32 : D)) Py_RETURN_NONE;
  rattn_decode_params p = {(int32_t)N, (int32_t)Hq, (int32_t)H, (int32_t)D, (int32_t)W, type_of(dt), 0.f, 0.f, 0};
  const float *gs, *gr;
  if (!gain_of(args[9], dev, Hq, D, gs) || !gain_of(args[10], dev, Hq, D, gr) || !PyFloat_CheckExact(args[11]) ||
      !PyFloat_CheckExact(args[12]) || !map_of(args[14], p.feature_map))
    Py_RETURN_NONE;
  p.softmax_scale = (float)PyFloat_AS_DOUBLE(args[11]);
  p.rms_eps = (float)PyFloat_AS_DOUBLE(args[12]);
  THPObjectPtr result;   // (made ahead of the step, as above)
  void* o;
  if (!output(args[13], *t[0], dev, false, result, o)) {
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  void* x[9];
  for (int i = 0; i < 9; ++i) x[i] = t[i]->data_ptr();
  rattn_status s;
  {
    NoGil others_run;
    size_t bytes = 0;
    s = g_cache.packed_bytes(&p, &bytes);
    if (s == RATTN_OK) {
      c10::DataPtr ws;
      if (bytes > 0) ws = c10::hip::HIPCachingAllocator::get()->allocate(bytes);
      s = g_cache.packed_step(&p, x[0], x[1], x[2], (const int32_t*)x[3], x[4], x[5], x[6], x[7], (float*)x[8], gs, gr, o, ws.get(), bytes,
                              stream_of(dev));
    }
  }
  return s == RATTN_OK ? result.release() : PyLong_FromLong(s);
}

// What a tree call's tensors have in common: k, v, parent, pos, rings, state, scales (NULL: none)
struct Tree {
  int dev = -1;
  rattn_tree_params p = {};
  void *k, *v, *kr, *vr, *ks = nullptr, *vs = nullptr, *state;
  const int32_t *parent, *pos;
};
bool tree_of(PyObject* k_, PyObject* v_, PyObject* parent_, PyObject* pos_, PyObject* kr_, PyObject* vr_, PyObject* state_, PyObject* ks_,
             PyObject* vs_, Tree& r) {
  const at::Tensor *k = tensor(k_), *v = tensor(v_), *parent = tensor(parent_), *pos = tensor(pos_), *kr = tensor(kr_), *vr = tensor(vr_), *state = tensor(state_);
  if (!k || !v || !parent || !pos || !kr || !vr || !state) return false;
  at::ScalarType dt;
  const int dev = device_of(k, dt);
  if (dev < 0 || k->dim() != 4 || kr->dim() != 4) return false;
  const int64_t N = k->size(0), M = k->size(1), H = k->size(2), D = k->size(3), W = kr->size(2);
  const bool packed = ks_ != Py_None;
  const at::ScalarType rt = packed ? CODES : dt;
  if (!plain4(k, dev, dt, N, M, H, D) || !plain4(v, dev, dt, N, M, H, D) || !plain(*parent, dev, at::kInt, 2) || parent->size(0) != N ||
      parent->size(1) != M || !ints(pos, dev, N) || !plain4(kr, dev, rt, N, H, W, D) || !plain4(vr, dev, rt, N, H, W, D) ||
      !plain4(state, dev, at::kFloat, N, H, D, D) || !small({N, M, H, D, W}) || packed != (vs_ != Py_None))
    return false;
  if (packed) {
    const at::Tensor *ks = tensor(ks_), *vs = tensor(vs_);
    if (!plain4(ks, dev, SCALES, N, H, W, D / 32) || !plain4(vs, dev, SCALES, N, H, W, D / 32)) return false;
    r.ks = ks->data_ptr();
    r.vs = vs->data_ptr();
  }
  r.dev = dev;
  r.p = {(int32_t)N, (int32_t)H, (int32_t)H, (int32_t)D, (int32_t)W, type_of(dt), (int32_t)M, 1.f, 1e-6f, 0};
  r.k = k->data_ptr(); r.v = v->data_ptr(); r.kr = kr->data_ptr(); r.vr = vr->data_ptr(); r.state = state->data_ptr();
  r.parent = (const int32_t*)parent->data_ptr(); r.pos = (const int32_t*)pos->data_ptr();
  return true;
}

// tree_step(q, k, v, parent, pos, k_ring, v_ring, state, gamma_swa, gamma_rla, softmax_scale, rms_eps, count, k_scale, v_scale, out,
// feature_map)
PyObject* do_tree_step(PyObject* const* args) {
  Tree r;
  if (!tree_of(args[1], args[2], args[3], args[4], args[5], args[6], args[7], args[13], args[14], r)) Py_RETURN_NONE;
  const at::Tensor *q = tensor(args[0]), *k = tensor(args[1]);
  const at::ScalarType dt = k->scalar_type();
  if (!q || !plain(*q, r.dev, dt, 4) || q->size(0) != r.p.N || q->size(1) != r.p.nodes || q->size(3) != r.p.D || !small({q->size(2)}))
    Py_RETURN_NONE;
  r.p.Hq = (int32_t)q->size(2);
  const int32_t* count = nullptr;
  if (args[12] != Py_None) {
    const at::Tensor* c = tensor(args[12]);
    if (!ints(c, r.dev, r.p.N)) Py_RETURN_NONE;
    count = (const int32_t*)c->data_ptr();
  }
  const float *gs, *gr;
  if (!gain_of(args[8], r.dev, r.p.Hq, r.p.D, gs) || !gain_of(args[9], r.dev, r.p.Hq, r.p.D, gr) || !PyFloat_CheckExact(args[10]) ||
      !PyFloat_CheckExact(args[11]) || !map_of(args[16], r.p.feature_map))
    Py_RETURN_NONE;
  r.p.softmax_scale = (float)PyFloat_AS_DOUBLE(args[10]);
  r.p.rms_eps = (float)PyFloat_AS_DOUBLE(args[11]);
  THPObjectPtr result;
  void* o;
  if (!output(args[15], *q, r.dev, true, result, o)) {   // (zero: a sequence may have rows, or nothing, without work)
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
  const void* qp = q->data_ptr();
  rattn_status s;
  {
    NoGil others_run;
    size_t bytes = 0;
    s = g_cache.tree_bytes(&r.p, r.ks != nullptr, &bytes);
    if (s == RATTN_OK) {
      c10::DataPtr ws;
      if (bytes > 0) ws = c10::hip::HIPCachingAllocator::get()->allocate(bytes);
      s = g_cache.tree_step(&r.p, qp, r.k, r.v, r.parent, count, r.pos, r.kr, r.ks, r.vr, r.vs, (const float*)r.state, gs, gr, o, ws.get(), bytes,
                            stream_of(r.dev));
    }
  }
  return s == RATTN_OK ? result.release() : PyLong_FromLong(s);
}

// tree_commit(k, v, parent, accepted, pos, k_ring, v_ring, state, k_scale, v_scale, feature_map): True
PyObject* do_tree_commit(PyObject* const* args) {
  Tree r;
  if (!tree_of(args[0], args[1], args[2], args[4], args[5], args[6], args[7], args[8], args[9], r) || !map_of(args[10], r.p.feature_map))
    Py_RETURN_NONE;
  const at::Tensor* acc = tensor(args[3]);
  if (!ints(acc, r.dev, r.p.N)) Py_RETURN_NONE;
  const int32_t* a = (const int32_t*)acc->data_ptr();
  rattn_status s;
  { NoGil others_run; s = g_cache.tree_commit(&r.p, r.k, r.v, r.parent, a, r.pos, r.kr, r.ks, r.vr, r.vs, (float*)r.state, stream_of(r.dev)); }
  if (s != RATTN_OK) return PyLong_FromLong(s);
  Py_RETURN_TRUE;
}

template <PyObject* (*F)(PyObject* const*), int ARGS> PyObject* cache_call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != ARGS || !g_cache.pack) return PyErr_Format(PyExc_TypeError, "takes %d arguments, after bind_cache", ARGS);
  try {
    return F(args);
  } catch (const std::exception&) {   // as in decode_step
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
  }
}
#define RATTN_FASTCALL(f) (PyCFunction)(void (*)(void))f

PyMethodDef g_methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"decode_step", (PyCFunction)(void (*)(void))decode_step, METH_FASTCALL, nullptr},
    {"bind_cache", RATTN_FASTCALL(bind_cache), METH_FASTCALL, nullptr},
    {"ring_pack", RATTN_FASTCALL((cache_call<do_pack, 3>)), METH_FASTCALL, nullptr},
    {"ring_unpack", RATTN_FASTCALL((cache_call<do_unpack, 5>)), METH_FASTCALL, nullptr},
    {"decode_step_packed", RATTN_FASTCALL((cache_call<do_packed_step, 15>)), METH_FASTCALL, nullptr},
    {"tree_step", RATTN_FASTCALL((cache_call<do_tree_step, 17>)), METH_FASTCALL, nullptr},
    {"tree_commit", RATTN_FASTCALL((cache_call<do_tree_commit, 11>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&g_module); }
