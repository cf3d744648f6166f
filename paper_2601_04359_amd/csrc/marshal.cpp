// Native marshalling of the binding's calls: what binding.py does with ctypes, for plain arguments.
//
// A small call spends most of its time on the host (one frame step of a small layer: 36 us of kernels behind 60 us
// of Python and launches), and a ctypes call with twenty arguments and the tensor queries in front of it cost 5 to
// 10 us.  Here the same checks and the same library call take under 1.  Arguments that are not plain (strided GPU
// tensors, built-in integers in 32-bit range, lists and tuples of them), and calls that the checks would refuse,
// return None: binding.py then takes its own path, which converts, or raises with the message.  The library's
// status comes back as an integer.  The entry points' addresses come from binding.py (bind), so both paths
// call the same loaded library.  The interpreter's lock is released around every library call.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/TensorBody.h>
#include <ATen/ops/empty.h>

#include <limits.h>
#include <stdint.h>

#include <initializer_list>
#include <vector>

#include "packcache.h"

namespace {

struct Library {
  decltype(&pc_rope3d) rope3d;
  decltype(&pc_score) score;
  decltype(&pc_compact) compact;
  decltype(&pc_compact_batch) compact_batch;
  decltype(&pc_frame_attn) frame_attn;
  decltype(&pc_frame_attn_workspace_bytes_for) attn_bytes;
  decltype(&pc_budget) budget;
} lib = {};
struct Q4Library {
  decltype(&pc_q4_store) store;
  decltype(&pc_q4_load) load;
  decltype(&pc_q4_attn) attn;
  decltype(&pc_q4_attn_workspace_bytes) attn_bytes;
  decltype(&pc_evict) evict;
  decltype(&pc_q4_evict) q4_evict;
  decltype(&pc_evict_workspace_bytes) evict_bytes;
} q4 = {};
PyObject* current_device = nullptr;   // torch's raw queries of the current device and of its stream
PyObject* raw_stream = nullptr;

// The lock comes back on every way out: an exception's way leads to a Python error.
template <class F>
auto unlocked(F&& call) {
  struct Lock {
    PyThreadState* state = PyEval_SaveThread();
    ~Lock() { PyEval_RestoreThread(state); }
  } lock;
  return call();
}

// ---- plain arguments -------------------------------------------------------------------------
const at::Tensor* plain(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  constexpr c10::DispatchKeySet wrapped({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchGradWrapper,
                                         c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::Functionalize,
                                         c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
                                         c10::DispatchKey::ZeroTensor});
  if (!t.defined() || !t.is_cuda() || t.layout() != c10::kStrided || t.key_set().has_any(wrapped)) return nullptr;
  return &t;
}
// rows dense, last dimension contiguous
bool rows_dense(const at::Tensor& t, int64_t dim) {
  return t.dim() == dim && t.stride(dim - 1) == 1 && t.stride(dim - 2) == t.size(dim - 1);
}
int dtype_code(const at::Tensor& t) {
  return t.scalar_type() == at::kFloat ? PC_F32 : t.scalar_type() == at::kBFloat16 ? PC_BF16 : -1;
}
bool as_int(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long long x = PyLong_AsLongLongAndOverflow(o, &over);
  if (over != 0 || x < INT32_MIN || x > INT32_MAX) return false;
  *v = static_cast<int32_t>(x);
  return true;
}
bool size_as_int(int64_t x, int* v) {
  *v = static_cast<int>(x);
  return x >= 0 && x <= INT32_MAX;
}
bool as_double(PyObject* o, double* v) {
  int32_t i;
  if (PyFloat_CheckExact(o)) {
    *v = PyFloat_AS_DOUBLE(o);
    return true;
  }
  if (!as_int(o, &i)) return false;
  *v = i;
  return true;
}
bool as_flag(PyObject* o, int* v) {
  *v = o == Py_True;
  return o == Py_True || o == Py_False;
}
bool is_table(PyObject* o) { return PyList_CheckExact(o) || PyTuple_CheckExact(o); }
bool as_ints(PyObject* o, Py_ssize_t n, std::vector<int32_t>& v) {
  if (!is_table(o) || PySequence_Fast_GET_SIZE(o) != n) return false;
  v.resize(n);
  for (Py_ssize_t i = 0; i < n; ++i)
    if (!as_int(PySequence_Fast_GET_ITEM(o, i), &v[i])) return false;
  return true;
}
bool as_segments(PyObject* o, std::vector<pc_segment>& v) {
  if (!is_table(o)) return false;
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
  v.resize(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject* s = PySequence_Fast_GET_ITEM(o, i);
    if (!is_table(s) || PySequence_Fast_GET_SIZE(s) != 4) return false;
    int32_t f[4];
    for (int k = 0; k < 4; ++k)
      if (!as_int(PySequence_Fast_GET_ITEM(s, k), &f[k])) return false;
    v[i] = {f[0], f[1], f[2], f[3]};
  }
  return n > 0;
}
PyObject* ints(const int32_t* v, Py_ssize_t n) {
  PyObject* list = PyList_New(n);
  for (Py_ssize_t i = 0; list && i < n; ++i) {
    PyObject* x = PyLong_FromLong(v[i]);
    if (!x) {
      Py_DECREF(list);
      return nullptr;
    }
    PyList_SET_ITEM(list, i, x);
  }
  return list;
}
// the current stream of the current device: what a launch without a stream argument would use
bool current_stream(void** out) {
  PyObject* device = PyObject_CallNoArgs(current_device);
  PyObject* handle = device ? PyObject_CallOneArg(raw_stream, device) : nullptr;
  Py_XDECREF(device);
  if (!handle) return false;
  *out = PyLong_AsVoidPtr(handle);
  Py_DECREF(handle);
  return !PyErr_Occurred();
}
// unbound, or a mode that wants to see every tensor method
bool ready() { return raw_stream != nullptr && !at::impl::torch_function_mode_enabled(); }

#define PLAIN_OR_NONE(cond) \
  if (!(cond)) Py_RETURN_NONE

// ---- calls: in the order of binding.py, positional ---------------------------------------------
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {   // 7 addresses, the two queries
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "bind: 9 arguments");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  lib = {reinterpret_cast<decltype(&pc_rope3d)>(p[0]),
         reinterpret_cast<decltype(&pc_score)>(p[1]),
         reinterpret_cast<decltype(&pc_compact)>(p[2]),
         reinterpret_cast<decltype(&pc_compact_batch)>(p[3]),
         reinterpret_cast<decltype(&pc_frame_attn)>(p[4]),
         reinterpret_cast<decltype(&pc_frame_attn_workspace_bytes_for)>(p[5]),
         reinterpret_cast<decltype(&pc_budget)>(p[6])};
  Py_INCREF(a[7]);
  Py_INCREF(a[8]);
  Py_XSETREF(current_device, a[7]);
  Py_XSETREF(raw_stream, a[8]);
  Py_RETURN_NONE;
}

PyObject* rope3d(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // x, pos, sections, base, out_scale
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 5 && ready());
  const at::Tensor *x = plain(a[0]), *pos = plain(a[1]);
  PLAIN_OR_NONE(x && pos && rows_dense(*x, 3) && is_table(a[2]) && PySequence_Fast_GET_SIZE(a[2]) >= 3);
  int32_t sec[3];
  for (int i = 0; i < 3; ++i) PLAIN_OR_NONE(as_int(PySequence_Fast_GET_ITEM(a[2], i), &sec[i]));
  double base, out_scale;
  int H, n, D;
  const int dt = dtype_code(*x);
  PLAIN_OR_NONE(dt >= 0 && as_double(a[3], &base) && as_double(a[4], &out_scale) && size_as_int(x->size(0), &H) &&
                size_as_int(x->size(1), &n) && size_as_int(x->size(2), &D));
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  void *xp = x->mutable_data_ptr(), *pp = pos->mutable_data_ptr();
  const int64_t stride = x->stride(0);
  return PyLong_FromLong(unlocked([&] {
    return lib.rope3d(xp, dt, H, n, D, stride, static_cast<int32_t*>(pp), sec[0], sec[1], sec[2], base, out_scale, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// Qs, K, Nk, scale, lse, score, share_heads, ws, q_rows, key_range
PyObject* score(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 10 && ready());
  const at::Tensor *Q = plain(a[0]), *K = plain(a[1]), *out = plain(a[5]), *ws = plain(a[7]);
  const at::Tensor *lse = nullptr, *rows = nullptr;
  PLAIN_OR_NONE(Q && K && out && ws && rows_dense(*Q, 3) && rows_dense(*K, 3) && out->dim() >= 1);
  PLAIN_OR_NONE(a[4] == Py_None || ((lse = plain(a[4])) && lse->dim() >= 1));
  PLAIN_OR_NONE(a[8] == Py_None || (rows = plain(a[8])));
  int32_t Nk, begin = 0, end = 0;
  double scale;
  int share, Hq, Hkv, n_qs, D;
  const int dt = dtype_code(*K);
  PLAIN_OR_NONE(dt >= 0 && as_int(a[2], &Nk) && as_double(a[3], &scale) && as_flag(a[6], &share) &&
                size_as_int(Q->size(0), &Hq) && size_as_int(K->size(0), &Hkv) && size_as_int(Q->size(2), &D) &&
                size_as_int(rows ? rows->numel() : Q->size(1), &n_qs));
  if (a[9] != Py_None)
    PLAIN_OR_NONE(is_table(a[9]) && PySequence_Fast_GET_SIZE(a[9]) >= 2 &&
                  as_int(PySequence_Fast_GET_ITEM(a[9], 0), &begin) && as_int(PySequence_Fast_GET_ITEM(a[9], 1), &end));
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  void *qp = Q->mutable_data_ptr(), *kp = K->mutable_data_ptr(), *op = out->mutable_data_ptr(), *wp = ws->mutable_data_ptr();
  void *lp = lse ? lse->mutable_data_ptr() : nullptr, *rp = rows ? rows->mutable_data_ptr() : nullptr;
  const int64_t qs = Q->stride(0), ks = K->stride(0), os = out->stride(0), ls = lse ? lse->stride(0) : 0;
  const size_t wn = ws->numel();
  return PyLong_FromLong(unlocked([&] {
    return lib.score(qp, kp, dt, Hq, Hkv, n_qs, Nk, D, qs, ks, static_cast<int32_t*>(rp), static_cast<float>(scale),
                     static_cast<float*>(lp), ls, static_cast<float*>(op), os, share, begin, end, wp, wn, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// What _check_kv_layout accepts, for one set of tensors ([L][H][cap][D] with layers, else [H][cap][D]).
bool cache_layout(const at::Tensor& K, const at::Tensor& V, const at::Tensor& pos, int64_t dim, bool share) {
  if (!rows_dense(K, dim) || !rows_dense(V, dim) || !rows_dense(pos, dim) || V.sizes() != K.sizes()) return false;
  for (int64_t i = 0; i < dim - 2; ++i)
    if (V.stride(i) != K.stride(i)) return false;
  return pos.size(dim - 1) == 3 && pos.size(dim - 3) == (share ? 1 : K.size(dim - 3));
}

// K, V, pos, score, segments, budgets, share_heads, out, idx, ws; the caches with a layer axis or without
PyObject* compact_call(PyObject* const* a, Py_ssize_t n_args, bool layers) {
  PLAIN_OR_NONE(n_args == 10 && ready());
  const int64_t dim = layers ? 4 : 3, head = dim - 3;
  const at::Tensor *K = plain(a[0]), *V = plain(a[1]), *pos = plain(a[2]), *sc = plain(a[3]), *ws = plain(a[9]);
  int share;
  PLAIN_OR_NONE(K && V && pos && sc && ws && as_flag(a[6], &share) && cache_layout(*K, *V, *pos, dim, share) &&
                sc->dim() > head);
  const at::Tensor *Ko = K, *Vo = V, *po = pos, *idx = nullptr;
  if (a[7] != Py_None) {
    PLAIN_OR_NONE(PyTuple_CheckExact(a[7]) && PyTuple_GET_SIZE(a[7]) == 3);
    Ko = plain(PyTuple_GET_ITEM(a[7], 0)), Vo = plain(PyTuple_GET_ITEM(a[7], 1)), po = plain(PyTuple_GET_ITEM(a[7], 2));
    PLAIN_OR_NONE(Ko && Vo && po && rows_dense(*Ko, dim) && rows_dense(*Vo, dim) && rows_dense(*po, dim) &&
                  Vo->sizes() == Ko->sizes() && po->size(dim - 1) == 3 && po->size(head) == (share ? 1 : K->size(head)));
    for (int64_t i = 0; i <= head; ++i) PLAIN_OR_NONE(Vo->stride(i) == Ko->stride(i));
  }
  PLAIN_OR_NONE(a[8] == Py_None || ((idx = plain(a[8])) && idx->dim() > head));
  std::vector<pc_segment> seg;
  std::vector<int32_t> budget;
  int L = 1, Hkv, D;
  const int dt = dtype_code(*K);
  PLAIN_OR_NONE(as_segments(a[4], seg) && as_ints(a[5], static_cast<Py_ssize_t>(seg.size()), budget) && dt >= 0 &&
                size_as_int(K->size(head), &Hkv) && size_as_int(K->size(dim - 1), &D) &&
                (!layers || size_as_int(K->size(0), &L)));
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  auto ptr = [](const at::Tensor* t) { return t ? t->mutable_data_ptr() : nullptr; };
  auto by_head = [&](const at::Tensor* t) { return t ? t->stride(head) : 0; };
  auto by_layer = [&](const at::Tensor* t) { return t && layers ? t->stride(0) : 0; };
  void *kp = ptr(K), *vp = ptr(V), *kop = ptr(Ko), *vop = ptr(Vo), *wp = ptr(ws);
  auto *pp = static_cast<int32_t*>(ptr(pos)), *pop = static_cast<int32_t*>(ptr(po)), *ip = static_cast<int32_t*>(ptr(idx));
  auto* sp = static_cast<float*>(ptr(sc));
  const size_t wn = ws->numel();
  const int n = static_cast<int>(seg.size());
  std::vector<pc_segment> seg_out(n);
  int32_t nk = 0;
  const int status = unlocked([&] {
    return layers ? lib.compact_batch(L, kp, vp, pp, dt, Hkv, D, by_head(K), by_layer(K), by_head(pos), by_layer(pos), sp,
                                      by_head(sc), by_layer(sc), seg.data(), n, budget.data(), share, kop, vop, pop,
                                      by_head(Ko), by_layer(Ko), by_head(po), by_layer(po), ip, by_head(idx), by_layer(idx),
                                      seg_out.data(), &nk, wp, wn, stream)
                  : lib.compact(kp, vp, pp, dt, Hkv, D, by_head(K), by_head(pos), sp, by_head(sc), seg.data(), n,
                                budget.data(), share, kop, vop, pop, by_head(Ko), by_head(po), ip, by_head(idx),
                                seg_out.data(), &nk, wp, wn, stream);
  });
  if (status != PC_OK) return PyLong_FromLong(status);
  PyObject* table = PyList_New(n);
  for (int i = 0; table && i < n; ++i) {
    PyObject* s = Py_BuildValue("(iiii)", seg_out[i].start, seg_out[i].len, seg_out[i].kind, seg_out[i].frame);
    if (!s) Py_CLEAR(table);
    else PyList_SET_ITEM(table, i, s);
  }
  return table ? Py_BuildValue("(Ni)", table, nk) : nullptr;
}
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return compact_call(a, n, false);
  END_HANDLE_TH_ERRORS
}
PyObject* compact_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return compact_call(a, n, true);
  END_HANDLE_TH_ERRORS
}

PyObject* frame_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // Q, K, V, Nk, scale, O, lse, ws
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 8 && ready());
  const at::Tensor *Q = plain(a[0]), *K = plain(a[1]), *V = plain(a[2]), *O = plain(a[5]), *lse = nullptr, *ws = nullptr;
  PLAIN_OR_NONE(Q && K && V && O && rows_dense(*Q, 3) && rows_dense(*K, 3) && rows_dense(*V, 3) &&
                K->stride(0) == V->stride(0) && O->dim() >= 1);
  int32_t Nk;
  double scale;
  int Hq, Hkv, Nq, D;
  const int dt = dtype_code(*Q);
  PLAIN_OR_NONE(dt >= 0 && as_int(a[3], &Nk) && as_double(a[4], &scale) && size_as_int(Q->size(0), &Hq) &&
                size_as_int(K->size(0), &Hkv) && size_as_int(Q->size(1), &Nq) && size_as_int(Q->size(2), &D));
  PLAIN_OR_NONE(a[6] == Py_None || ((lse = plain(a[6])) && lse->dim() == 2 && lse->size(0) == Hq && lse->size(1) == Nq &&
                                    lse->is_contiguous()));
  PLAIN_OR_NONE(a[7] == Py_None || (ws = plain(a[7])));
  at::Tensor own;   // a workspace of the call's own, from torch's stream-ordered allocator
  if (!ws) {
    const size_t bytes = lib.attn_bytes(dt, Hq, Hkv, Nq, Nk, D);
    if (bytes) {
      own = at::empty({static_cast<int64_t>(bytes < 16 ? 16 : bytes)},
                      at::TensorOptions().dtype(at::kByte).device(Q->device()));
      ws = &own;
    }
  }
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  void *qp = Q->mutable_data_ptr(), *kp = K->mutable_data_ptr(), *vp = V->mutable_data_ptr(), *op = O->mutable_data_ptr();
  void *lp = lse ? lse->mutable_data_ptr() : nullptr, *wp = ws ? ws->mutable_data_ptr() : nullptr;
  const int64_t qs = Q->stride(0), ks = K->stride(0), os = O->stride(0);
  const size_t wn = ws ? ws->numel() : 0;
  return PyLong_FromLong(unlocked([&] {
    return lib.frame_attn(qp, kp, vp, dt, Hq, Hkv, Nq, Nk, D, qs, ks, os, static_cast<float>(scale), op,
                          static_cast<float*>(lp), wp, wn, stream);
  }));
  END_HANDLE_TH_ERRORS
}

// ---- the cache in 4 bits, and eviction by accumulated weight -----------------------------------------
PyObject* bind_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {   // 7 addresses
  if (n != 7) {
    PyErr_SetString(PyExc_TypeError, "bind_q4: 7 arguments");
    return nullptr;
  }
  void* p[7];
  for (int i = 0; i < 7; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
  if (PyErr_Occurred()) return nullptr;
  q4 = {reinterpret_cast<decltype(&pc_q4_store)>(p[0]),
        reinterpret_cast<decltype(&pc_q4_load)>(p[1]),
        reinterpret_cast<decltype(&pc_q4_attn)>(p[2]),
        reinterpret_cast<decltype(&pc_q4_attn_workspace_bytes)>(p[3]),
        reinterpret_cast<decltype(&pc_evict)>(p[4]),
        reinterpret_cast<decltype(&pc_q4_evict)>(p[5]),
        reinterpret_cast<decltype(&pc_evict_workspace_bytes)>(p[6])};
  Py_RETURN_NONE;
}
bool ready_q4() { return ready() && q4.store != nullptr; }

// The current stream, and whether every tensor is on its device: calls go there.
struct Place {
  void* stream = nullptr;
  int device = -1;
  bool find() {
    PyObject* d = PyObject_CallNoArgs(current_device);
    if (!d) return false;
    device = static_cast<int>(PyLong_AsLong(d));
    PyObject* handle = PyObject_CallOneArg(raw_stream, d);
    Py_DECREF(d);
    if (!handle) return false;
    stream = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    return !PyErr_Occurred();
  }
  bool holds(std::initializer_list<const at::Tensor*> all) const {
    for (const at::Tensor* t : all)
      if (t && t->get_device() != device) return false;
    return true;
  }
};
// rows dense, or one row: what would lie between rows does not matter then
bool rows_follow(const at::Tensor& t) {
  return t.dim() == 3 && (t.size(2) <= 1 || t.stride(2) == 1) && (t.size(1) <= 1 || t.stride(1) == t.size(2));
}
bool optional(PyObject* o, const at::Tensor** t) { return o == Py_None || (*t = plain(o)) != nullptr; }
void* pointer(const at::Tensor* t) { return t ? t->mutable_data_ptr() : nullptr; }

// What binding.py's _q4_struct accepts, a tuple of four.
struct Cache4 {
  pc_q4_cache c;
  const at::Tensor* t[4];
  int H, cap, D;
  bool from(PyObject* o) {
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 4) return false;
    for (int i = 0; i < 4; ++i)
      if (!(t[i] = plain(PyTuple_GET_ITEM(o, i))) || t[i]->scalar_type() != at::kByte || !rows_dense(*t[i], 3)) return false;
    const at::Tensor &kc = *t[0], &ks = *t[1], &vc = *t[2], &vs = *t[3];
    if (vc.sizes() != kc.sizes() || vs.sizes() != ks.sizes() || ks.size(0) != kc.size(0) || ks.size(1) != kc.size(1) ||
        kc.size(2) != 16 * ks.size(2) || vc.stride(0) != kc.stride(0) || vs.stride(0) != ks.stride(0))
      return false;
    int half;
    if (!size_as_int(kc.size(0), &H) || !size_as_int(kc.size(1), &cap) || !size_as_int(kc.size(2), &half) || half > 1024) return false;
    D = 2 * half;
    auto bytes = [](const at::Tensor& x) { return static_cast<uint8_t*>(x.mutable_data_ptr()); };
    c = {bytes(kc), bytes(ks), bytes(vc), bytes(vs), kc.stride(0), ks.stride(0)};
    return true;
  }
  bool on(const Place& at) const { return at.holds({t[0], t[1], t[2], t[3]}); }
};

// Coordinates and sums as binding.py's _check_book takes them; Hsel 0: neither is there.
struct Book {
  const at::Tensor *pos = nullptr, *weights = nullptr;
  int Hsel = 0;
  bool from(PyObject* p, PyObject* w, int H, int64_t rows) {
    if (!optional(p, &pos) || !optional(w, &weights)) return false;
    int64_t n = 0;
    if (pos) {
      if (pos->scalar_type() != at::kInt || !rows_dense(*pos, 3) || pos->size(2) != 3 || pos->size(1) < rows) return false;
      n = pos->size(0);
    }
    if (weights) {
      if (weights->scalar_type() != at::kFloat || weights->dim() != 2 || weights->size(1) < rows ||
          (weights->size(1) > 1 && weights->stride(1) != 1) || (pos && weights->size(0) != n))
        return false;
      n = weights->size(0);
    }
    Hsel = static_cast<int>(n);
    return (!pos && !weights) || (n >= 1 && n <= H && H % n == 0);
  }
  int32_t* pos_at() const { return static_cast<int32_t*>(pointer(pos)); }
  float* weights_at() const { return static_cast<float*>(pointer(weights)); }
  int64_t pos_stride() const { return pos ? pos->stride(0) : 0; }
  int64_t weights_stride() const { return weights ? weights->stride(0) : 0; }
};
// a workspace of the call's own, from torch's stream-ordered allocator
at::Tensor make_workspace(size_t bytes, const at::Tensor& like) {
  return at::empty({static_cast<int64_t>(bytes < 16 ? 16 : bytes)}, at::TensorOptions().dtype(at::kByte).device(like.device()));
}

PyObject* q4_store(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // K, V, cache, row0, pos_new, pos, weights
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 7 && ready_q4());
  const at::Tensor *K = plain(a[0]), *V = plain(a[1]), *fresh = nullptr;
  Cache4 cache;
  Book book;
  int32_t row0;
  int n;
  PLAIN_OR_NONE(K && V && cache.from(a[2]) && as_int(a[3], &row0) && optional(a[4], &fresh) && rows_follow(*K) &&
                rows_follow(*V) && K->sizes() == V->sizes() && K->scalar_type() == V->scalar_type() &&
                K->size(0) == cache.H && K->size(2) == cache.D && size_as_int(K->size(1), &n) && row0 >= 0 &&
                static_cast<int64_t>(row0) + n <= cache.cap &&
                book.from(a[5], a[6], cache.H, static_cast<int64_t>(row0) + n) && !fresh == !book.pos);
  PLAIN_OR_NONE(!fresh || (fresh->scalar_type() == at::kInt && fresh->dim() == 2 && fresh->size(0) == n && fresh->size(1) == 3 &&
                           fresh->is_contiguous()));
  const int dt = dtype_code(*K);
  Place at;
  if (!at.find()) return nullptr;
  PLAIN_OR_NONE(dt >= 0 && cache.on(at) && at.holds({K, V, fresh, book.pos, book.weights}));
  void *kp = pointer(K), *vp = pointer(V);
  auto* np = static_cast<int32_t*>(pointer(fresh));
  const int64_t ks = K->stride(0), vs = V->stride(0);
  return PyLong_FromLong(unlocked([&] {
    return q4.store(kp, vp, dt, cache.H, n, cache.D, ks, vs, &cache.c, row0, np, book.pos_at(), book.pos_stride(),
                    book.weights_at(), book.weights_stride(), book.Hsel, at.stream);
  }));
  END_HANDLE_TH_ERRORS
}

PyObject* q4_load(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // cache, row0, K, V
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 4 && ready_q4());
  Cache4 cache;
  int32_t row0;
  const at::Tensor *K = nullptr, *V = nullptr;
  PLAIN_OR_NONE(cache.from(a[0]) && as_int(a[1], &row0) && optional(a[2], &K) && optional(a[3], &V) && (K || V));
  const at::Tensor& some = K ? *K : *V;
  int n;
  PLAIN_OR_NONE(some.dim() == 3 && size_as_int(some.size(1), &n) && row0 >= 0 && static_cast<int64_t>(row0) + n <= cache.cap);
  for (const at::Tensor* t : {K, V})
    PLAIN_OR_NONE(!t || (rows_follow(*t) && t->size(0) == cache.H && t->size(1) == n && t->size(2) == cache.D &&
                         t->scalar_type() == some.scalar_type()));
  const int dt = dtype_code(some);
  Place at;
  if (!at.find()) return nullptr;
  PLAIN_OR_NONE(dt >= 0 && cache.on(at) && at.holds({K, V}));
  void *kp = pointer(K), *vp = pointer(V);
  const int64_t ks = K ? K->stride(0) : 0, vs = V ? V->stride(0) : 0;
  return PyLong_FromLong(unlocked([&] {
    return q4.load(&cache.c, cache.H, row0, n, cache.D, dt, kp, vp, ks, vs, at.stream);
  }));
  END_HANDLE_TH_ERRORS
}

PyObject* q4_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // Q, cache, Nk, scale, O, lse, weights, decay, ws
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 9 && ready_q4());
  const at::Tensor *Q = plain(a[0]), *O = plain(a[4]), *lse = nullptr, *ws = nullptr;
  Cache4 cache;
  Book book;
  int32_t Nk;
  double scale, decay;
  int Hq, Nq;
  PLAIN_OR_NONE(Q && O && cache.from(a[1]) && as_int(a[2], &Nk) && as_double(a[3], &scale) && optional(a[5], &lse) &&
                as_double(a[7], &decay) && optional(a[8], &ws) && rows_follow(*Q) && rows_follow(*O) &&
                O->sizes() == Q->sizes() && O->scalar_type() == Q->scalar_type() && Q->size(2) == cache.D && cache.H > 0 &&
                size_as_int(Q->size(0), &Hq) && size_as_int(Q->size(1), &Nq) && Hq % cache.H == 0 && Nk >= 1 &&
                Nk <= cache.cap && book.from(Py_None, a[6], cache.H, Nk));
  PLAIN_OR_NONE(!lse || (lse->scalar_type() == at::kFloat && lse->dim() == 2 && lse->size(0) == Hq && lse->size(1) == Nq &&
                         lse->is_contiguous()));
  const int dt = dtype_code(*Q);
  Place at;
  if (!at.find()) return nullptr;
  PLAIN_OR_NONE(dt >= 0 && cache.on(at) && at.holds({Q, O, lse, book.weights, ws}));
  at::Tensor own;
  if (!ws) {
    const size_t bytes = q4.attn_bytes(dt, Hq, cache.H, Nq, Nk, cache.D, book.weights != nullptr);
    if (bytes) ws = &(own = make_workspace(bytes, *Q));
  }
  void *qp = pointer(Q), *op = pointer(O), *wp = pointer(ws);
  auto* lp = static_cast<float*>(pointer(lse));
  const int64_t qs = Q->stride(0), os = O->stride(0);
  const size_t wn = ws ? ws->nbytes() : 0;
  return PyLong_FromLong(unlocked([&] {
    return q4.attn(qp, &cache.c, dt, Hq, cache.H, Nq, Nk, cache.D, qs, os, static_cast<float>(scale), op, lp, book.weights_at(),
                   book.weights_stride(), book.Hsel, static_cast<float>(decay), wp, wn, at.stream);
  }));
  END_HANDLE_TH_ERRORS
}

// pos, weights, Nk, n_keep, n_anchor, recent_t, idx, ws from a[0] on
struct Eviction {
  Book book;
  int32_t Nk, n_keep, n_anchor, recent_t;
  const at::Tensor *idx = nullptr, *ws = nullptr;
  at::Tensor own;
  bool from(PyObject* const* a, int H, int64_t cap) {
    return as_int(a[2], &Nk) && as_int(a[3], &n_keep) && as_int(a[4], &n_anchor) && as_int(a[5], &recent_t) && a[1] != Py_None &&
           Nk >= 0 && Nk <= cap && H > 0 && book.from(a[0], a[1], H, Nk) && optional(a[6], &idx) && optional(a[7], &ws) &&
           (!idx || (idx->scalar_type() == at::kInt && idx->dim() == 2 && idx->size(0) == book.Hsel && idx->size(1) >= n_keep &&
                     (idx->size(1) <= 1 || idx->stride(1) == 1)));
  }
  void workspace(const at::Tensor& like) {
    const size_t bytes = ws ? 0 : q4.evict_bytes(book.Hsel, Nk, n_keep);
    if (bytes) ws = &(own = make_workspace(bytes, like));
  }
};

PyObject* evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // K, V, then as above
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 10 && ready_q4());
  const at::Tensor *K = plain(a[0]), *V = plain(a[1]);
  Eviction e;
  int H, D;
  PLAIN_OR_NONE(K && V && rows_dense(*K, 3) && rows_dense(*V, 3) && K->sizes() == V->sizes() &&
                K->scalar_type() == V->scalar_type() && size_as_int(K->size(0), &H) && size_as_int(K->size(2), &D) &&
                e.from(a + 2, H, K->size(1)));
  const int dt = dtype_code(*K);
  Place at;
  if (!at.find()) return nullptr;
  PLAIN_OR_NONE(dt >= 0 && at.holds({K, V, e.book.pos, e.book.weights, e.idx, e.ws}));
  e.workspace(*K);
  void *kp = pointer(K), *vp = pointer(V), *wp = pointer(e.ws);
  auto* ip = static_cast<int32_t*>(pointer(e.idx));
  const int64_t ks = K->stride(0), vs = V->stride(0), is = e.idx ? e.idx->stride(0) : 0;
  const size_t wn = e.ws ? e.ws->nbytes() : 0;
  return PyLong_FromLong(unlocked([&] {
    return q4.evict(kp, vp, dt, H, D, ks, vs, e.book.pos_at(), e.book.pos_stride(), e.book.weights_at(), e.book.weights_stride(),
                    e.book.Hsel, e.Nk, e.n_keep, e.n_anchor, e.recent_t, ip, is, wp, wn, at.stream);
  }));
  END_HANDLE_TH_ERRORS
}

PyObject* q4_evict(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // cache, then as above
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 9 && ready_q4());
  Cache4 cache;
  Eviction e;
  PLAIN_OR_NONE(cache.from(a[0]) && e.from(a + 1, cache.H, cache.cap));
  Place at;
  if (!at.find()) return nullptr;
  PLAIN_OR_NONE(cache.on(at) && at.holds({e.book.pos, e.book.weights, e.idx, e.ws}));
  e.workspace(*cache.t[0]);
  void* wp = pointer(e.ws);
  auto* ip = static_cast<int32_t*>(pointer(e.idx));
  const int64_t is = e.idx ? e.idx->stride(0) : 0;
  const size_t wn = e.ws ? e.ws->nbytes() : 0;
  return PyLong_FromLong(unlocked([&] {
    return q4.q4_evict(&cache.c, cache.H, cache.D, e.book.pos_at(), e.book.pos_stride(), e.book.weights_at(),
                       e.book.weights_stride(), e.book.Hsel, e.Nk, e.n_keep, e.n_anchor, e.recent_t, ip, is, wp, wn, at.stream);
  }));
  END_HANDLE_TH_ERRORS
}

// Rows start .. start + n - 1 of three caches as views: K, V, pos, dim, start, n
PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  PLAIN_OR_NONE(n_args == 6 && ready());
  int32_t dim, start, n;
  PLAIN_OR_NONE(as_int(a[3], &dim) && as_int(a[4], &start) && as_int(a[5], &n) && dim >= 0 && start >= 0 && n >= 0);
  const at::Tensor* t[3];
  for (int i = 0; i < 3; ++i)
    PLAIN_OR_NONE((t[i] = plain(a[i])) && t[i]->dim() > dim && static_cast<int64_t>(start) + n <= t[i]->size(dim));
  PyObject* views = PyTuple_New(3);
  for (int i = 0; views && i < 3; ++i) {
    PyObject* v = THPVariable_Wrap(t[i]->narrow(dim, start, n));
    if (!v) Py_CLEAR(views);
    else PyTuple_SET_ITEM(views, i, v);
  }
  return views;
  END_HANDLE_TH_ERRORS
}

// ---- tables (host only) ------------------------------------------------------------------------
PyObject* budget(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // mode, n_frame_tokens, n_past, gamma, b_min
  HANDLE_TH_ERRORS
  int32_t mode, n, n_past, b_min;
  double gamma;
  PLAIN_OR_NONE(n_args == 5 && lib.budget && as_int(a[0], &mode) && as_int(a[1], &n) && as_int(a[2], &n_past) &&
                as_double(a[3], &gamma) && as_int(a[4], &b_min) && n_past >= 0 && n_past <= 1 << 16);
  std::vector<int32_t> out(n_past + 1);
  const int status = lib.budget(mode, n, n_past, gamma, b_min, out.data());
  return status != PC_OK ? PyLong_FromLong(status) : ints(out.data(), n_past);
  END_HANDLE_TH_ERRORS
}

PyObject* segment_budgets(PyObject*, PyObject* const* a, Py_ssize_t n_args) {   // segments, by_distance
  HANDLE_TH_ERRORS
  std::vector<pc_segment> seg;
  PLAIN_OR_NONE(n_args == 2 && as_segments(a[0], seg) && is_table(a[1]));
  const Py_ssize_t n_by = PySequence_Fast_GET_SIZE(a[1]);
  std::vector<int32_t> out(seg.size());
  Py_ssize_t d = 0;
  for (size_t i = seg.size(); i-- > 0;) {
    out[i] = seg[i].len;
    if (seg[i].kind != PC_SEG_FRAME) continue;
    PLAIN_OR_NONE(d < n_by && as_int(PySequence_Fast_GET_ITEM(a[1], d), &out[i]));
    ++d;
  }
  return ints(out.data(), static_cast<Py_ssize_t>(out.size()));
  END_HANDLE_TH_ERRORS
}

// How many past frames a table holds: segments
PyObject* past_frames(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  std::vector<pc_segment> seg;
  PLAIN_OR_NONE(n_args == 1 && as_segments(a[0], seg));
  long n = 0;
  for (const pc_segment& s : seg) n += s.kind == PC_SEG_FRAME;
  return PyLong_FromLong(n);
  END_HANDLE_TH_ERRORS
}

// Rows from the first to the last past frame that is over its budget, False if none is: segments, budgets
PyObject* prunable_span(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  std::vector<pc_segment> seg;
  std::vector<int32_t> b;
  PLAIN_OR_NONE(n_args == 2 && as_segments(a[0], seg) && as_ints(a[1], static_cast<Py_ssize_t>(seg.size()), b));
  int64_t begin = -1, end = 0;
  for (size_t i = 0; i < seg.size(); ++i)
    if (seg[i].kind == PC_SEG_FRAME && b[i] < seg[i].len) {
      if (begin < 0) begin = seg[i].start;
      end = static_cast<int64_t>(seg[i].start) + seg[i].len;
    }
  if (begin < 0) Py_RETURN_FALSE;
  return Py_BuildValue("(LL)", static_cast<long long>(begin), static_cast<long long>(end));
  END_HANDLE_TH_ERRORS
}

#define ENTRY(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(bind),       ENTRY(rope3d),      ENTRY(score),  ENTRY(compact),
                         ENTRY(compact_batch), ENTRY(frame_attn), ENTRY(rows), ENTRY(budget), ENTRY(segment_budgets),
                         ENTRY(past_frames), ENTRY(prunable_span), ENTRY(bind_q4), ENTRY(q4_store), ENTRY(q4_load),
                         ENTRY(q4_attn), ENTRY(evict), ENTRY(q4_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// What this file was built against, for the loader to compare: it reads torch's tensors through inlined accessors
// and calls the library through the header's signatures, and neither is checked anywhere else.
PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&module);
  if (m && (PyModule_AddStringConstant(m, "torch_version", PC_TORCH_VERSION) < 0 ||
            PyModule_AddIntConstant(m, "pc_version", PC_VERSION) < 0))
    Py_CLEAR(m);
  return m;
}
