// The way from Python to the entry points that a layer's pass goes through (binding.py), for calls whose arguments are what they
// should be: plain tensors and plain ints.  Each function here reads the tensors' pointers, sizes and types, calls
// the C entry point on the current stream and returns its code; for anything else it returns None and has done nothing, and
// binding.py takes the general way, through ctypes, which also names the error.  What is checked is what the general way checks: that
// a quantiser's input lies in device memory with rows of unit stride, and the types of inputs and Y.  Every other tensor is a pointer.
//
// Why: a call through ctypes costs the host 1.7 us (a quantiser, 10 arguments) to 2.3 us (a layer, 19) before the launch, against
// 3.4 us of the runtime's own, and a decode pass of two calls was bound by that.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>

#include "../../include/serq.h"
#include "../../include/serq_kv.h"

namespace {

decltype(&serq_quantize_act) f_quantize_act;
decltype(&serq_swiglu_quantize_act) f_swiglu_quantize_act;
decltype(&serq_mx_quantize_act) f_mx_quantize_act;
decltype(&serq_mx_swiglu_quantize_act) f_mx_swiglu_quantize_act;
decltype(&serq_quantize_act_asym) f_quantize_act_asym;
decltype(&serq_linear) f_linear;
decltype(&serq_mx_linear) f_mx_linear;
decltype(&serq_g128_linear) f_g128_linear;
decltype(&serq_kv_append) f_kv_append;
decltype(&serq_paged_attn) f_paged_attn;

// Arguments of one call; `ok` falls once one of them is not the plain thing.
struct Args {
  PyObject* const* a;
  bool ok = !at::impl::torch_function_mode_enabled();

  const at::Tensor* tensor(int i) {                    // a plain tensor or parameter, of any type and any number of dimensions
    if (!THPVariable_CheckExact(a[i])) { ok = false; return nullptr; }
    return &THPVariable_Unpack(a[i]);
  }
  void* ptr(int i) {                                   // of a tensor
    const at::Tensor* t = ok ? tensor(i) : nullptr;
    return t ? t->data_ptr() : nullptr;
  }
  void* ptr_or_none(int i) { return a[i] == Py_None ? nullptr : ptr(i); }
  int64_t integer(int i) {
    int over = 1;
    long long v = 0;
    if (PyLong_CheckExact(a[i])) v = PyLong_AsLongLongAndOverflow(a[i], &over);
    if (over) ok = false;
    return v;
  }
  int integer32(int i) {
    const int64_t v = integer(i);
    if (v != (int)v) ok = false;
    return (int)v;
  }
  int dtype(const at::Tensor& t) {
    switch (t.scalar_type()) {
      case at::kFloat: return SERQ_F32;
      case at::kHalf: return SERQ_F16;
      case at::kBFloat16: return SERQ_BF16;
      default: ok = false; return 0;
    }
  }
  // [M, K] activations with unit inner stride
  struct Rows { void* p; int dt; int64_t M, K, ld; };
  Rows rows(int i) {
    Rows r{};
    const at::Tensor* t = ok ? tensor(i) : nullptr;
    if (!t || !t->is_cuda() || t->dim() != 2 || t->stride(1) != 1) { ok = false; return r; }
    r = {t->data_ptr(), dtype(*t), t->size(0), t->size(1), 0};
    r.ld = r.M > 0 ? t->stride(0) : r.K;
    return r;
  }
  // the two halves of a gated product, alike in shape and type
  void alike(const Rows& g, const Rows& u) {
    if (g.M != u.M || g.K != u.K || g.dt != u.dt) ok = false;
  }
};

void* stream() { return (void*)c10::hip::getCurrentHIPStream().stream(); }

// n arguments in; `read` takes them and returns the call, which is made if everything was plain.
// The interpreter lock is given up for the call proper, as ctypes does: a launch waits where the queue is full, and what it waits for
// may be a host function that needs the lock.  The caller's frame holds the arguments meanwhile.  (Host time of a decode pass of two
// calls, lock held / given up: 7.9 / 8.0 us.)
template <class F>
PyObject* run(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, const F& read) {
  if (n != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments expected", want);
    return nullptr;
  }
  int rc = 0;
  PyThreadState* unlocked = nullptr;
  try {
    Args x{a};
    const auto call = read(x);
    if (!x.ok) Py_RETURN_NONE;
    void* const st = stream();
    unlocked = PyEval_SaveThread();
    rc = call(st);
  } catch (...) {                                      // (a tensor without storage, for instance: the general way says which)
    if (unlocked) PyEval_RestoreThread(unlocked);
    Py_RETURN_NONE;
  }
  PyEval_RestoreThread(unlocked);
  return PyLong_FromLong(rc);
}

PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {        // X, s_inv, abits, Xq, scale
  return run(a, n, 5, [](Args& x) {
    const Args::Rows X = x.rows(0);
    const float* s = (const float*)x.ptr_or_none(1);
    const int abits = x.integer32(2);
    void* xq = x.ptr(3);
    float* sc = (float*)x.ptr(4);
    return [=](void* st) { return f_quantize_act(X.p, X.dt, s, X.M, X.K, X.ld, abits, xq, sc, st); };
  });
}

PyObject* swiglu_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {  // G, U, s_inv, abits, Xq, scale
  return run(a, n, 6, [](Args& x) {
    const Args::Rows G = x.rows(0), U = x.rows(1);
    const float* s = (const float*)x.ptr_or_none(2);
    const int abits = x.integer32(3);
    void* xq = x.ptr(4);
    float* sc = (float*)x.ptr(5);
    x.alike(G, U);
    return [=](void* st) { return f_swiglu_quantize_act(G.p, U.p, G.dt, s, G.M, G.K, G.ld, U.ld, abits, xq, sc, st); };
  });
}

PyObject* mx_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {     // X, s_inv, Xq, xsc
  return run(a, n, 4, [](Args& x) {
    const Args::Rows X = x.rows(0);
    const float* s = (const float*)x.ptr_or_none(1);
    void* xq = x.ptr(2);
    uint8_t* sc = (uint8_t*)x.ptr(3);
    return [=](void* st) { return f_mx_quantize_act(X.p, X.dt, s, X.M, X.K, X.ld, xq, sc, st); };
  });
}

PyObject* mx_swiglu_quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n) {   // G, U, s_inv, Xq, xsc
  return run(a, n, 5, [](Args& x) {
    const Args::Rows G = x.rows(0), U = x.rows(1);
    const float* s = (const float*)x.ptr_or_none(2);
    void* xq = x.ptr(3);
    uint8_t* sc = (uint8_t*)x.ptr(4);
    x.alike(G, U);
    return [=](void* st) { return f_mx_swiglu_quantize_act(G.p, U.p, G.dt, s, G.M, G.K, G.ld, U.ld, xq, sc, st); };
  });
}

PyObject* quantize_act_asym(PyObject*, PyObject* const* a, Py_ssize_t n) {   // X, s_inv, abits, Xq, scale, zero
  return run(a, n, 6, [](Args& x) {
    const Args::Rows X = x.rows(0);
    const float* s = (const float*)x.ptr_or_none(1);
    const int abits = x.integer32(2);
    void* xq = x.ptr(3);
    float* sc = (float*)x.ptr(4);
    int32_t* z = (int32_t*)x.ptr(5);
    return [=](void* st) { return f_quantize_act_asym(X.p, X.dt, s, X.M, X.K, X.ld, abits, xq, sc, z, st); };
  });
}

// Y: a tensor of a type the library has, and its row stride
struct Out { void* p; int dt; int64_t ld; };
Out output(Args& x, int i) {
  Out y{};
  const at::Tensor* t = x.ok ? x.tensor(i) : nullptr;
  if (!t || t->dim() < 1) { x.ok = false; return y; }
  y = {t->data_ptr(), x.dtype(*t), t->stride(0)};
  return y;
}
struct Room { void* p; size_t n; };
Room workspace(Args& x, int i) {
  Room r{};
  if (x.a[i] == Py_None) return r;
  const at::Tensor* t = x.ok ? x.tensor(i) : nullptr;
  if (t) r = {t->data_ptr(), (size_t)t->numel()};
  return r;
}

// Xq, scale, abits, Wq, wscale, s_begin, r, Rp, r_dtype, M, N, K, Y, ws, flags
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 15, [](Args& x) {
    const void* xq = x.ptr(0);
    const float* sc = (const float*)x.ptr(1);
    const int abits = x.integer32(2);
    const void* wq = x.ptr(3);
    const float* wsc = (const float*)x.ptr(4);
    const int s0 = x.integer32(5), r = x.integer32(6);
    const void* rp = x.ptr_or_none(7);
    const int rdt = x.integer32(8);
    const int64_t M = x.integer(9), N = x.integer(10), K = x.integer(11);
    const Out y = output(x, 12);
    const Room w = workspace(x, 13);
    const int flags = x.integer32(14);
    return [=](void* st) { return f_linear(xq, sc, abits, wq, wsc, s0, r, rp, rdt, M, N, K, y.p, y.dt, y.ld, w.p, w.n, flags, st); };
  });
}

// Xq, xsc, Wq, wsc, s_begin, r, Rq, rsc, M, N, K, Y, ws, flags
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 14, [](Args& x) {
    const void* xq = x.ptr(0);
    const uint8_t* xsc = (const uint8_t*)x.ptr(1);
    const void* wq = x.ptr(2);
    const uint8_t* wsc = (const uint8_t*)x.ptr(3);
    const int s0 = x.integer32(4), r = x.integer32(5);
    const void* rq = x.ptr_or_none(6);
    const uint8_t* rsc = (const uint8_t*)x.ptr_or_none(7);
    const int64_t M = x.integer(8), N = x.integer(9), K = x.integer(10);
    const Out y = output(x, 11);
    const Room w = workspace(x, 12);
    const int flags = x.integer32(13);
    return [=](void* st) { return f_mx_linear(xq, xsc, wq, wsc, s0, r, rq, rsc, M, N, K, y.p, y.dt, M > 0 ? y.ld : N, w.p, w.n, flags, st); };
  });
}

// Xq, scale, zero, abits, Wq, gscale, wsum, s_begin, r, Rp, r_dtype, M, N, K, Y, flags
PyObject* g128_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 16, [](Args& x) {
    const void* xq = x.ptr(0);
    const float* sc = (const float*)x.ptr(1);
    const int32_t* z = (const int32_t*)x.ptr_or_none(2);
    const int abits = x.integer32(3);
    const void *wq = x.ptr(4), *gsc = x.ptr(5);
    const float* wsum = (const float*)x.ptr(6);
    const int s0 = x.integer32(7), r = x.integer32(8);
    const void* rp = x.ptr_or_none(9);
    const int rdt = x.integer32(10);
    const int64_t M = x.integer(11), N = x.integer(12), K = x.integer(13);
    const Out y = output(x, 14);
    const int flags = x.integer32(15);
    return [=](void* st) { return f_g128_linear(xq, sc, z, abits, wq, gsc, wsum, s0, r, rp, rdt, M, N, K, y.p, y.dt, y.ld, flags, st); };
  });
}

// ---- the paged cache: here every tensor's type and sizes are checked, as the general way does -------------------------------------
// [tokens, heads, dim] with unit inner stride, in device memory
struct Heads { void* p; int dt; int64_t T, H, D, ld, ldh; };
Heads heads(Args& x, int i) {
  Heads h{};
  const at::Tensor* t = x.ok ? x.tensor(i) : nullptr;
  if (!t || !t->is_cuda() || t->dim() != 3 || (t->stride(2) != 1 && t->numel() > 0)) { x.ok = false; return h; }
  h = {t->data_ptr(), x.dtype(*t), t->size(0), t->size(1), t->size(2), t->stride(0), t->stride(1)};
  if (h.dt == SERQ_F32) x.ok = false;
  return h;
}
const at::Tensor* typed(Args& x, int i, at::ScalarType type, int64_t dims) {
  const at::Tensor* t = x.ok ? x.tensor(i) : nullptr;
  if (!t || !t->is_cuda() || t->scalar_type() != type || t->dim() != dims || (t->numel() > 0 && t->stride(dims - 1) != 1)) {
    x.ok = false;
    return nullptr;
  }
  return t;
}
const float* scales(Args& x, int i, int64_t n) {
  if (!x.ok || x.a[i] == Py_None) return nullptr;
  const at::Tensor* t = typed(x, i, at::kFloat, 1);
  if (!t || t->size(0) != n) { x.ok = false; return nullptr; }
  return (const float*)t->data_ptr();
}
// K, V, table, cu_q, kv_len from argument i on; k_scale, v_scale from argument s on
struct Cache { serq_kv_cache c; serq_kv_batch b; };
Cache cache(Args& x, int i, int s, const Heads& q) {
  Cache r{};
  const at::Tensor *K = x.ok ? x.tensor(i) : nullptr, *V = x.ok ? x.tensor(i + 1) : nullptr;
  const at::Tensor *tb = typed(x, i + 2, at::kInt, 2), *cu = typed(x, i + 3, at::kInt, 1), *len = typed(x, i + 4, at::kInt, 1);
  if (!x.ok) return r;
  const bool f8 = K->scalar_type() == at::kFloat8_e4m3fn;
  const int64_t B = len->size(0);
  if (!K->is_cuda() || !V->is_cuda() || K->dim() != 4 || V->dim() != 4 || K->sizes() != V->sizes() || K->scalar_type() != V->scalar_type() ||
      (K->numel() > 0 && (K->stride(3) != 1 || V->stride(3) != 1)) || (!f8 && x.dtype(*K) != q.dt) || cu->size(0) != B + 1 ||
      tb->size(0) != B || K->size(3) != q.D || B > 65536 || tb->size(1) > 0x7fffffff || K->size(1) > 65536 || K->size(2) > 65536 || q.D > 65536) {
    x.ok = false;
    return r;
  }
  r.c = {K->data_ptr(), V->data_ptr(), scales(x, s, K->size(2)), scales(x, s + 1, K->size(2)), K->stride(0), K->stride(1), K->stride(2),
         V->stride(0), V->stride(1), V->stride(2), K->size(0), (int32_t)K->size(1), (int32_t)K->size(2), (int32_t)K->size(3),
         f8 ? SERQ_F8 : q.dt};
  r.b = {(const int32_t*)cu->data_ptr(), (const int32_t*)len->data_ptr(), (const int32_t*)tb->data_ptr(),
         B <= 1 ? std::max(tb->stride(0), tb->size(1)) : tb->stride(0), q.T, (int32_t)tb->size(1), (int32_t)B};
  return r;
}
bool same_rows(const Heads& a, const Heads& b) { return a.T == b.T && a.D == b.D && a.dt == b.dt; }

// q, k, v, K, V, table, cu_q, kv_len, cos, sin, interleaved, positions, k_scale, v_scale, q_out
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 15, [](Args& x) {
    Heads q{}, qo{};
    const Heads k = heads(x, 1), v = heads(x, 2);
    if (x.a[0] != Py_None) {
      q = heads(x, 0);
      qo = heads(x, 14);
      if (!same_rows(q, k) || !same_rows(qo, k) || q.H != qo.H || q.H > 65536) x.ok = false;
    }
    const Cache c = cache(x, 3, 12, k);
    const float *cs = nullptr, *sn = nullptr;
    int64_t rows = 0, rot = 0;
    if (x.a[8] != Py_None) {
      const at::Tensor *ct = typed(x, 8, at::kFloat, 2), *st = typed(x, 9, at::kFloat, 2);
      if (x.ok && (!ct->is_contiguous() || !st->is_contiguous() || ct->sizes() != st->sizes() || ct->size(1) > 65536)) x.ok = false;
      if (x.ok) {
        cs = (const float*)ct->data_ptr();
        sn = (const float*)st->data_ptr();
        rows = ct->size(0);
        rot = 2 * ct->size(1);
      }
    } else if (x.a[9] != Py_None) {
      x.ok = false;
    }
    const int inter = x.integer32(10);
    const int32_t* pos = nullptr;
    if (x.a[11] != Py_None) {
      const at::Tensor* t = typed(x, 11, at::kInt, 1);
      if (t && t->size(0) < k.T) x.ok = false;
      if (t) pos = (const int32_t*)t->data_ptr();
    }
    if (!same_rows(k, v) || k.H != c.c.heads || v.H != c.c.heads) x.ok = false;
    return [=](void* st) {
      return f_kv_append(q.p, q.ld, q.ldh, (int)q.H, k.p, k.ld, k.ldh, v.p, v.ld, v.ldh, k.dt, cs, sn, rows, (int)rot, inter, pos, &c.c, &c.b,
                         qo.p, qo.ld, qo.ldh, st);
    };
  });
}

// q, K, V, table, cu_q, kv_len, max_q, max_kv, scale, window, k_scale, v_scale, out, lse, ws
PyObject* paged_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return run(a, n, 15, [](Args& x) {
    const Heads q = heads(x, 0), o = heads(x, 12);
    const Cache c = cache(x, 1, 10, q);
    const int max_q = x.integer32(6), window = x.integer32(9);
    const int64_t max_kv = x.integer(7);
    float scale = 0.0f;
    if (PyFloat_CheckExact(x.a[8])) scale = (float)PyFloat_AS_DOUBLE(x.a[8]);
    else x.ok = false;
    float* lse = nullptr;
    if (x.a[13] != Py_None) {
      const at::Tensor* t = typed(x, 13, at::kFloat, 2);
      if (t && (!t->is_contiguous() || t->size(0) != q.T || t->size(1) != q.H)) x.ok = false;
      if (t) lse = (float*)t->data_ptr();
    }
    Room w{};
    if (x.a[14] != Py_None) {
      const at::Tensor* t = x.ok ? x.tensor(14) : nullptr;
      if (t && (!t->is_cuda() || t->scalar_type() != at::kByte || !t->is_contiguous())) x.ok = false;
      if (t && x.ok) w = {t->data_ptr(), (size_t)t->numel()};
    }
    if (!same_rows(q, o) || q.H != o.H || q.H > 65536) x.ok = false;
    return [=](void* st) {
      return f_paged_attn(q.p, q.ld, q.ldh, (int)q.H, q.dt, &c.c, &c.b, max_q, max_kv, scale, window, o.p, o.ld, o.ldh, lse, w.p, w.n, st);
    };
  });
}

// the addresses of the entry points, in the order of the declarations above
PyObject* bind_slots(void** const* slots, Py_ssize_t count, PyObject* const* a, Py_ssize_t n) {
  if (n != count) {
    PyErr_SetString(PyExc_TypeError, "one address per entry point expected");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < n; ++i) {
    void* p = PyLong_AsVoidPtr(a[i]);
    if (!p) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null address");
      return nullptr;
    }
    *slots[i] = p;
  }
  Py_RETURN_NONE;
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void** const slots[] = {(void**)&f_quantize_act, (void**)&f_swiglu_quantize_act, (void**)&f_mx_quantize_act,
                          (void**)&f_mx_swiglu_quantize_act, (void**)&f_quantize_act_asym, (void**)&f_linear,
                          (void**)&f_mx_linear, (void**)&f_g128_linear};
  return bind_slots(slots, sizeof(slots) / sizeof(slots[0]), a, n);
}
PyObject* bind_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void** const slots[] = {(void**)&f_kv_append, (void**)&f_paged_attn};
  return bind_slots(slots, sizeof(slots) / sizeof(slots[0]), a, n);
}

#define SERQ_FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SERQ_FAST(bind), SERQ_FAST(quantize_act), SERQ_FAST(swiglu_quantize_act), SERQ_FAST(mx_quantize_act),
                         SERQ_FAST(mx_swiglu_quantize_act), SERQ_FAST(quantize_act_asym), SERQ_FAST(linear),
                         SERQ_FAST(mx_linear), SERQ_FAST(g128_linear), SERQ_FAST(bind_kv), SERQ_FAST(kv_append),
                         SERQ_FAST(paged_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) { return PyModule_Create(&module); }
