// CPython module behind the package's tensor functions: checks the tensors,
// allocates what the caller did not give, and calls the C ABI on the current
// stream.  The host cost of a call bounds every small problem: the launch
// itself takes about 3.5 us, and the same checks and conversions in Python
// with ctypes took another 8 to 10 (per call on the smallest problems, before
// and after: prefill 11.7 and 4.9 us, decode with its output and workspace
// given 12.1 and 3.4, L2 norm 11.9 and 5.1, RMSNorm 13.8 and 6.5).
//
// A call that is not plainly valid (a wrong shape or type, a subclass, a
// stream argument, an unusual scalar) returns None from here, and the Python
// function goes through its own checks, which raise the errors.  A returned
// int is the C ABI's error status.

#include <Python.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <initializer_list>
#include <utility>

#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/attn.h"
#include "../../include/kv4.h"
#include "../../include/norms.h"
#include "../../include/rope.h"

namespace {

// A plain contiguous GPU tensor, or nullptr.
const at::Tensor* plain(PyObject* obj) {
  if (!THPVariable_CheckExact(obj)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(obj);
  return t.layout() == c10::kStrided && t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}

// Every size fits the C ABI's int arguments.
bool ints(const at::Tensor& t) {
  for (int64_t n : t.sizes())
    if (n > INT_MAX) return false;
  return true;
}

bool number(PyObject* obj, float& x) {
  if (PyFloat_CheckExact(obj)) x = (float)PyFloat_AS_DOUBLE(obj);
  else if (PyLong_CheckExact(obj)) {
    const double d = PyLong_AsDouble(obj);
    if (d == -1.0 && PyErr_Occurred()) {
      PyErr_Clear();
      return false;
    }
    x = (float)d;
  } else return false;
  return true;
}

// A Python int that fits.
bool whole(PyObject* obj, int& x) {
  if (!PyLong_CheckExact(obj)) return false;
  int over = 0;
  const long long v = PyLong_AsLongLongAndOverflow(obj, &over);
  if (over || v < INT_MIN || v > INT_MAX) return false;
  x = (int)v;
  return true;
}

bool truth(PyObject* obj, bool& x) {
  if (!PyBool_Check(obj)) return false;
  x = obj == Py_True;
  return true;
}

hipStream_t stream() { return c10::hip::getCurrentHIPStream().stream(); }

PyObject* none() { Py_RETURN_NONE; }

// Run f (a C ABI call) without the interpreter lock.
template <typename F>
int unlocked(F&& f) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  return rc;
}

// The given output object, or a new reference to the allocated tensor.
PyObject* result(int rc, PyObject* given, at::Tensor&& made) {
  if (rc != ATTN_OK) return PyLong_FromLong(rc);
  if (given != Py_None) {
    Py_INCREF(given);
    return given;
  }
  return THPVariable_Wrap(std::move(made));
}

struct Attn {
  const at::Tensor *q, *k, *v;
  at::Tensor o;
  const float* slopes = nullptr;
  attn_dtype dtype;
  int B, Hq, Hkv, Lq, Lk, D;
  float scale;
};

// The arguments shared by the attention calls; false if not plainly valid.
bool attn_args(PyObject* q, PyObject* k, PyObject* v, PyObject* o, PyObject* scale, PyObject* slopes, Attn& a) {
  a.q = plain(q);
  a.k = plain(k);
  a.v = plain(v);
  if (!a.q || !a.k || !a.v || a.q->dim() != 4 || a.k->dim() != 4) return false;
  const auto dt = a.q->scalar_type();
  if ((dt != at::kHalf && dt != at::kBFloat16) || a.k->scalar_type() != dt || a.v->scalar_type() != dt) return false;
  if (a.k->sizes() != a.v->sizes() || a.k->size(0) != a.q->size(0) || a.k->size(3) != a.q->size(3)) return false;
  if (!ints(*a.q) || !ints(*a.k)) return false;
  a.dtype = dt == at::kHalf ? ATTN_F16 : ATTN_BF16;
  a.B = (int)a.q->size(0);
  a.Hq = (int)a.q->size(1);
  a.Lq = (int)a.q->size(2);
  a.D = (int)a.q->size(3);
  a.Hkv = (int)a.k->size(1);
  a.Lk = (int)a.k->size(2);
  if (slopes != Py_None) {
    const at::Tensor* s = plain(slopes);
    if (!s || s->scalar_type() != at::kFloat || s->numel() != a.Hq) return false;
    a.slopes = static_cast<const float*>(s->data_ptr());
  }
  if (scale == Py_None) {
    if (a.D < 1) return false;
    a.scale = (float)(1.0 / std::sqrt((double)a.D));
  } else if (!number(scale, a.scale)) return false;
  if (o != Py_None) {
    const at::Tensor* t = plain(o);
    if (!t || t->scalar_type() != dt || t->sizes() != a.q->sizes()) return false;
    a.o = *t;
  } else {
    a.o = at::empty_like(*a.q);
  }
  return true;
}

// (q, k, v, o, causal, scale, alibi_slopes, softcap, window, stream)
PyObject* py_attn_fwd(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Attn a;
  bool causal;
  float cap = 0.f;
  int window = 0;
  if (n != 10 || x[9] != Py_None || !truth(x[4], causal)) return none();
  if (x[8] != Py_None && !whole(x[8], window)) return none();
  if (x[7] != Py_None && !number(x[7], cap)) return none();
  if (!attn_args(x[0], x[1], x[2], x[3], x[5], x[6], a)) return none();
  const void *q = a.q->data_ptr(), *k = a.k->data_ptr(), *v = a.v->data_ptr();
  void* o = a.o.data_ptr();
  // Few rows against many keys: a workspace, which lives on this stream like
  // the call itself (so not for tensors on another device).  Where memory has
  // run out the call does without it.
  at::Tensor ws;
  size_t bytes = 0;
  const int S = attn_fwd_num_splits(a.B, a.Hq, a.Hkv, a.Lq, a.Lk, a.D, causal, window);
  if (S > 1 && a.q->device().index() == c10::hip::getCurrentHIPStream().device_index()) {
    bytes = attn_fwd_workspace_bytes(a.B, a.Hq, a.Lq, a.D, S);
    try {
      ws = at::empty({(int64_t)bytes}, a.q->options().dtype(at::kByte));
    } catch (const c10::OutOfMemoryError&) {
      bytes = 0;
    }
  }
  void* w = bytes ? ws.data_ptr() : nullptr;
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return attn_fwd_split(q, k, v, o, a.B, a.Hq, a.Hkv, a.Lq, a.Lk, a.D, causal, a.scale, a.slopes, cap, window, w,
                          bytes, a.dtype, s);
  });
  return result(rc, x[3], std::move(a.o));
  END_HANDLE_TH_ERRORS
}

// (q, k, v, o, scale, alibi_slopes, softcap, num_splits, workspace, stream)
PyObject* py_attn_decode(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Attn a;
  float cap = 0.f;
  int splits;
  if (n != 10 || x[9] != Py_None || !whole(x[7], splits)) return none();
  if (x[6] != Py_None && !number(x[6], cap)) return none();
  at::Tensor ws;
  if (x[8] != Py_None) {
    const at::Tensor* t = plain(x[8]);
    if (!t) return none();
    ws = *t;
  }
  if (!attn_args(x[0], x[1], x[2], x[3], x[4], x[5], a) || a.Lq != 1) return none();
  if (!ws.defined()) {
    const int S = splits ? splits : attn_decode_num_splits(a.B, a.Hq, a.Hkv, a.Lk, a.D);
    const size_t need = attn_decode_workspace_bytes(a.B, a.Hq, a.D, std::max(S, 1));
    ws = at::empty({(int64_t)std::max<size_t>(need, 16)}, a.q->options().dtype(at::kByte));
  }
  const void *q = a.q->data_ptr(), *k = a.k->data_ptr(), *v = a.v->data_ptr();
  void *o = a.o.data_ptr(), *w = ws.data_ptr();
  const size_t bytes = ws.nbytes();
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return attn_decode_mod(q, k, v, o, a.B, a.Hq, a.Hkv, a.Lk, a.D, a.scale, a.slopes, cap, splits, w, bytes, a.dtype,
                           s);
  });
  return result(rc, x[3], std::move(a.o));
  END_HANDLE_TH_ERRORS
}

// (q, k, v, o, scale, alibi_slopes, softcap, num_splits, stream)
PyObject* py_attn_decode_noalloc(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Attn a;
  float cap = 0.f;
  int splits;
  if (n != 9 || x[8] != Py_None || !whole(x[7], splits)) return none();
  if (x[6] != Py_None && !number(x[6], cap)) return none();
  if (!attn_args(x[0], x[1], x[2], x[3], x[4], x[5], a) || a.Lq != 1) return none();
  const void *q = a.q->data_ptr(), *k = a.k->data_ptr(), *v = a.v->data_ptr();
  void* o = a.o.data_ptr();
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return attn_decode_noalloc(q, k, v, o, a.B, a.Hq, a.Hkv, a.Lk, a.D, a.scale, a.slopes, cap, splits, a.dtype, s);
  });
  return result(rc, x[3], std::move(a.o));
  END_HANDLE_TH_ERRORS
}

struct Norm {
  const at::Tensor* x;
  at::Tensor ws, out, y;
  norm_dtype dtype;
  int N, M, chunks;
};

bool norm_args(PyObject* px, PyObject* pout, PyObject* chunks, PyObject* workspace, bool rms, PyObject* py, Norm& a) {
  a.x = plain(px);
  if (!a.x || a.x->dim() != 2 || !ints(*a.x) || !whole(chunks, a.chunks)) return false;
  const auto dt = a.x->scalar_type();
  if (dt == at::kHalf) a.dtype = NORM_F16;
  else if (dt == at::kBFloat16) a.dtype = NORM_BF16;
  else if (dt == at::kFloat) a.dtype = NORM_F32;
  else return false;
  a.N = (int)a.x->size(0);
  a.M = (int)a.x->size(1);
  if (pout != Py_None) {
    const at::Tensor* t = plain(pout);
    if (!t || t->scalar_type() != at::kFloat || t->numel() != a.N) return false;
    a.out = *t;
  }
  if (rms && py != Py_None) {
    const at::Tensor* t = plain(py);
    if (!t || t->scalar_type() != dt || t->sizes() != a.x->sizes()) return false;
    a.y = *t;
  }
  if (workspace != Py_None) {
    const at::Tensor* t = plain(workspace);
    if (!t) return false;
    a.ws = *t;
  }
  const auto opt = a.x->options();
  if (!a.ws.defined()) {
    const int C = a.chunks ? a.chunks : norm_chunks(rms, a.N, a.M, a.dtype);
    a.ws = at::empty({(int64_t)std::max<size_t>(norm_workspace_bytes(a.N, std::max(C, 1)), 16)}, opt.dtype(at::kByte));
  }
  if (rms && !a.y.defined()) a.y = at::empty_like(*a.x);
  if (!a.out.defined()) a.out = at::empty({(int64_t)a.N}, opt.dtype(at::kFloat));
  return true;
}

// (x, out, chunks, workspace, stream)
PyObject* py_norm_l2(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Norm a;
  if (n != 5 || x[4] != Py_None || !norm_args(x[0], x[1], x[2], x[3], false, nullptr, a)) return none();
  const void* px = a.x->data_ptr();
  float* out = static_cast<float*>(a.out.data_ptr());
  void* w = a.ws.data_ptr();
  const size_t bytes = a.ws.nbytes();
  const hipStream_t s = stream();
  const int rc = unlocked([&] { return norm_l2(px, out, a.N, a.M, a.dtype, a.chunks, w, bytes, s); });
  return result(rc, x[1], std::move(a.out));
  END_HANDLE_TH_ERRORS
}

// (x, y, rowmax, eps, chunks, workspace, stream) -> (y, rowmax)
PyObject* py_rmsnorm_rowmax(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Norm a;
  float eps;
  if (n != 7 || x[6] != Py_None || !number(x[3], eps) || !norm_args(x[0], x[2], x[4], x[5], true, x[1], a))
    return none();
  const void* px = a.x->data_ptr();
  void *y = a.y.data_ptr(), *w = a.ws.data_ptr();
  float* out = static_cast<float*>(a.out.data_ptr());
  const size_t bytes = a.ws.nbytes();
  const hipStream_t s = stream();
  const int rc =
      unlocked([&] { return rmsnorm_rowmax(px, y, out, a.N, a.M, eps, a.dtype, a.chunks, w, bytes, s); });
  if (rc != ATTN_OK) return PyLong_FromLong(rc);
  PyObject* r = PyTuple_New(2);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, result(rc, x[1], std::move(a.y)));
  PyTuple_SET_ITEM(r, 1, result(rc, x[2], std::move(a.out)));
  return r;
  END_HANDLE_TH_ERRORS
}

// A tensor on the current device, contiguous unless `strided`; nullptr otherwise.
const at::Tensor* here(PyObject* obj, bool strided = false) {
  if (!THPVariable_CheckExact(obj)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(obj);
  if (t.layout() != c10::kStrided || !t.is_cuda() || (!strided && !t.is_contiguous()) || !ints(t)) return nullptr;
  return t.device().index() == c10::hip::getCurrentHIPStream().device_index() ? &t : nullptr;
}

// The same, of a type and shape.
const at::Tensor* here(PyObject* obj, at::ScalarType type, at::IntArrayRef shape) {
  const at::Tensor* t = here(obj);
  return t && t->scalar_type() == type && t->sizes() == shape ? t : nullptr;
}

// [B, H, L, D] whose rows are contiguous, and its strides of batches, heads and
// tokens (0 where there is one alone).
const at::Tensor* rows(PyObject* obj, long long (&strides)[3]) {
  const at::Tensor* t = here(obj, true);
  if (!t || t->dim() != 4 || (t->size(3) != 1 && t->stride(3) != 1)) return nullptr;
  for (int i = 0; i < 3; ++i) strides[i] = t->size(i) > 1 ? t->stride(i) : 0;
  return t;
}

// A new contiguous tensor on the current device, from PyTorch's allocator: what
// at::empty makes, without its dispatch (0.5 us each against 0.75).
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
  return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}

// The given output of that type and shape, or a new one; false if the given one is not plain.
bool output(PyObject* obj, const at::Tensor& like, at::ScalarType type, at::IntArrayRef shape, at::Tensor& out) {
  if (obj == Py_None) {
    out = fresh(shape, type, like);
    return true;
  }
  const at::Tensor* t = here(obj, type, shape);
  if (t) out = *t;
  return t != nullptr;
}

// Whether the memory that two tensors span has a common part.
bool overlap(const at::Tensor& a, const at::Tensor& b) {
  if (!a.numel() || !b.numel()) return false;
  const auto end = [](const at::Tensor& t) {
    int64_t n = 1;
    for (int64_t i = 0; i < t.dim(); ++i) n += (t.size(i) - 1) * t.stride(i);
    return static_cast<const char*>(t.data_ptr()) + n * t.element_size();
  };
  return a.data_ptr() < end(b) && b.data_ptr() < end(a);
}

// A tuple of outputs, or the error status.
PyObject* results(int rc, std::initializer_list<std::pair<PyObject*, at::Tensor*>> outs) {
  if (rc != ATTN_OK) return PyLong_FromLong(rc);
  PyObject* r = PyTuple_New((Py_ssize_t)outs.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (const auto& [given, made] : outs) {
    PyObject* o = made ? result(rc, given, std::move(*made)) : none();
    if (!o) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// (q, k, positions, freqs, q_out, k_out, interleaved, magnitude, bwd, stream) -> (q_out, k_out)
PyObject* py_rope(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  bool inter, bwd;
  float magnitude;
  long long qs[3], ks[3];
  if (n != 10 || x[9] != Py_None || !truth(x[6], inter) || !truth(x[8], bwd) || !number(x[7], magnitude)) return none();
  const at::Tensor* q = rows(x[0], qs);
  if (!q) return none();
  const at::Tensor* k = nullptr;
  if (x[1] != Py_None && !(k = rows(x[1], ks))) return none();
  if (!k && x[5] != Py_None) return none();
  const auto type = q->scalar_type();
  rope_dtype dtype;
  if (type == at::kHalf) dtype = ROPE_F16;
  else if (type == at::kBFloat16) dtype = ROPE_BF16;
  else if (type == at::kFloat) dtype = ROPE_F32;
  else return none();
  const int64_t B = q->size(0), L = q->size(2), D = q->size(3);
  if (k && (k->scalar_type() != type || k->size(0) != B || k->size(2) != L || k->size(3) != D)) return none();
  const at::Tensor *pos = here(x[2]), *freqs = here(x[3]);
  if (!pos || !freqs || freqs->scalar_type() != at::kDouble || freqs->dim() != 1) return none();
  if (pos->scalar_type() != at::kInt && pos->scalar_type() != at::kLong) return none();
  const bool each = pos->dim() == 2 && pos->size(0) == B && pos->size(1) == L;
  if (!each && !(pos->dim() == 1 && pos->size(0) == L)) return none();
  if (freqs->size(0) > INT_MAX / 2) return none();
  at::Tensor qo, ko;
  if (!output(x[4], *q, type, q->sizes(), qo) || (k && !output(x[5], *q, type, k->sizes(), ko))) return none();
  // An output that is given shares memory with nothing, or is its input.
  const auto apart = [&](const at::Tensor& o, const at::Tensor& x, const at::Tensor* other, const at::Tensor& out) {
    return ((o.data_ptr() == x.data_ptr() && x.is_contiguous()) || !overlap(o, x)) && (!other || !overlap(o, *other)) &&
           (!out.defined() || !overlap(o, out));
  };
  if (x[4] != Py_None && !apart(qo, *q, k, ko)) return none();
  if (x[5] != Py_None && !apart(ko, *k, q, qo)) return none();
  const void *qp = q->data_ptr(), *kp = k ? k->data_ptr() : nullptr, *pp = pos->data_ptr();
  void *qop = qo.data_ptr(), *kop = k ? ko.data_ptr() : nullptr;
  const double* fp = static_cast<const double*>(freqs->data_ptr());
  const int Hq = (int)q->size(1), Hkv = k ? (int)k->size(1) : 0, R = 2 * (int)freqs->size(0);
  const int bits = pos->scalar_type() == at::kLong ? 64 : 32;
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return (bwd ? rope_bwd : rope_fwd)(qp, qs, qop, Hq, kp, k ? ks : nullptr, kop, Hkv, (int)B, (int)L, (int)D, pp,
                                       bits, each ? L : 0, fp, R, inter, magnitude, dtype, s);
  });
  return results(rc, {{x[4], &qo}, {x[5], k ? &ko : nullptr}});
  END_HANDLE_TH_ERRORS
}

// (lens, counts, table, free_pages, page, L, slots, positions, new_lens, taken, stream) -> the last four
PyObject* py_kv_slots(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int page, L;
  if (n != 11 || x[10] != Py_None || !whole(x[4], page) || !whole(x[5], L) || L < 1) return none();
  const at::Tensor *lens = here(x[0]), *counts = here(x[1]), *table = here(x[2]), *pages = here(x[3]);
  if (!lens || !counts || !table || !pages || lens->dim() != 1 || table->dim() != 2 || pages->dim() != 1) return none();
  const int64_t B = lens->size(0), M = table->size(1);
  if (counts->sizes() != lens->sizes() || table->size(0) != B) return none();
  for (const at::Tensor* t : {lens, counts, table, pages})
    if (t->scalar_type() != at::kInt) return none();
  at::Tensor out[4];
  if (!output(x[6], *lens, at::kLong, {B, L}, out[0]) || !output(x[7], *lens, at::kInt, {B, L}, out[1]) ||
      !output(x[8], *lens, at::kInt, {B}, out[2]) || !output(x[9], *lens, at::kInt, {1}, out[3]))
    return none();
  for (const at::Tensor* t : {lens, counts, pages})
    if (overlap(*table, *t)) return none();
  for (int i = 0; i < 4; ++i)
    if (x[6 + i] != Py_None) {
      for (const at::Tensor* t : {lens, counts, table, pages})
        if (overlap(out[i], *t)) return none();
      for (int j = 0; j < i; ++j)
        if (overlap(out[i], out[j])) return none();
    }
  const int* pt[3] = {static_cast<const int*>(lens->data_ptr()), static_cast<const int*>(counts->data_ptr()),
                      static_cast<const int*>(pages->data_ptr())};
  int* tp = static_cast<int*>(table->data_ptr());
  long long* sp = static_cast<long long*>(out[0].data_ptr());
  int* op[3] = {static_cast<int*>(out[1].data_ptr()), static_cast<int*>(out[2].data_ptr()),
                static_cast<int*>(out[3].data_ptr())};
  const int F = (int)pages->size(0);
  const hipStream_t s = stream();
  const int rc = unlocked(
      [&] { return kv_slots(pt[0], pt[1], tp, pt[2], F, (int)B, (int)M, page, L, sp, op[0], op[1], op[2], s); });
  return results(rc, {{x[6], &out[0]}, {x[7], &out[1]}, {x[8], &out[2]}, {x[9], &out[3]}});
  END_HANDLE_TH_ERRORS
}

// Tokens of a page of a cache [pages, H, bytes], 0 if it is none of head dim D.
int cache_page(const at::Tensor& cache, int D) {
  if (cache.scalar_type() != at::kByte || cache.dim() != 3 || (D != 64 && D != 128)) return 0;
  const int64_t page = cache.size(2) * 16 / (17 * D);
  return page > 0 && page <= INT_MAX && kv4_page_bytes((int)page, D) == (size_t)cache.size(2) ? (int)page : 0;
}

// (k, v, cache, slots, stream) -> cache
PyObject* py_kv4_append(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  long long ks[3], vs[3];
  if (n != 5 || x[4] != Py_None) return none();
  const at::Tensor *k = rows(x[0], ks), *v = rows(x[1], vs), *cache = here(x[2]);
  if (!k || !v || !cache || k->sizes() != v->sizes()) return none();
  const auto type = k->scalar_type();
  if ((type != at::kHalf && type != at::kBFloat16) || v->scalar_type() != type) return none();
  const int B = (int)k->size(0), H = (int)k->size(1), L = (int)k->size(2), D = (int)k->size(3);
  const int page = cache_page(*cache, D);
  const at::Tensor* slots = here(x[3], at::kLong, {B, L});
  if (!page || cache->size(1) != H || !slots) return none();
  const void *kp = k->data_ptr(), *vp = v->data_ptr();
  void* cp = cache->data_ptr();
  const long long* sp = static_cast<const long long*>(slots->data_ptr());
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return kv4_append(kp, ks, vp, vs, cp, sp, B, H, L, D, (int)cache->size(0), page,
                      type == at::kHalf ? ATTN_F16 : ATTN_BF16, s);
  });
  if (rc != ATTN_OK) return PyLong_FromLong(rc);
  Py_INCREF(x[2]);
  return x[2];
  END_HANDLE_TH_ERRORS
}

// (cache, table, lens, L, D, dtype, k, v, starts, stream) -> (k, v)
PyObject* py_kv4_load(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int L, D;
  if (n != 10 || x[9] != Py_None || !whole(x[3], L) || !whole(x[4], D) || L < 1 || !THPDtype_Check(x[5])) return none();
  const auto type = reinterpret_cast<THPDtype*>(x[5])->scalar_type;
  if (type != at::kHalf && type != at::kBFloat16) return none();
  const at::Tensor *cache = here(x[0]), *table = here(x[1]);
  if (!cache || !table || table->dim() != 2 || table->scalar_type() != at::kInt) return none();
  const int page = cache_page(*cache, D);
  const int64_t B = table->size(0);
  const at::Tensor *lens = here(x[2], at::kInt, {B}), *starts = nullptr;
  if (!page || !lens || (x[8] != Py_None && !(starts = here(x[8], at::kInt, {B})))) return none();
  at::Tensor k, v;
  const int64_t shape[4] = {B, cache->size(1), L, D};
  if (!output(x[6], *cache, type, shape, k) || !output(x[7], *cache, type, shape, v)) return none();
  const void* cp = cache->data_ptr();
  const int *tp = static_cast<const int*>(table->data_ptr()), *lp = static_cast<const int*>(lens->data_ptr()),
            *sp = starts ? static_cast<const int*>(starts->data_ptr()) : nullptr;
  void *kp = k.data_ptr(), *vp = v.data_ptr();
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return kv4_load(cp, tp, sp, lp, kp, vp, (int)B, (int)shape[1], L, D, (int)cache->size(0), page,
                    (int)table->size(1), type == at::kHalf ? ATTN_F16 : ATTN_BF16, s);
  });
  return results(rc, {{x[6], &k}, {x[7], &v}});
  END_HANDLE_TH_ERRORS
}

// (q, cache, table, lens, o, scale, alibi_slopes, softcap, window, workspace, stream)
PyObject* py_attn_decode_kv4(PyObject*, PyObject* const* x, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  float cap = 0.f, scale;
  int window = 0;
  if (n != 11 || x[10] != Py_None) return none();
  if (x[7] != Py_None && !number(x[7], cap)) return none();
  if (x[8] != Py_None && !whole(x[8], window)) return none();
  const at::Tensor *q = here(x[0]), *cache = here(x[1]), *table = here(x[2]);
  if (!q || !cache || !table || q->dim() != 4 || q->size(2) != 1 || table->dim() != 2) return none();
  const auto type = q->scalar_type();
  if ((type != at::kHalf && type != at::kBFloat16) || table->scalar_type() != at::kInt) return none();
  const int64_t B = q->size(0);
  const int Hq = (int)q->size(1), D = (int)q->size(3), page = cache_page(*cache, D);
  const at::Tensor* lens = here(x[3], at::kInt, {B});
  if (!page || !lens || table->size(0) != B) return none();
  const float* slopes = nullptr;
  if (x[6] != Py_None) {
    const at::Tensor* t = here(x[6]);
    if (!t || t->scalar_type() != at::kFloat || t->numel() != Hq) return none();
    slopes = static_cast<const float*>(t->data_ptr());
  }
  if (x[5] == Py_None) scale = (float)(1.0 / std::sqrt((double)D));
  else if (!number(x[5], scale)) return none();
  at::Tensor o, ws;
  if (!output(x[4], *q, type, q->sizes(), o)) return none();
  if (x[9] != Py_None) {
    const at::Tensor* t = here(x[9]);
    if (!t) return none();
    ws = *t;
  } else {
    const size_t need = attn_decode_kv4_workspace_bytes((int)B, Hq, (int)cache->size(1), D);
    ws = fresh({(int64_t)std::max<size_t>(need, 16)}, at::kByte, *q);
  }
  const void *qp = q->data_ptr(), *cp = cache->data_ptr();
  const int *tp = static_cast<const int*>(table->data_ptr()), *lp = static_cast<const int*>(lens->data_ptr());
  void *op = o.data_ptr(), *wp = ws.data_ptr();
  const size_t bytes = ws.nbytes();
  const hipStream_t s = stream();
  const int rc = unlocked([&] {
    return attn_decode_kv4(qp, cp, tp, lp, op, (int)B, Hq, (int)cache->size(1), D, (int)cache->size(0), page,
                           (int)table->size(1), scale, slopes, cap, window, wp, bytes,
                           type == at::kHalf ? ATTN_F16 : ATTN_BF16, s);
  });
  return result(rc, x[4], std::move(o));
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

PyMethodDef methods[] = {
    {"attn_fwd", fast<py_attn_fwd>(), METH_FASTCALL, nullptr},
    {"attn_decode", fast<py_attn_decode>(), METH_FASTCALL, nullptr},
    {"attn_decode_noalloc", fast<py_attn_decode_noalloc>(), METH_FASTCALL, nullptr},
    {"norm_l2", fast<py_norm_l2>(), METH_FASTCALL, nullptr},
    {"rmsnorm_rowmax", fast<py_rmsnorm_rowmax>(), METH_FASTCALL, nullptr},
    {"rope", fast<py_rope>(), METH_FASTCALL, nullptr},
    {"kv_slots", fast<py_kv_slots>(), METH_FASTCALL, nullptr},
    {"kv4_append", fast<py_kv4_append>(), METH_FASTCALL, nullptr},
    {"kv4_load", fast<py_kv4_load>(), METH_FASTCALL, nullptr},
    {"attn_decode_kv4", fast<py_attn_decode_kv4>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
