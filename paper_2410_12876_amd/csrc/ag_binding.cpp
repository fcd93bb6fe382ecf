// The binding's per-call work: reads shapes, dtypes and addresses of the tensor arguments and makes the C call.
//
// A decode step on short caches is under ten microseconds of device time, so what the host spends per call is part of
// the step: looking the stream up through torch.cuda (2.9 us), checking and fetching a dozen addresses one Python call at
// a time (4 us) and ctypes' conversion of fifteen arguments (2.7 us) was more than the two kernel launches cost.  The
// same work on the tensors' own structures takes well under a microsecond.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ag.h"

namespace {

struct bad_arg {};  // a Python exception has been set

[[noreturn]] void fail(PyObject *type, const char *msg) {
  PyErr_SetString(type, msg);
  throw bad_arg();
}

const at::Tensor &tensor(PyObject *o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is expected");
  return THPVariable_Unpack(o);
}

// Device address of an argument: None stays NULL, an integer is taken as the address itself.
void *ptr(PyObject *o) {
  if (o == Py_None) return nullptr;
  if (THPVariable_Check(o)) {
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_contiguous()) fail(PyExc_ValueError, "tensor arguments must be contiguous");
    return t.data_ptr();
  }
  if (!PyLong_Check(o)) fail(PyExc_TypeError, "a tensor, an address or None is expected");
  void *p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw bad_arg();
  return p;
}
template <typename T> T *ptr_as(PyObject *o) { return static_cast<T *>(ptr(o)); }

int int_of(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw bad_arg();
  return (int)v;
}
int64_t int64_of(PyObject *o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw bad_arg();
  return v;
}
float float_of(PyObject *o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw bad_arg();
  return (float)v;
}

ag_dtype dtype_of(const at::Tensor &t) {
  if (t.scalar_type() == at::kBFloat16) return AG_BF16;
  if (t.scalar_type() == at::kFloat) return AG_F32;
  PyErr_Format(PyExc_ValueError, "unsupported tensor dtype %s", c10::toString(t.scalar_type()));
  throw bad_arg();
}

int64_t dim(const at::Tensor &t, int want, int i) {
  if (t.dim() != want) fail(PyExc_ValueError, "a tensor argument has the wrong number of dimensions");
  return t.size(i);
}

// A size of a tensor of which nothing else is looked at: it may have any number of dimensions beyond that one.
int64_t size_of(const at::Tensor &t, int i) {
  if (t.dim() <= i) fail(PyExc_IndexError, "a tensor argument has too few dimensions");
  return t.size(i);
}

// The struct behind a ctypes structure (None: NULL).  The caller holds a reference to it for the length of the call.
template <typename T> T *struct_of(PyObject *o) {
  if (o == Py_None) return nullptr;
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw bad_arg();
  void *p = b.buf;
  const bool fits = b.len == (Py_ssize_t)sizeof(T);
  PyBuffer_Release(&b);
  if (!fits) fail(PyExc_TypeError, "a structure of another type");
  return static_cast<T *>(p);
}

// stream argument: None = torch's current stream, an integer = the handle, else an object with a cuda_stream attribute
void *stream_of(PyObject *o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  if (PyLong_Check(o)) return ptr(o);
  PyObject *a = PyObject_GetAttrString(o, "cuda_stream");
  if (!a) throw bad_arg();
  void *p = PyLong_AsVoidPtr(a);
  Py_DECREF(a);
  if (!p && PyErr_Occurred()) throw bad_arg();
  return p;
}

// Runs the C call without the interpreter lock (a launch can wait for room in the queue) and returns its status.
template <typename F> PyObject *call(F &&f) {
  ag_status st;
  Py_BEGIN_ALLOW_THREADS st = f();
  Py_END_ALLOW_THREADS return PyLong_FromLong((long)st);
}

// Every function takes (context, stream, arguments of the Python entry point...).
#define AG_BINDING(name, count)                                                                          \
  PyObject *name##_(ag_ctx *ctx, void *s, PyObject *const *a);                                            \
  PyObject *name(PyObject *, PyObject *const *a, Py_ssize_t n) {                                          \
    try {                                                                                                \
      if (n != 2 + (count)) fail(PyExc_TypeError, #name ": wrong number of arguments");                    \
      ag_ctx *ctx = ptr_as<ag_ctx>(a[0]);                                                                 \
      return name##_(ctx, stream_of(a[1]), a + 2);                                                        \
    } catch (const bad_arg &) {                                                                          \
      return nullptr;                                                                                    \
    } catch (const std::exception &e) {                                                                  \
      PyErr_SetString(PyExc_RuntimeError, e.what());                                                      \
      return nullptr;                                                                                    \
    }                                                                                                    \
  }                                                                                                      \
  PyObject *name##_(ag_ctx *ctx, void *s, PyObject *const *a)

// feat, w_gate, bias, tau, n_sink, logits_out, flags_out
AG_BINDING(gate, 7) {
  const at::Tensor &x = tensor(a[0]), &w = tensor(a[1]);
  const int B = dim(x, 3, 0), L = dim(x, 3, 1), d = dim(x, 3, 2), H = size_of(w, 1), n_sink = int_of(a[4]);
  const ag_dtype dt = dtype_of(x);
  const void *xp = ptr(a[0]), *wp = ptr(a[1]);
  const float *bias = ptr_as<float>(a[2]), tau = float_of(a[3]);
  float *logits = ptr_as<float>(a[5]);
  uint8_t *flags = ptr_as<uint8_t>(a[6]);
  return call([&] { return ag_gate(ctx, s, xp, dt, B, L, d, wp, bias, H, tau, n_sink, logits, flags); });
}

// h, norm_w, eps, w_gate, bias, tau, n_sink, x_out, logits_out, flags_out
AG_BINDING(rmsnorm_gate, 10) {
  const at::Tensor &h = tensor(a[0]), &w = tensor(a[3]);
  const int B = dim(h, 3, 0), L = dim(h, 3, 1), d = dim(h, 3, 2), H = size_of(w, 1), n_sink = int_of(a[6]);
  const ag_dtype dt = dtype_of(h);
  const void *hp = ptr(a[0]), *g = ptr(a[1]), *wp = ptr(a[3]);
  const float eps = float_of(a[2]), *bias = ptr_as<float>(a[4]), tau = float_of(a[5]);
  void *xo = ptr(a[7]);
  float *logits = ptr_as<float>(a[8]);
  uint8_t *flags = ptr_as<uint8_t>(a[9]);
  return call([&] { return ag_rmsnorm_gate(ctx, s, hp, dt, B, L, d, g, eps, wp, bias, H, tau, n_sink, xo, logits, flags); });
}

// k, v, flags, pos0, cache
AG_BINDING(compact_kv, 5) {
  const int L = size_of(tensor(a[0]), 2), pos0 = int_of(a[3]);
  const void *k = ptr(a[0]), *v = ptr(a[1]);
  const uint8_t *f = ptr_as<uint8_t>(a[2]);
  ag_kv_cache *c = struct_of<ag_kv_cache>(a[4]);
  return call([&] { return ag_compact_kv(ctx, s, k, v, f, L, pos0, c); });
}

// flags, room, total_rows, row_off, rows_needed
AG_BINDING(pack_row_off, 5) {
  const at::Tensor &f = tensor(a[0]);
  const int B = dim(f, 3, 0), H = dim(f, 3, 1), L = dim(f, 3, 2), room = int_of(a[1]);
  const int64_t total = int64_of(a[2]);
  const uint8_t *fp = ptr_as<uint8_t>(a[0]);
  int64_t *ro = ptr_as<int64_t>(a[3]), *need = ptr_as<int64_t>(a[4]);
  return call([&] { return ag_pack_row_off(ctx, s, fp, B, H, L, room, total, ro, need); });
}

// x, w_kv, flags, pos0, kv_out, cache
AG_BINDING(project_compact_kv, 6) {
  const at::Tensor &x = tensor(a[0]);
  const int B = dim(x, 3, 0), L = dim(x, 3, 1), d = dim(x, 3, 2), pos0 = int_of(a[3]);
  const ag_dtype dt = dtype_of(x);
  const void *xp = ptr(a[0]), *w = ptr(a[1]);
  const uint8_t *f = ptr_as<uint8_t>(a[2]);
  void *kv = ptr(a[4]);
  ag_kv_cache *c = struct_of<ag_kv_cache>(a[5]);
  return call([&] { return ag_project_compact_kv(ctx, s, xp, dt, B, L, d, w, f, pos0, kv, c); });
}

// q, k, v, flags, scale, cache, n_recent, out
AG_BINDING(prefill_attn, 8) {
  const at::Tensor &q = tensor(a[0]);
  const int B = dim(q, 4, 0), Hq = dim(q, 4, 1), L = dim(q, 4, 2), D = dim(q, 4, 3), Hkv = size_of(tensor(a[1]), 1), n = int_of(a[6]);
  const ag_dtype dt = dtype_of(q);
  const void *qp = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = ptr_as<uint8_t>(a[3]);
  const float scale = float_of(a[4]);
  const ag_kv_cache *c = struct_of<ag_kv_cache>(a[5]);
  void *out = ptr(a[7]);
  return call([&] { return ag_prefill_attn_recent(ctx, s, qp, k, v, f, B, L, Hq, Hkv, D, dt, scale, c, n, out); });
}

// q, k, v, flags, scale, pos0, cache, n_recent, out
AG_BINDING(compact_prefill_attn, 9) {
  const at::Tensor &q = tensor(a[0]);
  const int B = dim(q, 4, 0), Hq = dim(q, 4, 1), L = dim(q, 4, 2), D = dim(q, 4, 3), Hkv = size_of(tensor(a[1]), 1);
  const int pos0 = int_of(a[5]), n = int_of(a[7]);
  const ag_dtype dt = dtype_of(q);
  const void *qp = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = ptr_as<uint8_t>(a[3]);
  const float scale = float_of(a[4]);
  ag_kv_cache *c = struct_of<ag_kv_cache>(a[6]);
  void *out = ptr(a[8]);
  return call([&] { return ag_compact_prefill_attn(ctx, s, qp, k, v, f, B, L, Hq, Hkv, D, dt, scale, pos0, c, n, out); });
}

// q, k_new, v_new, new_flags, pos, scale, cache, ring, out
AG_BINDING(decode_attn, 9) {
  const at::Tensor &q = tensor(a[0]);
  const int Hq = size_of(q, 1), pos = int_of(a[4]);
  const void *qp = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = ptr_as<uint8_t>(a[3]);
  const float scale = float_of(a[5]);
  ag_kv_cache *c = struct_of<ag_kv_cache>(a[6]);
  ag_recent_ring *r = struct_of<ag_recent_ring>(a[7]);
  void *out = ptr(a[8]);
  return call([&] { return ag_decode_attn_recent(ctx, s, qp, k, v, f, pos, Hq, scale, c, r, out); });
}

// q, k_new, v_new, new_flags, pos, scale, cache, out
AG_BINDING(decode_attn_static, 8) {
  const at::Tensor &q = tensor(a[0]);
  const int Hq = size_of(q, 1), pos = int_of(a[4]);
  const void *qp = ptr(a[0]), *k = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = ptr_as<uint8_t>(a[3]);
  const float scale = float_of(a[5]);
  ag_kv_cache *c = struct_of<ag_kv_cache>(a[6]);
  void *out = ptr(a[7]);
  return call([&] { return ag_decode_attn_static(ctx, s, qp, k, v, f, pos, Hq, scale, c, out); });
}

// k, v, flags, pos0, ring
AG_BINDING(recent_fill, 5) {
  const at::Tensor &k = tensor(a[0]);
  const int B = dim(k, 4, 0), H = dim(k, 4, 1), L = dim(k, 4, 2), D = dim(k, 4, 3), pos0 = int_of(a[3]);
  const ag_dtype dt = dtype_of(k);
  const void *kp = ptr(a[0]), *v = ptr(a[1]);
  const uint8_t *f = ptr_as<uint8_t>(a[2]);
  ag_recent_ring *r = struct_of<ag_recent_ring>(a[4]);
  return call([&] { return ag_recent_fill(ctx, s, kp, v, f, B, L, H, D, dt, pos0, r); });
}

// x, w_qkv, h_prime, d_prime, w_o, bias, tau, n_sink, logits_out, flags_out
AG_BINDING(gate_mha, 10) {
  const at::Tensor &x = tensor(a[0]), &wo = tensor(a[4]);
  const int B = dim(x, 3, 0), L = dim(x, 3, 1), d = dim(x, 3, 2), H = size_of(wo, 1);
  const int hp = int_of(a[2]), dp = int_of(a[3]), n_sink = int_of(a[7]);
  const ag_dtype dt = dtype_of(x);
  const void *xp = ptr(a[0]), *w = ptr(a[1]), *wop = ptr(a[4]);
  const float *bias = ptr_as<float>(a[5]), tau = float_of(a[6]);
  float *logits = ptr_as<float>(a[8]);
  uint8_t *flags = ptr_as<uint8_t>(a[9]);
  return call([&] { return ag_gate_mha(ctx, s, xp, dt, B, L, d, w, hp, dp, wop, bias, H, tau, n_sink, logits, flags); });
}

void like(const at::Tensor &t, const at::Tensor &other, const char *msg) {
  if (t.scalar_type() != other.scalar_type() || t.sizes() != other.sizes()) fail(PyExc_ValueError, msg);
}
// One byte for each of a call's n tokens of the units, or None.
const uint8_t *flags_of(PyObject *o, int64_t n) {
  if (THPVariable_Check(o) && (tensor(o).element_size() != 1 || tensor(o).numel() != n))
    fail(PyExc_ValueError, "flags are not one byte for every token of every KV head");
  return ptr_as<uint8_t>(o);
}

// q, k, rope, q_out, k_out
AG_BINDING(rotate, 5) {
  const at::Tensor &q = tensor(a[0]);
  const int B = dim(q, 4, 0), Hq = dim(q, 4, 1), L = dim(q, 4, 2), D = dim(q, 4, 3);
  int Hkv = 0;
  if (a[1] != Py_None) {
    const at::Tensor &k = tensor(a[1]);
    Hkv = dim(k, 4, 1);
    if (k.scalar_type() != q.scalar_type() || k.size(0) != B || k.size(2) != L || k.size(3) != D)
      fail(PyExc_ValueError, "rotate: q and k differ in more than their heads");
    if (THPVariable_Check(a[4])) like(tensor(a[4]), k, "rotate: k_out and k differ");
  }
  if (THPVariable_Check(a[3])) like(tensor(a[3]), q, "rotate: q_out and q differ");
  const ag_dtype dt = dtype_of(q);
  const void *qp = ptr(a[0]), *k = ptr(a[1]);
  const ag_rope *r = struct_of<ag_rope>(a[2]);
  void *qo = ptr(a[3]), *ko = ptr(a[4]);
  return call([&] { return ag_rotate(ctx, s, qp, k, dt, B, Hq, Hkv, L, D, r, qo, ko); });
}

// The shape of a call's tensors against the cache's: [B, Hkv, (L,) D] in bf16.
void like_cache(const at::Tensor &t, const ag_q8_cache *c, int dims) {
  if (t.scalar_type() != at::kBFloat16) fail(PyExc_ValueError, "the paged 8-bit cache takes bf16 tensors");
  if (c && (dim(t, dims, 0) != c->B || t.size(1) != c->Hkv || t.size(dims - 1) != c->D))
    fail(PyExc_ValueError, "a tensor's shape differs from the cache's");
}

// k, v, flags, rope, cache
AG_BINDING(q8_append, 5) {
  const at::Tensor &k = tensor(a[0]);
  const int L = dim(k, 4, 2);
  const ag_rope *r = struct_of<ag_rope>(a[3]);
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[4]);
  like_cache(k, c, 4);
  like(tensor(a[1]), k, "k and v differ");
  const void *kp = ptr(a[0]), *v = ptr(a[1]);
  const uint8_t *f = flags_of(a[2], k.size(0) * k.size(1) * L);
  return call([&] { return ag_q8_append(ctx, s, kp, v, f, L, r, c); });
}

// q, k, v, flags, rope, scale, cache, out
AG_BINDING(q8_prefill_attn, 8) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
  const int Hq = dim(q, 4, 1), L = dim(q, 4, 2);
  const ag_rope *r = struct_of<ag_rope>(a[4]);
  const float scale = float_of(a[5]);
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[6]);
  like_cache(k, c, 4);
  like(tensor(a[2]), k, "k and v differ");
  like(tensor(a[7]), q, "out and q differ");
  if (q.scalar_type() != k.scalar_type() || q.size(0) != k.size(0) || k.size(2) != L || q.size(3) != k.size(3))
    fail(PyExc_ValueError, "q and k differ in more than their heads");
  const void *qp = ptr(a[0]), *kp = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = flags_of(a[3], k.size(0) * k.size(1) * L);
  void *out = ptr(a[7]);
  return call([&] { return ag_q8_prefill_attn(ctx, s, qp, kp, v, f, L, Hq, r, scale, c, out); });
}

// q, k_new, v_new, new_flags, rope, scale, cache, out
AG_BINDING(q8_decode_attn, 8) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
  const int Hq = dim(q, 3, 1);
  const ag_rope *r = struct_of<ag_rope>(a[4]);
  const float scale = float_of(a[5]);
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[6]);
  like_cache(k, c, 3);
  like(tensor(a[2]), k, "k_new and v_new differ");
  like(tensor(a[7]), q, "out and q differ");
  if (q.scalar_type() != k.scalar_type() || q.size(0) != k.size(0) || q.size(2) != k.size(2))
    fail(PyExc_ValueError, "q and k_new differ in more than their heads");
  const void *qp = ptr(a[0]), *kp = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = flags_of(a[3], k.size(0) * k.size(1));
  void *out = ptr(a[7]);
  return call([&] { return ag_q8_decode_attn(ctx, s, qp, kp, v, f, Hq, r, scale, c, out); });
}

// int32 numbers, n of them.
int32_t *ints_of(PyObject *o, int64_t n, const char *msg) {
  const at::Tensor &t = tensor(o);
  if (t.scalar_type() != at::kInt || t.numel() != n) fail(PyExc_ValueError, msg);
  return ptr_as<int32_t>(o);
}

// q, k, q_weight, k_weight, eps, rope, q_out, k_out
AG_BINDING(norm_rotate, 8) {
  const at::Tensor &q = tensor(a[0]);
  const int B = dim(q, 4, 0), Hq = dim(q, 4, 1), L = dim(q, 4, 2), D = dim(q, 4, 3);
  int Hkv = 0;
  if (a[1] != Py_None) {
    const at::Tensor &k = tensor(a[1]);
    Hkv = dim(k, 4, 1);
    if (k.scalar_type() != q.scalar_type() || k.size(0) != B || k.size(2) != L || k.size(3) != D)
      fail(PyExc_ValueError, "norm_rotate: q and k differ in more than their heads");
    if (THPVariable_Check(a[7])) like(tensor(a[7]), k, "norm_rotate: k_out and k differ");
  }
  for (int i = 2; i < 4; ++i)
    if (THPVariable_Check(a[i]) && (tensor(a[i]).scalar_type() != q.scalar_type() || tensor(a[i]).numel() != D))
      fail(PyExc_ValueError, "norm_rotate: a weight is not one value of the vectors' type for each of theirs");
  if (THPVariable_Check(a[6])) like(tensor(a[6]), q, "norm_rotate: q_out and q differ");
  const ag_dtype dt = dtype_of(q);
  const void *qp = ptr(a[0]), *k = ptr(a[1]), *qw = ptr(a[2]), *kw = ptr(a[3]);
  const float eps = float_of(a[4]);
  const ag_rope *r = struct_of<ag_rope>(a[5]);
  void *qo = ptr(a[6]), *ko = ptr(a[7]);
  return call([&] { return ag_norm_rotate(ctx, s, qp, k, dt, B, Hq, Hkv, L, D, qw, kw, eps, r, qo, ko); });
}

// q, k, v, flags, parent, rope, scale, cache, out
AG_BINDING(q8_tree_attn, 9) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
  const int Hq = dim(q, 4, 1), L = dim(q, 4, 2);
  const ag_rope *r = struct_of<ag_rope>(a[5]);
  const float scale = float_of(a[6]);
  const ag_q8_cache *c = struct_of<ag_q8_cache>(a[7]);
  like_cache(k, c, 4);
  like(tensor(a[2]), k, "k and v differ");
  like(tensor(a[8]), q, "out and q differ");
  if (q.scalar_type() != k.scalar_type() || q.size(0) != k.size(0) || k.size(2) != L || q.size(3) != k.size(3))
    fail(PyExc_ValueError, "q and k differ in more than their heads");
  const void *qp = ptr(a[0]), *kp = ptr(a[1]), *v = ptr(a[2]);
  const uint8_t *f = flags_of(a[3], k.size(0) * k.size(1) * L);
  const int32_t *parent = ints_of(a[4], k.size(0) * L, "parent is not an int32 number for every node");
  void *out = ptr(a[8]);
  return call([&] { return ag_q8_tree_attn(ctx, s, qp, kp, v, f, parent, L, Hq, r, scale, c, out); });
}

// k, v, flags, parent, last, rope, cache
AG_BINDING(q8_tree_append, 7) {
  const at::Tensor &k = tensor(a[0]);
  const int L = dim(k, 4, 2);
  const ag_rope *r = struct_of<ag_rope>(a[5]);
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[6]);
  like_cache(k, c, 4);
  like(tensor(a[1]), k, "k and v differ");
  const void *kp = ptr(a[0]), *v = ptr(a[1]);
  const uint8_t *f = flags_of(a[2], k.size(0) * k.size(1) * L);
  const int32_t *parent = ints_of(a[3], k.size(0) * L, "parent is not an int32 number for every node");
  const int32_t *last = ints_of(a[4], k.size(0), "last is not an int32 number for every sequence");
  return call([&] { return ag_q8_tree_append(ctx, s, kp, v, f, parent, last, L, r, c); });
}

int32_t *ref_of(PyObject *o, const ag_q8_cache *c) { return ints_of(o, c ? c->n_pages : 0, "not an int32 number for every page"); }

// cache, ref, rows
AG_BINDING(q8_reserve, 3) {
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[0]);
  int32_t *ref = ref_of(a[1], c);
  const int64_t rows = int64_of(a[2]);
  if (rows > 0x7fffffff) fail(PyExc_ValueError, "rows does not fit");
  return call([&] { return ag_q8_reserve(ctx, s, c, ref, rows < 0 ? -1 : (int)rows); });
}

// src, parent, dst, ref
AG_BINDING(q8_fork, 4) {
  const ag_q8_cache *from = struct_of<ag_q8_cache>(a[0]);
  ag_q8_cache *to = struct_of<ag_q8_cache>(a[2]);
  const int32_t *parent = ints_of(a[1], to ? to->B : 0, "parent is not an int32 number for every sequence of dst");
  int32_t *ref = ref_of(a[3], from);
  return call([&] { return ag_q8_fork(ctx, s, from, parent, to, ref); });
}

// cache, ref, which
AG_BINDING(q8_release, 3) {
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[0]);
  int32_t *ref = ref_of(a[1], c);
  if (THPVariable_Check(a[2]) && (tensor(a[2]).element_size() != 1 || tensor(a[2]).numel() != (c ? c->B : 0)))
    fail(PyExc_ValueError, "which is not one byte for every sequence");
  const uint8_t *which = ptr_as<uint8_t>(a[2]);
  return call([&] { return ag_q8_release(ctx, s, c, ref, which); });
}

// cache, ref, moved, used
AG_BINDING(q8_compact_pages, 4) {
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[0]);
  int32_t *ref = ref_of(a[1], c), *moved = ref_of(a[2], c), *used = ints_of(a[3], 1, "used is not one int32 number");
  return call([&] { return ag_q8_compact_pages(ctx, s, c, ref, moved, used); });
}

// cache, moved
AG_BINDING(q8_remap, 2) {
  ag_q8_cache *c = struct_of<ag_q8_cache>(a[0]);
  const int32_t *moved = ref_of(a[1], c);
  return call([&] { return ag_q8_remap(ctx, s, c, moved); });
}

#define AG_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {AG_METHOD(gate), AG_METHOD(rmsnorm_gate), AG_METHOD(compact_kv), AG_METHOD(pack_row_off),
                         AG_METHOD(project_compact_kv), AG_METHOD(prefill_attn), AG_METHOD(compact_prefill_attn),
                         AG_METHOD(decode_attn), AG_METHOD(decode_attn_static), AG_METHOD(recent_fill), AG_METHOD(gate_mha),
                         AG_METHOD(rotate), AG_METHOD(q8_append), AG_METHOD(q8_prefill_attn), AG_METHOD(q8_decode_attn),
                         AG_METHOD(norm_rotate), AG_METHOD(q8_tree_attn), AG_METHOD(q8_tree_append), AG_METHOD(q8_reserve),
                         AG_METHOD(q8_fork), AG_METHOD(q8_release), AG_METHOD(q8_compact_pages), AG_METHOD(q8_remap),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Calls into libag on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
