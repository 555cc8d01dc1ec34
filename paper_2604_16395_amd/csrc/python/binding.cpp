// Argument marshalling of the per-step calls (append, plan, attention, merge, rotation, linear attention, read-back) for the Python
// package, through the CPython API: a step of small sizes is bound by what the host does between
// its launches, and building the argument structs through ctypes took 9 of the 14 us of a call.
// Every pointer, length and stream is read from the objects on each call; nothing is kept.
//
// Each function returns the library's status, or None where an argument is not of the plain form
// expected here (another type, layout or element type): the caller then takes the ctypes path,
// which words the errors.  The library's functions are handed over as addresses by setup(), so
// that this module follows the library that the package loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstring>

#include "s2l.h"

namespace {

struct Entry {
  s2l_status (*append)(const s2l_kv_cache*, const s2l_batch*, const void*, const void*, void*);
  s2l_status (*plan)(const s2l_batch*, int32_t, int32_t, const s2l_plan_opts*, void*, size_t, s2l_plan_info*, void*);
  s2l_status (*attn[3])(const s2l_kv_cache*, const s2l_batch*, const void*, int32_t, float, void*, float*,
                        const s2l_plan_info*, void*, size_t, void*);   // attention, quantised Q, without the merge
  s2l_status (*fused)(const s2l_kv_cache*, const s2l_batch*, const void*, const void*, const void*, int32_t, float,
                      void*, float*, const s2l_plan_info*, void*, size_t, int32_t*, void*);
  s2l_status (*reduce)(const s2l_batch*, int32_t, void*, float*, const s2l_plan_info*, const void*, size_t, void*);
  decltype(&s2l_rope_qk) rope_qk;
  decltype(&s2l_rope_kv_append) rope_append;
  decltype(&s2l_linear_attn) linear;
  decltype(&s2l_norm_rope_qk) norm_rope_qk;
  decltype(&s2l_norm_rope_kv_append) norm_rope_append;
  decltype(&s2l_kv_read) read;
} lib;

PyObject *tensor_type, *cache_type, *batch_type, *opts_type, *info_type, *stream_type, *bf16, *f32, *u8, *is_initialized, *get_device, *get_stream,
    *rope_type, *state_type, *i32, *norm_type, *parameter_type;
PyObject *s_dtype, *s_data_ptr, *s_is_contiguous, *s_shape, *s_numel, *s_k_pages, *s_v_pages, *s_k_scale, *s_v_scale,
    *s_fp8, *s_prefix_host, *s_chunk_host, *s_tables_host, *s_prefix_lens, *s_chunk_lens, *s_cu_chunk, *s_block_tables,
    *s_cuda_stream, *s_stride, *s_get_device, *s_inv_freq, *s_positions, *s_pair_axis, *s_adjacent, *s_scale, *s_states, *s_log_decay,
    *s_slot_in, *s_slot_out, *s_mxfp4, *s_q_weight, *s_k_weight, *s_eps, *s_offset, *s_dim;

// Owned reference, released at the end of the scope.
struct Ref {
  PyObject* o;
  explicit Ref(PyObject* p) : o(p) {}
  Ref(const Ref&) = delete;
  ~Ref() { Py_XDECREF(o); }
  explicit operator bool() const { return o != nullptr; }
};

bool to_ptr(PyObject* number, void** p) {
  *p = PyLong_AsVoidPtr(number);
  return !PyErr_Occurred();
}

bool data_ptr(PyObject* t, void** p) {
  const Ref v(PyObject_CallMethodNoArgs(t, s_data_ptr));
  return v && PyLong_CheckExact(v.o) && to_ptr(v.o, p);
}

// A contiguous tensor of the element type; None only where allowed (a NULL pointer).
bool tensor(PyObject* t, PyObject* dtype, void** p, bool none_ok = false) {
  *p = nullptr;
  if (t == Py_None) return none_ok;
  if ((PyObject*)Py_TYPE(t) != tensor_type) return false;
  const Ref d(PyObject_GetAttr(t, s_dtype));
  if (!d || d.o != dtype) return false;
  const Ref c(PyObject_CallMethodNoArgs(t, s_is_contiguous));
  return c && c.o == Py_True && data_ptr(t, p);
}

bool attr_data_ptr(PyObject* o, PyObject* name, void** p) {
  const Ref t(PyObject_GetAttr(o, name));
  return t && (PyObject*)Py_TYPE(t.o) == tensor_type && data_ptr(t.o, p);
}

bool numel(PyObject* t, size_t* n) {
  const Ref v(PyObject_CallMethodNoArgs(t, s_numel));
  if (!v) return false;
  *n = PyLong_AsSize_t(v.o);
  return !PyErr_Occurred();
}

// A contiguous int32 buffer held by an attribute (a numpy array).
struct HostArray {
  Py_buffer b{};
  bool held = false;
  ~HostArray() {
    if (held) PyBuffer_Release(&b);
  }
  bool take(PyObject* o, PyObject* name, int ndim) {
    const Ref a(PyObject_GetAttr(o, name));
    if (!a || PyObject_GetBuffer(a.o, &b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) return false;
    held = true;
    return b.ndim == ndim && b.itemsize == 4 && b.format && b.format[0] == 'i' && b.format[1] == 0;
  }
};

struct BatchArg {
  s2l_batch c{};
  HostArray prefix, chunk;
  bool take(PyObject* o) {
    if ((PyObject*)Py_TYPE(o) != batch_type) return false;
    HostArray tables;
    void* p[4];
    if (!prefix.take(o, s_prefix_host, 1) || !chunk.take(o, s_chunk_host, 1) || !tables.take(o, s_tables_host, 2) ||
        chunk.b.shape[0] != prefix.b.shape[0] || tables.b.shape[1] > INT32_MAX ||
        !attr_data_ptr(o, s_prefix_lens, &p[0]) || !attr_data_ptr(o, s_chunk_lens, &p[1]) ||
        !attr_data_ptr(o, s_cu_chunk, &p[2]) || !attr_data_ptr(o, s_block_tables, &p[3]))
      return false;
    c.num_reqs = (int32_t)prefix.b.shape[0];
    c.max_pages_per_req = (int32_t)tables.b.shape[1];
    c.prefix_lens = static_cast<const int32_t*>(p[0]);
    c.chunk_lens = static_cast<const int32_t*>(p[1]);
    c.cu_chunk = static_cast<const int32_t*>(p[2]);
    c.block_tables = static_cast<const int32_t*>(p[3]);
    c.prefix_lens_host = static_cast<const int32_t*>(prefix.b.buf);
    c.chunk_lens_host = static_cast<const int32_t*>(chunk.b.buf);
    return true;
  }
};

bool cache_arg(PyObject* o, s2l_kv_cache* c) {
  if ((PyObject*)Py_TYPE(o) != cache_type) return false;
  *c = s2l_kv_cache{};
  const Ref k(PyObject_GetAttr(o, s_k_pages)), fp8(PyObject_GetAttr(o, s_fp8));
  if (!k || !fp8 || (PyObject*)Py_TYPE(k.o) != tensor_type || (fp8.o != Py_True && fp8.o != Py_False)) return false;
  const Ref shape(PyObject_GetAttr(k.o, s_shape)), mx(PyObject_GetAttr(o, s_mxfp4));
  if (!shape || !mx || !PyTuple_Check(shape.o) || PyTuple_GET_SIZE(shape.o) != (mx.o == Py_True ? 3 : 4)) return false;
  int32_t n[4];
  for (int i = 0; i < (int)PyTuple_GET_SIZE(shape.o); ++i) {
    const long long x = PyLong_AsLongLong(PyTuple_GET_ITEM(shape.o, i));
    if (PyErr_Occurred() || x < 0 || x > INT32_MAX) return false;
    n[i] = (int32_t)x;
  }
  void *ks = nullptr, *vs = nullptr;
  if (mx.o == Py_True) {   // both pools in full, as they may be others than those that the cache was made of
    const Ref v(PyObject_GetAttr(o, s_v_pages));
    if (n[2] != S2L_MXFP4_RUN_BYTES || fp8.o == Py_True || !v || !tensor(k.o, u8, &c->k_pages) || !tensor(v.o, u8, &c->v_pages)) return false;
    const Ref v_shape(PyObject_GetAttr(v.o, s_shape));
    if (!v_shape || PyObject_RichCompareBool(shape.o, v_shape.o, Py_EQ) != 1) return false;
    n[2] = S2L_PAGE_SIZE;
    n[3] = S2L_HEAD_DIM;
  } else if (!data_ptr(k.o, &c->k_pages) || !attr_data_ptr(o, s_v_pages, &c->v_pages)) {
    return false;
  }
  if (fp8.o == Py_True && (!attr_data_ptr(o, s_k_scale, &ks) || !attr_data_ptr(o, s_v_scale, &vs))) return false;
  c->k_scale = static_cast<const float*>(ks);
  c->v_scale = static_cast<const float*>(vs);
  c->num_pages = n[0];
  c->num_kv_heads = n[1];
  c->page_size = n[2];
  c->head_dim = n[3];
  c->dtype = mx.o == Py_True ? S2L_KV_MXFP4 : fp8.o == Py_True ? S2L_KV_FP8_E4M3 : S2L_KV_BF16;
  return true;
}

// None: the current stream of the current device (number `dev`, where the caller has it); a number; or a torch.cuda.Stream.
bool stream_arg(PyObject* s, void** p, long dev = -1) {
  if (s == Py_None && dev >= 0) {
    const Ref number(PyLong_FromLong(dev));
    const Ref raw(number ? PyObject_CallOneArg(get_stream, number.o) : nullptr);
    return raw && to_ptr(raw.o, p);
  }
  if (s == Py_None) {
    const Ref ready(PyObject_CallNoArgs(is_initialized));
    if (!ready || ready.o != Py_True) return false;
    const Ref dev(PyObject_CallNoArgs(get_device));
    if (!dev) return false;
    const Ref raw(PyObject_CallOneArg(get_stream, dev.o));
    return raw && to_ptr(raw.o, p);
  }
  if (PyLong_CheckExact(s)) return to_ptr(s, p);
  if (PyObject_IsInstance(s, stream_type) != 1) return false;
  const Ref raw(PyObject_GetAttr(s, s_cuda_stream));
  return raw && PyLong_CheckExact(raw.o) && to_ptr(raw.o, p);
}

// A ctypes structure of exactly this type; None only where allowed.
template <typename T>
struct StructArg {
  Py_buffer b{};
  bool held = false;
  T* p = nullptr;
  ~StructArg() {
    if (held) PyBuffer_Release(&b);
  }
  bool take(PyObject* o, PyObject* type, bool none_ok = false) {
    if (o == Py_None) return none_ok;
    if ((PyObject*)Py_TYPE(o) != type || PyObject_GetBuffer(o, &b, PyBUF_WRITABLE) != 0) return false;
    held = true;
    p = static_cast<T*>(b.buf);
    return b.len == (Py_ssize_t)sizeof(T);
  }
};

bool int_arg(PyObject* o, int32_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  const long x = PyLong_AsLong(o);
  if (PyErr_Occurred() || x < INT32_MIN || x > INT32_MAX) return false;
  *v = (int32_t)x;
  return true;
}

// The current device's index; none before the GPU is in use.
bool current_device(long* dev) {
  const Ref ready(PyObject_CallNoArgs(is_initialized));
  if (!ready || ready.o != Py_True) return false;
  const Ref d(PyObject_CallNoArgs(get_device));
  if (!d) return false;
  *dev = PyLong_AsLong(d.o);
  return !PyErr_Occurred();
}
bool on_device(PyObject* t, long dev) {
  const Ref d(PyObject_CallMethodNoArgs(t, s_get_device));
  return d && PyLong_AsLong(d.o) == dev && !PyErr_Occurred();
}

// Shape and strides, in elements, of a tensor of `ndim` dimensions.
bool layout(PyObject* t, int ndim, int64_t* shape, int64_t* stride) {
  const Ref sh(PyObject_GetAttr(t, s_shape)), st(PyObject_CallMethodNoArgs(t, s_stride));
  if (!sh || !st || !PyTuple_Check(sh.o) || !PyTuple_Check(st.o) || PyTuple_GET_SIZE(sh.o) != ndim || PyTuple_GET_SIZE(st.o) != ndim)
    return false;
  for (int i = 0; i < ndim; ++i) {
    shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh.o, i));
    stride[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(st.o, i));
  }
  return !PyErr_Occurred();
}

// Shape of a tensor of three dimensions.
bool shape3(PyObject* t, int64_t* shape) {
  const Ref sh(PyObject_GetAttr(t, s_shape));
  if (!sh || !PyTuple_Check(sh.o) || PyTuple_GET_SIZE(sh.o) != 3) return false;
  for (int i = 0; i < 3; ++i) shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(sh.o, i));
  return !PyErr_Occurred();
}
bool is_vector(PyObject* t) {
  const Ref d(PyObject_CallMethodNoArgs(t, s_dim));
  return d && PyLong_AsLong(d.o) == 1 && !PyErr_Occurred();
}

// A device tensor of rows [>= tokens][heads][128], each row's heads contiguous.
struct Rows {
  void* p = nullptr;
  int64_t stride = 0;
  int32_t heads = 0;
  bool take(PyObject* t, int64_t tokens, long dev) {
    int64_t n[3], s[3];
    if ((PyObject*)Py_TYPE(t) != tensor_type) return false;
    const Ref d(PyObject_GetAttr(t, s_dtype));
    if (!d || d.o != bf16 || !layout(t, 3, n, s) || n[0] < tokens || n[1] > INT32_MAX || n[2] != S2L_HEAD_DIM || s[2] != 1 ||
        (n[1] > 1 && s[1] != S2L_HEAD_DIM) || !on_device(t, dev) || !data_ptr(t, &p))
      return false;
    stride = s[0];
    heads = (int32_t)n[1];
    return true;
  }
};

int64_t total_tokens(const s2l_batch& b) {
  int64_t n = 0;
  for (int32_t r = 0; r < b.num_reqs; ++r) n += b.chunk_lens_host[r] > 0 ? b.chunk_lens_host[r] : 0;
  return n;
}

// The batch, on the current device.
bool batch_on_device(PyObject* o, BatchArg* batch, int64_t* tokens, long* dev) {
  if (!current_device(dev) || !batch->take(o)) return false;
  const Ref c(PyObject_GetAttr(o, s_chunk_lens));
  *tokens = total_tokens(batch->c);
  return c && on_device(c.o, *dev);
}

// An attribute that is a contiguous device tensor of `dtype`; its element count.
bool attr_tensor(PyObject* o, PyObject* name, PyObject* dtype, long dev, void** p, size_t* n) {
  const Ref t(PyObject_GetAttr(o, name));
  return t && tensor(t.o, dtype, p) && numel(t.o, n) && on_device(t.o, dev);
}

// The cache's pages, and the scales that e4m3 pages come with, are on the device.
bool cache_on_device(PyObject* o, const s2l_kv_cache& c, long dev) {
  PyObject* const names[] = {s_k_pages, s_v_pages, s_k_scale, s_v_scale};
  for (int i = 0; i < (c.dtype == S2L_KV_FP8_E4M3 ? 4 : 2); ++i) {
    const Ref t(PyObject_GetAttr(o, names[i]));
    if (!t || !on_device(t.o, dev)) return false;
  }
  return true;
}

bool rope_arg(PyObject* o, int64_t tokens, long dev, s2l_rope* r) {
  if ((PyObject*)Py_TYPE(o) != rope_type) return false;
  *r = s2l_rope{};
  void* f;
  size_t pairs;
  if (!attr_tensor(o, s_inv_freq, f32, dev, &f, &pairs) || pairs > 64) return false;
  r->inv_freq = static_cast<const float*>(f);
  r->rot_dim = 2 * (int32_t)pairs;
  r->num_axes = 1;
  const Ref pos(PyObject_GetAttr(o, s_positions)), axis(PyObject_GetAttr(o, s_pair_axis)), adj(PyObject_GetAttr(o, s_adjacent)),
      scale(PyObject_GetAttr(o, s_scale));
  if (!pos || !axis || !adj || !scale || !PyBytes_CheckExact(axis.o) || PyBytes_GET_SIZE(axis.o) != sizeof r->pair_axis ||
      !PyFloat_CheckExact(scale.o) || (adj.o != Py_True && adj.o != Py_False))
    return false;
  std::memcpy(r->pair_axis, PyBytes_AS_STRING(axis.o), sizeof r->pair_axis);
  r->flags = adj.o == Py_True ? S2L_ROPE_ADJACENT : 0;
  r->scale = (float)PyFloat_AS_DOUBLE(scale.o);
  if (pos.o == Py_None) return true;
  if ((PyObject*)Py_TYPE(pos.o) != tensor_type) return false;
  const Ref d(PyObject_GetAttr(pos.o, s_dtype));
  int64_t n[2] = {1, 0}, s[2] = {0, 1};
  void* p;
  if (!d || d.o != i32 || (!layout(pos.o, 2, n, s) && !layout(pos.o, 1, n + 1, s + 1)) || n[0] < 1 || n[0] > S2L_ROPE_MAX_AXES || n[1] < tokens || s[1] != 1 || s[0] < 0 ||
      !on_device(pos.o, dev) || !data_ptr(pos.o, &p))
    return false;
  r->positions = static_cast<const int32_t*>(p);
  r->pos_stride = s[0];
  r->num_axes = (int32_t)n[0];
  return true;
}

// A QKNorm's weight: None, or a contiguous device vector of 128 (a tensor, or a module's parameter) of the type that
// `dtype` names, which the first weight sets.
bool weight_arg(PyObject* o, PyObject* name, long dev, int32_t* dtype, const void** w) {
  const Ref t(PyObject_GetAttr(o, name));
  *w = nullptr;
  if (!t || t.o == Py_None) return t.o == Py_None;
  if ((PyObject*)Py_TYPE(t.o) != tensor_type && (PyObject*)Py_TYPE(t.o) != parameter_type) return false;
  const Ref d(PyObject_GetAttr(t.o, s_dtype)), c(PyObject_CallMethodNoArgs(t.o, s_is_contiguous));
  const int32_t type = d.o == f32 ? S2L_NORM_FP32 : d.o == bf16 ? S2L_NORM_BF16 : -1;
  void* p;
  size_t n;
  if (type < 0 || (*dtype >= 0 && type != *dtype) || c.o != Py_True || !numel(t.o, &n) || n != S2L_HEAD_DIM || !is_vector(t.o) ||
      !on_device(t.o, dev) || !data_ptr(t.o, &p))
    return false;
  *dtype = type;
  *w = p;
  return true;
}

bool norm_arg(PyObject* o, long dev, s2l_qk_norm* n) {
  if ((PyObject*)Py_TYPE(o) != norm_type) return false;
  *n = s2l_qk_norm{};
  int32_t dtype = -1;
  const Ref eps(PyObject_GetAttr(o, s_eps)), offset(PyObject_GetAttr(o, s_offset));
  if (!eps || !offset || !PyFloat_CheckExact(eps.o) || !PyFloat_CheckExact(offset.o) ||
      !weight_arg(o, s_q_weight, dev, &dtype, &n->q_weight) || !weight_arg(o, s_k_weight, dev, &dtype, &n->k_weight))
    return false;
  n->eps = (float)PyFloat_AS_DOUBLE(eps.o);
  n->offset = (float)PyFloat_AS_DOUBLE(offset.o);
  n->weight_dtype = dtype < 0 ? S2L_NORM_BF16 : dtype;
  return true;
}

PyObject* general() {   // not the plain form: whatever was raised on the way does not count
  PyErr_Clear();
  Py_RETURN_NONE;
}

template <typename F>
PyObject* call(F f) {
  s2l_status st;
  Py_BEGIN_ALLOW_THREADS st = f();
  Py_END_ALLOW_THREADS return PyLong_FromLong(st);
}

// (cache, batch, k_new, v_new, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  s2l_kv_cache cache;
  BatchArg batch;
  void *k, *v, *stream;
  if (n != 5 || !tensor(a[2], bf16, &k) || !tensor(a[3], bf16, &v) || !cache_arg(a[0], &cache) || !batch.take(a[1]) ||
      !stream_arg(a[4], &stream))
    return general();
  return call([&] { return lib.append(&cache, &batch.c, k, v, stream); });
}

// (batch, hq, hkv, opts, workspace, info, stream)
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
  BatchArg batch;
  StructArg<s2l_plan_opts> opts;
  StructArg<s2l_plan_info> info;
  int32_t hq, hkv;
  void *ws, *stream;
  size_t bytes;
  if (n != 7 || !batch.take(a[0]) || !int_arg(a[1], &hq) || !int_arg(a[2], &hkv) || !opts.take(a[3], opts_type, true) ||
      !tensor(a[4], u8, &ws) || !numel(a[4], &bytes) || !info.take(a[5], info_type) || !stream_arg(a[6], &stream))
    return general();
  return call([&] { return lib.plan(&batch.c, hq, hkv, opts.p, ws, bytes, info.p, stream); });
}

struct AttnArgs {
  s2l_kv_cache cache;
  BatchArg batch;
  StructArg<s2l_plan_info> plan;
  void *q, *out, *lse, *ws, *stream;
  int32_t hq;
  size_t bytes;
  float scale;
  // (cache, batch, q, hq, scale, out, lse, plan, workspace, stream)
  bool take(PyObject* const* a) {
    if (!tensor(a[2], bf16, &q) || !tensor(a[5], bf16, &out) || !tensor(a[6], f32, &lse, true) ||
        !tensor(a[8], u8, &ws) || !numel(a[8], &bytes) || !cache_arg(a[0], &cache) || !batch.take(a[1]) ||
        !int_arg(a[3], &hq) || !PyFloat_CheckExact(a[4]) || !plan.take(a[7], info_type) || !stream_arg(a[9], &stream))
      return false;
    scale = (float)PyFloat_AS_DOUBLE(a[4]);
    return true;
  }
};

// (which, cache, batch, q, hq, scale, out, lse, plan, workspace, stream)
PyObject* attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  AttnArgs x;
  int32_t which;
  if (n != 11 || !int_arg(a[0], &which) || which < 0 || which > 2 || !x.take(a + 1)) return general();
  return call([&] {
    return lib.attn[which](&x.cache, &x.batch.c, x.q, x.hq, x.scale, x.out, static_cast<float*>(x.lse), x.plan.p, x.ws,
                           x.bytes, x.stream);
  });
}

// (cache, batch, q, hq, scale, out, lse, plan, workspace, stream, k_new, v_new): (status, fused)
PyObject* fused(PyObject*, PyObject* const* a, Py_ssize_t n) {
  AttnArgs x;
  void *k, *v;
  if (n != 12 || !tensor(a[10], bf16, &k) || !tensor(a[11], bf16, &v) || !x.take(a)) return general();
  int32_t used = 0;
  s2l_status st;
  Py_BEGIN_ALLOW_THREADS st = lib.fused(&x.cache, &x.batch.c, k, v, x.q, x.hq, x.scale, x.out,
                                        static_cast<float*>(x.lse), x.plan.p, x.ws, x.bytes, &used, x.stream);
  Py_END_ALLOW_THREADS return Py_BuildValue("(iO)", (int)st, used ? Py_True : Py_False);
}

// (batch, hq, out, lse, plan, workspace, stream)
PyObject* reduce(PyObject*, PyObject* const* a, Py_ssize_t n) {
  BatchArg batch;
  StructArg<s2l_plan_info> info;
  int32_t hq;
  void *out, *lse, *ws, *stream;
  size_t bytes;
  if (n != 7 || !tensor(a[2], bf16, &out) || !tensor(a[3], f32, &lse, true) || !tensor(a[5], u8, &ws) ||
      !numel(a[5], &bytes) || !batch.take(a[0]) || !int_arg(a[1], &hq) || !info.take(a[4], info_type) || !stream_arg(a[6], &stream))
    return general();
  return call([&] { return lib.reduce(&batch.c, hq, out, static_cast<float*>(lse), info.p, ws, bytes, stream); });
}

// (batch, rope, q, q_out, k, k_out, stream), with a norm after the batch for norm_rope_qk
PyObject* rotate(PyObject* const* a, Py_ssize_t n, bool normed) {
  BatchArg batch;
  s2l_rope rope;
  s2l_qk_norm norm;
  Rows q, q_out, k, k_out;
  int64_t tokens;
  long dev;
  void* stream;
  if (n != 7 + normed || !batch_on_device(a[0], &batch, &tokens, &dev) || (normed && !norm_arg(a[1], dev, &norm))) return general();
  a += normed;
  if (!rope_arg(a[1], tokens, dev, &rope) || !q.take(a[2], tokens, dev) || !q_out.take(a[3], tokens, dev) || q.heads != q_out.heads ||
      !stream_arg(a[6], &stream, dev))
    return general();
  if (a[4] != Py_None && (!k.take(a[4], tokens, dev) || !k_out.take(a[5], tokens, dev) || k.heads != k_out.heads)) return general();
  return call([&] {
    return normed ? lib.norm_rope_qk(&batch.c, &norm, &rope, q.p, q.stride, q.heads, q_out.p, q_out.stride, k.p, k.stride, k.heads,
                                     k_out.p, k_out.stride, stream)
                  : lib.rope_qk(&batch.c, &rope, q.p, q.stride, q.heads, q_out.p, q_out.stride, k.p, k.stride, k.heads, k_out.p,
                                k_out.stride, stream);
  });
}
PyObject* rope_qk(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotate(a, n, false); }
PyObject* norm_rope_qk(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotate(a, n, true); }

// (cache, batch, rope, q, q_out, k, v, stream), with a norm after the batch for norm_rope_append
PyObject* rotate_append(PyObject* const* a, Py_ssize_t n, bool normed) {
  s2l_kv_cache cache;
  BatchArg batch;
  s2l_rope rope;
  s2l_qk_norm norm;
  Rows q, q_out, k, v;
  int64_t tokens;
  long dev;
  void* stream;
  if (n != 8 + normed || !cache_arg(a[0], &cache) || !batch_on_device(a[1], &batch, &tokens, &dev) ||
      !cache_on_device(a[0], cache, dev) || (normed && !norm_arg(a[2], dev, &norm)))
    return general();
  a += normed;
  if (!rope_arg(a[2], tokens, dev, &rope) || !k.take(a[5], tokens, dev) || !v.take(a[6], tokens, dev) ||
      k.heads != cache.num_kv_heads || v.heads != k.heads || !stream_arg(a[7], &stream, dev))
    return general();
  if (a[3] != Py_None && (!q.take(a[3], tokens, dev) || !q_out.take(a[4], tokens, dev) || q.heads != q_out.heads)) return general();
  return call([&] {
    return normed ? lib.norm_rope_append(&cache, &batch.c, &norm, &rope, q.p, q.stride, q.heads, q_out.p, q_out.stride, k.p, k.stride,
                                         v.p, v.stride, stream)
                  : lib.rope_append(&cache, &batch.c, &rope, q.p, q.stride, q.heads, q_out.p, q_out.stride, k.p, k.stride, v.p,
                                    v.stride, stream);
  });
}
PyObject* rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotate_append(a, n, false); }
PyObject* norm_rope_append(PyObject*, PyObject* const* a, Py_ssize_t n) { return rotate_append(a, n, true); }

// (cache, batch, part, cu_out, k_out, v_out, stream)
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  s2l_kv_cache cache;
  BatchArg batch;
  int32_t part;
  int64_t tokens, rows[3], more[3];
  long dev;
  void *cu, *k, *v, *stream;
  size_t offsets;
  if (n != 7 || !cache_arg(a[0], &cache) || !batch_on_device(a[1], &batch, &tokens, &dev) || !cache_on_device(a[0], cache, dev) ||
      !int_arg(a[2], &part) || !tensor(a[3], i32, &cu) || !numel(a[3], &offsets) || !on_device(a[3], dev) || !is_vector(a[3]) ||
      offsets < (size_t)batch.c.num_reqs || !tensor(a[4], bf16, &k) || !on_device(a[4], dev) || !shape3(a[4], rows) ||
      !tensor(a[5], bf16, &v) || !on_device(a[5], dev) || !shape3(a[5], more) || rows[0] != more[0] ||
      rows[1] != cache.num_kv_heads || more[1] != rows[1] || rows[2] != S2L_HEAD_DIM || more[2] != S2L_HEAD_DIM || !stream_arg(a[6], &stream, dev))
    return general();
  return call([&] { return lib.read(&cache, &batch.c, part, static_cast<const int32_t*>(cu), k, v, rows[0], stream); });
}

// (state, batch, q, k, v, scale, out, workspace, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  BatchArg batch;
  Rows q, k, v, out;
  int64_t tokens, shape[4], stride[4];
  long dev;
  size_t in_slots, out_slots, decays, elements, bytes = 0;
  void *in, *slots, *states, *decay, *ws = nullptr, *st;
  if (n != 9 || (PyObject*)Py_TYPE(a[0]) != state_type || !batch_on_device(a[1], &batch, &tokens, &dev) || !q.take(a[2], tokens, dev) ||
      !k.take(a[3], tokens, dev) || !v.take(a[4], tokens, dev) || !PyFloat_CheckExact(a[5]) || !out.take(a[6], tokens, dev) ||
      k.heads != v.heads || q.heads != out.heads || !stream_arg(a[8], &st, dev) ||
      !attr_tensor(a[0], s_slot_in, i32, dev, &in, &in_slots) || !attr_tensor(a[0], s_slot_out, i32, dev, &slots, &out_slots) ||
      !attr_tensor(a[0], s_log_decay, f32, dev, &decay, &decays) || !attr_tensor(a[0], s_states, f32, dev, &states, &elements))
    return general();
  if (a[7] != Py_None && (!tensor(a[7], u8, &ws) || !numel(a[7], &bytes) || !on_device(a[7], dev))) return general();
  const Ref all(PyObject_GetAttr(a[0], s_states));
  if (!all || !layout(all.o, 4, shape, stride) || shape[0] > INT32_MAX || shape[1] != q.heads || decays != (size_t)q.heads ||
      shape[2] != S2L_HEAD_DIM || shape[3] != S2L_HEAD_DIM || in_slots != (size_t)batch.c.num_reqs || out_slots != in_slots)
    return general();
  const s2l_linear_state state = {static_cast<float*>(states), static_cast<const float*>(decay), static_cast<const int32_t*>(in),
                                  static_cast<const int32_t*>(slots), (int32_t)shape[0], q.heads};
  const float scale = (float)PyFloat_AS_DOUBLE(a[5]);
  return call([&] {
    return lib.linear(&state, &batch.c, q.p, q.stride, k.p, k.stride, v.p, v.stride, k.heads, scale, out.p, out.stride, ws, bytes, st);
  });
}

// (types and dtypes and torch functions as a tuple, entry point addresses as a tuple)
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* f[13];
  PyObject** o[] = {&tensor_type, &cache_type, &batch_type, &opts_type, &info_type, &stream_type,
                    &bf16, &f32, &u8, &is_initialized, &get_device, &get_stream, &rope_type, &state_type, &i32, &norm_type, &parameter_type};
  if (n != 2 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 17 || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 13) {
    PyErr_SetString(PyExc_TypeError, "setup(objects, addresses)");
    return nullptr;
  }
  for (int i = 0; i < 13; ++i)
    if (!to_ptr(PyTuple_GET_ITEM(a[1], i), &f[i])) return nullptr;
  for (int i = 0; i < 17; ++i) {
    Py_INCREF(PyTuple_GET_ITEM(a[0], i));
    Py_XSETREF(*o[i], PyTuple_GET_ITEM(a[0], i));
  }
  lib.append = reinterpret_cast<decltype(lib.append)>(f[0]);
  lib.plan = reinterpret_cast<decltype(lib.plan)>(f[1]);
  for (int i = 0; i < 3; ++i) lib.attn[i] = reinterpret_cast<decltype(lib.attn[0])>(f[2 + i]);
  lib.fused = reinterpret_cast<decltype(lib.fused)>(f[5]);
  lib.reduce = reinterpret_cast<decltype(lib.reduce)>(f[6]);
  lib.rope_qk = reinterpret_cast<decltype(lib.rope_qk)>(f[7]);
  lib.rope_append = reinterpret_cast<decltype(lib.rope_append)>(f[8]);
  lib.linear = reinterpret_cast<decltype(lib.linear)>(f[9]);
  lib.norm_rope_qk = reinterpret_cast<decltype(lib.norm_rope_qk)>(f[10]);
  lib.norm_rope_append = reinterpret_cast<decltype(lib.norm_rope_append)>(f[11]);
  lib.read = reinterpret_cast<decltype(lib.read)>(f[12]);
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(setup), FAST(append), FAST(plan), FAST(attn), FAST(fused), FAST(reduce), FAST(rope_qk),
                         FAST(rope_append), FAST(linear), FAST(norm_rope_qk), FAST(norm_rope_append), FAST(read), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Argument marshalling of the per-step calls.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) {
  const struct {
    PyObject** o;
    const char* s;
  } names[] = {{&s_dtype, "dtype"}, {&s_data_ptr, "data_ptr"}, {&s_is_contiguous, "is_contiguous"}, {&s_shape, "shape"},
               {&s_numel, "numel"}, {&s_k_pages, "k_pages"}, {&s_v_pages, "v_pages"}, {&s_k_scale, "k_scale"},
               {&s_v_scale, "v_scale"}, {&s_fp8, "fp8"}, {&s_prefix_host, "prefix_host"}, {&s_chunk_host, "chunk_host"},
               {&s_tables_host, "tables_host"}, {&s_prefix_lens, "prefix_lens"}, {&s_chunk_lens, "chunk_lens"},
               {&s_cu_chunk, "cu_chunk"}, {&s_block_tables, "block_tables"}, {&s_cuda_stream, "cuda_stream"},
               {&s_stride, "stride"}, {&s_get_device, "get_device"}, {&s_inv_freq, "inv_freq"}, {&s_positions, "positions"},
               {&s_pair_axis, "pair_axis"}, {&s_adjacent, "adjacent"}, {&s_scale, "scale"}, {&s_states, "states"},
               {&s_log_decay, "log_decay"}, {&s_slot_in, "slot_in"}, {&s_slot_out, "slot_out"}, {&s_mxfp4, "mxfp4"},
               {&s_q_weight, "q_weight"}, {&s_k_weight, "k_weight"}, {&s_eps, "eps"}, {&s_offset, "offset"}, {&s_dim, "dim"}};
  for (const auto& n : names)
    if (!(*n.o = PyUnicode_InternFromString(n.s))) return nullptr;
  return PyModule_Create(&module);
}
