// The key/value cache calls of include/rrs.h on torch tensors: a CPython module that checks the
// tensors, allocates outputs and workspaces from torch's caching allocator and makes the C call
// on the current HIP stream. No computation. In C++ because a decode step makes these calls once
// per layer: with the same checks in Python a call took 10 to 15 us of host time (append 11.2,
// attention 9.9, eviction 15.2), more than the kernels of a short cache; here 5.2, 4.7 and 7.6,
// most of it the launch.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "rrs.h"

namespace {

PyObject* g_rrs_error = nullptr;  // RRSError(code, where)

// A Python exception is set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const std::string& what) {
  PyErr_SetString(type, what.c_str());
  throw Raised{};
}

std::string text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + (s.size() == 1 ? ",)" : ")");
}

const char* text(at::ScalarType t) {
  switch (t) {
    case at::kHalf: return "torch.float16";
    case at::kFloat: return "torch.float32";
    case at::kInt: return "torch.int32";
    case at::kByte: return "torch.uint8";
    case at::kBool: return "torch.bool";
    case at::kFloat8_e4m3fn: return "torch.float8_e4m3fn";
    default: return c10::toString(t);
  }
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(name) + " must be a torch.Tensor");
  return THPVariable_Unpack(o);
}

// The GPU that a call is for: that of the tensor which says so.
at::Device gpu_of(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda())
    raise(PyExc_ValueError,
          std::string(name) + " must be a GPU tensor, got " + t.device().str());
  return t.device();
}

const at::Tensor& gpu_tensor(PyObject* o, const char* name, at::ScalarType dtype, at::Device on) {
  const at::Tensor& t = tensor(o, name);
  if (t.device() != on)
    raise(PyExc_ValueError,
          std::string(name) + " must be on " + on.str() + ", got " + t.device().str());
  if (t.scalar_type() != dtype)
    raise(PyExc_TypeError, std::string(name) + " must be " + text(dtype) + ", got " +
                               text(t.scalar_type()));
  return t;
}

// The device pointer of a contiguous tensor of this type and shape on this GPU.
void* dev(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape,
          at::Device on) {
  const at::Tensor& t = gpu_tensor(o, name, dtype, on);
  if (t.sizes() != shape)
    raise(PyExc_ValueError, std::string(name) + " must have shape " + text(shape) + ", got " +
                                text(t.sizes()));
  if (!t.is_contiguous()) raise(PyExc_ValueError, std::string(name) + " must be contiguous");
  return t.data_ptr();
}
void* dev_or_null(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape,
                  at::Device on) {
  return o == Py_None ? nullptr : dev(o, name, dtype, shape, on);
}

int to_int(PyObject* o, const char* name) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < INT32_MIN || v > INT32_MAX)
    raise(PyExc_ValueError, std::string(name) + " is out of range");
  return (int)v;
}

bool to_bool(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised{};
  return v != 0;
}

void arguments(Py_ssize_t got, Py_ssize_t want, const char* name) {
  if (got != want) raise(PyExc_TypeError, std::string(name) + ": wrong number of arguments");
}

PyObject* check(rrs_status s, const char* where, PyObject* result) {
  if (s == RRS_OK) return result;
  Py_XDECREF(result);
  if (PyObject* e = PyObject_CallFunction(g_rrs_error, "is", (int)s, where)) {
    PyErr_SetObject(g_rrs_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}

// The call's device made current, and its current stream.
struct Launch {
  c10::DeviceGuard guard;
  void* stream;
  explicit Launch(at::Device on)
      : guard(on), stream(c10::hip::getCurrentHIPStream(on.index()).stream()) {}
};

struct Cache {
  rrs_kv_cache c{};
  int64_t heads, dim, sequences, capacity;

  // a: k, v, table, k_scale, v_scale
  Cache(PyObject* const* a, at::Device on) {
    const at::Tensor& k = tensor(a[0], "k");
    const at::Tensor& table = tensor(a[2], "table");
    if (k.dim() != 4 || table.dim() != 2)
      raise(PyExc_ValueError, "cache: k must have 4 dimensions and table 2");
    const auto s = k.sizes();
    c.table = static_cast<const int32_t*>(dev(a[2], "table", at::kInt, table.sizes(), on));
    const bool fp8 = k.scalar_type() == at::kFloat8_e4m3fn;
    const bool int4 = !fp8 && (a[3] != Py_None || a[4] != Py_None);
    const auto type = fp8 ? at::kFloat8_e4m3fn : int4 ? at::kByte : at::kHalf;
    c.k = dev(a[0], "k", type, s, on);
    c.v = dev(a[1], "v", type, s, on);
    if (int4 || fp8) {
      const int64_t per_page[3] = {s[0], s[1], fp8 ? s[2] / 16 : s[2]};
      c.k_scale = dev(a[3], "k_scale", at::kHalf, per_page, on);
      c.v_scale = dev(a[4], "v_scale", at::kHalf, per_page, on);
    }
    for (const int64_t x : {s[0], s[1], s[2], 2 * s[3], table.size(0), table.size(1)})
      if (x > INT32_MAX) raise(PyExc_ValueError, "cache: a size is out of range");
    heads = s[1];
    dim = int4 ? 2 * s[3] : s[3];
    sequences = table.size(0);
    capacity = table.size(1) * s[2];
    c.format = fp8 ? RRS_KV_FP8 : int4 ? RRS_KV_INT4 : RRS_KV_F16;
    c.pages = (int32_t)s[0];
    c.kv_heads = (int32_t)heads;
    c.page_size = (int32_t)s[2];
    c.head_dim = (int32_t)dim;
    c.sequences = (int32_t)sequences;
    c.max_pages = (int32_t)table.size(1);
  }

  int bound(PyObject* max_length) const {
    if (max_length != Py_None) return to_int(max_length, "max_length");
    return (int)std::min<int64_t>(capacity, INT32_MAX);
  }
};

// The caller's workspace, or one from the caching allocator on the current stream (which the
// call's launches use too, so the memory is not handed out again before they ran).
struct Workspace {
  at::Tensor keep;
  void* p = nullptr;
  size_t bytes = 0;
  Workspace(PyObject* o, size_t need, at::Device on) {
    if (o != Py_None) {
      const at::Tensor& t = tensor(o, "workspace");
      if (t.device() != on || !t.is_contiguous())
        raise(PyExc_ValueError, "workspace must be contiguous and on " + on.str());
      p = t.data_ptr();
      bytes = t.nbytes();
    } else if (need > 0) {
      keep = at::empty({(int64_t)need}, at::TensorOptions().device(on).dtype(at::kByte));
      p = keep.data_ptr();
      bytes = need;
    }
  }
};

// The memory of an argument, for calls whose outputs may not share any with what they still read.
struct Span {
  const char* name;
  const void* p;
  size_t bytes;
  bool meets(const Span& o) const {
    const char *a = static_cast<const char*>(p), *b = static_cast<const char*>(o.p);
    return bytes > 0 && o.bytes > 0 && a < b + o.bytes && b < a + bytes;
  }
};

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// The first `outputs` spans share memory with none of the others.
void apart(const char* call, const Span* spans, size_t outputs, size_t count) {
  for (size_t i = 0; i < outputs; ++i)
    for (size_t j = i + 1; j < count; ++j)
      if (spans[i].meets(spans[j]))
        raise(PyExc_ValueError, std::string(call) + ": " + spans[i].name + " and " +
                                    spans[j].name + " must not overlap");
}

// A tuple of new tensors.
PyObject* wrap_all(const at::Tensor* t, int n) {
  PyObject* r = PyTuple_New(n);
  for (int i = 0; r && i < n; ++i) {
    PyObject* x = wrap(t[i]);
    if (!x) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i, x);
  }
  return r;
}

// int32 outputs: new ones, or those of the caller's tuple.
struct Int32Out {
  at::Tensor made[6];
  int32_t* p[6];
  Int32Out(PyObject* out, const char* const* names, const std::vector<int64_t>* shapes, int n,
           const at::Tensor& like, at::Device on, const char* what) {
    if (out != Py_None && (!PyTuple_Check(out) || PyTuple_GET_SIZE(out) != n))
      raise(PyExc_TypeError, what);
    for (int i = 0; i < n; ++i) {
      if (out == Py_None) {
        made[i] = at::empty(shapes[i], like.options());
        p[i] = static_cast<int32_t*>(made[i].data_ptr());
      } else {
        p[i] = static_cast<int32_t*>(
            dev(PyTuple_GET_ITEM(out, i), names[i], at::kInt, shapes[i], on));
      }
    }
  }
};

#define RRS_CALL(name)                                                              \
  PyObject* name##_body(PyObject* const* a, Py_ssize_t n);                          \
  PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n) {                     \
    HANDLE_TH_ERRORS                                                                \
    try {                                                                           \
      return name##_body(a, n);                                                     \
    } catch (const Raised&) {                                                       \
      return nullptr;                                                               \
    }                                                                               \
    END_HANDLE_TH_ERRORS                                                            \
  }                                                                                 \
  PyObject* name##_body(PyObject* const* a, Py_ssize_t n)

// qkv, positions, rope, cache (5), seq, slot, heads, sections, interleaved, weights, slot_pos, out
RRS_CALL(rope_kv_append) {
  arguments(n, 16, "rope_kv_append");
  const at::Device on = gpu_of(a[0], "qkv");
  const Cache cache(a + 3, on);
  const int heads = to_int(a[10], "heads");
  const int64_t width = (heads + 2 * cache.heads) * cache.dim;
  const at::Tensor& qkv = tensor(a[0], "qkv");
  if (qkv.scalar_type() != at::kHalf || qkv.dim() != 2 ||
      qkv.size(1) != width || qkv.stride(1) != 1)
    raise(PyExc_ValueError, "qkv must be a float16 GPU tensor (M, " + std::to_string(width) +
                                ") with unit column stride");
  const int64_t M = qkv.size(0);
  if (M > INT32_MAX) raise(PyExc_ValueError, "qkv has too many rows");
  const at::Tensor& positions = tensor(a[1], "positions");
  const int64_t axes = positions.dim() == 2 ? positions.size(1) : 0;
  const void* pp = dev(a[1], "positions", at::kInt, {M, axes}, on);
  const at::Tensor& rope = gpu_tensor(a[2], "rope", at::kFloat, on);
  if (rope.dim() != 2 || rope.size(0) > INT32_MAX || rope.size(1) > INT32_MAX)
    raise(PyExc_ValueError, "rope must have shape (positions, rotary dim)");
  dev(a[2], "rope", at::kFloat, rope.sizes(), on);
  int32_t sections[4] = {};
  if (a[11] == Py_None) {
    if (axes != 1)
      raise(PyExc_ValueError, "sections must name " + std::to_string(axes) + " axes");
    sections[0] = (int32_t)(rope.size(1) / 2);
  } else {
    PyObject* list = PySequence_Fast(a[11], "sections must be a sequence of ints");
    if (!list) throw Raised{};
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(list);
    bool good = count == axes && count <= 4;
    for (Py_ssize_t i = 0; good && i < count; ++i) {
      const long v = PyLong_AsLong(PySequence_Fast_GET_ITEM(list, i));
      good = !(v == -1 && PyErr_Occurred()) && v >= INT32_MIN && v <= INT32_MAX;
      sections[i] = (int32_t)v;
    }
    Py_DECREF(list);
    if (PyErr_Occurred()) throw Raised{};
    if (!good)
      raise(PyExc_ValueError, "sections must name " + std::to_string(axes) + " axes, at most 4");
  }
  const void* sp = dev(a[8], "seq", at::kInt, {M}, on);
  const void* tp = dev(a[9], "slot", at::kInt, {M}, on);
  const int64_t slots[3] = {cache.sequences, cache.heads, cache.capacity};
  void* wp = dev_or_null(a[13], "weights", at::kFloat, slots, on);
  void* op = dev_or_null(a[14], "slot_pos", at::kInt, slots, on);
  at::Tensor made;
  void* qp;
  if (a[15] == Py_None) {
    if (heads < 0) raise(PyExc_ValueError, "heads must be positive");
    made = at::empty({M, heads, cache.dim}, qkv.options());
    qp = made.data_ptr();
  } else {
    qp = dev(a[15], "out", at::kHalf, {M, heads, cache.dim}, on);
  }
  const Launch launch(on);
  const rrs_status s = rrs_rope_kv_append(
      qkv.data_ptr(), M > 1 ? qkv.stride(0) : width, (int)M, heads,
      static_cast<const int32_t*>(pp), (int)axes, sections,
      static_cast<const float*>(rope.data_ptr()), (int)rope.size(0), (int)rope.size(1),
      to_bool(a[12]) ? RRS_ROPE_INTERLEAVED : 0, &cache.c, static_cast<const int32_t*>(sp),
      static_cast<const int32_t*>(tp), qp, static_cast<float*>(wp), static_cast<int32_t*>(op),
      launch.stream);
  if (s != RRS_OK) return check(s, "rrs_rope_kv_append", nullptr);
  return a[15] == Py_None ? wrap(made) : Py_NewRef(a[15]);
}

// Q, cache (5), lengths, max_length, scale, mask, weights, return_lse, workspace, out
RRS_CALL(paged_attention) {
  arguments(n, 14, "paged_attention");
  const at::Device on = gpu_of(a[0], "Q");
  const Cache cache(a + 1, on);
  const at::Tensor& Q = tensor(a[0], "Q");
  const int64_t B = cache.sequences, heads = Q.dim() == 3 ? Q.size(1) : 0;
  if (heads > INT32_MAX) raise(PyExc_ValueError, "Q has too many heads");
  const int64_t shape[3] = {B, heads, cache.dim};
  const void* qp = dev(a[0], "Q", at::kHalf, shape, on);
  const void* lp = dev(a[6], "lengths", at::kInt, {B}, on);
  const int top = cache.bound(a[7]);
  double scale = 1.0 / std::sqrt((double)cache.dim);
  if (a[8] != Py_None) {
    scale = PyFloat_AsDouble(a[8]);
    if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
  }
  const void* mp = dev_or_null(a[9], "mask", at::kBool, {B, cache.capacity}, on);
  void* wp = dev_or_null(a[10], "weights", at::kFloat, {B, cache.heads, cache.capacity}, on);
  const bool want_lse = to_bool(a[11]);
  at::Tensor made, lse;
  void* yp;
  if (a[13] == Py_None) {
    made = at::empty(shape, Q.options());
    yp = made.data_ptr();
  } else {
    yp = dev(a[13], "out", at::kHalf, shape, on);
  }
  if (want_lse) lse = at::empty({B, heads}, Q.options().dtype(at::kFloat));
  const size_t need =
      a[12] == Py_None
          ? rrs_paged_attention_workspace_bytes(&cache.c, (int)heads, top, wp != nullptr)
          : 0;
  const Workspace ws(a[12], need, on);
  const Launch launch(on);
  const rrs_status s = rrs_paged_attention(
      qp, (int)heads, &cache.c, static_cast<const int32_t*>(lp), top, (float)scale,
      static_cast<const uint8_t*>(mp), static_cast<float*>(wp), yp,
      want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, ws.p, ws.bytes, launch.stream);
  if (s != RRS_OK) return check(s, "rrs_paged_attention", nullptr);
  PyObject* y = a[13] == Py_None ? wrap(made) : Py_NewRef(a[13]);
  if (!want_lse || !y) return y;
  PyObject* l = wrap(lse);
  PyObject* both = l ? PyTuple_Pack(2, y, l) : nullptr;
  Py_DECREF(y);
  Py_XDECREF(l);
  return both;
}

// Q, cache (5), row_start, lengths, max_tokens, max_length, scale, mask, return_lse, workspace, out
RRS_CALL(prompt_attention) {
  arguments(n, 15, "prompt_attention");
  const at::Device on = gpu_of(a[0], "Q");
  const Cache cache(a + 1, on);
  const at::Tensor& Q = tensor(a[0], "Q");
  const int64_t B = cache.sequences, M = Q.dim() == 3 ? Q.size(0) : 0;
  const int64_t heads = Q.dim() == 3 ? Q.size(1) : 0;
  if (heads > INT32_MAX || M > INT32_MAX) raise(PyExc_ValueError, "Q is too large");
  const int64_t shape[3] = {M, heads, cache.dim};
  const void* qp = dev(a[0], "Q", at::kHalf, shape, on);
  const void* sp = dev(a[6], "row_start", at::kInt, {B + 1}, on);
  const void* lp = dev(a[7], "lengths", at::kInt, {B}, on);
  const int tokens = a[8] == Py_None ? (int)M : to_int(a[8], "max_tokens");
  const int top = cache.bound(a[9]);
  double scale = 1.0 / std::sqrt((double)cache.dim);
  if (a[10] != Py_None) {
    scale = PyFloat_AsDouble(a[10]);
    if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
  }
  const void* mp = dev_or_null(a[11], "mask", at::kBool, {B, cache.capacity}, on);
  const bool want_lse = to_bool(a[12]);
  at::Tensor made, lse;
  void* yp;
  if (a[14] == Py_None) {
    made = at::empty(shape, Q.options());
    yp = made.data_ptr();
  } else {
    yp = dev(a[14], "out", at::kHalf, shape, on);
  }
  if (want_lse) lse = at::empty({M, heads}, Q.options().dtype(at::kFloat));
  const size_t need = rrs_prompt_attention_workspace_bytes(&cache.c, (int)heads, tokens, top);
  const Workspace ws(a[13], need, on);
  const size_t rows = (size_t)(M * heads * cache.dim) * 2;
  if (a[13] != Py_None || a[14] != Py_None) {
    const size_t pool = THPVariable_Unpack(a[1]).nbytes();
    const size_t scales = a[4] == Py_None ? 0 : THPVariable_Unpack(a[4]).nbytes();
    const Span spans[] = {{"workspace", ws.p, need},
                          {"out", yp, rows},
                          {"Q", qp, rows},
                          {"row_start", sp, (size_t)(B + 1) * 4},
                          {"lengths", lp, (size_t)B * 4},
                          {"mask", mp, mp ? (size_t)(B * cache.capacity) : 0},
                          {"table", cache.c.table, (size_t)B * cache.c.max_pages * 4},
                          {"k", cache.c.k, pool},
                          {"v", cache.c.v, pool},
                          {"k_scale", cache.c.k_scale, scales},
                          {"v_scale", cache.c.v_scale, scales}};
    apart("prompt_attention", spans, 2, sizeof(spans) / sizeof(spans[0]));
  }
  const Launch launch(on);
  const rrs_status s = rrs_prompt_attention(
      qp, (int)M, (int)heads, &cache.c, static_cast<const int32_t*>(sp), tokens,
      static_cast<const int32_t*>(lp), top, (float)scale, static_cast<const uint8_t*>(mp), yp,
      want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, ws.p, ws.bytes, launch.stream);
  if (s != RRS_OK) return check(s, "rrs_prompt_attention", nullptr);
  PyObject* y = a[14] == Py_None ? wrap(made) : Py_NewRef(a[14]);
  if (!want_lse || !y) return y;
  PyObject* l = wrap(lse);
  PyObject* both = l ? PyTuple_Pack(2, y, l) : nullptr;
  Py_DECREF(y);
  Py_XDECREF(l);
  return both;
}

// cache (5), heads, max_tokens, max_length
RRS_CALL(prompt_attention_workspace_bytes) {
  arguments(n, 8, "prompt_attention_workspace_bytes");
  const Cache cache(a, gpu_of(a[0], "k"));
  return PyLong_FromSize_t(rrs_prompt_attention_workspace_bytes(
      &cache.c, to_int(a[5], "heads"), to_int(a[6], "max_tokens"), to_int(a[7], "max_length")));
}

// cache (5), heads, max_length, with_weights
RRS_CALL(paged_attention_workspace_bytes) {
  arguments(n, 8, "paged_attention_workspace_bytes");
  const Cache cache(a, gpu_of(a[0], "k"));
  return PyLong_FromSize_t(rrs_paged_attention_workspace_bytes(
      &cache.c, to_int(a[5], "heads"), to_int(a[6], "max_length"), to_bool(a[7])));
}

// cache (5), lengths, weights, slot_pos, keep_from, budget, max_length, out, workspace
RRS_CALL(kv_evict) {
  arguments(n, 13, "kv_evict");
  const at::Device on = gpu_of(a[5], "lengths");
  const Cache cache(a, on);
  const int64_t B = cache.sequences, h = cache.heads, cap = cache.capacity;
  const void* lp = dev(a[5], "lengths", at::kInt, {B}, on);
  const void* wp = dev(a[6], "weights", at::kFloat, {B, h, cap}, on);
  const void* pp = dev(a[7], "slot_pos", at::kInt, {B, h, cap}, on);
  const void* fp = dev(a[8], "keep_from", at::kInt, {B}, on);
  const int budget = to_int(a[9], "budget"), top = cache.bound(a[10]);
  if (budget < 1 || budget > cap)
    raise(PyExc_ValueError, "budget must be in [1, " + std::to_string(cap) + "], got " +
                                std::to_string(budget));
  const at::Tensor& lengths = THPVariable_Unpack(a[5]);
  const size_t need = rrs_kv_evict_workspace_bytes(&cache.c, top, budget);
  const Workspace ws(a[12], need, on);
  at::Tensor made[4];
  void* out[4];
  if (a[11] == Py_None) {
    made[0] = at::empty({B, h, budget}, lengths.options());
    made[1] = at::empty({B}, lengths.options());
    made[2] = at::empty({B, h, cap}, lengths.options().dtype(at::kFloat));
    made[3] = at::empty({B, h, cap}, lengths.options());
    for (int i = 0; i < 4; ++i) out[i] = made[i].data_ptr();
  } else {
    if (!PyTuple_Check(a[11]) || PyTuple_GET_SIZE(a[11]) != 4)
      raise(PyExc_TypeError, "out must be a tuple (kept, lengths, weights, slot_pos)");
    out[0] = dev(PyTuple_GET_ITEM(a[11], 0), "kept", at::kInt, {B, h, budget}, on);
    out[1] = dev(PyTuple_GET_ITEM(a[11], 1), "new_lengths", at::kInt, {B}, on);
    out[2] = dev(PyTuple_GET_ITEM(a[11], 2), "weights_out", at::kFloat, {B, h, cap}, on);
    out[3] = dev(PyTuple_GET_ITEM(a[11], 3), "pos_out", at::kInt, {B, h, cap}, on);
  }
  // The kernels read the inputs and the cache while they write, in any order.
  if (a[11] != Py_None || a[12] != Py_None) {
    const size_t row = (size_t)B * h, all = row * cap * 4, pool = THPVariable_Unpack(a[0]).nbytes();
    const size_t scales = a[3] == Py_None ? 0 : THPVariable_Unpack(a[3]).nbytes();
    const Span spans[] = {{"workspace", ws.p, need},
                          {"kept", out[0], row * budget * 4},
                          {"new_lengths", out[1], (size_t)B * 4},
                          {"weights_out", out[2], all},
                          {"pos_out", out[3], all},
                          {"lengths", lp, (size_t)B * 4},
                          {"weights", wp, all},
                          {"slot_pos", pp, all},
                          {"keep_from", fp, (size_t)B * 4},
                          {"table", cache.c.table, (size_t)B * cache.c.max_pages * 4},
                          {"k", cache.c.k, pool},
                          {"v", cache.c.v, pool},
                          {"k_scale", cache.c.k_scale, scales},
                          {"v_scale", cache.c.v_scale, scales}};
    const size_t count = sizeof(spans) / sizeof(spans[0]);
    for (size_t i = 0; i < 5; ++i)
      for (size_t j = i + 1; j < count; ++j)
        if (spans[i].meets(spans[j]))
          raise(PyExc_ValueError, std::string("kv_evict: ") + spans[i].name + " and " +
                                      spans[j].name + " must not overlap");
  }
  const Launch launch(on);
  const rrs_status s = rrs_kv_evict(
      &cache.c, static_cast<const int32_t*>(lp), top, static_cast<const float*>(wp),
      static_cast<const int32_t*>(pp), static_cast<const int32_t*>(fp), budget,
      static_cast<int32_t*>(out[0]), static_cast<int32_t*>(out[1]), static_cast<float*>(out[2]),
      static_cast<int32_t*>(out[3]), ws.p, ws.bytes, launch.stream);
  if (s != RRS_OK) return check(s, "rrs_kv_evict", nullptr);
  if (a[11] != Py_None) return Py_NewRef(a[11]);
  PyObject* r = PyTuple_New(4);
  for (int i = 0; r && i < 4; ++i) {
    PyObject* t = wrap(made[i]);
    if (!t) {
      Py_DECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i, t);
  }
  return r;
}

// cache (5), max_length, budget
RRS_CALL(kv_evict_workspace_bytes) {
  arguments(n, 7, "kv_evict_workspace_bytes");
  const Cache cache(a, gpu_of(a[0], "k"));
  return PyLong_FromSize_t(rrs_kv_evict_workspace_bytes(&cache.c, to_int(a[5], "max_length"),
                                                        to_int(a[6], "budget")));
}

// cache (5), lengths, max_length, out
RRS_CALL(kv_read) {
  arguments(n, 8, "kv_read");
  const at::Device on = gpu_of(a[5], "lengths");
  const Cache cache(a, on);
  const int64_t B = cache.sequences;
  const void* lp = dev(a[5], "lengths", at::kInt, {B}, on);
  const at::Tensor& lengths = THPVariable_Unpack(a[5]);
  const int top = cache.bound(a[6]);
  if (top < 1 || top > cache.capacity)
    raise(PyExc_ValueError, "max_length must be in [1, " + std::to_string(cache.capacity) +
                                "], got " + std::to_string(top));
  const int64_t shape[4] = {B, cache.heads, top, cache.dim};
  at::Tensor made[2];
  void* out[2];
  if (a[7] == Py_None) {
    for (int i = 0; i < 2; ++i) {
      made[i] = at::empty(shape, lengths.options().dtype(at::kHalf));
      out[i] = made[i].data_ptr();
    }
  } else {
    if (!PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != 2)
      raise(PyExc_TypeError, "out must be a tuple (K, V)");
    out[0] = dev(PyTuple_GET_ITEM(a[7], 0), "K", at::kHalf, shape, on);
    out[1] = dev(PyTuple_GET_ITEM(a[7], 1), "V", at::kHalf, shape, on);
  }
  const Launch launch(on);
  const rrs_status s = rrs_kv_read(&cache.c, static_cast<const int32_t*>(lp), top, out[0], out[1],
                                   launch.stream);
  if (s != RRS_OK) return check(s, "rrs_kv_read", nullptr);
  if (a[7] != Py_None) return Py_NewRef(a[7]);
  PyObject* k = wrap(made[0]);
  PyObject* v = k ? wrap(made[1]) : nullptr;
  PyObject* both = v ? PyTuple_Pack(2, k, v) : nullptr;
  Py_XDECREF(k);
  Py_XDECREF(v);
  return both;
}

// table, lengths, parent, room, pages, page_size, out, workspace
RRS_CALL(kv_fork) {
  arguments(n, 8, "kv_fork");
  const at::Device on = gpu_of(a[0], "table");
  const at::Tensor& table = tensor(a[0], "table");
  if (table.dim() != 2) raise(PyExc_ValueError, "table must have 2 dimensions");
  const int32_t* tp = static_cast<const int32_t*>(dev(a[0], "table", at::kInt, table.sizes(), on));
  const int64_t S = table.size(0), C = table.size(1);
  if (S > INT32_MAX || C > INT32_MAX) raise(PyExc_ValueError, "table is too large");
  const void* lp = dev(a[1], "lengths", at::kInt, {S}, on);
  const void* pp = dev_or_null(a[2], "parent", at::kInt, {S}, on);
  const void* rp = dev(a[3], "room", at::kInt, {S}, on);
  const int pages = to_int(a[4], "pages"), page_size = to_int(a[5], "page_size");
  static const char* const names[] = {"table_out", "lengths_out", "room_out", "src", "dst", "count"};
  const std::vector<int64_t> shapes[] = {{S, C}, {S}, {S}, {S}, {S}, {2}};
  const Int32Out out(a[6], names, shapes, 6, table, on,
                     "out must be a tuple (table, lengths, room, src, dst, count)");
  const size_t need = rrs_kv_fork_workspace_bytes((int)S, (int)C, page_size, pages);
  const Workspace ws(a[7], need, on);
  if (a[6] != Py_None || a[7] != Py_None) {
    const size_t row = (size_t)S * 4, all = (size_t)S * C * 4;
    const Span spans[] = {{"workspace", ws.p, need}, {names[0], out.p[0], all},
                          {names[1], out.p[1], row}, {names[2], out.p[2], row},
                          {names[3], out.p[3], row}, {names[4], out.p[4], row},
                          {names[5], out.p[5], 8},   {"table", tp, all},
                          {"lengths", lp, row},      {"parent", pp, pp ? row : 0},
                          {"room", rp, row}};
    apart("kv_fork", spans, 7, sizeof(spans) / sizeof(spans[0]));
  }
  const Launch launch(on);
  const rrs_status s =
      rrs_kv_fork(tp, (int)S, (int)C, page_size, pages, static_cast<const int32_t*>(lp),
                  static_cast<const int32_t*>(pp), static_cast<const int32_t*>(rp), out.p[0],
                  out.p[1], out.p[2], out.p[3], out.p[4], out.p[5], ws.p, ws.bytes, launch.stream);
  if (s != RRS_OK) return check(s, "rrs_kv_fork", nullptr);
  return a[6] != Py_None ? Py_NewRef(a[6]) : wrap_all(out.made, 6);
}

// table, lengths, pages, page_size, out, workspace
RRS_CALL(kv_compact) {
  arguments(n, 6, "kv_compact");
  const at::Device on = gpu_of(a[0], "table");
  const at::Tensor& table = tensor(a[0], "table");
  if (table.dim() != 2) raise(PyExc_ValueError, "table must have 2 dimensions");
  const int32_t* tp = static_cast<const int32_t*>(dev(a[0], "table", at::kInt, table.sizes(), on));
  const int64_t S = table.size(0), C = table.size(1);
  if (S > INT32_MAX || C > INT32_MAX) raise(PyExc_ValueError, "table is too large");
  const void* lp = dev(a[1], "lengths", at::kInt, {S}, on);
  const int pages = to_int(a[2], "pages"), page_size = to_int(a[3], "page_size");
  if (pages < 1) raise(PyExc_ValueError, "pages must be positive");
  const int64_t moves = std::max(1, pages / 2);
  static const char* const names[] = {"table_out", "src", "dst", "count"};
  const std::vector<int64_t> shapes[] = {{S, C}, {moves}, {moves}, {2}};
  const Int32Out out(a[4], names, shapes, 4, table, on,
                     "out must be a tuple (table, src, dst, count)");
  const size_t need = rrs_kv_compact_workspace_bytes((int)S, (int)C, page_size, pages);
  const Workspace ws(a[5], need, on);
  if (a[4] != Py_None || a[5] != Py_None) {
    const size_t all = (size_t)S * C * 4, list = (size_t)moves * 4;
    const Span spans[] = {{"workspace", ws.p, need}, {names[0], out.p[0], all},
                          {names[1], out.p[1], list}, {names[2], out.p[2], list},
                          {names[3], out.p[3], 8},    {"table", tp, all},
                          {"lengths", lp, (size_t)S * 4}};
    apart("kv_compact", spans, 5, sizeof(spans) / sizeof(spans[0]));
  }
  const Launch launch(on);
  const rrs_status s = rrs_kv_compact(tp, (int)S, (int)C, page_size, pages,
                                      static_cast<const int32_t*>(lp), out.p[0], out.p[1],
                                      out.p[2], out.p[3], ws.p, ws.bytes, launch.stream);
  if (s != RRS_OK) return check(s, "rrs_kv_compact", nullptr);
  return a[4] != Py_None ? Py_NewRef(a[4]) : wrap_all(out.made, 4);
}

// sequences, max_pages, page_size, pages
RRS_CALL(kv_fork_workspace_bytes) {
  arguments(n, 4, "kv_fork_workspace_bytes");
  return PyLong_FromSize_t(
      rrs_kv_fork_workspace_bytes(to_int(a[0], "sequences"), to_int(a[1], "max_pages"),
                                  to_int(a[2], "page_size"), to_int(a[3], "pages")));
}
RRS_CALL(kv_compact_workspace_bytes) {
  arguments(n, 4, "kv_compact_workspace_bytes");
  return PyLong_FromSize_t(
      rrs_kv_compact_workspace_bytes(to_int(a[0], "sequences"), to_int(a[1], "max_pages"),
                                     to_int(a[2], "page_size"), to_int(a[3], "pages")));
}

// cache (5), src, dst, count
RRS_CALL(kv_copy_pages) {
  arguments(n, 8, "kv_copy_pages");
  const at::Device on = gpu_of(a[0], "k");
  const Cache cache(a, on);
  const at::Tensor& src = tensor(a[5], "src");
  const int64_t pairs = src.dim() == 1 ? src.size(0) : -1;
  if (pairs < 0 || pairs > INT32_MAX) raise(PyExc_ValueError, "src must have 1 dimension");
  const void* sp = dev(a[5], "src", at::kInt, {pairs}, on);
  const void* dp = dev(a[6], "dst", at::kInt, {pairs}, on);
  const void* cp = nullptr;
  if (a[7] != Py_None) {
    const at::Tensor& count = gpu_tensor(a[7], "count", at::kInt, on);
    if (count.numel() < 1) raise(PyExc_ValueError, "count must not be empty");
    cp = dev(a[7], "count", at::kInt, count.sizes(), on);
  }
  if (pairs == 0) Py_RETURN_NONE;
  // The lists are read while pages are written.
  const size_t pool = THPVariable_Unpack(a[0]).nbytes();
  const size_t scales = a[3] == Py_None ? 0 : THPVariable_Unpack(a[3]).nbytes();
  const Span spans[] = {{"k", cache.c.k, pool},
                        {"v", cache.c.v, pool},
                        {"k_scale", cache.c.k_scale, scales},
                        {"v_scale", cache.c.v_scale, scales},
                        {"src", sp, (size_t)pairs * 4},
                        {"dst", dp, (size_t)pairs * 4},
                        {"count", cp, cp ? (size_t)4 : 0}};
  apart("kv_copy_pages", spans, 4, sizeof(spans) / sizeof(spans[0]));
  const Launch launch(on);
  return check(rrs_kv_copy_pages(&cache.c, static_cast<const int32_t*>(sp),
                                 static_cast<const int32_t*>(dp), (int)pairs,
                                 static_cast<const int32_t*>(cp), launch.stream),
               "rrs_kv_copy_pages", Py_NewRef(Py_None));
}

// The exception type for a status other than RRS_OK.
PyObject* set_error(PyObject*, PyObject* type) {
  Py_INCREF(type);
  Py_XSETREF(g_rrs_error, type);
  Py_RETURN_NONE;
}

#define RRS_METHOD(name) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {RRS_METHOD(rope_kv_append),
                          RRS_METHOD(paged_attention),
                          RRS_METHOD(paged_attention_workspace_bytes),
                          RRS_METHOD(kv_evict),
                          RRS_METHOD(kv_evict_workspace_bytes),
                          RRS_METHOD(kv_read),
                          RRS_METHOD(prompt_attention),
                          RRS_METHOD(prompt_attention_workspace_bytes),
                          RRS_METHOD(kv_fork),
                          RRS_METHOD(kv_fork_workspace_bytes),
                          RRS_METHOD(kv_compact),
                          RRS_METHOD(kv_compact_workspace_bytes),
                          RRS_METHOD(kv_copy_pages),
                          {"set_error", set_error, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&kModule); }
