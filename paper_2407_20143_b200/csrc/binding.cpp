// torch tensors to the C calls of the decoding operators.
//
// One token's step is a few microseconds of GPU work per call, less than marshalling tensors through Python
// takes (7 to 11 us a call measured with ctypes, 3 to 4 with this module), so their arguments are checked
// and turned into descriptors here.  The module knows the C calls by the addresses that bind() is given; it
// holds no state but those and the exception class.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <string>
#include <type_traits>

#include "bcp.h"

namespace {

decltype(&bcp_rope) g_rope;
decltype(&bcp_rope_axes) g_rope_axes;
decltype(&bcp_kv_write) g_write;
decltype(&bcp_kv_write_axes) g_write_axes;
decltype(&bcp_kv_read) g_read;
decltype(&bcp_kv_attend) g_attend;
decltype(&bcp_kv_attend_shared) g_shared;
decltype(&bcp_verify_drafts) g_verify;
decltype(&bcp_last_error) g_last_error;
PyObject* g_error;  // BcpError

// Raises BcpError(code, message); returns NULL.
PyObject* raise(int code, const char* fmt, ...) {
  char text[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(text, sizeof text, fmt, ap);
  va_end(ap);
  PyObject* e = PyObject_CallFunction(g_error, "is", code, text);
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  return nullptr;
}
PyObject* result(int rc) {
  if (rc != BCP_OK) return raise(rc, "%s", g_last_error());
  Py_RETURN_NONE;
}

const at::Tensor* tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) {
    raise(BCP_ERR_INVALID, "%s is not a tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

// The device of a call: its first tensor's, which has to be the current one.
bool device_of(PyObject* o, const char* name, int* device) {
  const at::Tensor* t = tensor(o, name);
  if (!t) return false;
  if (!t->is_cuda()) {
    raise(BCP_ERR_INVALID, "%s is not on a CUDA device", name);
    return false;
  }
  *device = t->get_device();
  const int current = c10::cuda::current_device();
  if (*device != current) {
    raise(BCP_ERR_INVALID, "%s is on cuda:%d, but cuda:%d is the current device", name, *device, current);
    return false;
  }
  return true;
}

bool on_device(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }

// The calls leave no trace in autograd's graph: a result without history would end a gradient without a word.
bool no_gradient(const at::Tensor& t, const char* name) {
  if (!t.requires_grad() || !c10::GradMode::is_enabled()) return true;
  raise(BCP_ERR_INVALID, "%s requires a gradient, which this call does not record (rope() does): detach it, or call under torch.no_grad()", name);
  return false;
}

// Counts a write, so that autograd notices where the values from before are still wanted.
void written(PyObject* o) {
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
template <typename... Tensors>
PyObject* result_in(int rc, Tensors... outputs) {
  if (rc == BCP_OK) (written(outputs), ...);
  return result(rc);
}

bool heads(PyObject* o, const char* name, int device, int64_t tokens, int64_t dim, bcp_heads* h) {
  const at::Tensor* p = tensor(o, name);
  if (!p) return false;
  const at::Tensor& t = *p;
  if (!no_gradient(t, name)) return false;
  if (t.dim() != 3) {
    raise(BCP_ERR_INVALID, "%s has %d dimensions; [tokens, heads, head_dim] expected", name, int(t.dim()));
    return false;
  }
  switch (t.scalar_type()) {
    case at::kFloat: h->type = BCP_F32; break;
    case at::kBFloat16: h->type = BCP_BF16; break;
    case at::kHalf: h->type = BCP_F16; break;
    default:
      raise(BCP_ERR_INVALID, "%s is neither float32, bfloat16 nor float16", name);
      return false;
  }
  if (!on_device(t, device)) {
    raise(BCP_ERR_INVALID, "%s is on another device", name);
    return false;
  }
  if (t.size(0) != tokens || t.size(2) != dim) {
    raise(BCP_ERR_MISMATCH, "%s has shape (%lld, %lld, %lld); %lld tokens and vectors of %lld expected", name, (long long)t.size(0),
          (long long)t.size(1), (long long)t.size(2), (long long)tokens, (long long)dim);
    return false;
  }
  if (dim > 1 && t.stride(2) != 1) {
    raise(BCP_ERR_INVALID, "the elements of %s's vectors are not contiguous", name);
    return false;
  }
  if (t.size(1) > 65536) {
    raise(BCP_ERR_INVALID, "%s has %lld heads", name, (long long)t.size(1));
    return false;
  }
  h->data = t.data_ptr();
  // a dimension of one element may carry any stride
  h->token_stride = t.size(0) > 1 ? t.stride(0) : 0;
  h->head_stride = t.size(1) > 1 ? t.stride(1) : 0;
  h->n_heads = uint32_t(t.size(1));
  return true;
}

// A contiguous tensor of indices (or sums) of the given type and shape (n1 < 0: one dimension).
void* index(PyObject* o, const char* name, int device, at::ScalarType type, int64_t n0, int64_t n1 = -1) {
  static char empty[1];  // what a tensor without elements points to is not read
  const at::Tensor* p = tensor(o, name);
  if (!p) return nullptr;
  const at::Tensor& t = *p;
  if (!no_gradient(t, name)) return nullptr;
  if (t.scalar_type() != type || !on_device(t, device)) {
    raise(BCP_ERR_INVALID, "%s must be %s on cuda:%d", name, c10::toString(type), device);
    return nullptr;
  }
  if (t.dim() != (n1 < 0 ? 1 : 2) || t.size(0) != n0 || (n1 >= 0 && t.size(1) != n1) || !t.is_contiguous()) {
    if (n1 < 0)
      raise(BCP_ERR_MISMATCH, "%s must be contiguous, of shape [%lld]", name, (long long)n0);
    else
      raise(BCP_ERR_MISMATCH, "%s must be contiguous, of shape [%lld, %lld]", name, (long long)n0, (long long)n1);
    return nullptr;
  }
  return t.numel() ? t.data_ptr() : empty;
}

// None: the current stream of the device; else a raw handle.
bool stream_of(PyObject* o, int device, void** stream) {
  if (o == Py_None) {
    *stream = c10::cuda::getCurrentCUDAStream(static_cast<c10::DeviceIndex>(device)).stream();
    return true;
  }
  *stream = PyLong_AsVoidPtr(o);
  return !PyErr_Occurred();
}

bool same_device(int device, PyObject* owner, const char* name) {
  if (PyLong_AsLong(owner) == device) return true;
  if (!PyErr_Occurred()) raise(BCP_ERR_INVALID, "%s is on another device", name);
  return false;
}

bool arguments(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, want);
  return n == want;
}

// Positions of each axis, rows of [axes, tokens]; the map gets the stride between them.
void* axis_positions(PyObject* o, int device, int64_t tokens, bcp_rope_axes_map* axes) {
  static char empty[1];
  const at::Tensor* p = tensor(o, "positions");
  if (!p) return nullptr;
  const at::Tensor& t = *p;
  if (t.scalar_type() != at::kLong || !on_device(t, device)) {
    raise(BCP_ERR_INVALID, "positions must be %s on cuda:%d", c10::toString(at::kLong), device);
    return nullptr;
  }
  if (t.dim() != 2 || t.size(0) != axes->n_axes || t.size(1) != tokens || (tokens > 1 && t.stride(1) != 1)) {
    raise(BCP_ERR_MISMATCH, "positions must be of shape [%u, %lld] with contiguous rows, one for each axis", axes->n_axes, (long long)tokens);
    return nullptr;
  }
  axes->axis_stride = t.stride(0);
  return t.numel() ? t.data_ptr() : empty;
}

// rope(table, table device, x, x2 or None, out, out2 or None, positions, transpose, stream[, axes])
PyObject* py_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, n == 10 ? 10 : 9)) return nullptr;
  int device;
  if (!device_of(a[2], "x", &device) || !same_device(device, a[1], "the table")) return nullptr;
  const at::Tensor& x = THPVariable_Unpack(a[2]);
  if (x.dim() != 3) return raise(BCP_ERR_INVALID, "x has %d dimensions; [tokens, heads, head_dim] expected", int(x.dim()));
  const int64_t tokens = x.size(0), dim = x.size(2);
  if (dim > int64_t(BCP_MAX_HEAD_DIM)) return raise(BCP_ERR_INVALID, "vectors of %lld elements; at most %u", (long long)dim, BCP_MAX_HEAD_DIM);
  bcp_heads h[4];
  const bool two = a[3] != Py_None;
  if (!heads(a[2], "x", device, tokens, dim, &h[0]) || !heads(a[4], "out", device, tokens, dim, &h[1])) return nullptr;
  if (two && (!heads(a[3], "x", device, tokens, dim, &h[2]) || !heads(a[5], "out", device, tokens, dim, &h[3]))) return nullptr;
  bcp_rope_axes_map axes;
  const bool by_axes = n == 10;
  if (by_axes) axes = *static_cast<const bcp_rope_axes_map*>(PyLong_AsVoidPtr(a[9]));
  void* const positions = by_axes ? axis_positions(a[6], device, tokens, &axes) : index(a[6], "positions", device, at::kLong, tokens);
  void* stream;
  if (!positions || !stream_of(a[8], device, &stream)) return nullptr;
  const bcp_rope_table* const table = static_cast<const bcp_rope_table*>(PyLong_AsVoidPtr(a[0]));
  const int64_t* const at = static_cast<const int64_t*>(positions);
  const int rc = by_axes ? g_rope_axes(&h[0], &h[1], two ? &h[2] : nullptr, two ? &h[3] : nullptr, uint32_t(dim), tokens, table, &axes, at,
                                       a[7] == Py_True, stream)
                         : g_rope(&h[0], &h[1], two ? &h[2] : nullptr, two ? &h[3] : nullptr, uint32_t(dim), tokens, table, at,
                                  a[7] == Py_True, stream);
  return two ? result_in(rc, a[4], a[5]) : result_in(rc, a[4]);
}

// kv_write(cache, cache device, k, v, slots, table or None, table device, positions or None, stream, the cache's keys, its values
// [, axes])
PyObject* py_kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, n == 12 ? 12 : 11)) return nullptr;
  const bcp_kv_cache* cache = static_cast<const bcp_kv_cache*>(PyLong_AsVoidPtr(a[0]));
  int device;
  if (!device_of(a[2], "k", &device) || !same_device(device, a[1], "the cache")) return nullptr;
  const bool turn = a[5] != Py_None;
  if (turn != (a[7] != Py_None)) return raise(BCP_ERR_INVALID, "rope and positions go together");
  if (turn && !same_device(device, a[6], "the table")) return nullptr;
  const at::Tensor& first = THPVariable_Unpack(a[2]);
  const int64_t tokens = first.dim() ? first.size(0) : 0;
  bcp_heads k, v;
  if (!heads(a[2], "k", device, tokens, cache->head_dim, &k) || !heads(a[3], "v", device, tokens, cache->head_dim, &v)) return nullptr;
  void* const slots = index(a[4], "slots", device, at::kLong, tokens);
  bcp_rope_axes_map axes;
  const bool by_axes = n == 12;
  if (by_axes) axes = *static_cast<const bcp_rope_axes_map*>(PyLong_AsVoidPtr(a[11]));
  void* positions = nullptr;
  if (slots && turn) positions = by_axes ? axis_positions(a[7], device, tokens, &axes) : index(a[7], "positions", device, at::kLong, tokens);
  void* stream;
  if (!slots || (turn && !positions) || !stream_of(a[8], device, &stream)) return nullptr;
  const bcp_rope_table* const table = turn ? static_cast<const bcp_rope_table*>(PyLong_AsVoidPtr(a[5])) : nullptr;
  const int64_t *const to = static_cast<const int64_t*>(slots), *const at = static_cast<const int64_t*>(positions);
  return result_in(by_axes ? g_write_axes(cache, &k, &v, to, tokens, table, &axes, at, stream) : g_write(cache, &k, &v, to, tokens, table, at, stream),
                   a[9], a[10]);
}

// kv_read(cache, cache device, slots, k, v, stream)
PyObject* py_kv_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 6)) return nullptr;
  const bcp_kv_cache* cache = static_cast<const bcp_kv_cache*>(PyLong_AsVoidPtr(a[0]));
  int device;
  if (!device_of(a[2], "slots", &device) || !same_device(device, a[1], "the cache")) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(a[2]);
  const int64_t tokens = t.dim() ? t.size(0) : 0;
  void* const slots = index(a[2], "slots", device, at::kLong, tokens);
  bcp_heads k, v;
  void* stream;
  if (!slots || !heads(a[3], "k", device, tokens, cache->head_dim, &k) || !heads(a[4], "v", device, tokens, cache->head_dim, &v) ||
      !stream_of(a[5], device, &stream))
    return nullptr;
  return result_in(g_read(cache, static_cast<const int64_t*>(slots), tokens, &k, &v, stream), a[3], a[4]);
}

// kv_attend(cache, cache device, q, out, lse, block_table, lengths, scale, window, workspace, its bytes, its device, stream)
PyObject* py_kv_attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 13)) return nullptr;
  const bcp_kv_cache* cache = static_cast<const bcp_kv_cache*>(PyLong_AsVoidPtr(a[0]));
  int device;
  if (!device_of(a[2], "q", &device) || !same_device(device, a[1], "the cache") || !same_device(device, a[11], "the workspace")) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(a[2]);
  if (t.dim() != 3) return raise(BCP_ERR_INVALID, "q has %d dimensions; [sequences, heads, head_dim] expected", int(t.dim()));
  const int64_t seqs = t.size(0);
  if (seqs > 0x7fffffff) return raise(BCP_ERR_INVALID, "%lld sequences", (long long)seqs);
  bcp_heads q, out;
  if (!heads(a[2], "q", device, seqs, cache->head_dim, &q) || !heads(a[3], "out", device, seqs, cache->head_dim, &out)) return nullptr;
  void* const lse = index(a[4], "lse", device, at::kFloat, seqs, t.size(1));
  void* const lengths = lse ? index(a[6], "lengths", device, at::kInt, seqs) : nullptr;
  const at::Tensor* const table = lengths ? tensor(a[5], "block_table") : nullptr;
  if (!table) return nullptr;
  if (table->dim() != 2 || table->size(0) != seqs || table->scalar_type() != at::kInt || !on_device(*table, device) ||
      (table->size(1) > 1 && table->stride(1) != 1) || table->size(1) > 0x7fffffff)
    return raise(BCP_ERR_INVALID, "block_table must be an int32 tensor [%lld, width] on cuda:%d with contiguous rows", (long long)seqs, device);
  const double scale = PyFloat_AsDouble(a[7]);
  const long long window = PyLong_AsLongLong(a[8]);
  const uint64_t bytes = PyLong_AsUnsignedLongLong(a[10]);
  if (PyErr_Occurred()) return nullptr;
  if (window < 0) return raise(BCP_ERR_INVALID, "window %lld is negative", window);
  void* stream;
  if (!stream_of(a[12], device, &stream)) return nullptr;
  static int32_t no_pages[1];  // a table without columns is not read
  return result_in(g_attend(cache, &q, &out, static_cast<float*>(lse), uint32_t(seqs),
                            table->numel() ? static_cast<const int32_t*>(table->data_ptr()) : no_pages, seqs > 1 ? table->stride(0) : table->size(1),
                            uint32_t(table->size(1)), static_cast<const int32_t*>(lengths), float(scale),
                            uint32_t(window > 0x7fffffff ? 0x7fffffff : window), PyLong_AsVoidPtr(a[9]), bytes, stream),
                   a[3], a[4]);
}

// A block table: int32 rows, contiguous; what a table without columns points to is not read.
struct Table {
  const int32_t* data;
  int64_t stride;
  uint32_t width;
};
bool block_table(PyObject* o, const char* name, int device, int64_t rows, Table* out) {
  static int32_t no_pages[1];
  const at::Tensor* const t = tensor(o, name);
  if (!t) return false;
  if (t->dim() != 2 || (rows >= 0 && t->size(0) != rows) || t->scalar_type() != at::kInt || !on_device(*t, device) ||
      (t->size(1) > 1 && t->stride(1) != 1) || t->size(0) > 0x7fffffff || t->size(1) > 0x7fffffff) {
    raise(BCP_ERR_INVALID, "%s must be an int32 tensor [%s, width] on cuda:%d with contiguous rows", name,
          rows >= 0 ? std::to_string(rows).c_str() : "prefixes", device);
    return false;
  }
  out->data = t->numel() ? static_cast<const int32_t*>(t->data_ptr()) : no_pages;
  out->stride = t->size(0) > 1 ? t->stride(0) : t->size(1);
  out->width = uint32_t(t->size(1));
  return true;
}

// kv_attend_shared(cache, cache device, q, out, lse, prefix_table, prefix_lengths, starts, block_table, lengths, scale, workspace, its bytes,
// its device, stream)
PyObject* py_kv_attend_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 15)) return nullptr;
  const bcp_kv_cache* cache = static_cast<const bcp_kv_cache*>(PyLong_AsVoidPtr(a[0]));
  int device;
  if (!device_of(a[2], "q", &device) || !same_device(device, a[1], "the cache") || !same_device(device, a[13], "the workspace")) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(a[2]);
  if (t.dim() != 3) return raise(BCP_ERR_INVALID, "q has %d dimensions; [sequences, heads, head_dim] expected", int(t.dim()));
  const int64_t seqs = t.size(0);
  if (seqs > 0x7fffffff) return raise(BCP_ERR_INVALID, "%lld sequences", (long long)seqs);
  bcp_heads q, out;
  if (!heads(a[2], "q", device, seqs, cache->head_dim, &q) || !heads(a[3], "out", device, seqs, cache->head_dim, &out)) return nullptr;
  void* const lse = index(a[4], "lse", device, at::kFloat, seqs, t.size(1));
  Table prefix, own;
  if (!lse || !block_table(a[5], "prefix_table", device, -1, &prefix) || !block_table(a[8], "block_table", device, seqs, &own)) return nullptr;
  const int64_t prefixes = THPVariable_Unpack(a[5]).size(0);
  void* const prefix_lengths = index(a[6], "prefix_lengths", device, at::kInt, prefixes);
  void* const starts = prefix_lengths ? index(a[7], "starts", device, at::kInt, prefixes + 1) : nullptr;
  void* const lengths = starts ? index(a[9], "lengths", device, at::kInt, seqs) : nullptr;
  if (!lengths) return nullptr;
  const double scale = PyFloat_AsDouble(a[10]);
  const uint64_t bytes = PyLong_AsUnsignedLongLong(a[12]);
  if (PyErr_Occurred()) return nullptr;
  void* stream;
  if (!stream_of(a[14], device, &stream)) return nullptr;
  return result_in(g_shared(cache, &q, &out, static_cast<float*>(lse), uint32_t(seqs), prefix.data, prefix.stride, prefix.width,
                            static_cast<const int32_t*>(prefix_lengths), static_cast<const int32_t*>(starts), uint32_t(prefixes), own.data, own.stride,
                            own.width, static_cast<const int32_t*>(lengths), float(scale), PyLong_AsVoidPtr(a[11]), bytes, stream),
                   a[3], a[4]);
}

// Rows over the vocabulary [sequences, rows, vocab].
bool vocab_rows(PyObject* o, const char* name, int device, int64_t seqs, int64_t rows, int64_t vocab, bcp_vocab_rows* r) {
  const at::Tensor* p = tensor(o, name);
  if (!p) return false;
  const at::Tensor& t = *p;
  if (!no_gradient(t, name)) return false;
  switch (t.scalar_type()) {
    case at::kFloat: r->type = BCP_F32; break;
    case at::kBFloat16: r->type = BCP_BF16; break;
    case at::kHalf: r->type = BCP_F16; break;
    default:
      raise(BCP_ERR_INVALID, "%s is neither float32, bfloat16 nor float16", name);
      return false;
  }
  if (!on_device(t, device)) {
    raise(BCP_ERR_INVALID, "%s is on another device", name);
    return false;
  }
  if (t.dim() != 3 || t.size(0) != seqs || t.size(1) != rows || t.size(2) != vocab || (vocab > 1 && t.stride(2) != 1)) {
    raise(BCP_ERR_MISMATCH, "%s must be of shape [%lld, %lld, %lld] with contiguous rows", name, (long long)seqs, (long long)rows, (long long)vocab);
    return false;
  }
  static char empty[16] __attribute__((aligned(16)));  // what a tensor without elements points to is not read
  r->data = t.numel() ? t.data_ptr() : empty;
  r->seq_stride = seqs > 1 ? t.stride(0) : 0, r->row_stride = rows > 1 ? t.stride(1) : 0;
  r->reserved = 0;
  return true;
}

// verify(target, draft or None, drafts, uniform, temperature or None, probabilities, tokens, accepted, stream)
PyObject* py_verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (!arguments(n, 9)) return nullptr;
  int device;
  if (!device_of(a[0], "target", &device)) return nullptr;
  const at::Tensor& z = THPVariable_Unpack(a[0]);
  if (z.dim() != 3 || z.size(1) < 1) return raise(BCP_ERR_INVALID, "target must be [sequences, drafts + 1, vocabulary]");
  const int64_t seqs = z.size(0), drafts = z.size(1) - 1, vocab = z.size(2);
  if (seqs > 0x7fffffff || drafts > int64_t(BCP_MAX_DRAFTS) || vocab > int64_t(BCP_MAX_VOCAB))
    return raise(BCP_ERR_INVALID, "%lld sequences of %lld drafts and a vocabulary of %lld; at most %u drafts and %u tokens", (long long)seqs,
                 (long long)drafts, (long long)vocab, BCP_MAX_DRAFTS, BCP_MAX_VOCAB);
  bcp_vocab_rows target, draft;
  const bool certain = a[1] == Py_None;
  if (!vocab_rows(a[0], "target", device, seqs, drafts + 1, vocab, &target)) return nullptr;
  if (!certain && !vocab_rows(a[1], "draft", device, seqs, drafts, vocab, &draft)) return nullptr;
  void* const x = index(a[2], "drafts", device, at::kLong, seqs, drafts);
  void* const u = x ? index(a[3], "uniform", device, at::kFloat, seqs, drafts + 1) : nullptr;
  void* const t = u && a[4] != Py_None ? index(a[4], "temperature", device, at::kFloat, seqs) : nullptr;
  if (!u || (a[4] != Py_None && !t)) return nullptr;
  void* const tokens = index(a[6], "out", device, at::kLong, seqs, drafts + 1);
  void* const accepted = tokens ? index(a[7], "accepted", device, at::kInt, seqs) : nullptr;
  const int probabilities = PyObject_IsTrue(a[5]);
  void* stream;
  if (!accepted || probabilities < 0 || !stream_of(a[8], device, &stream)) return nullptr;
  return result_in(g_verify(&target, certain ? nullptr : &draft, uint32_t(seqs), uint32_t(drafts), uint32_t(vocab), static_cast<const int64_t*>(x),
                            static_cast<const float*>(u), static_cast<const float*>(t), probabilities, static_cast<int64_t*>(tokens),
                            static_cast<int32_t*>(accepted), stream),
                   a[6], a[7]);
}

// bind(BcpError, addresses of bcp_rope, bcp_rope_axes, bcp_kv_write, bcp_kv_write_axes, bcp_kv_read, bcp_kv_attend,
// bcp_kv_attend_shared, bcp_verify_drafts, bcp_last_error)
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr int kCalls = 9;
  if (!arguments(n, 1 + kCalls)) return nullptr;
  void* f[kCalls];
  for (int i = 0; i < kCalls; ++i) f[i] = PyLong_AsVoidPtr(a[i + 1]);
  if (PyErr_Occurred()) return nullptr;
  Py_INCREF(a[0]);
  Py_XDECREF(g_error);
  g_error = a[0];
  int i = 0;
  auto next = [&](auto& call) { call = reinterpret_cast<std::remove_reference_t<decltype(call)>>(f[i++]); };
  next(g_rope), next(g_rope_axes), next(g_write), next(g_write_axes), next(g_read), next(g_attend), next(g_shared), next(g_verify), next(g_last_error);
  Py_RETURN_NONE;
}

// C++ exceptions (torch's checks) must not reach the interpreter.
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(self, a, n);
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}
template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
constexpr PyMethodDef method(const char* name) {
  return PyMethodDef{name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F>)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method<py_bind>("bind"),       method<py_rope>("rope"),           method<py_kv_write>("kv_write"),
                           method<py_kv_read>("kv_read"), method<py_kv_attend>("kv_attend"),
                           method<py_kv_attend_shared>("kv_attend_shared"), method<py_verify>("verify"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&g_module); }
