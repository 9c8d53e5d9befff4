// Argument marshalling, in C++, of the cache calls that a generation loop makes every step (binding.py: kv_update, kv_append,
// kv_read, kv_attention).  For a single request the GPU is done in four to five microseconds a call; marshalled by ctypes a
// call took 7 to 12 on the host, 3.3 of them the launch.  Nothing but addresses, sizes, checks and output tensors passes here: the calls
// are libmoin.so's, whose addresses binding.py hands over.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <string>

#include "../../include/moin.h"

namespace {

decltype(&moin_kv_update) f_update;
decltype(&moin_kv_append) f_append;
decltype(&moin_kv_read) f_read;
decltype(&moin_kv_attention_workspace_bytes) f_ws;
decltype(&moin_kv_attention) f_attention;
PyObject* g_error;

struct Refused {};   // a Python exception is set

[[noreturn]] void refuse(const std::string& why) {
  PyErr_SetString(g_error, why.c_str());
  throw Refused();
}
std::string shown(const at::Tensor& t) {
  std::string s = "[";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + "] of " + c10::toString(t.scalar_type()) + " on " + t.device().str();
}
const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) refuse("expected a tensor, got " + std::string(Py_TYPE(o)->tp_name));
  return THPVariable_Unpack(o);
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int32_t size32(PyObject* o) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) refuse("a size of " + std::to_string(v) + " does not fit 32 bits");
  return (int32_t)v;
}
// The library launches on the current device.
bool here(const at::Tensor& t) { return t.is_cuda() && t.get_device() == c10::cuda::current_device(); }
void holder_here(PyObject* device) {   // of a cache, of tables
  const int64_t d = integer(device);
  if (d != c10::cuda::current_device())
    refuse("the cache or tables are on device " + std::to_string(d) + ", the current one is " + std::to_string(c10::cuda::current_device()));
}
// int32 vector of n entries; None: no vector
int32_t* vec(PyObject* o, int64_t n) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kInt || t.numel() != n || !t.is_contiguous() || !here(t))
    refuse("expected " + std::to_string(n) + " contiguous int32 values on the current CUDA device, got " + shown(t));
  return static_cast<int32_t*>(t.data_ptr());
}
int32_t length(const at::Tensor& t) {
  if (t.dim() < 1 || t.size(0) > INT32_MAX) refuse("expected a vector, got " + shown(t));
  return (int32_t)t.size(0);
}
// [T, heads, dim] bf16 (or [T, heads * dim]) whose tokens may lie apart
struct Rows { void* p; int64_t stride; };
Rows rows_of(const at::Tensor& t, int64_t T, int64_t heads, int64_t dim) {
  if (t.scalar_type() != at::kBFloat16 || !here(t) || t.dim() < 2 || t.dim() > 3 || t.size(0) != T ||
      (t.dim() == 3 ? t.size(1) != heads || t.size(2) != dim : t.size(1) != heads * dim))
    refuse("expected bf16 [" + std::to_string(T) + ", " + std::to_string(heads) + ", " + std::to_string(dim) + "] on the current CUDA device, got " + shown(t));
  if (t.is_contiguous()) return {t.data_ptr(), heads * dim};
  if (t.stride(-1) != 1 || (t.dim() == 3 && heads > 1 && t.stride(1) != dim)) refuse("the heads of a token must lie side by side");
  return {t.data_ptr(), T > 1 ? t.stride(0) : heads * dim};
}
// Do rows of `width` elements share memory?  (Queries and results may be parts of the rows of one tensor.)
bool share(const Rows& a, const Rows& b, int64_t T, int64_t width) {
  const int64_t off = (static_cast<char*>(b.p) - static_cast<char*>(a.p)) / 2;   // elements; both are 16-bit, 16-byte aligned (or refused)
  if (T == 0 || off >= (T - 1) * a.stride + width || -off >= (T - 1) * b.stride + width) return false;
  if (a.stride != b.stride) return true;
  const int64_t in = ((off % a.stride) + a.stride) % a.stride;
  return in < width || a.stride - in < width;
}
// [positions, dim / 2, 2] fp32
struct Rope { const float* p; int32_t n; };
Rope rope_of(PyObject* o, int64_t dim) {
  if (o == Py_None) return {nullptr, 0};
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != at::kFloat || !here(t) || !t.is_contiguous() || t.dim() != 3 || t.size(1) * 2 != dim || t.size(2) != 2 || t.size(0) > INT32_MAX)
    refuse("expected a contiguous float32 table [positions, " + std::to_string(dim / 2) + ", 2] on the current CUDA device, got " + shown(t));
  return {static_cast<const float*>(t.data_ptr()), (int32_t)t.size(0)};
}
cudaStream_t stream_of(PyObject* o) {   // None: the current one
  return o == Py_None ? c10::cuda::getCurrentCUDAStream().stream() : reinterpret_cast<cudaStream_t>((intptr_t)integer(o));
}

// A new bf16 tensor beside `like` (on the current CUDA device: the caller has looked) for a call on `stream`, without the dispatcher.
// Its memory belongs to that stream: of a block of the current one, pending work may be anywhere.
at::Tensor fresh(at::IntArrayRef size, const at::Tensor& like, PyObject* stream) {
  auto make = [&] { return at::Tensor(at::detail::empty_cuda(size, at::kBFloat16, like.device(), std::nullopt)); };
  if (stream == Py_None) return make();
  const c10::cuda::CUDAStreamGuard guard(c10::cuda::getStreamFromExternal(stream_of(stream), like.get_device()));
  return make();
}

template <class F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F&& body) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return nullptr;
  }
  try {
    return body();
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    Py_INCREF(a[0]);
    g_error = a[0];
    f_update = reinterpret_cast<decltype(f_update)>((intptr_t)integer(a[1]));
    f_append = reinterpret_cast<decltype(f_append)>((intptr_t)integer(a[2]));
    f_read = reinterpret_cast<decltype(f_read)>((intptr_t)integer(a[3]));
    f_ws = reinterpret_cast<decltype(f_ws)>((intptr_t)integer(a[4]));
    f_attention = reinterpret_cast<decltype(f_attention)>((intptr_t)integer(a[5]));
    Py_RETURN_NONE;
  });
}

// (tables, batch, rows, want, lens_out, n_free_out, stream, their device) -> status; structs by address
PyObject* update(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    holder_here(a[7]);
    const auto* tables = reinterpret_cast<const moin_kv_tables*>((intptr_t)integer(a[0]));
    const auto* batch = reinterpret_cast<const moin_kv_batch*>((intptr_t)integer(a[1]));
    return PyLong_FromLong(f_update(tables, vec(a[2], batch->R), vec(a[3], batch->R), batch, vec(a[4], tables->n_rows), vec(a[5], 1), stream_of(a[6])));
  });
}

// (cache, slot, k, v, pos, rope, stream, the cache's device) -> status
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 8, [&] {
    holder_here(a[7]);
    const auto* kv = reinterpret_cast<const moin_kv*>((intptr_t)integer(a[0]));
    const int32_t T = length(tensor(a[1]));
    const Rows k = rows_of(tensor(a[2]), T, kv->n_kv_heads, kv->head_dim), v = rows_of(tensor(a[3]), T, kv->n_kv_heads, kv->head_dim);
    const Rope rope = rope_of(a[5], kv->head_dim);
    return PyLong_FromLong(f_append(kv, vec(a[1], T), k.p, k.stride, v.p, v.stride, vec(a[4], T), rope.p, rope.n, T, stream_of(a[6])));
  });
}

// (cache, slot, k, v, stream, the cache's device) -> (status, k, v); None for k or v: a new tensor
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    holder_here(a[5]);
    const auto* kv = reinterpret_cast<const moin_kv*>((intptr_t)integer(a[0]));
    const at::Tensor& slot = tensor(a[1]);
    const int32_t T = length(slot);
    const int32_t* s = vec(a[1], T);
    auto out = [&](PyObject* o) { return o == Py_None ? fresh({T, kv->n_kv_heads, kv->head_dim}, slot, a[4]) : tensor(o); };
    const at::Tensor k = out(a[2]), v = out(a[3]);
    const Rows kr = rows_of(k, T, kv->n_kv_heads, kv->head_dim), vr = rows_of(v, T, kv->n_kv_heads, kv->head_dim);
    const int32_t st = f_read(kv, s, kr.p, kr.stride, vr.p, vr.stride, T, stream_of(a[4]));
    return Py_BuildValue("(iNN)", (int)st, THPVariable_Wrap(k), THPVariable_Wrap(v));
  });
}

// (cache, tables, q, cu_q, kv_len, max_q, max_kv, rows, scale, rope, out, stream, device) -> (status, out); None for out: a new tensor, for
// scale: 1 / sqrt(head_dim).  The scratch is a block of the caching allocator that belongs to the stream: given back when the call
// has returned, it is handed out again only to work behind it.
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&] {
    holder_here(a[12]);
    const auto* kv = reinterpret_cast<const moin_kv*>((intptr_t)integer(a[0]));
    const auto* tables = reinterpret_cast<const moin_kv_tables*>((intptr_t)integer(a[1]));
    const at::Tensor& q = tensor(a[2]);
    if (q.dim() != 3) refuse("expected q as [tokens, heads, head_dim], got " + shown(q));
    const int32_t T = length(q), R = length(tensor(a[4]));
    if (q.size(1) > INT32_MAX) refuse("too many heads");
    const int32_t heads = (int32_t)q.size(1);
    const Rows qr = rows_of(q, T, heads, kv->head_dim);
    const at::Tensor out = a[10] == Py_None ? fresh(q.sizes(), q, a[11]) : tensor(a[10]);
    const Rows outr = rows_of(out, T, heads, kv->head_dim);
    if (a[10] != Py_None && share(qr, outr, T, (int64_t)heads * kv->head_dim)) refuse("out may not overlap q: other parts of the call still read it");
    const Rope rope = rope_of(a[9], kv->head_dim);
    int32_t max_q = size32(a[5]);
    if (max_q < 1 || max_q > T) max_q = T;
    int32_t max_kv = size32(a[6]);
    const int64_t capacity = (int64_t)tables->max_pages * tables->page_tokens;
    if (max_kv < 1 || max_kv > capacity) max_kv = (int32_t)std::min<int64_t>(capacity, INT32_MAX);
    double scale = 0;
    if (a[8] != Py_None) {
      scale = PyFloat_AsDouble(a[8]);
      if (PyErr_Occurred()) throw Refused();
    } else {
      scale = kv->head_dim == 64 ? 0.125 : 0.08838834764831845;
    }
    const int32_t *cu = vec(a[3], (int64_t)R + 1), *len = vec(a[4], R), *rows = vec(a[7], R);
    const cudaStream_t s = stream_of(a[11]);
    const size_t bytes = f_ws(R, T, max_q, max_kv, heads, kv->n_kv_heads, kv->head_dim);
    void* ws = c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(bytes, s);
    const int32_t st = f_attention(kv, tables, rows, cu, len, R, T, max_q, max_kv, qr.p, qr.stride, heads, (float)scale, rope.p, rope.n, outr.p,
                                   outr.stride, ws, bytes, s);
    c10::cuda::CUDACachingAllocator::raw_delete(ws);
    return Py_BuildValue("(iN)", (int)st, THPVariable_Wrap(out));
  });
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init), FAST(update), FAST(append), FAST(read), FAST(attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_steps", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__steps() { return PyModule_Create(&module); }
