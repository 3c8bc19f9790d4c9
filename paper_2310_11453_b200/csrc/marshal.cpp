// Compiled argument marshalling for the attention operators (module _marshal, used by binding.py).
//
// A decode step makes several of these calls per layer, each a few microseconds of device time; looking at seven tensors,
// allocating outputs and converting twenty arguments costs 10 microseconds from Python and about 3 from here.  The
// functions check what the Python wrappers document, allocate what was not given, and call the C entry points (whose
// addresses binding.py hands over from the library it loaded).  They return the result, or the bl_status as a number
// where it is not BL_OK; argument errors are ValueError and TypeError.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "../../include/bitlinear.h"

namespace {

using at::Tensor;

struct Entry {
  decltype(&bitlinear_qk_norm_rope) norm_rope;
  decltype(&bitlinear_attention_window) window;
  decltype(&bitlinear_kv4_page_bytes) page_bytes;
  decltype(&bitlinear_kv4_append) append;
  decltype(&bitlinear_kv4_read) read;
  decltype(&bitlinear_attention_kv4) kv4;
  decltype(&bitlinear_attention_kv4_ws_bytes) kv4_ws;
  decltype(&bitlinear_kv4_copy_pages) copy_pages;
} entry;

struct TypeError : std::runtime_error { using std::runtime_error::runtime_error; };

const Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw TypeError(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
std::string shape_of(const Tensor& t) {
  std::string s = "(";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  return s + ")";
}
void check_place(const Tensor& t, const char* name, c10::Device dev, at::ScalarType type) {
  if (!t.is_cuda() || t.device() != dev)
    throw std::invalid_argument(std::string(name) + " is on " + t.device().str() + ", expected a CUDA tensor on the device of the first argument");
  if (t.scalar_type() != type)
    throw TypeError(std::string(name) + " is " + c10::toString(t.scalar_type()) + ", expected " + c10::toString(type));
}
// A token matrix [rows, width] whose rows are contiguous; returns its row stride (of a single row, which has none, any that serves).
int64_t rows_of(const Tensor& t, const char* name, c10::Device dev, at::ScalarType type, int64_t rows, int64_t width) {
  check_place(t, name, dev, type);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != width || t.stride(1) != 1)
    throw std::invalid_argument(std::string(name) + " has shape " + shape_of(t) + ", expected (" + std::to_string(rows) + ", " +
                                std::to_string(width) + ") with the values of a row contiguous");
  return rows > 1 ? t.stride(0) : (width + 7) / 8 * 8;
}
// A contiguous tensor of n values in the given shape (second < 0: one dimension).
void* flat(const Tensor& t, const char* name, c10::Device dev, at::ScalarType type, int64_t first, int64_t second = -1) {
  check_place(t, name, dev, type);
  const bool fits = second < 0 ? t.dim() == 1 && t.size(0) == first : t.dim() == 2 && t.size(0) == first && t.size(1) == second;
  if (!fits || !t.is_contiguous())
    throw std::invalid_argument(std::string(name) + " has shape " + shape_of(t) + ", expected a contiguous (" + std::to_string(first) +
                                (second < 0 ? ",)" : ", " + std::to_string(second) + ")"));
  return t.data_ptr();
}
int64_t whole(PyObject* o, const char* name) {
  const int64_t v = PyLong_Check(o) ? PyLong_AsLongLong(o) : (PyIndex_Check(o) ? PyNumber_AsSsize_t(o, PyExc_OverflowError) : -1);
  if (PyErr_Occurred()) throw python_error();
  if (!PyLong_Check(o) && !PyIndex_Check(o)) throw TypeError(std::string(name) + " must be a whole number");
  return v;
}
int small(PyObject* o, const char* name) {
  const int64_t v = whole(o, name);
  if (v < INT32_MIN || v > INT32_MAX) throw std::invalid_argument(std::string(name) + " does not fit 32 bits");
  return (int)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}
bl_dtype type_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return BL_F32;
    case at::kHalf: return BL_F16;
    case at::kBFloat16: return BL_BF16;
    default: throw TypeError(std::string("unsupported dtype ") + c10::toString(t));
  }
}
c10::Device cuda_device(const Tensor& t, const char* name) {
  if (!t.is_cuda()) throw std::invalid_argument(std::string(name) + " is on " + t.device().str() + ", expected a CUDA tensor");
  return t.device();
}
void* stream_of(c10::Device dev) { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }
void want(Py_ssize_t have, Py_ssize_t n) {
  if (have != n) throw TypeError("expected " + std::to_string(n) + " arguments, got " + std::to_string(have));
}
PyObject* status(bl_status st) { return PyLong_FromLong((long)st); }

// Runs f and turns what it throws into a Python error.
template <typename F> PyObject* guarded(F f) {
  try {
    return f();
  } catch (python_error& e) {
    e.restore();
  } catch (const TypeError& e) {
    PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// The result of a call that may have allocated it: the given object, or the new tensor.
PyObject* given_or(PyObject* given, const Tensor& made) {
  if (given != Py_None) { Py_INCREF(given); return given; }
  return THPVariable_Wrap(made);
}

// q, k, positions, inv_freq, heads, kv_heads, head_dim, wq, wk, eps, interleaved, q_out, k_out
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 13);
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &pos = tensor(a[2], "positions"), &freq = tensor(a[3], "inv_freq");
    const int heads = small(a[4], "heads"), kv = small(a[5], "kv_heads"), dim = small(a[6], "head_dim");
    const c10::Device dev = cuda_device(q, "q");
    const auto type = q.scalar_type();
    const bl_dtype code = type_code(type);
    const int64_t T = q.dim() > 0 ? q.size(0) : 0, wide = (int64_t)heads * dim, narrow = (int64_t)kv * dim, half = freq.numel();
    const int64_t ld_q = rows_of(q, "q", dev, type, T, wide), ld_k = rows_of(k, "k", dev, type, T, narrow);
    void *pp = flat(pos, "positions", dev, at::kInt, T), *fp = flat(freq, "inv_freq", dev, at::kFloat, half);
    void *w1 = a[7] == Py_None ? nullptr : flat(tensor(a[7], "wq"), "wq", dev, type, dim);
    void *w2 = a[8] == Py_None ? nullptr : flat(tensor(a[8], "wk"), "wk", dev, type, dim);
    const float eps = real(a[9]);
    const int inter = PyObject_IsTrue(a[10]);
    if (inter < 0) throw python_error();
    const c10::cuda::CUDAGuard guard(dev);
    const Tensor qo = a[11] == Py_None ? at::empty({T, wide}, q.options()) : tensor(a[11], "q_out");
    const Tensor ko = a[12] == Py_None ? at::empty({T, narrow}, k.options()) : tensor(a[12], "k_out");
    const int64_t ld_qo = rows_of(qo, "q_out", dev, type, T, wide), ld_ko = rows_of(ko, "k_out", dev, type, T, narrow);
    if (2 * half > INT32_MAX) throw std::invalid_argument("inv_freq is too long");
    const bl_status st = entry.norm_rope(q.data_ptr(), k.data_ptr(), code, T, heads, kv, dim, ld_q, ld_k, w1, w2, eps, (int)(2 * half), inter,
                                         (const float*)fp, (const int32_t*)pp, qo.data_ptr(), ko.data_ptr(), ld_qo, ld_ko, stream_of(dev));
    if (st != BL_OK) return status(st);
    PyObject* r = PyTuple_New(2);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, given_or(a[11], qo));
    PyTuple_SET_ITEM(r, 1, given_or(a[12], ko));
    return r;
  });
}

// q, k, v, batch, seq, heads, kv_heads, head_dim, window, sinks, cu_q, cu_k, seq_k, scale, o
PyObject* window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 15);
    const Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const int batch = small(a[3], "batch");
    const int64_t seq = whole(a[4], "seq");
    const int heads = small(a[5], "heads"), kv = small(a[6], "kv_heads"), dim = small(a[7], "head_dim");
    const int win = small(a[8], "window"), sinks = small(a[9], "sinks");
    const c10::Device dev = cuda_device(q, "q");
    const auto type = q.scalar_type();
    const bl_dtype code = type_code(type);
    const int64_t rows = q.dim() > 0 ? q.size(0) : 0, rows_k = k.dim() > 0 ? k.size(0) : 0;
    // Keys with offsets of their own are bounded by the rows of k: the bound of the queries would cut their last tokens off and
    // shift every position.
    const int64_t seq_k = a[12] != Py_None ? whole(a[12], "seq_k") : a[11] == Py_None ? seq : rows_k;
    const int64_t wide = (int64_t)heads * dim, narrow = (int64_t)kv * dim;
    const int64_t ld_q = rows_of(q, "q", dev, type, rows, wide), ld_k = rows_of(k, "k", dev, type, rows_k, narrow);
    const int64_t ld_v = rows_of(v, "v", dev, type, rows_k, narrow);
    void* c1 = a[10] == Py_None ? nullptr : flat(tensor(a[10], "cu_q"), "cu_q", dev, at::kInt, (int64_t)batch + 1);
    void* c2 = a[11] == Py_None ? nullptr : flat(tensor(a[11], "cu_k"), "cu_k", dev, at::kInt, (int64_t)batch + 1);
    const float scale = real(a[13]);
    const c10::cuda::CUDAGuard guard(dev);
    const Tensor o = a[14] == Py_None ? at::empty({rows, wide}, q.options()) : tensor(a[14], "o");
    const int64_t ld_o = rows_of(o, "o", dev, type, rows, wide);
    const bl_status st = entry.window(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), code, batch, (const int32_t*)c1, (const int32_t*)c2,
                                      seq, seq_k, rows, rows_k, heads, kv, dim, ld_q, ld_k, ld_v, ld_o, win, sinks, scale, stream_of(dev));
    return st != BL_OK ? status(st) : given_or(a[14], o);
  });
}

// pages, page_size, kv_heads, head_dim, dtype: the first five arguments of every call on a cache
struct Cache {
  bl_kv4_cache c;
  c10::Device dev;
  at::ScalarType type;
  const Tensor& pages;
  int64_t width;
  explicit Cache(PyObject* const* a) : dev(c10::kCPU), type(at::kHalf), pages(tensor(a[0], "pages")) {
    dev = cuda_device(pages, "pages");
    c.page_size = small(a[1], "page_size"); c.kv_heads = small(a[2], "kv_heads"); c.head_dim = small(a[3], "head_dim");
    const int code = small(a[4], "dtype");
    if (code != BL_F16 && code != BL_BF16) throw TypeError("unsupported dtype of the cache");
    c.dtype = (bl_dtype)code;
    type = code == BL_F16 ? at::kHalf : at::kBFloat16;
    const int64_t bytes = (int64_t)entry.page_bytes(c.page_size, c.kv_heads, c.head_dim);
    if (bytes == 0) throw std::invalid_argument("unsupported cache sizes");
    c.num_pages = pages.dim() == 2 ? pages.size(0) : -1;
    c.pages = flat(pages, "pages", dev, at::kByte, c.num_pages, bytes);
    width = (int64_t)c.kv_heads * c.head_dim;
  }
};

// cache (5): whether it can be used at all
PyObject* cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 5);
    const Cache c(a);
    Py_RETURN_NONE;
  });
}

// cache (5), k, v, slots
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 8);
    const Cache c(a);
    const Tensor &k = tensor(a[5], "k"), &v = tensor(a[6], "v"), &slots = tensor(a[7], "slots");
    const int64_t T = k.dim() > 0 ? k.size(0) : 0;
    const int64_t ld_k = rows_of(k, "k", c.dev, c.type, T, c.width), ld_v = rows_of(v, "v", c.dev, c.type, T, c.width);
    void* sp = flat(slots, "slots", c.dev, at::kLong, T);
    const c10::cuda::CUDAGuard guard(c.dev);
    const bl_status st = entry.append(&c.c, k.data_ptr(), v.data_ptr(), T, ld_k, ld_v, (const int64_t*)sp, stream_of(c.dev));
    if (st != BL_OK) return status(st);
    Py_RETURN_NONE;
  });
}

// cache (5), slots, k, v
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 8);
    const Cache c(a);
    const Tensor& slots = tensor(a[5], "slots");
    const int64_t T = slots.dim() > 0 ? slots.size(0) : 0;
    const c10::cuda::CUDAGuard guard(c.dev);
    const auto options = c.pages.options().dtype(c.type);
    const Tensor k = a[6] == Py_None ? at::zeros({T, c.width}, options) : tensor(a[6], "k");
    const Tensor v = a[7] == Py_None ? at::zeros({T, c.width}, options) : tensor(a[7], "v");
    const int64_t ld_k = rows_of(k, "k", c.dev, c.type, T, c.width), ld_v = rows_of(v, "v", c.dev, c.type, T, c.width);
    void* sp = flat(slots, "slots", c.dev, at::kLong, T);
    const bl_status st = entry.read(&c.c, k.data_ptr(), v.data_ptr(), T, ld_k, ld_v, (const int64_t*)sp, stream_of(c.dev));
    if (st != BL_OK) return status(st);
    PyObject* r = PyTuple_New(2);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, given_or(a[6], k));
    PyTuple_SET_ITEM(r, 1, given_or(a[7], v));
    return r;
  });
}

// cache (5), q, block_table, lens, batch, n_q, heads, window, sinks, scale, o, ws
PyObject* kv4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 16);
    const Cache c(a);
    const Tensor &q = tensor(a[5], "q"), &table = tensor(a[6], "block_table"), &lens = tensor(a[7], "lens");
    const int batch = small(a[8], "batch"), n_q = small(a[9], "n_q"), heads = small(a[10], "heads");
    const int win = small(a[11], "window"), sinks = small(a[12], "sinks");
    const float scale = real(a[13]);
    const int64_t rows = (int64_t)batch * n_q, width = (int64_t)heads * c.c.head_dim;
    const int64_t ld_q = rows_of(q, "q", c.dev, c.type, rows, width);
    const int64_t max_pages = table.dim() == 2 ? table.size(1) : 0;
    void *tp = flat(table, "block_table", c.dev, at::kInt, batch, max_pages), *lp = flat(lens, "lens", c.dev, at::kInt, batch);
    const c10::cuda::CUDAGuard guard(c.dev);
    const Tensor o = a[14] == Py_None ? at::empty({rows, width}, q.options()) : tensor(a[14], "o");
    const int64_t ld_o = rows_of(o, "o", c.dev, c.type, rows, width);
    const int64_t need = (int64_t)entry.kv4_ws(batch, n_q, heads, c.c.kv_heads, c.c.head_dim);
    const Tensor ws = a[15] == Py_None ? at::empty({std::max<int64_t>(need, 256)}, c.pages.options()) : tensor(a[15], "ws");
    void* wp = flat(ws, "ws", c.dev, at::kByte, ws.numel());
    const bl_status st = entry.kv4(q.data_ptr(), batch, n_q, heads, ld_q, &c.c, (const int32_t*)tp, max_pages, (const int32_t*)lp, win, sinks,
                                   scale, o.data_ptr(), ld_o, wp, (size_t)ws.numel(), stream_of(c.dev));
    return st != BL_OK ? status(st) : given_or(a[14], o);
  });
}

// pages, pairs
PyObject* copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 2);
    const Tensor &pages = tensor(a[0], "pages"), &pairs = tensor(a[1], "pairs");
    const c10::Device dev = cuda_device(pages, "pages");
    check_place(pages, "pages", dev, at::kByte);
    if ((pages.dim() != 2 && pages.dim() != 3) || !pages.is_contiguous())
      throw std::invalid_argument("pages has shape " + shape_of(pages) + ", expected a contiguous [num_pages, bytes] or [layers, num_pages, bytes]");
    const int64_t num = pages.size(-2), bytes = pages.size(-1), layers = pages.dim() == 3 ? pages.size(0) : 1;
    const int64_t count = pairs.dim() == 2 ? pairs.size(0) : 0;
    void* pp = flat(pairs, "pairs", dev, at::kInt, count, 2);
    if (layers > INT32_MAX) throw std::invalid_argument("pages has too many layers");
    const c10::cuda::CUDAGuard guard(dev);
    const bl_status st = entry.copy_pages(pages.data_ptr(), (size_t)bytes, num, (int)layers, (size_t)(num * bytes), (const int32_t*)pp, count,
                                          stream_of(dev));
    if (st != BL_OK) return status(st);
    Py_INCREF(a[0]);
    return a[0];
  });
}

// Addresses of the C entry points, in the order of Entry.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 8);
    void* p[8];
    for (int i = 0; i < 8; ++i) {
      p[i] = PyLong_AsVoidPtr(a[i]);
      if (PyErr_Occurred()) throw python_error();
      if (!p[i]) throw std::invalid_argument("no address");
    }
    entry.norm_rope = reinterpret_cast<decltype(entry.norm_rope)>(p[0]);
    entry.window = reinterpret_cast<decltype(entry.window)>(p[1]);
    entry.page_bytes = reinterpret_cast<decltype(entry.page_bytes)>(p[2]);
    entry.append = reinterpret_cast<decltype(entry.append)>(p[3]);
    entry.read = reinterpret_cast<decltype(entry.read)>(p[4]);
    entry.kv4 = reinterpret_cast<decltype(entry.kv4)>(p[5]);
    entry.kv4_ws = reinterpret_cast<decltype(entry.kv4_ws)>(p[6]);
    entry.copy_pages = reinterpret_cast<decltype(entry.copy_pages)>(p[7]);
    Py_RETURN_NONE;
  });
}

#define FAST(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&name)), METH_FASTCALL, doc}
PyMethodDef methods[] = {FAST(bind, "Hands over the addresses of the C entry points."),
                         FAST(norm_rope, "bitlinear_qk_norm_rope"),
                         FAST(window, "bitlinear_attention_window"),
                         FAST(cache, "Checks a cache."),
                         FAST(append, "bitlinear_kv4_append"),
                         FAST(read, "bitlinear_kv4_read"),
                         FAST(kv4, "bitlinear_attention_kv4"),
                         FAST(copy_pages, "bitlinear_kv4_copy_pages"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Compiled argument marshalling of the attention operators.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
