// Compiled argument marshalling for the attention operators and the 8-bit layers (module _marshal, used by binding.py).
//
// A decode step makes several of these calls per layer, each a few microseconds of device time; looking at seven tensors,
// allocating outputs and converting twenty arguments costs 10 microseconds from Python and about 3 from here.  The
// functions check what the Python wrappers document, allocate what was not given, and call the C entry points (whose
// addresses binding.py hands over from the library it loaded).  They return the result, or the bl_status as a number
// where it is not BL_OK; argument errors are ValueError and TypeError.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/TensorImpl.h>
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
  decltype(&bitlinear_rms_norm_quant) norm_quant;
  decltype(&bitlinear_matmul_i8) matmul_i8;
  decltype(&bitlinear_route_topk) route;
  decltype(&bitlinear_route_topk_ws_bytes) route_ws;
  decltype(&bitlinear_matmul_grouped) grouped;
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

bool given(PyObject* o) { return o != Py_None; }
// An output: a given tensor, a new one for True, none for None or False.
Tensor output(PyObject* o, const char* name, int64_t rows, int64_t width, at::TensorOptions options) {
  if (o == Py_None || o == Py_False) return Tensor();
  if (o == Py_True) return at::empty({rows, width}, options);
  return tensor(o, name);
}
// Like rows_of, for a matrix whose rows take any stride; a stride that no row uses is the width, rounded up to `unit`.
int64_t any_rows_of(const Tensor& t, const char* name, c10::Device dev, at::ScalarType type, int64_t rows, int64_t width, int64_t unit) {
  check_place(t, name, dev, type);
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != width || (t.stride(1) != 1 && width > 1))
    throw std::invalid_argument(std::string(name) + " has shape " + shape_of(t) + ", expected (" + std::to_string(rows) + ", " +
                                std::to_string(width) + ") with the values of a row contiguous");
  return rows > 1 ? t.stride(0) : (width + unit - 1) / unit * unit;
}
PyObject* wrapped(PyObject* o, const Tensor& t) {
  if (o == Py_True) return THPVariable_Wrap(t);
  if (o == Py_False) o = Py_None;
  Py_INCREF(o);
  return o;
}
at::ScalarType scalar_type(PyObject* o) {                       // of a BL_* code
  switch (small(o, "dtype")) {
    case BL_F32: return at::kFloat;
    case BL_F16: return at::kHalf;
    case BL_BF16: return at::kBFloat16;
    default: throw TypeError("unsupported dtype");
  }
}
int truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw python_error();
  return v;
}

// One allocation for several small tensors that belong together: an allocation costs about as much as the rest of a call's marshalling.
// Each keeps the memory of all alive, so only up to kPooled bytes.
constexpr int64_t kPooled = 1 << 20;
struct Pool {
  Tensor bytes;
  int64_t used = 0;
  static int64_t room(int64_t n) { return (n + 15) / 16 * 16; }
  Tensor take(at::IntArrayRef sizes, at::ScalarType type) {
    int64_t n = c10::elementSize(type);
    Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(bytes.storage()), bytes.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(used / n);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    for (const int64_t s : sizes) n *= s;
    used += room(n);
    return t;
  }
};

// x, weight, eps, residual, rows, row_weights, h, y, x_q, scale
PyObject* norm_quant(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 10);
    const Tensor& x = tensor(a[0], "x");
    const c10::Device dev = cuda_device(x, "x");
    const auto type = x.scalar_type();
    const bl_dtype code = type_code(type);
    if (x.dim() != 2) throw std::invalid_argument("x has shape " + shape_of(x) + ", expected (rows, K)");
    const int64_t x_rows = x.size(0), K = x.size(1), ld_x = any_rows_of(x, "x", dev, type, x_rows, K, 8);
    const float eps = real(a[2]);
    int64_t T = x_rows, top_k = 0;
    void *rp = nullptr, *wp = nullptr;
    if (given(a[4])) {
      const Tensor& rows = tensor(a[4], "rows");
      if (rows.dim() != 2) throw std::invalid_argument("rows has shape " + shape_of(rows) + ", expected (T, top_k)");
      T = rows.size(0); top_k = rows.size(1);
      rp = flat(rows, "rows", dev, at::kInt, T, top_k);
      if (T > 0 && top_k > INT32_MAX) throw std::invalid_argument("rows is too wide");
      if (given(a[5])) wp = flat(tensor(a[5], "row_weights"), "row_weights", dev, at::kFloat, T, top_k);
    } else if (given(a[5])) {
      throw std::invalid_argument("row_weights without rows");
    }
    void* weight = given(a[1]) ? flat(tensor(a[1], "weight"), "weight", dev, type, K) : nullptr;
    const void* res = nullptr;
    int64_t ld_res = 0;
    if (given(a[3])) {
      const Tensor& r = tensor(a[3], "residual");
      ld_res = any_rows_of(r, "residual", dev, type, T, K, 8);
      res = r.data_ptr();
    }
    const c10::cuda::CUDAGuard guard(dev);
    const Tensor h = output(a[6], "h", T, K, x.options()), y = output(a[7], "y", T, K, x.options());
    Tensor q, scale;
    if (a[8] == Py_True && !given(a[9]) && T * K + 4 * T <= kPooled) {      // new codes and new scales
      Pool pool{at::empty({Pool::room(T * K) + Pool::room(4 * T)}, x.options().dtype(at::kByte))};
      q = pool.take({T, K}, at::kChar);
      scale = pool.take({T}, at::kFloat);
    } else {
      q = output(a[8], "x_q", T, K, x.options().dtype(at::kChar));
      if (q.defined()) scale = given(a[9]) ? tensor(a[9], "scale") : at::empty({T}, x.options().dtype(at::kFloat));
    }
    const int64_t ld_h = h.defined() ? any_rows_of(h, "h", dev, type, T, K, 8) : 0, ld_y = y.defined() ? any_rows_of(y, "y", dev, type, T, K, 8) : 0;
    const int64_t ld_q = q.defined() ? any_rows_of(q, "x_q", dev, at::kChar, T, K, 8) : 0;
    void* sp = q.defined() ? flat(scale, "scale", dev, at::kFloat, T) : nullptr;
    auto at_of = [](const Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    const bl_status st = entry.norm_quant(x.data_ptr(), code, x_rows, T, K, ld_x, (const int32_t*)rp, (const float*)wp, (int)top_k, res, ld_res,
                                          weight, eps, at_of(h), ld_h, at_of(y), ld_y, (int8_t*)at_of(q), ld_q, (float*)sp, stream_of(dev));
    if (st != BL_OK) return status(st);
    PyObject* r = PyTuple_New(4);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, wrapped(a[8], q));
    PyTuple_SET_ITEM(r, 1, q.defined() ? given_or(a[9], scale) : wrapped(Py_None, Tensor()));
    PyTuple_SET_ITEM(r, 2, wrapped(a[6], h));
    PyTuple_SET_ITEM(r, 3, wrapped(a[7], y));
    return r;
  });
}

// x_q, x_scale, w_q, w_scale, dtype, bias, relu, residual, y
PyObject* matmul_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 9);
    const Tensor &x = tensor(a[0], "x_q"), &w = tensor(a[2], "w_q");
    const c10::Device dev = cuda_device(x, "x_q");
    if (x.dim() != 2 || w.dim() != 2) throw std::invalid_argument("x_q and w_q must have two dimensions");
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
    const int64_t ld_x = any_rows_of(x, "x_q", dev, at::kChar, M, K, 16), ld_w = any_rows_of(w, "w_q", dev, at::kChar, N, K, 16);
    void* xs = given(a[1]) ? flat(tensor(a[1], "x_scale"), "x_scale", dev, at::kFloat, M) : nullptr;
    void* ws = given(a[3]) ? flat(tensor(a[3], "w_scale"), "w_scale", dev, at::kFloat, N) : nullptr;
    const auto type = given(a[8]) ? tensor(a[8], "y").scalar_type() : scalar_type(a[4]);
    void* bias = given(a[5]) ? flat(tensor(a[5], "bias"), "bias", dev, type, N) : nullptr;
    const int relu = truth(a[6]);
    const void* res = nullptr;
    int64_t ld_res = 0;
    if (given(a[7])) {
      const Tensor& r = tensor(a[7], "residual");
      ld_res = any_rows_of(r, "residual", dev, type, M, N, 1);
      res = r.data_ptr();
    }
    const c10::cuda::CUDAGuard guard(dev);
    const Tensor y = given(a[8]) ? tensor(a[8], "y") : at::empty({M, N}, x.options().dtype(type));
    const int64_t ld_y = any_rows_of(y, "y", dev, type, M, N, 1);
    const bl_status st = entry.matmul_i8((const int8_t*)x.data_ptr(), M, K, N, ld_x, (const float*)xs, (const int8_t*)w.data_ptr(), ld_w,
                                         (const float*)ws, bias, relu, res, ld_res, y.data_ptr(), type_code(type), ld_y, stream_of(dev));
    return st != BL_OK ? status(st) : given_or(a[8], y);
  });
}

// logits, top_k, normalise, positions, ws, chosen, weights, offsets, rows, places
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 10);
    const Tensor& z = tensor(a[0], "logits");
    const c10::Device dev = cuda_device(z, "logits");
    const auto type = z.scalar_type();
    const bl_dtype code = type_code(type);
    if (z.dim() != 2) throw std::invalid_argument("logits has shape " + shape_of(z) + ", expected (T, experts)");
    const int64_t T = z.size(0), E = z.size(1), ld = any_rows_of(z, "logits", dev, type, T, E, 1);
    const int k = small(a[1], "top_k"), normalise = truth(a[2]);
    if (E > INT32_MAX || k < 1 || k > E || k > 32) throw std::invalid_argument("top_k must be 1..32 and at most the number of experts");
    void* pos = given(a[3]) ? flat(tensor(a[3], "positions"), "positions", dev, at::kInt, T) : nullptr;
    const c10::cuda::CUDAGuard guard(dev);
    const int64_t need = (int64_t)entry.route_ws(T, (int)E), pairs = Pool::room(4 * T * k), list = Pool::room(4 * (E + 1));
    // new outputs come from one allocation
    const bool news[5] = {!given(a[5]), !given(a[6]), !given(a[7]), !given(a[8]), !given(a[9])};
    const int64_t room = (news[0] + news[1] + news[3] + news[4]) * pairs + news[2] * list;
    const bool pooled = room > 0 && room <= kPooled;
    Pool pool;
    if (pooled) pool.bytes = at::empty({room}, z.options().dtype(at::kByte));
    auto out = [&](int i, const char* name, at::IntArrayRef sizes, at::ScalarType type) {
      return !news[i] ? tensor(a[5 + i], name) : pooled ? pool.take(sizes, type) : at::empty(sizes, z.options().dtype(type));
    };
    const Tensor chosen = out(0, "chosen", {T, k}, at::kInt), weights = out(1, "weights", {T, k}, at::kFloat);
    const Tensor offsets = out(2, "offsets", {E + 1}, at::kInt), rows = out(3, "rows", {T * k}, at::kInt);
    const Tensor places = out(4, "places", {T, k}, at::kInt);
    void *cp = flat(chosen, "chosen", dev, at::kInt, T, k), *wp = flat(weights, "weights", dev, at::kFloat, T, k);
    void *op = flat(offsets, "offsets", dev, at::kInt, E + 1), *rp = flat(rows, "rows", dev, at::kInt, T * k);
    void* pp = flat(places, "places", dev, at::kInt, T, k);
    Tensor ws;
    if (given(a[4])) { ws = tensor(a[4], "ws"); (void)flat(ws, "ws", dev, at::kByte, ws.numel()); }
    else if (need > 0) ws = at::empty({need}, z.options().dtype(at::kByte));
    const bl_status st = entry.route(z.data_ptr(), code, T, (int)E, ld, k, normalise, (const int32_t*)pos, (int32_t*)cp, (float*)wp, (int32_t*)op,
                                     (int32_t*)rp, (int32_t*)pp, ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? (size_t)ws.numel() : 0,
                                     stream_of(dev));
    if (st != BL_OK) return status(st);
    PyObject* r = PyTuple_New(5);
    if (!r) throw python_error();
    PyTuple_SET_ITEM(r, 0, given_or(a[5], chosen));
    PyTuple_SET_ITEM(r, 1, given_or(a[6], weights));
    PyTuple_SET_ITEM(r, 2, given_or(a[7], offsets));
    PyTuple_SET_ITEM(r, 3, given_or(a[8], rows));
    PyTuple_SET_ITEM(r, 4, given_or(a[9], places));
    return r;
  });
}

// x, w, offsets, rows, x_scale, w_scale, bias, relu, dtype, y
PyObject* grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 10);
    const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w"), &offsets = tensor(a[2], "offsets");
    const c10::Device dev = cuda_device(x, "x");
    const auto type = x.scalar_type();
    const bool codes = type == at::kChar;
    if (!codes && type != at::kHalf && type != at::kBFloat16) throw TypeError(std::string("x is ") + c10::toString(type) + ", expected int8, fp16 or bf16");
    const int64_t unit = codes ? 16 : 8;
    if (x.dim() != 2 || w.dim() != 3) throw std::invalid_argument("x must have two dimensions and w three");
    const int64_t x_rows = x.size(0), K = x.size(1), E = w.size(0), N = w.size(1);
    const int64_t ld_x = any_rows_of(x, "x", dev, type, x_rows, K, unit);
    check_place(w, "w", dev, type);
    if (w.size(2) != K || w.stride(2) != 1) throw std::invalid_argument("w has shape " + shape_of(w) + ", expected (experts, N, K) with the values of a row contiguous");
    if (E < 1 || E > INT32_MAX) throw std::invalid_argument("w has no experts, or too many");
    const int64_t ld_w = N > 1 ? w.stride(1) : E > 1 ? w.stride(0) : (K + unit - 1) / unit * unit;
    void* op = flat(offsets, "offsets", dev, at::kInt, E + 1);
    const int64_t R = given(a[3]) ? tensor(a[3], "rows").numel() : x_rows;
    void* rp = given(a[3]) ? flat(tensor(a[3], "rows"), "rows", dev, at::kInt, R) : nullptr;
    void* xs = given(a[4]) ? flat(tensor(a[4], "x_scale"), "x_scale", dev, at::kFloat, x_rows) : nullptr;
    void* ws = given(a[5]) ? flat(tensor(a[5], "w_scale"), "w_scale", dev, at::kFloat, E, N) : nullptr;
    const auto ytype = given(a[9]) ? tensor(a[9], "y").scalar_type() : given(a[8]) ? scalar_type(a[8]) : codes ? at::kBFloat16 : type;
    void* bias = given(a[6]) ? flat(tensor(a[6], "bias"), "bias", dev, ytype, E, N) : nullptr;
    const int relu = truth(a[7]);
    const c10::cuda::CUDAGuard guard(dev);
    const Tensor y = given(a[9]) ? tensor(a[9], "y") : at::empty({R, N}, x.options().dtype(ytype));
    const int64_t ld_y = any_rows_of(y, "y", dev, ytype, R, N, 1);
    const bl_status st = entry.grouped(x.data_ptr(), codes ? BL_I8 : type_code(type), x_rows, K, N, ld_x, (const float*)xs, w.data_ptr(), ld_w,
                                       w.stride(0), (const float*)ws, (int)E, (const int32_t*)op, (const int32_t*)rp, R, bias, relu, y.data_ptr(),
                                       type_code(ytype), ld_y, stream_of(dev));
    return st != BL_OK ? status(st) : given_or(a[9], y);
  });
}

// Addresses of the C entry points, in the order of Entry.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    want(n, 13);
    void* p[13];
    for (int i = 0; i < 13; ++i) {
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
    entry.norm_quant = reinterpret_cast<decltype(entry.norm_quant)>(p[8]);
    entry.matmul_i8 = reinterpret_cast<decltype(entry.matmul_i8)>(p[9]);
    entry.route = reinterpret_cast<decltype(entry.route)>(p[10]);
    entry.route_ws = reinterpret_cast<decltype(entry.route_ws)>(p[11]);
    entry.grouped = reinterpret_cast<decltype(entry.grouped)>(p[12]);
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
                         FAST(norm_quant, "bitlinear_rms_norm_quant"),
                         FAST(matmul_i8, "bitlinear_matmul_i8"),
                         FAST(route, "bitlinear_route_topk"),
                         FAST(grouped, "bitlinear_matmul_grouped"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Compiled argument marshalling of the attention operators and the 8-bit layers.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
