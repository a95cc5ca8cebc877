// The torch side of the operators on device tensors: what a call has to check, allocate and look up before it enters the C ABI,
// in C++ because small calls are all host time (turning four tokens took the host 8.3 us through ctypes and torch's Python calls and
// takes it 4.2 here, of which the launch is 2; a product 6.6 and 4.4).  Python functions in the module `_tensors`; tensors.py
// documents and wraps them.  A function returns its result, or the library's code as an int where that is not 0, and raises
// ValueError for arguments that do not fit.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/ops/empty_strided.h>
#include <c10/core/AutogradState.h>
#include <hip/hip_runtime_api.h>
#include <torch/csrc/autograd/python_variable.h>
#include <cmath>
#include <exception>
#include <optional>
#include <stdexcept>
#include <string>
#include "../../include/pahq.h"

namespace {
using at::Tensor;

struct Refused : std::exception {
  std::string text;
  explicit Refused(std::string t) : text(std::move(t)) {}
  const char* what() const noexcept override { return text.c_str(); }
};
inline void need(bool ok, const char* text) {
  if (!ok) throw Refused(text);
}
struct PythonError {};           // an exception is set already

// `t` has a forward-mode derivative that its next operation is expected to carry on
bool has_tangent(const Tensor& t) { return t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode(); }

const Tensor& tensor(PyObject* o, const char* text) {
  need(THPVariable_Check(o), text);
  const Tensor& t = THPVariable_Unpack(o);
  need(t.layout() == at::kStrided && !t.is_neg(), "tensors: strided, their values as they lie in memory");
  // read or written as plain memory it would lose the tangent, or keep one that is no longer its own
  need(!has_tangent(t), "a tangent (forward-mode derivative): not carried here");
  return t;
}
long long number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return v;
}
int dtype_of(at::ScalarType t) {
  return t == at::kFloat ? PAHQ_F32 : t == at::kBFloat16 ? PAHQ_BF16 : t == at::kHalf ? PAHQ_F16 : -1;
}
constexpr at::ScalarType TYPES[3] = {at::kFloat, at::kBFloat16, at::kHalf};
bool tracked(const Tensor& t) { return t.requires_grad() && at::GradMode::is_enabled(); }

// Elements from row to row of a matrix whose rows are contiguous, -1 if they are not.  Of a single row or column torch reports
// any stride.
int64_t row_stride(const Tensor& t) {
  const int64_t rows = t.size(0), cols = t.size(1);
  if (t.is_contiguous() || (rows <= 1 && (cols <= 1 || t.stride(1) == 1))) return cols ? cols : 1;
  return (t.stride(1) == 1 || cols <= 1) && t.stride(0) >= cols ? t.stride(0) : -1;
}
int32_t size32(int64_t n) {
  need(n <= INT32_MAX, "at most 2^31 - 1 in a direction");
  return (int32_t)n;
}

// The device of the operands made current for a call, and its current stream.
struct On {
  int before = -1;
  hipStream_t stream;
  explicit On(at::DeviceIndex device) {
    int now = 0;
    if (hipGetDevice(&now) != hipSuccess) throw std::runtime_error("no current device");
    if (now != device) {
      if (hipSetDevice(device) != hipSuccess) throw std::runtime_error("the operands' device cannot be made current");
      before = now;
    }
    stream = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(device).stream();
  }
  ~On() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

// A matrix in 4 bits as tensors.py hands it over: (address of codes, of scales, rows, cols, device index)
struct Held {
  uint8_t *codes, *scales;
  int64_t rows, cols;
  at::DeviceIndex device;
  explicit Held(PyObject* o) {
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 5, "an Mx4");
    codes = (uint8_t*)(uintptr_t)number(PyTuple_GET_ITEM(o, 0));
    scales = (uint8_t*)(uintptr_t)number(PyTuple_GET_ITEM(o, 1));
    rows = number(PyTuple_GET_ITEM(o, 2));
    cols = number(PyTuple_GET_ITEM(o, 3));
    device = (at::DeviceIndex)number(PyTuple_GET_ITEM(o, 4));
  }
};
// `t` was written: a backward pass that kept its former values has to notice
void written(const Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
bool on(const Tensor& t, at::DeviceIndex device) { return t.is_cuda() && t.get_device() == device; }

// `o` checked as the result [rows][cols], or a new tensor of TYPES[dtype] where it is None
Tensor result(PyObject* o, int dtype, int64_t rows, int64_t cols, at::DeviceIndex device, int64_t* ld) {
  if (o == Py_None) {
    need(dtype >= 0 && dtype < 3, "dtype: float32, bfloat16 or float16");
    *ld = cols ? cols : 1;
    return at::empty_strided({rows, cols}, {*ld, 1}, at::TensorOptions().dtype(TYPES[dtype]).device(at::Device(at::kCUDA, device)));
  }
  const Tensor& t = tensor(o, "out: a tensor");
  if (!(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && dtype_of(t.scalar_type()) >= 0 && on(t, device) && !tracked(t) &&
        (*ld = row_stride(t)) >= 0))
    throw Refused("out: [" + std::to_string(rows) + "][" + std::to_string(cols) +
                  "] in float32, bfloat16 or float16, rows contiguous, on the operands' device, without a gradient");
  return t;
}

// (x, down, out): out None -> (memory of codes and scales, a Held tuple of it); out a Held tuple -> None
PyObject* mx4_quantize(PyObject* const* a) {
  const Tensor& given = tensor(a[0], "x: a tensor");
  need(given.is_cuda() && given.dim() == 2 && dtype_of(given.scalar_type()) >= 0, "x: a matrix in float32, bfloat16 or float16 on the device");
  need(!tracked(given), "rounding to 4 bits has no gradient: detach x");
  bool down = a[1] == Py_True;
  std::optional<Tensor> turned;
  int64_t ld = row_stride(given);
  if (ld < 0) {                     // a transposed view: the other direction of its base
    turned = given.t();
    down = !down;
    ld = row_stride(*turned);
    need(ld >= 0, "x: rows or columns contiguous, not overlapping");
  }
  const Tensor& x = turned ? *turned : given;
  const int64_t rows = x.size(down ? 1 : 0), cols = x.size(down ? 0 : 1);
  need(cols >= 1, "rows of at least one element");
  const at::DeviceIndex device = x.get_device();
  Tensor both;
  uint8_t *codes, *scales;
  if (a[2] == Py_None) {
    const int64_t groups = (cols + 255) / 256;
    both = at::empty({rows * groups * 136}, at::TensorOptions().dtype(at::kByte).device(x.device()));
    codes = (uint8_t*)both.data_ptr();
    scales = codes + rows * groups * 128;
  } else {
    const Held out(a[2]);
    need(out.rows == rows && out.cols == cols && out.device == device, "out: of the result's shape, on x's device");
    codes = out.codes;
    scales = out.scales;
  }
  if (rows) {
    const On current(device);
    const int rc = pahq_mx4_quantize(current.stream, x.data_ptr(), dtype_of(x.scalar_type()), size32(rows), size32(cols), ld,
                                     down ? PAHQ_MX4_BY_COLUMNS : PAHQ_MX4_BY_ROWS, codes, scales);
    if (rc) return PyLong_FromLong(rc);
  }
  if (a[2] != Py_None) Py_RETURN_NONE;
  return Py_BuildValue("(N(KKLLi))", THPVariable_Wrap(both), (unsigned long long)(uintptr_t)codes, (unsigned long long)(uintptr_t)scales, (long long)rows,
                       (long long)cols, (int)device);
}

// (q, dtype, out)
PyObject* mx4_dequantize(PyObject* const* a) {
  const Held q(a[0]);
  int64_t ld;
  const Tensor out = result(a[2], (int)number(a[1]), q.rows, q.cols, q.device, &ld);
  if (q.rows) {
    const On current(q.device);
    const int rc = pahq_mx4_dequantize(current.stream, q.codes, q.scales, size32(q.rows), size32(q.cols), out.data_ptr(), dtype_of(out.scalar_type()), ld);
    if (rc) return PyLong_FromLong(rc);
    written(out);
  }
  return THPVariable_Wrap(out);
}

// (a, w, bias, residual, dtype, out)
PyObject* mx4_gemm(PyObject* const* a) {
  const Held x(a[0]), w(a[1]);
  need(x.cols == w.cols && x.device == w.device, "a [m][k] and w [n][k] on one device");
  int64_t ld, ld_res = 0;
  const Tensor out = result(a[5], (int)number(a[4]), x.rows, w.rows, x.device, &ld);
  const float* bias = nullptr;
  const void* residual = nullptr;
  if (a[2] != Py_None) {
    const Tensor& b = tensor(a[2], "bias: a tensor");
    need(b.scalar_type() == at::kFloat && b.dim() == 1 && b.size(0) == w.rows && on(b, x.device) && b.is_contiguous() && !tracked(b),
         "bias: float32 [n], contiguous, on the operands' device, without a gradient");
    bias = (const float*)b.data_ptr();
  }
  if (a[3] != Py_None) {
    const Tensor& r = tensor(a[3], "residual: a tensor");
    need(r.dim() == 2 && r.size(0) == x.rows && r.size(1) == w.rows && r.scalar_type() == out.scalar_type() && on(r, x.device) && !tracked(r) &&
             (ld_res = row_stride(r)) >= 0,
         "residual: [m][n] of the result's dtype, rows contiguous, on the operands' device, without a gradient");
    residual = r.data_ptr();
  }
  if (x.rows && w.rows) {
    const On current(x.device);
    const int rc = pahq_mx4_gemm(current.stream, x.codes, x.scales, w.codes, w.scales, size32(x.rows), size32(w.rows), size32(x.cols), bias, residual, ld_res,
                                 out.data_ptr(), dtype_of(out.scalar_type()), ld);
    if (rc) return PyLong_FromLong(rc);
    written(out);
  }
  return THPVariable_Wrap(out);
}

// Strides of tokens and heads; of a single one torch reports any
void head_strides(const Tensor& t, int64_t* token, int64_t* head) {
  const int64_t heads = t.size(1), d = t.size(2);
  need(d <= 1 || t.stride(2) == 1, "the elements of a head: contiguous");
  *head = heads <= 1 ? d : t.stride(1);
  *token = t.size(0) <= 1 ? (heads > 1 ? (heads - 1) * *head : 0) + d : t.stride(0);
}

// (x, positions, table, layout, magnitude, inverse, out)
PyObject* rotary(PyObject* const* a) {
  const Tensor& x = tensor(a[0], "x: a tensor");
  need(x.is_cuda() && x.dim() == 3 && dtype_of(x.scalar_type()) >= 0, "x: [tokens][heads][d_head] in float32, bfloat16 or float16 on the device");
  const int64_t tokens = x.size(0), heads = x.size(1), d = x.size(2);
  const at::DeviceIndex device = x.get_device();
  const Tensor &positions = tensor(a[1], "positions: a tensor"), &table = tensor(a[2], "table: a tensor");
  need(positions.scalar_type() == at::kLong && positions.dim() == 1 && positions.size(0) == tokens && on(positions, device) && positions.is_contiguous(),
       "positions: int64 [tokens], contiguous, on x's device");
  need(table.scalar_type() == at::kLong && table.dim() == 1 && on(table, device) && table.is_contiguous() && table.numel() >= 1 && 2 * table.numel() <= d,
       "table: from rotary_table, on x's device, for at most d_head elements");
  const double magnitude = real(a[4]);
  Tensor out;
  if (a[6] == Py_None) {
    out = at::empty_like(x, x.options(), at::MemoryFormat::Contiguous);
  } else {
    out = tensor(a[6], "out: a tensor");
    need(out.sizes() == x.sizes() && out.scalar_type() == x.scalar_type() && on(out, device), "out: of x's shape and dtype, on its device");
  }
  if (tokens && heads) {
    int64_t xt, xh, ot, oh;
    head_strides(x, &xt, &xh);
    head_strides(out, &ot, &oh);
    const On current(device);
    const int rc = pahq_rotary(current.stream, x.data_ptr(), dtype_of(x.scalar_type()), size32(tokens), size32(heads), size32(d), xt, xh,
                               (const int64_t*)positions.data_ptr(), (const uint64_t*)table.data_ptr(), (int32_t)(2 * table.numel()), (int32_t)number(a[3]),
                               (float)magnitude, a[5] == Py_True, out.data_ptr(), ot, oh);
    if (rc) return PyLong_FromLong(rc);
    written(out);
  }
  return THPVariable_Wrap(out);
}

// The first five arguments of every call on a cache: keys, values, starts, lengths, pages
struct Paged {
  Tensor keys, values;
  pahq_kv_cache cache = {};
  pahq_kv_batch batch = {};
  at::DeviceIndex device;
  Paged(PyObject* const* a, bool read_only) : keys(tensor(a[0], "keys: a tensor")), values(tensor(a[1], "values: a tensor")) {
    device = keys.get_device();
    need(keys.is_cuda() && keys.dim() == 4 && keys.sizes() == values.sizes() && keys.scalar_type() == values.scalar_type() && on(values, device) &&
             dtype_of(keys.scalar_type()) >= 0 && keys.size(0) >= 1 && keys.size(1) >= 1 && keys.size(2) >= 1 && keys.size(3) >= 1,
         "keys and values: [pages][heads][page_size][d_head] in float32, bfloat16 or float16 on one device");
    need(!tracked(keys) && !tracked(values), read_only ? "a cache has no gradient: detach it" : "keys and values: without a gradient");
    int64_t s[3];
    for (int i = 0; i < 3; i++) {         // of a single one torch reports any stride
      s[i] = keys.size(i) > 1 ? keys.stride(i) : 0;
      need(s[i] == (values.size(i) > 1 ? values.stride(i) : 0), "keys and values: with the same strides");
    }
    need((keys.stride(3) == 1 && values.stride(3) == 1) || keys.size(3) == 1, "the elements of a row: contiguous");
    cache = {keys.data_ptr(), values.data_ptr(), dtype_of(keys.scalar_type()), size32(keys.size(0)), size32(keys.size(2)), size32(keys.size(1)),
             size32(keys.size(3)), s[0], s[1], s[2]};
    const Tensor &starts = tensor(a[2], "starts: a tensor"), &lengths = tensor(a[3], "lengths: a tensor"), &pages = tensor(a[4], "pages: a tensor");
    need(starts.scalar_type() == at::kInt && starts.dim() == 1 && starts.size(0) >= 1 && on(starts, device) && starts.is_contiguous(),
         "starts: int32 [batch + 1], contiguous, on the cache's device");
    need(lengths.scalar_type() == at::kInt && lengths.dim() == 1 && lengths.size(0) == starts.size(0) - 1 && on(lengths, device) && lengths.is_contiguous(),
         "lengths: int32 [batch], contiguous, on the cache's device");
    int64_t ld = 0;
    need(pages.scalar_type() == at::kInt && pages.dim() == 2 && pages.size(0) == lengths.size(0) && on(pages, device) && (ld = row_stride(pages)) >= 0,
         "pages: int32 [batch][width], rows contiguous, on the cache's device");
    batch = {(const int32_t*)starts.data_ptr(), (const int32_t*)lengths.data_ptr(), (const int32_t*)pages.data_ptr(), size32(lengths.size(0)),
             size32(pages.size(1)), ld, 0};
  }
  // rows [tokens][heads][d_head] of the cache's dtype; heads 0: any number
  pahq_kv_rows rows(const Tensor& t, int64_t tokens, int64_t heads, const char* text) const {
    need(t.dim() == 3 && (tokens < 0 || t.size(0) == tokens) && (heads ? t.size(1) == heads : t.size(1) >= 1) && t.size(2) == cache.d_head &&
             t.scalar_type() == keys.scalar_type() && on(t, device) && !tracked(t),
         text);
    pahq_kv_rows r = {t.data_ptr(), 0, 0};
    head_strides(t, &r.token, &r.head);
    return r;
  }
};

// (keys, values, starts, lengths, pages, k, v, positions, table, layout, magnitude, q, out)
PyObject* kv_append(PyObject* const* a) {
  Paged p(a, false);
  const Tensor &k = tensor(a[5], "k: a tensor"), &v = tensor(a[6], "v: a tensor");
  const pahq_kv_rows kr = p.rows(k, -1, p.cache.heads, "k: [tokens][cache heads][d_head] of the cache's dtype, on its device, without a gradient");
  const int64_t tokens = k.size(0);
  p.batch.tokens = size32(tokens);
  const pahq_kv_rows vr = p.rows(v, tokens, p.cache.heads, "v: [tokens][cache heads][d_head] of the cache's dtype, on its device, without a gradient");
  const int64_t* positions = nullptr;
  const uint64_t* table = nullptr;
  int64_t pairs = 0;
  if (a[7] != Py_None) {
    const Tensor& t = tensor(a[7], "positions: a tensor");
    need(t.scalar_type() == at::kLong && t.dim() == 1 && t.size(0) == tokens && on(t, p.device) && t.is_contiguous(),
         "positions: int64 [tokens], contiguous, on the cache's device");
    positions = (const int64_t*)t.data_ptr();
  }
  if (a[8] != Py_None) {
    const Tensor& t = tensor(a[8], "table: a tensor");
    need(t.scalar_type() == at::kLong && t.dim() == 1 && on(t, p.device) && t.is_contiguous() && t.numel() >= 1 && 2 * t.numel() <= p.cache.d_head,
         "table: from rotary_table, on the cache's device, for at most d_head elements");
    table = (const uint64_t*)t.data_ptr();
    pairs = t.numel();
  }
  const float magnitude = (float)real(a[10]);
  Tensor out;
  pahq_kv_rows qr = {}, outr = {};
  int32_t q_heads = 0;
  if (a[11] != Py_None) {
    const Tensor& q = tensor(a[11], "q: a tensor");
    qr = p.rows(q, tokens, 0, "q: [tokens][heads][d_head] of the cache's dtype, on its device, without a gradient");
    q_heads = size32(q.size(1));
    out = a[12] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(a[12], "out: a tensor");
    outr = p.rows(out, tokens, q_heads, "out: of q's shape and dtype, on its device, without a gradient");
  } else {
    need(a[12] == Py_None, "out: for q only");
  }
  if (tokens && p.batch.batch) {
    const On current(p.device);
    const int rc = pahq_kv_append(current.stream, &p.cache, &p.batch, &kr, &vr, positions, table, (int32_t)(2 * pairs), (int32_t)number(a[9]), magnitude,
                                  q_heads ? &qr : nullptr, q_heads, q_heads ? &outr : nullptr);
    if (rc) return PyLong_FromLong(rc);
    written(p.keys);
    written(p.values);
    if (q_heads) written(out);
  }
  if (!q_heads) Py_RETURN_NONE;
  return THPVariable_Wrap(out);
}

// (keys, values, starts, lengths, pages, q, tree, scale, out)
PyObject* kv_attention(PyObject* const* a) {
  Paged p(a, true);
  const Tensor& q = tensor(a[5], "q: a tensor");
  const pahq_kv_rows qr = p.rows(q, -1, 0, "q: [tokens][heads][d_head] of the cache's dtype, on its device, without a gradient");
  const int64_t tokens = q.size(0), heads = q.size(1);
  need(heads % p.cache.heads == 0, "q: a multiple of the cache's heads");
  p.batch.tokens = size32(tokens);
  const uint64_t* tree = nullptr;
  int32_t words = 0;
  if (a[6] != Py_None) {
    const Tensor& t = tensor(a[6], "tree: a tensor");
    need(t.scalar_type() == at::kLong && t.dim() == 2 && t.size(0) == tokens && t.size(1) >= 1 && on(t, p.device) && t.is_contiguous(),
         "tree: int64 [tokens][words], contiguous, on the cache's device");
    tree = (const uint64_t*)t.data_ptr();
    words = size32(t.size(1));
  }
  const float scale = a[7] == Py_None ? (float)(1.0 / std::sqrt((double)p.cache.d_head)) : (float)real(a[7]);
  const Tensor out = a[8] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(a[8], "out: a tensor");
  const pahq_kv_rows outr = p.rows(out, tokens, heads, "out: of q's shape and dtype, on its device, without a gradient");
  if (tokens && p.batch.batch) {
    const On current(p.device);
    size_t bytes = 0;
    int rc = pahq_kv_attention_workspace(&p.cache, &p.batch, size32(heads), &bytes);
    if (rc) return PyLong_FromLong(rc);
    Tensor space;
    if (bytes) space = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
    rc = pahq_kv_attention(current.stream, &p.cache, &p.batch, &qr, size32(heads), tree, words, scale, &outr, bytes ? space.data_ptr() : nullptr, bytes);
    if (rc) return PyLong_FromLong(rc);
    written(out);
  }
  return THPVariable_Wrap(out);
}

// (keys, values, starts, lengths, pages, paths, out)
PyObject* kv_keep(PyObject* const* a) {
  Paged p(a, false);
  const int64_t batch = p.batch.batch;
  const Tensor& paths = tensor(a[5], "paths: a tensor");
  need(paths.scalar_type() == at::kInt && paths.dim() == 2 && paths.size(0) == batch && on(paths, p.device) && paths.is_contiguous(),
       "paths: int32 [batch][depth], contiguous, on the cache's device");
  const Tensor out = a[6] == Py_None ? at::empty({batch}, paths.options()) : tensor(a[6], "out: a tensor");
  need(out.scalar_type() == at::kInt && out.dim() == 1 && out.size(0) == batch && on(out, p.device) && out.is_contiguous(),
       "out: int32 [batch], contiguous, on the cache's device");
  p.batch.tokens = INT32_MAX;
  if (batch) {
    const On current(p.device);
    const int rc = pahq_kv_keep(current.stream, &p.cache, &p.batch, (const int32_t*)paths.data_ptr(), size32(paths.size(1)), (int32_t*)out.data_ptr());
    if (rc) return PyLong_FromLong(rc);
    written(p.keys);
    written(p.values);
    written(out);
  }
  return THPVariable_Wrap(out);
}

void set_error_of_torch(const char* name, const char* text) {
  PyObject* const torch = PyImport_ImportModule("torch");
  PyObject* const error = torch ? PyObject_GetAttrString(torch, name) : nullptr;
  if (error) PyErr_SetString(error, text);
  Py_XDECREF(error);
  Py_XDECREF(torch);
}

// Arguments counted, C++ exceptions turned into Python's
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments", N);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const PythonError&) {
  } catch (const Refused& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::OutOfMemoryError& e) {          // under torch's own name, for programs that make room and try again
    set_error_of_torch("OutOfMemoryError", e.what_without_backtrace());
  } catch (const c10::Error& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown error");
  }
  return nullptr;
}
#define ENTRY(f, n) {#f, (PyCFunction)(void (*)())entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(mx4_quantize, 3), ENTRY(mx4_dequantize, 3), ENTRY(mx4_gemm, 6), ENTRY(rotary, 7),
                         ENTRY(kv_append, 13), ENTRY(kv_attention, 9), ENTRY(kv_keep, 7), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
