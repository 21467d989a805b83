// Argument marshalling of the calls that serve single tokens, where a call is as long as the host needs for it: checks, output
// allocation and the library call in one native function each.  (From Python, field by field, a norm of four rows took 20 us of host time
// for 4 us of GPU time, an append and a read 50 for 13.)  The functions of api.py of the same names give defaults and say what they mean.
// Every function returns the library's status first; arguments that are no such tensors raise here.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sp.h"

namespace {

struct Raised {};      // a Python exception is set

[[noreturn]] void value_error(const char* format, const char* what) {
  PyErr_Format(PyExc_ValueError, format, what);
  throw Raised();
}
const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
    throw Raised();
  }
  return THPVariable_Unpack(o);
}
void on_device(const at::Tensor& t, int dev) {
  if (t.is_cuda() && t.get_device() == dev) return;
  if (!t.is_cuda()) PyErr_SetString(PyExc_RuntimeError, "libsp operates on CUDA tensors only (there is no CPU path)");
  else PyErr_SetString(PyExc_ValueError, "the tensors of a call must be on one device");
  throw Raised();
}
// Index of the device of a call's first tensor, which has to be the current one (the kernels run on its current stream).
int current_device(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (!t.is_cuda()) on_device(t, 0);
  const int dev = (int)t.get_device();
  if (dev != (int)c10::cuda::current_device()) {
    PyErr_SetString(PyExc_ValueError, "the tensors of a call must be on the current CUDA device");
    throw Raised();
  }
  return dev;
}
void* stream_of(int dev) { return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }

int32_t code_of(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return SP_F32;
    case at::kBFloat16: return SP_BF16;
    case at::kDouble: return SP_F64;
    case at::kFloat8_e4m3fn: return SP_E4M3;
    default: return -1;
  }
}
// Matrix view of a 2-D tensor whose rows are contiguous.
sp_mat rows(const at::Tensor& t, int dev, const char* what, bool eight = false) {
  on_device(t, dev);
  const int32_t code = code_of(t.scalar_type());
  const char* kind = eight ? "%s must be a row-major 2-D tensor of float8_e4m3fn" : "%s must be a row-major 2-D tensor of fp32 or bf16";
  if (code < 0 || eight != (code == SP_E4M3) || t.dim() != 2) value_error(kind, what);
  const int64_t n = t.size(0), cols = t.size(1), ld = t.stride(0);
  if (t.stride(1) != 1 && cols > 1) value_error(kind, what);
  return sp_mat{t.data_ptr(), code, 0, n, cols, n > 1 ? ld : (cols > ld ? cols : ld)};
}
sp_mat rows(PyObject* o, int dev, const char* what, bool eight = false) { return rows(tensor(o, what), dev, what, eight); }
// Address of a contiguous vector, null for None.
template <typename T>
T* vector(PyObject* o, at::ScalarType type, int64_t n, int dev, const char* what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, what);
  on_device(t, dev);
  if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous %s with %lld entries", what, type == at::kInt ? "int32" : "float32", (long long)n);
    throw Raised();
  }
  return (T*)t.data_ptr();
}
at::TensorOptions on(at::ScalarType type, int dev) { return at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)dev)); }
at::Tensor empty(at::IntArrayRef size, at::ScalarType type, int dev) { return at::empty(size, on(type, dev)); }
// [n, cols] whose rows start on 16 bytes (a slice of a wider matrix would be the same, 3 us later)
at::Tensor rows_of_16_bytes(int64_t n, int64_t cols, at::ScalarType type, int dev) {
  const int64_t per = 16 / (int64_t)c10::elementSize(type), wide = (cols + per - 1) / per * per;
  return wide == cols ? empty({n, cols}, type, dev) : at::empty_strided({n, cols}, {wide, 1}, on(type, dev));
}
struct Workspace {
  at::Tensor t;
  void* ptr = nullptr;
  size_t bytes = 0;
  Workspace(PyObject* given, size_t need, int dev) {
    if (given != Py_None) {
      t = tensor(given, "ws");
      on_device(t, dev);
    } else if (need > 0) {
      t = empty({(int64_t)need}, at::kByte, dev);
    } else {
      return;
    }
    ptr = t.data_ptr();
    bytes = t.nbytes();
  }
};
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw Raised();
  return v != 0;
}
double number(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised();
  return v;
}
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised();
  return v;
}
int32_t integer32(PyObject* o, const char* what) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) value_error("%s is out of range", what);
  return (int32_t)v;
}
PyObject* wrapped(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
// (status, tensors ...): a tensor that is not defined is None
PyObject* answer(sp_status status, std::initializer_list<at::Tensor> list) {
  PyObject* r = PyTuple_New(1 + (Py_ssize_t)list.size());
  if (!r) throw Raised();
  PyTuple_SET_ITEM(r, 0, PyLong_FromLong((long)status));
  Py_ssize_t i = 1;
  for (const at::Tensor& t : list) PyTuple_SET_ITEM(r, i++, wrapped(t));
  return r;
}

// X, weight, eps, residual, h_out, out, eight, want_rstd
PyObject* rms_norm(PyObject* const* a) {
  const int dev = current_device(a[0], "X");
  const at::Tensor& X = tensor(a[0], "X");
  const sp_mat x = rows(X, dev, "X");
  sp_mat r{}, h{};
  at::Tensor H;
  if (a[3] != Py_None) {
    r = rows(a[3], dev, "residual");
    H = a[4] == Py_None ? rows_of_16_bytes(x.rows, x.cols, tensor(a[3], "residual").scalar_type(), dev) : tensor(a[4], "h_out");
  } else if (a[4] != Py_None) {
    H = tensor(a[4], "h_out");
  }
  if (H.defined()) h = rows(H, dev, "h_out");
  at::Tensor Y = a[5] == Py_None ? rows_of_16_bytes(x.rows, x.cols, truth(a[6]) ? at::kFloat8_e4m3fn : X.scalar_type(), dev) : tensor(a[5], "out");
  const bool eight = Y.scalar_type() == at::kFloat8_e4m3fn;
  const sp_mat y = rows(Y, dev, "out", eight);
  at::Tensor scale, rstd;
  if (eight) scale = empty({x.rows}, at::kFloat, dev);
  if (truth(a[7])) rstd = empty({x.rows}, at::kFloat, dev);
  const sp_status s = sp_rms_norm(&x, a[3] == Py_None ? nullptr : &r, vector<float>(a[1], at::kFloat, x.cols, dev, "weight"), number(a[2]),
                                  H.defined() ? &h : nullptr, &y, eight ? (float*)scale.data_ptr() : nullptr,
                                  rstd.defined() ? (float*)rstd.data_ptr() : nullptr, stream_of(dev));
  return answer(s, {Y, H, scale, rstd});
}

// dY, H, weight, rstd, eps, d_stream, want_weight, out, ws
PyObject* rms_norm_grad(PyObject* const* a) {
  const int dev = current_device(a[0], "dY");
  const sp_mat g = rows(a[0], dev, "dY"), h = rows(a[1], dev, "H");
  at::Tensor X = a[7] == Py_None ? rows_of_16_bytes(g.rows, g.cols, tensor(a[1], "H").scalar_type(), dev) : tensor(a[7], "out");
  const sp_mat x = rows(X, dev, "out");
  sp_mat d{};
  if (a[5] != Py_None) d = rows(a[5], dev, "d_stream");
  const bool weight = truth(a[6]);
  at::Tensor dw;
  if (weight) dw = empty({g.cols}, at::kFloat, dev);
  const Workspace ws(a[8], weight ? sp_rms_norm_grad_bytes(g.rows, g.cols) : 0, dev);
  const sp_status s = sp_rms_norm_grad(&g, &h, vector<float>(a[2], at::kFloat, g.cols, dev, "weight"),
                                       vector<float>(a[3], at::kFloat, g.rows, dev, "rstd"), number(a[4]), a[5] == Py_None ? nullptr : &d, &x,
                                       weight ? (float*)dw.data_ptr() : nullptr, ws.ptr, ws.bytes, stream_of(dev));
  return answer(s, {X, dw});
}

// X, x_scale, W, w_scale, bias, act, other, combine, out, f32, status
PyObject* linear_e4m3(PyObject* const* a) {
  const int dev = current_device(a[0], "X");
  const sp_mat x = rows(a[0], dev, "X", true), w = rows(a[2], dev, "W", true);
  at::Tensor Y = a[8] == Py_None ? rows_of_16_bytes(x.rows, w.rows, truth(a[9]) ? at::kFloat : at::kBFloat16, dev) : tensor(a[8], "out");
  const sp_mat y = rows(Y, dev, "out");
  sp_mat o{};
  if (a[6] != Py_None) o = rows(a[6], dev, "other");
  const sp_status s = sp_linear_e4m3(&x, vector<float>(a[1], at::kFloat, x.rows, dev, "x_scale"), &w,
                                     vector<float>(a[3], at::kFloat, w.rows, dev, "w_scale"), vector<float>(a[4], at::kFloat, w.rows, dev, "bias"),
                                     integer32(a[5], "act"), a[6] == Py_None ? nullptr : &o, integer32(a[7], "combine"), &y,
                                     vector<int32_t>(a[10], at::kInt, 4, dev, "status"), stream_of(dev));
  return answer(s, {Y});
}

// k, v, k_scale, v_scale, table, lens at a[0 .. 5]
sp_kv_cache cache_of(PyObject* const* a, int dev) {
  const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
  const bool four = k.scalar_type() == at::kByte;
  if (!four && k.scalar_type() != at::kBFloat16) value_error("%s are bf16 or uint8", "pages");
  if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
    value_error("%s must be [n_pages, n_kv_heads, page_len, d_head] of one shape and dtype", "k and v");
  sp_kv_cache c = {};
  const int64_t d_head = four ? 2 * k.size(3) : k.size(3);
  for (int i = 0; i < 3; ++i)
    if (k.size(i) > INT32_MAX) value_error("%s is out of range", "the number of pages, heads or tokens");
  if (d_head > INT32_MAX) value_error("%s is out of range", "d_head");
  c.kind = four ? SP_CACHE_4BIT : SP_CACHE_BF16;
  c.n_pages = (int32_t)k.size(0); c.n_kv_heads = (int32_t)k.size(1); c.page_len = (int32_t)k.size(2); c.d_head = (int32_t)d_head;
  const auto step = [&](const at::Tensor& t) {
    on_device(t, dev);
    int64_t inner = 1;
    for (int64_t i = t.dim() - 1; i > 0; --i) {
      if (t.stride(i) != inner && t.size(i) > 1) value_error("%s must be contiguous", "the entries of a page");
      inner *= t.size(i);
    }
    return (t.size(0) > 1 ? t.stride(0) : inner) * (int64_t)t.element_size();
  };
  c.step = step(k);
  bool equal = step(v) == c.step;
  if (four) {
    const at::Tensor &ks = tensor(a[2], "k_scale"), &vs = tensor(a[3], "v_scale");
    const int64_t want[5] = {k.size(0), k.size(1), k.size(2), d_head / SP_CACHE_GROUP, 2};
    for (const at::Tensor* t : {&ks, &vs})
      if (t->scalar_type() != at::kBFloat16 || t->sizes() != at::IntArrayRef(want, 5))
        value_error("%s must be bf16 [n_pages, n_kv_heads, page_len, d_head / 64, 2]", "k_scale and v_scale");
    c.scale_step = step(ks);
    equal = equal && step(vs) == c.scale_step;
    c.k_scale = ks.data_ptr(); c.v_scale = vs.data_ptr();
  }
  if (!equal) value_error("%s lie equally far apart, and so do those of their scales", "the pages of k and v");
  c.k = k.data_ptr(); c.v = v.data_ptr();
  const at::Tensor& table = tensor(a[4], "table");
  on_device(table, dev);
  if (table.dim() != 2 || table.scalar_type() != at::kInt || (table.stride(1) != 1 && table.size(1) > 1))
    value_error("%s must be int32 [n_seq, pages] with contiguous rows", "table");
  if (table.size(0) > INT32_MAX || table.size(1) > INT32_MAX) value_error("%s is out of range", "the size of table");
  c.n_seq = (int32_t)table.size(0);
  c.max_pages = (int32_t)table.size(1);
  c.table = (const int32_t*)table.data_ptr();
  c.table_ld = c.n_seq > 1 ? table.stride(0) : c.max_pages;
  c.lens = vector<int32_t>(a[5], at::kInt, c.n_seq, dev, "lens");
  return c;
}
// Offsets [n_seq + 1]
const int32_t* offsets(PyObject* o, int64_t n_seq, int dev, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.numel() != n_seq + 1) value_error("%s, table and lens are of one number of sequences", what);
  return vector<int32_t>(o, at::kInt, n_seq + 1, dev, what);
}

// k, v, k_scale, v_scale (all None: no pages), table, lens, K, V, cu, Q, inv_freq, neighbours, positions, q_out, k_out, want_k, status, d_head
PyObject* cache_append(PyObject* const* a) {
  const int dev = current_device(a[6], "K");
  sp_cache_append_args args = {};
  args.K = rows(a[6], dev, "K");
  const int64_t N = args.K.rows, n_seq = tensor(a[8], "cu").numel() - 1;
  if (n_seq < 0 || n_seq > INT32_MAX) value_error("%s holds n_seq + 1 offsets", "cu");
  sp_kv_cache c = {};
  if (a[0] != Py_None) {
    c = cache_of(a, dev);
    args.V = rows(a[7], dev, "V");
  } else {
    const int64_t d_head = a[17] == Py_None ? 0 : integer(a[17]);
    if (d_head < 1 || args.K.cols % d_head != 0 || args.K.cols / d_head > INT32_MAX) value_error("%s of the keys", "d_head");
    c.d_head = (int32_t)d_head;
    c.n_kv_heads = (int32_t)(args.K.cols / d_head);
    c.n_seq = (int32_t)n_seq;
    c.lens = vector<int32_t>(a[5], at::kInt, n_seq, dev, "lens");
  }
  args.cu = offsets(a[8], c.n_seq, dev, "cu");
  at::Tensor q_out, k_out;
  if (a[9] != Py_None) {
    const at::Tensor& Q = tensor(a[9], "Q");
    args.Q = rows(Q, dev, "Q");
    q_out = a[13] == Py_None ? empty({N, args.Q.cols}, Q.scalar_type(), dev) : tensor(a[13], "q_out");
    args.Q_out = rows(q_out, dev, "q_out");
    args.n_heads = c.d_head > 0 ? (int32_t)(args.Q.cols / c.d_head) : 0;
  }
  if (a[14] != Py_None) k_out = tensor(a[14], "k_out");
  else if (truth(a[15])) k_out = empty({N, args.K.cols}, tensor(a[6], "K").scalar_type(), dev);
  if (k_out.defined()) args.K_out = rows(k_out, dev, "k_out");
  if (a[10] != Py_None) {
    const int64_t n = tensor(a[10], "inv_freq").numel();
    if (n > INT32_MAX / 2) value_error("%s is out of range", "the number of frequencies");
    args.turned = (int32_t)(2 * n);
    if (n > 0) args.inv_freq = vector<float>(a[10], at::kFloat, n, dev, "inv_freq");
  }
  args.neighbours = truth(a[11]) ? 1 : 0;
  args.positions = vector<int32_t>(a[12], at::kInt, N, dev, "positions");
  const sp_status s = sp_cache_append(&c, &args, vector<int32_t>(a[16], at::kInt, 4, dev, "status"), stream_of(dev));
  return answer(s, {q_out, k_out});
}

// k, v, k_scale, v_scale, table, lens, cu, rows, f32, K, V, status
PyObject* cache_read(PyObject* const* a) {
  const int dev = current_device(a[0], "k");
  const sp_kv_cache c = cache_of(a, dev);
  const int64_t n = integer(a[7]), cols = (int64_t)c.n_kv_heads * c.d_head;
  if (n < 0) value_error("%s is negative", "the number of rows");
  const at::ScalarType type = truth(a[8]) ? at::kFloat : at::kBFloat16;
  at::Tensor K = a[9] == Py_None ? empty({n, cols}, type, dev) : tensor(a[9], "K");
  at::Tensor V = a[10] == Py_None ? empty({n, cols}, type, dev) : tensor(a[10], "V");
  const sp_mat k = rows(K, dev, "K"), v = rows(V, dev, "V");
  const sp_status s = sp_cache_read(&c, offsets(a[6], c.n_seq, dev, "cu"), &k, &v, vector<int32_t>(a[11], at::kInt, 4, dev, "status"), stream_of(dev));
  return answer(s, {K, V});
}

// k, v, k_scale, v_scale, table, lens, Q, cu_q, n_heads, causal, scale (None: 1 / sqrt(d_head)), max_keys, out, lse, want_lse, ws, status
PyObject* cache_attention(PyObject* const* a) {
  const int dev = current_device(a[6], "Q");
  const sp_kv_cache c = cache_of(a, dev);
  const at::Tensor& Q = tensor(a[6], "Q");
  const sp_mat q = rows(Q, dev, "Q");
  const int32_t n_heads = integer32(a[8], "n_heads");
  at::Tensor O = a[12] == Py_None ? empty({q.rows, q.cols}, Q.scalar_type(), dev) : tensor(a[12], "out");
  const sp_mat o = rows(O, dev, "out");
  at::Tensor lse;
  if (a[13] != Py_None) lse = tensor(a[13], "lse");
  else if (truth(a[14])) lse = empty({q.rows, n_heads < 0 ? 0 : n_heads}, at::kFloat, dev);
  float* lse_ptr = nullptr;
  if (lse.defined()) {
    on_device(lse, dev);
    if (lse.scalar_type() != at::kFloat || lse.numel() != q.rows * n_heads || !lse.is_contiguous())
      value_error("%s must be contiguous float32 [rows of Q, n_heads]", "lse");
    lse_ptr = (float*)lse.data_ptr();
  }
  const int64_t max_keys = integer(a[11]);
  const double scale = a[10] == Py_None ? 1.0 / std::sqrt((double)(c.d_head > 0 ? c.d_head : 1)) : number(a[10]);
  const Workspace ws(a[15], sp_cache_attention_bytes(q.rows, c.n_seq, n_heads, c.n_kv_heads, c.d_head, q.dtype, c.max_pages, c.page_len, max_keys), dev);
  const sp_status s = sp_cache_attention(&c, &q, offsets(a[7], c.n_seq, dev, "cu_q"), n_heads, truth(a[9]) ? 1 : 0, scale, max_keys, &o, lse_ptr,
                                         vector<int32_t>(a[16], at::kInt, 4, dev, "status"), ws.ptr, ws.bytes, stream_of(dev));
  return answer(s, {O, lse});
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, n);
    return nullptr;
  }
  HANDLE_TH_ERRORS                         // (an allocation that fails is torch's own error)
  try {
    return F(args);
  } catch (const Raised&) {
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
template <PyObject* (*F)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
  return PyMethodDef{name, (PyCFunction)(void (*)(void))entry<F, N>, METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<rms_norm, 8>("rms_norm"),
                         method<rms_norm_grad, 9>("rms_norm_grad"),
                         method<linear_e4m3, 11>("linear_e4m3"),
                         method<cache_append, 18>("cache_append"),
                         method<cache_read, 12>("cache_read"),
                         method<cache_attention, 17>("cache_attention"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }
