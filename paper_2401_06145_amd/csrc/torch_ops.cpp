// The transformer operators for torch tensors: checks of the arguments, the outputs' memory and
// the current stream, then one call of the C-ABI.  A binding in C++ because a new token's
// kernels take about 3 us each: argument checks, allocations and the call from Python
// (ctypes) took 9 to 13 us, and take 4 to 8 here.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <sstream>

#include "spconv.h"

namespace {

constexpr int64_t kScaleBlock = 128;  // columns of an 8-bit row that share a scale

struct Api {
  decltype(&spconv_rms_norm) rms_norm = nullptr;
  decltype(&spconv_scaled_linear) scaled_linear = nullptr;
  decltype(&spconv_attention) attention = nullptr;
  decltype(&spconv_attention_workspace_bytes) workspace = nullptr;
  decltype(&spconv_rotate_heads) rotate_heads = nullptr;
  decltype(&spconv_cache_write) cache_write = nullptr;
  decltype(&spconv_cache_read) cache_read = nullptr;
  decltype(&spconv_cached_attention) cached_attention = nullptr;
  decltype(&spconv_cached_attention_workspace_bytes) cached_workspace = nullptr;
  PyObject* check = nullptr;  // (status, name): raises the library's error
} api;

// bind(functions..., check): the library's functions as addresses, in the order of Api.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr int kFunctions = 9;
  if (n != kFunctions + 1) {
    PyErr_SetString(PyExc_TypeError, "bind takes 10 arguments");
    return nullptr;
  }
  void* at[kFunctions];
  for (int i = 0; i < kFunctions; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
  if (PyErr_Occurred()) return nullptr;
  int i = 0;
  const auto take = [&](auto& f) { f = reinterpret_cast<std::decay_t<decltype(f)>>(at[i++]); };
  take(api.rms_norm);
  take(api.scaled_linear);
  take(api.attention);
  take(api.workspace);
  take(api.rotate_heads);
  take(api.cache_write);
  take(api.cache_read);
  take(api.cached_attention);
  take(api.cached_workspace);
  Py_XDECREF(api.check);
  Py_INCREF(args[kFunctions]);
  api.check = args[kFunctions];
  Py_RETURN_NONE;
}

// The error that a call ends with; `what` names the argument.
struct Refused : std::runtime_error {
  using std::runtime_error::runtime_error;
};
[[noreturn]] void refuse(const char* what, const std::string& wanted, const at::Tensor& t) {
  std::ostringstream s;
  s << what << ": expected " << wanted << ", got " << t.scalar_type() << " " << t.sizes() << " with strides " << t.strides();
  throw Refused(s.str());
}
std::string shape(std::initializer_list<int64_t> v) {
  std::ostringstream s;
  s << at::IntArrayRef(v.begin(), v.size());
  return s.str();
}

bool tensor(PyObject* o) { return THPVariable_Check(o); }
// A tensor whose derivatives nobody asks for: there are none to give.
const at::Tensor& get(PyObject* o, const char* what) {
  if (!tensor(o)) throw Refused(std::string(what) + ": expected a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if ((t.requires_grad() && at::GradMode::is_enabled()) || t._fw_grad(0).defined())
    throw Refused(std::string(what) + ": requires a gradient, and this operator is forward only (use torch.no_grad() or detach())");
  return t;
}

int dtype_of(at::ScalarType t, const char* what) {
  switch (t) {
    case at::kFloat: return SPCONV_F32;
    case at::kHalf: return SPCONV_F16;
    case at::kBFloat16: return SPCONV_BF16;
    default: throw Refused(std::string(what) + ": " + c10::toString(t) + " is not one of the layers' types");
  }
}

// Rows [n][c] whose columns follow each other; their stride (of a single row, torch's may be anything).
int64_t rows(const at::Tensor& t, const char* what, at::ScalarType dtype, int64_t n, int64_t c) {
  if (t.scalar_type() != dtype || t.dim() != 2 || t.size(0) != n || t.size(1) != c || (c > 1 && t.stride(1) != 1))
    refuse(what, std::string("rows ") + shape({n, c}) + " of " + c10::toString(dtype), t);
  return n > 1 ? t.stride(0) : c;
}
void heads(const at::Tensor& t, const char* what, at::ScalarType dtype, int64_t d) {
  if (t.scalar_type() != dtype || t.dim() != 3 || t.size(2) != d || t.stride(2) != 1)
    refuse(what, "[rows][heads][" + std::to_string(d) + "] of " + c10::toString(dtype), t);
}
// Strides of rows and of heads; those of a single row or head are never used, and may be anything.
struct Strides {
  int64_t row, head;
};
Strides strides(const at::Tensor& t) {
  const int64_t d = t.size(2);
  return {t.size(0) > 1 ? t.stride(0) : t.size(1) * d, t.size(1) > 1 ? t.stride(1) : d};
}
template <typename T>
const T* array(PyObject* o, const char* what, at::ScalarType dtype, std::initializer_list<int64_t> size, at::Device device) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = get(o, what);
  if (t.scalar_type() != dtype || t.sizes() != at::IntArrayRef(size.begin(), size.size()) || !t.is_contiguous())
    refuse(what, std::string("contiguous ") + c10::toString(dtype) + " " + shape(size), t);
  if (t.device() != device) throw Refused(std::string(what) + ": on another device");
  return static_cast<const T*>(t.data_ptr());
}
void same_device(const at::Tensor& first, std::initializer_list<const at::Tensor*> others) {
  if (!first.is_cuda()) throw Refused("expected tensors on a GPU");
  for (const at::Tensor* t : others)
    if (t && t->device() != first.device()) throw Refused("tensors on different devices");
}
void* stream_of(const at::Tensor& t) { return c10::hip::getCurrentHIPStream(t.device().index()).stream(); }
at::Tensor empty(at::IntArrayRef size, at::ScalarType dtype, const at::Tensor& like) {
  return at::Tensor(at::detail::empty_cuda(size, dtype, like.device(), std::nullopt));
}

// The library's status as a Python error; whether there is one.
bool failed(int status, const char* name) {
  if (status == SPCONV_OK) return false;
  PyObject* r = PyObject_CallFunction(api.check, "is", status, name);
  if (r) {
    Py_DECREF(r);
    PyErr_SetString(PyExc_RuntimeError, name);
  }
  return true;
}

bool truth(PyObject* o) { return PyObject_IsTrue(o) == 1; }
int whole(PyObject* o) {
  const long v = PyLong_AsLong(o);
  if (PyErr_Occurred()) throw python_error();
  if (v < INT32_MIN || v > INT32_MAX) throw Refused("a length of more than 31 bits");
  return (int)v;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw python_error();
  return (float)v;
}

#define SPC_BEGIN                                                     \
  HANDLE_TH_ERRORS                                                    \
  try {                                                               \
    if (!api.check) throw Refused("the library is not loaded");
#define SPC_END                                     \
  }                                                 \
  catch (const Refused& e) {                        \
    PyErr_SetString(PyExc_ValueError, e.what());    \
    return nullptr;                                 \
  }                                                 \
  END_HANDLE_TH_ERRORS

// rms_norm(x, gamma, residual or None, eps, bits8) -> (y, scale or None, sum or None)
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 5) throw Refused("rms_norm takes 5 arguments");
  const at::Tensor& x = get(args[0], "x");
  if (x.dim() != 2) refuse("x", "rows", x);
  const int64_t n = x.size(0), c = x.size(1);
  if (c > INT32_MAX) throw Refused("x: more than 2^31 - 1 columns");
  const at::ScalarType t = x.scalar_type();
  const int dtype = dtype_of(t, "x");
  const int64_t ld_x = rows(x, "x", t, n, c);
  const void* gamma = array<void>(args[1], "gamma", t, {c}, x.device());
  const bool bits8 = truth(args[4]);
  at::Tensor sum, scale;
  const at::Tensor* res = nullptr;
  int64_t ld_res = 0;
  if (args[2] != Py_None) {
    res = &get(args[2], "residual");
    ld_res = rows(*res, "residual", t, n, c);
  }
  same_device(x, {res});
  const c10::OptionalDeviceGuard guard(x.device());
  const int64_t blocks = (c + kScaleBlock - 1) / kScaleBlock;
  if (res) sum = empty({n, c}, t, x);
  at::Tensor y = empty({n, c}, bits8 ? at::kFloat8_e4m3fn : t, x);
  if (bits8) scale = empty({n, blocks}, at::kFloat, x);
  if (failed(api.rms_norm(x.data_ptr(), ld_x, res ? res->data_ptr() : nullptr, ld_res, gamma, res ? sum.data_ptr() : nullptr,
                          c, y.data_ptr(), c, bits8 ? static_cast<float*>(scale.data_ptr()) : nullptr, blocks, n, (int)c,
                          dtype, bits8, real(args[3]), stream_of(x)),
             "spconv_rms_norm"))
    return nullptr;
  PyObject* out = PyTuple_New(3);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(y)));
  PyTuple_SET_ITEM(out, 1, bits8 ? THPVariable_Wrap(std::move(scale)) : (Py_INCREF(Py_None), Py_None));
  PyTuple_SET_ITEM(out, 2, res ? THPVariable_Wrap(std::move(sum)) : (Py_INCREF(Py_None), Py_None));
  return out;
  SPC_END
}

// scaled_linear(x, x_scale, w, w_scale, dtype, relu, exact) -> y
PyObject* scaled_linear(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 7) throw Refused("scaled_linear takes 7 arguments");
  const at::Tensor &x = get(args[0], "x"), &xs = get(args[1], "x_scale"), &w = get(args[2], "w"), &ws = get(args[3], "w_scale");
  if (x.dim() != 2) refuse("x", "rows", x);
  if (w.dim() != 2) refuse("w", "rows", w);
  if (!THPDtype_Check(args[4])) throw Refused("dtype: expected a torch.dtype");
  const at::ScalarType t = reinterpret_cast<THPDtype*>(args[4])->scalar_type;
  const int dtype = dtype_of(t, "dtype");
  const int64_t m = x.size(0), k = x.size(1), n = w.size(0), kb = (k + kScaleBlock - 1) / kScaleBlock;
  const int64_t ld_x = rows(x, "x", at::kFloat8_e4m3fn, m, k), ld_w = rows(w, "w", at::kFloat8_e4m3fn, n, k);
  const int64_t ld_xs = rows(xs, "x_scale", at::kFloat, m, kb);
  const int64_t ld_ws = rows(ws, "w_scale", at::kFloat, (n + kScaleBlock - 1) / kScaleBlock, kb);
  if (n > INT32_MAX || k > INT32_MAX) throw Refused("more than 2^31 - 1 columns or outputs");
  same_device(x, {&xs, &w, &ws});
  const c10::OptionalDeviceGuard guard(x.device());
  at::Tensor y = empty({m, n}, t, x);
  if (failed(api.scaled_linear(x.data_ptr(), ld_x, static_cast<const float*>(xs.data_ptr()), ld_xs, w.data_ptr(), ld_w,
                               static_cast<const float*>(ws.data_ptr()), ld_ws, y.data_ptr(), n, m, (int)n, (int)k, dtype,
                               truth(args[5]), truth(args[6]), stream_of(x)),
             "spconv_scaled_linear"))
    return nullptr;
  return THPVariable_Wrap(std::move(y));
  SPC_END
}

// attention(q, k, v, q_start, k_start, max_q, max_k, k_len, prefix, causal, scale or None, cap, slopes,
//           q_pos, k_pos) -> out
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 15) throw Refused("attention takes 15 arguments");
  const at::Tensor &q = get(args[0], "q"), &k = get(args[1], "k"), &v = get(args[2], "v");
  const at::Tensor& q_start = get(args[3], "q_start");
  if (q.dim() != 3) refuse("q", "[rows][heads][width]", q);
  const at::ScalarType t = q.scalar_type();
  spconv_attention_args a = {};
  a.dtype = dtype_of(t, "q");
  const int64_t d = q.size(2);
  heads(q, "q", t, d);
  heads(k, "k", t, d);
  heads(v, "v", t, d);
  if (v.sizes() != k.sizes()) refuse("v", "k's shape", v);
  if (q_start.dim() != 1 || q_start.size(0) < 1) refuse("q_start", "contiguous Int [docs + 1]", q_start);
  const int64_t docs = q_start.size(0) - 1;
  if (q.size(1) > INT32_MAX || k.size(1) > INT32_MAX || d > INT32_MAX || docs > INT32_MAX) throw Refused("sizes of more than 31 bits");
  a.n_q = q.size(0), a.n_k = k.size(0), a.n_docs = (int)docs;
  a.heads = (int)q.size(1), a.kv_heads = (int)k.size(1), a.head_dim = (int)d;
  a.d_q_start = array<int32_t>(args[3], "q_start", at::kInt, {docs + 1}, q.device());
  a.d_k_start = array<int32_t>(args[4], "k_start", at::kInt, {docs + 1}, q.device());
  a.max_q = whole(args[5]), a.max_k = whole(args[6]);
  a.d_k_len = array<int32_t>(args[7], "k_len", at::kInt, {docs}, q.device());
  a.d_prefix = array<int32_t>(args[8], "prefix", at::kInt, {docs}, q.device());
  a.causal = truth(args[9]);
  a.scale = args[10] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : real(args[10]);
  a.cap = real(args[11]);
  a.d_slopes = array<float>(args[12], "slopes", at::kFloat, {q.size(1)}, q.device());
  a.d_q_pos = array<int32_t>(args[13], "q_pos", at::kInt, {a.n_q, 4}, q.device());
  a.d_k_pos = array<int32_t>(args[14], "k_pos", at::kInt, {a.n_k, 4}, q.device());
  same_device(q, {&k, &v});
  const c10::OptionalDeviceGuard guard(q.device());
  at::Tensor out = empty(q.sizes(), t, q);
  a.d_q = q.data_ptr(), a.d_k = k.data_ptr(), a.d_v = v.data_ptr(), a.d_out = out.data_ptr();
  const Strides sq = strides(q), sk = strides(k), sv = strides(v), so = strides(out);
  a.q_row = sq.row, a.q_head = sq.head, a.k_row = sk.row, a.k_head = sk.head;
  a.v_row = sv.row, a.v_head = sv.head, a.out_row = so.row, a.out_head = so.head;
  const size_t need = api.workspace(&a);
  at::Tensor workspace;
  if (need) workspace = empty({(int64_t)need}, at::kByte, q);
  if (failed(api.attention(&a, need ? workspace.data_ptr() : nullptr, need, stream_of(q)), "spconv_attention")) return nullptr;
  return THPVariable_Wrap(std::move(out));
  SPC_END
}

// rotate_heads(q, k or None, pos, freq, q_gamma, k_gamma, eps, interleaved, gain) -> (q, k or None)
PyObject* rotate_heads(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 9) throw Refused("rotate_heads takes 9 arguments");
  const at::Tensor &q = get(args[0], "q"), &pos = get(args[2], "pos"), &freq = get(args[3], "freq");
  if (q.dim() != 3) refuse("q", "[rows][heads][width]", q);
  const at::ScalarType t = q.scalar_type();
  spconv_rotation r = {};
  r.dtype = dtype_of(t, "q");
  const int64_t n = q.size(0), d = q.size(2);
  heads(q, "q", t, d);
  const at::Tensor* k = args[1] == Py_None ? nullptr : &get(args[1], "k");
  if (k) {
    heads(*k, "k", t, d);
    if (k->size(0) != n) refuse("k", "as many rows as q", *k);
  }
  if (pos.dim() < 1 || pos.dim() > 2) refuse("pos", "contiguous Int [rows] or [rows][4]", pos);
  if (freq.dim() != 1) refuse("freq", "contiguous Double [rotated / 2]", freq);
  if (q.size(1) > INT32_MAX || d > INT32_MAX || freq.size(0) > INT32_MAX / 2 || (k && k->size(1) > INT32_MAX))
    throw Refused("sizes of more than 31 bits");
  r.n = n, r.heads = (int)q.size(1), r.kv_heads = k ? (int)k->size(1) : 0, r.head_dim = (int)d;
  r.rotated = 2 * (int)freq.size(0);
  r.voxels = pos.dim() == 2;
  r.d_pos = r.voxels ? array<int32_t>(args[2], "pos", at::kInt, {n, 4}, q.device())
                     : array<int32_t>(args[2], "pos", at::kInt, {n}, q.device());
  r.d_freq = array<double>(args[3], "freq", at::kDouble, {freq.size(0)}, q.device());
  r.d_q_gamma = array<void>(args[4], "q_gamma", t, {d}, q.device());
  r.d_k_gamma = array<void>(args[5], "k_gamma", t, {d}, q.device());
  r.eps = real(args[6]), r.interleaved = truth(args[7]), r.gain = real(args[8]);
  same_device(q, {k});
  const c10::OptionalDeviceGuard guard(q.device());
  at::Tensor q_out = empty(q.sizes(), t, q), k_out;
  if (k) k_out = empty(k->sizes(), t, q);
  const auto place = [](const at::Tensor& x, int64_t* row, int64_t* head) {
    const Strides s = strides(x);
    *row = s.row, *head = s.head;
  };
  r.d_q = q.data_ptr(), r.d_q_out = q_out.data_ptr();
  place(q, &r.q_row, &r.q_head);
  place(q_out, &r.q_out_row, &r.q_out_head);
  if (k) {
    r.d_k = k->data_ptr(), r.d_k_out = k_out.data_ptr();
    place(*k, &r.k_row, &r.k_head);
    place(k_out, &r.k_out_row, &r.k_out_head);
  }
  if (failed(api.rotate_heads(&r, stream_of(q)), "spconv_rotate_heads")) return nullptr;
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(q_out)));
  PyTuple_SET_ITEM(out, 1, k ? THPVariable_Wrap(std::move(k_out)) : (Py_INCREF(Py_None), Py_None));
  return out;
  SPC_END
}

// The pages of args[0..3] (keys, values, their scales or None), and the table args[table].
struct Pages {
  spconv_pages p = {};
  const at::Tensor* k;
  bool bits8;
};
Pages get_pages(PyObject* const* args, PyObject* table_arg) {
  Pages g;
  const at::Tensor &k = get(args[0], "pages of keys"), &v = get(args[1], "pages of values"), &table = get(table_arg, "table");
  g.k = &k;
  if (k.dim() != 4) refuse("pages of keys", "[pages][heads][rows][width]", k);
  g.bits8 = k.scalar_type() == at::kFloat8_e4m3fn;
  const int64_t pages = k.size(0), heads = k.size(1), page = k.size(2), d = k.size(3);
  if (heads > INT32_MAX || page > INT32_MAX || d > INT32_MAX) throw Refused("sizes of more than 31 bits");
  if (v.scalar_type() != k.scalar_type() || v.sizes() != k.sizes()) refuse("pages of values", "the keys' shape and type", v);
  if (!k.is_contiguous() || !v.is_contiguous()) throw Refused("pages: not contiguous");
  if ((args[2] != Py_None) != g.bits8 || (args[3] != Py_None) != g.bits8)
    throw Refused("scales belong to pages of 8 bits (Float8_e4m3fn), and to no others");
  if (v.device() != k.device()) throw Refused("tensors on different devices");
  g.p.d_k = k.data_ptr(), g.p.d_v = v.data_ptr();
  g.p.d_k_scale = const_cast<float*>(array<float>(args[2], "scales of keys", at::kFloat, {pages, heads, page}, k.device()));
  g.p.d_v_scale = const_cast<float*>(array<float>(args[3], "scales of values", at::kFloat, {pages, heads, page}, k.device()));
  if (table.dim() != 2 || table.size(0) > INT32_MAX || table.size(1) > INT32_MAX) refuse("table", "contiguous Int [docs][pages]", table);
  g.p.d_table = array<int32_t>(table_arg, "table", at::kInt, {table.size(0), table.size(1)}, k.device());
  g.p.n_pages = pages, g.p.n_docs = (int)table.size(0), g.p.table_row = (int)table.size(1);
  g.p.page = (int)page, g.p.kv_heads = (int)heads, g.p.head_dim = (int)d;
  // no page has no address, but is still one of 8 bits
  static float nothing;
  if (g.bits8 && !g.p.d_k_scale) g.p.d_k_scale = g.p.d_v_scale = &nothing;
  return g;
}
void same_type(const Pages& g, at::ScalarType t) {
  if (!g.bits8 && g.k->scalar_type() != t)
    throw Refused(std::string("pages of ") + c10::toString(g.k->scalar_type()) + " and rows of " + c10::toString(t));
}

// cache_write(pages of keys, of values, scales of keys, of values, k, v, q_start, k_len, table)
PyObject* cache_write(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 9) throw Refused("cache_write takes 9 arguments");
  const Pages g = get_pages(args, args[8]);
  const at::Tensor &k = get(args[4], "k"), &v = get(args[5], "v");
  const at::ScalarType t = k.scalar_type();
  const int dtype = dtype_of(t, "k");
  same_type(g, t);
  heads(k, "k", t, g.p.head_dim);
  heads(v, "v", t, g.p.head_dim);
  if (k.size(1) != g.p.kv_heads) refuse("k", "the pages' heads", k);
  if (v.sizes() != k.sizes()) refuse("v", "k's shape", v);
  const int64_t docs = g.p.n_docs;
  get(args[6], "q_start"), get(args[7], "k_len");
  const int32_t* start = array<int32_t>(args[6], "q_start", at::kInt, {docs + 1}, k.device());
  const int32_t* len = array<int32_t>(args[7], "k_len", at::kInt, {docs}, k.device());
  same_device(k, {&v, g.k});
  const c10::OptionalDeviceGuard guard(k.device());
  const Strides sk = strides(k), sv = strides(v);
  if (failed(api.cache_write(&g.p, k.data_ptr(), sk.row, sk.head, v.data_ptr(), sv.row, sv.head, start, len, k.size(0), dtype,
                             stream_of(k)),
             "spconv_cache_write"))
    return nullptr;
  Py_RETURN_NONE;
  SPC_END
}

// cache_read(pages of keys, of values, scales of keys, of values, start, table, rows, dtype) -> (k, v)
PyObject* cache_read(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 8) throw Refused("cache_read takes 8 arguments");
  const Pages g = get_pages(args, args[5]);
  if (!THPDtype_Check(args[7])) throw Refused("dtype: expected a torch.dtype");
  const at::ScalarType t = reinterpret_cast<THPDtype*>(args[7])->scalar_type;
  const int dtype = dtype_of(t, "dtype");
  same_type(g, t);
  get(args[4], "start");
  const int32_t* start = array<int32_t>(args[4], "start", at::kInt, {(int64_t)g.p.n_docs + 1}, g.k->device());
  const int64_t rows = whole(args[6]);
  if (rows < 0) throw Refused("rows: negative");
  same_device(*g.k, {});
  const c10::OptionalDeviceGuard guard(g.k->device());
  at::Tensor k = empty({rows, g.p.kv_heads, g.p.head_dim}, t, *g.k), v = empty(k.sizes(), t, *g.k);
  const Strides s = strides(k);
  if (failed(api.cache_read(&g.p, k.data_ptr(), s.row, s.head, v.data_ptr(), s.row, s.head, start, rows, dtype, stream_of(*g.k)),
             "spconv_cache_read"))
    return nullptr;
  PyObject* out = PyTuple_New(2);
  if (!out) return nullptr;
  PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(std::move(k)));
  PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(std::move(v)));
  return out;
  SPC_END
}

// cached_attention(pages of keys, of values, scales of keys, of values, q, q_start, k_len, table, max_q, max_k,
//                  prefix, causal, scale or None, cap, slopes) -> out
PyObject* cached_attention(PyObject*, PyObject* const* args, Py_ssize_t count) {
  SPC_BEGIN
  if (count != 15) throw Refused("cached_attention takes 15 arguments");
  const Pages g = get_pages(args, args[7]);
  const at::Tensor& q = get(args[4], "q");
  if (q.dim() != 3) refuse("q", "[rows][heads][width]", q);
  const at::ScalarType t = q.scalar_type();
  spconv_attention_args a = {};
  a.dtype = dtype_of(t, "q");
  same_type(g, t);
  heads(q, "q", t, g.p.head_dim);
  const int64_t docs = g.p.n_docs;
  if (q.size(1) > INT32_MAX) throw Refused("sizes of more than 31 bits");
  a.n_q = q.size(0), a.n_docs = g.p.n_docs;
  a.heads = (int)q.size(1), a.kv_heads = g.p.kv_heads, a.head_dim = g.p.head_dim;
  get(args[5], "q_start"), get(args[6], "k_len");
  a.d_q_start = array<int32_t>(args[5], "q_start", at::kInt, {docs + 1}, q.device());
  a.d_k_len = array<int32_t>(args[6], "k_len", at::kInt, {docs}, q.device());
  a.max_q = whole(args[8]), a.max_k = whole(args[9]);
  a.d_prefix = array<int32_t>(args[10], "prefix", at::kInt, {docs}, q.device());
  a.causal = truth(args[11]);
  a.scale = args[12] == Py_None ? (float)(1.0 / std::sqrt((double)a.head_dim)) : real(args[12]);
  a.cap = real(args[13]);
  a.d_slopes = array<float>(args[14], "slopes", at::kFloat, {q.size(1)}, q.device());
  same_device(q, {g.k});
  const c10::OptionalDeviceGuard guard(q.device());
  at::Tensor out = empty(q.sizes(), t, q);
  a.d_q = q.data_ptr(), a.d_out = out.data_ptr();
  const Strides sq = strides(q), so = strides(out);
  a.q_row = sq.row, a.q_head = sq.head, a.out_row = so.row, a.out_head = so.head;
  const size_t need = api.cached_workspace(&g.p, &a);
  at::Tensor workspace;
  if (need) workspace = empty({(int64_t)need}, at::kByte, q);
  if (failed(api.cached_attention(&g.p, &a, need ? workspace.data_ptr() : nullptr, need, stream_of(q)),
             "spconv_cached_attention"))
    return nullptr;
  return THPVariable_Wrap(std::move(out));
  SPC_END
}

#define SPC_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SPC_METHOD(bind), SPC_METHOD(rms_norm), SPC_METHOD(scaled_linear), SPC_METHOD(attention),
                         SPC_METHOD(rotate_heads), SPC_METHOD(cache_write), SPC_METHOD(cache_read),
                         SPC_METHOD(cached_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_ops() { return PyModule_Create(&module); }
