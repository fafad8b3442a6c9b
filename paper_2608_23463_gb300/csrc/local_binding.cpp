// Native part of local.py: checks tensors, allocates results and calls the C
// ABI (include/proxyformer.h) of the local stream's operators on the current
// stream of the tensors' device.  Where a token or two is served the kernels
// take 2 to 8 us; the same work in Python through ctypes took 11 a call, 4 so.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "proxyformer.h"

namespace {

PyObject* g_error = nullptr;  // ProxyFormerError(status, message)

// A Python exception is set.
struct Raised {};

[[noreturn]] void raise(pf_status s, const std::string& msg) {
  PyObject* e = PyObject_CallFunction(g_error, "is", (int)s, msg.c_str());
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  }
  throw Raised{};
}

void check(pf_status s) {
  if (s != PF_OK) raise(s, pf_last_error());
}

bool none(PyObject* o) { return o == Py_None; }

const at::Tensor& tensor(const char* name, PyObject* o) {
  if (!THPVariable_Check(o)) raise(PF_ERR_INVALID_ARG, std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}

template <class T>
T* address(PyObject* o) {
  return reinterpret_cast<T*>(integer(o));
}

// A matrix as the library takes it: [rows, width] on the GPU, the values of a row side
// by side.
struct Rows {
  void* p;
  int64_t ld;
};
Rows rows_of(const char* name, const at::Tensor& t, int64_t rows, int64_t width, at::ScalarType type,
             c10::Device dev) {
  if (t.dim() != 2 || t.size(0) != rows || t.size(1) != width || t.scalar_type() != type ||
      !t.is_cuda() || t.device() != dev || (width > 1 && t.stride(1) != 1))
    raise(PF_ERR_INVALID_ARG, std::string(name) + " must be a [" + std::to_string(rows) + ", " +
                                  std::to_string(width) + "] " + c10::toString(type) +
                                  " matrix with contiguous rows on one GPU");
  return {t.data_ptr(), rows > 1 ? t.stride(0) : width};  // the stride of a single row says nothing
}

// Contiguous values of a type; null for None.
template <class T>
T* values(const char* name, PyObject* o, at::IntArrayRef shape, at::ScalarType type, c10::Device dev) {
  if (none(o)) return nullptr;
  const at::Tensor& t = tensor(name, o);
  if (t.sizes() != shape || t.scalar_type() != type || t.device() != dev || !t.is_contiguous())
    raise(PF_ERR_INVALID_ARG, std::string(name) + " has another shape, type or device than it needs");
  return static_cast<T*>(t.data_ptr());
}

// Scratch of an object, read and written on the current stream.  The object may drop it while
// that stream still uses it: its memory then waits for the stream, whichever it was made on.
void* bytes(const char* name, PyObject* o, c10::Device dev, size_t* n) {
  if (none(o)) {
    *n = 0;
    return nullptr;
  }
  const at::Tensor& t = tensor(name, o);
  if (t.scalar_type() != at::kByte || t.device() != dev || !t.is_contiguous())
    raise(PF_ERR_INVALID_ARG, std::string(name) + " must be contiguous bytes on the tensors' GPU");
  c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(),
                                                c10::cuda::getCurrentCUDAStream(dev.index()));
  *n = (size_t)t.numel();
  return t.data_ptr();
}

c10::Device cuda_device(const char* name, const at::Tensor& t) {
  if (!t.is_cuda()) raise(PF_ERR_INVALID_ARG, std::string(name) + " must be on a GPU");
  return t.device();
}

at::Tensor new_rows(int64_t rows, int64_t width, at::ScalarType type, c10::Device dev) {
  return at::empty({rows, width}, at::TensorOptions().dtype(type).device(dev));
}

// A result: the given tensor, or a new one.
at::Tensor result(PyObject* o, int64_t rows, int64_t width, at::ScalarType type, c10::Device dev) {
  return none(o) ? new_rows(rows, width, type, dev) : tensor("out", o);
}

// The call, without the interpreter's lock (it waits where the device's queue is full).
template <class F>
void call(c10::Device dev, F f) {
  const c10::cuda::CUDAGuard guard(dev);
  void* stream = c10::cuda::getCurrentCUDAStream(dev.index()).stream();
  pf_status s;
  Py_BEGIN_ALLOW_THREADS;
  s = f(stream);
  Py_END_ALLOW_THREADS;
  check(s);
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }

// Python's tuple of the results; those of a null tensor are None.
template <class... T>
PyObject* tuple(const T&... t) {
  PyObject* o = PyTuple_New(sizeof...(t));
  if (!o) throw Raised{};
  Py_ssize_t i = 0;
  auto put = [&](const at::Tensor& x) {
    PyObject* v = x.defined() ? wrap(x) : (Py_INCREF(Py_None), Py_None);
    PyTuple_SET_ITEM(o, i++, v);
    return v != nullptr;
  };
  if (!(put(t) && ...)) {
    Py_DECREF(o);
    throw Raised{};
  }
  return o;
}

at::ScalarType type_of(const pf_qk_desc& d) { return d.dtype == PF_F32 ? at::kFloat : at::kBFloat16; }

int64_t row_count(const char* name, const at::Tensor& t) {
  if (t.dim() != 2) raise(PF_ERR_INVALID_ARG, std::string(name) + " must be a matrix");
  return t.size(0);
}

pf_qkv qk_rows(const pf_qk_desc& d, int64_t n, const char* nq, const at::Tensor& q, const char* nk,
               const at::Tensor& k, c10::Device dev) {
  const Rows a = rows_of(nq, q, n, (int64_t)d.n_heads * d.dh, type_of(d), dev);
  const Rows b = rows_of(nk, k, n, (int64_t)d.n_kv * d.dh, type_of(d), dev);
  return {a.p, b.p, nullptr, a.ld, b.ld, 0};
}

// rope_fwd(desc, q, k, L, w_q, w_k, pos, out_q, out_k) -> (q, k)
PyObject* rope_fwd(PyObject* const* a) {
  const pf_qk_desc& d = *address<pf_qk_desc>(a[0]);
  const at::Tensor &q = tensor("q", a[1]), &k = tensor("k", a[2]);
  const c10::Device dev = cuda_device("q", q);
  const int64_t n = row_count("q", q), L = none(a[3]) ? std::max<int64_t>(n, 1) : integer(a[3]);
  const pf_qkv x = qk_rows(d, n, "q", q, "k", k, dev);
  const float* w_q = values<float>("w_q", a[4], {d.dh}, at::kFloat, dev);
  const float* w_k = values<float>("w_k", a[5], {d.dh}, at::kFloat, dev);
  const int32_t* pos = values<int32_t>("pos", a[6], {n, d.n_axes}, at::kInt, dev);
  const at::Tensor oq = result(a[7], n, q.size(1), type_of(d), dev),
                   ok = result(a[8], n, k.size(1), type_of(d), dev);
  const pf_qkv o = qk_rows(d, n, "out q", oq, "out k", ok, dev);
  call(dev, [&](void* s) { return pf_qk_rope_fwd(&d, n, L, &x, w_q, w_k, pos, &o, s); });
  return tuple(oq, ok);
}

// rope_bwd(desc, q, k, dq, dk, L, w_q, w_k, pos, out_q, out_k, ws) -> (dq, dk, dw_q, dw_k)
PyObject* rope_bwd(PyObject* const* a) {
  const pf_qk_desc& d = *address<pf_qk_desc>(a[0]);
  const at::Tensor &q = tensor("q", a[1]), &k = tensor("k", a[2]);
  const c10::Device dev = cuda_device("q", q);
  const int64_t n = row_count("q", q), L = none(a[5]) ? std::max<int64_t>(n, 1) : integer(a[5]);
  const pf_qkv x = qk_rows(d, n, "q", q, "k", k, dev);
  const pf_qkv g = qk_rows(d, n, "dq", tensor("dq", a[3]), "dk", tensor("dk", a[4]), dev);
  const float* w_q = values<float>("w_q", a[6], {d.dh}, at::kFloat, dev);
  const float* w_k = values<float>("w_k", a[7], {d.dh}, at::kFloat, dev);
  const int32_t* pos = values<int32_t>("pos", a[8], {n, d.n_axes}, at::kInt, dev);
  const at::Tensor oq = result(a[9], n, q.size(1), type_of(d), dev),
                   ok = result(a[10], n, k.size(1), type_of(d), dev);
  const pf_qkv o = qk_rows(d, n, "out q", oq, "out k", ok, dev);
  const auto weights = at::TensorOptions().dtype(at::kFloat).device(dev);
  at::Tensor dw_q, dw_k;
  if (w_q) dw_q = at::empty({d.dh}, weights);
  if (w_k) dw_k = at::empty({d.dh}, weights);
  float* g_q = w_q ? dw_q.data_ptr<float>() : nullptr;
  float* g_k = w_k ? dw_k.data_ptr<float>() : nullptr;
  size_t size;
  void* ws = bytes("ws", a[11], dev, &size);
  call(dev, [&](void* s) {
    return pf_qk_rope_bwd(&d, n, L, &x, w_q, w_k, pos, &g, &o, g_q, g_k, ws, size, s);
  });
  return tuple(oq, ok, dw_q, dw_k);
}

pf_qkv window_rows(const pf_window_desc& d, const char* const* names, const at::Tensor& q,
                   const at::Tensor& k, const at::Tensor& v, c10::Device dev) {
  const int64_t n = (int64_t)d.batch * d.L, nk = (int64_t)d.n_kv * d.dh;
  const Rows a = rows_of(names[0], q, n, (int64_t)d.n_heads * d.dh, at::kBFloat16, dev);
  const Rows b = rows_of(names[1], k, n, nk, at::kBFloat16, dev);
  const Rows c = rows_of(names[2], v, n, nk, at::kBFloat16, dev);
  return {a.p, b.p, c.p, a.ld, b.ld, c.ld};
}
const char* const kInputs[] = {"q", "k", "v"};
const char* const kGradients[] = {"dq", "dk", "dv"};

// window_fwd(desc, q, k, v, out, size of saved or 0) -> (out, saved or None)
PyObject* window_fwd(PyObject* const* a) {
  const pf_window_desc& d = *address<pf_window_desc>(a[0]);
  const at::Tensor &q = tensor("q", a[1]), &k = tensor("k", a[2]), &v = tensor("v", a[3]);
  const c10::Device dev = cuda_device("q", q);
  const int64_t n = (int64_t)d.batch * d.L, nq = (int64_t)d.n_heads * d.dh, size = integer(a[5]);
  const pf_qkv x = window_rows(d, kInputs, q, k, v, dev);
  const at::Tensor out = result(a[4], n, nq, at::kBFloat16, dev);
  const Rows o = rows_of("out", out, n, nq, at::kBFloat16, dev);
  at::Tensor saved;
  if (size > 0) saved = at::empty({size}, at::TensorOptions().dtype(at::kByte).device(dev));
  void* keep = size > 0 ? saved.data_ptr() : nullptr;
  call(dev, [&](void* s) { return pf_window_attn_fwd(&d, &x, o.p, o.ld, keep, s); });
  return tuple(out, saved);
}

// window_bwd(desc, q, k, v, out, dout, saved, dq, dk, dv, ws) -> (dq, dk, dv)
PyObject* window_bwd(PyObject* const* a) {
  const pf_window_desc& d = *address<pf_window_desc>(a[0]);
  const at::Tensor &q = tensor("q", a[1]), &k = tensor("k", a[2]), &v = tensor("v", a[3]);
  const c10::Device dev = cuda_device("q", q);
  const int64_t n = (int64_t)d.batch * d.L, nq = (int64_t)d.n_heads * d.dh, nk = (int64_t)d.n_kv * d.dh;
  const pf_qkv x = window_rows(d, kInputs, q, k, v, dev);
  const Rows o = rows_of("out", tensor("out", a[4]), n, nq, at::kBFloat16, dev);
  const Rows g = rows_of("dout", tensor("dout", a[5]), n, nq, at::kBFloat16, dev);
  size_t kept, size;
  const void* saved = bytes("saved", a[6], dev, &kept);
  if (kept < pf_window_attn_saved_size(&d))
    raise(PF_ERR_INVALID_ARG, "backward needs what a forward with train=True has saved");
  const at::Tensor dq = result(a[7], n, nq, at::kBFloat16, dev),
                   dk = result(a[8], n, nk, at::kBFloat16, dev),
                   dv = result(a[9], n, nk, at::kBFloat16, dev);
  const pf_qkv dx = window_rows(d, kGradients, dq, dk, dv, dev);
  void* ws = bytes("ws", a[10], dev, &size);
  call(dev, [&](void* s) {
    return pf_window_attn_bwd(&d, &x, o.p, o.ld, saved, g.p, g.ld, &dx, ws, size, s);
  });
  return tuple(dq, dk, dv);
}

// paged_append(desc, qk_desc, cache, len, q or None, k, v, w_q, w_k, start, pos, out) -> q or None
PyObject* paged_append(PyObject* const* a) {
  const pf_paged_desc& d = *address<pf_paged_desc>(a[0]);
  const pf_qk_desc& r = *address<pf_qk_desc>(a[1]);
  pf_paged_cache* cache = address<pf_paged_cache>(a[2]);
  const at::Tensor &k = tensor("k", a[5]), &v = tensor("v", a[6]);
  const c10::Device dev = cuda_device("k", k);
  values<int32_t>("len", a[3], {d.batch}, at::kInt, dev);  // the cache is on that GPU
  const int64_t n = row_count("k", k), nq = (int64_t)d.n_heads * d.dh, nk = (int64_t)d.n_kv * d.dh;
  const Rows kr = rows_of("k", k, n, nk, at::kBFloat16, dev), vr = rows_of("v", v, n, nk, at::kBFloat16, dev);
  Rows qr{nullptr, 0}, o{nullptr, 0};
  at::Tensor out;
  if (!none(a[4])) {
    qr = rows_of("q", tensor("q", a[4]), n, nq, at::kBFloat16, dev);
    out = result(a[11], n, nq, at::kBFloat16, dev);
    o = rows_of("out", out, n, nq, at::kBFloat16, dev);
  }
  const float* w_q = values<float>("w_q", a[7], {r.dh}, at::kFloat, dev);
  const float* w_k = values<float>("w_k", a[8], {r.dh}, at::kFloat, dev);
  const int32_t* start = values<int32_t>("start", a[9], {d.batch + 1}, at::kInt, dev);
  const int32_t* pos = values<int32_t>("pos", a[10], {n, r.n_axes}, at::kInt, dev);
  const pf_qkv x = {qr.p, kr.p, vr.p, qr.ld, kr.ld, vr.ld};
  call(dev, [&](void* s) {
    return pf_paged_append(&d, &r, n, &x, w_q, w_k, start, pos, cache, o.p, o.ld, s);
  });
  if (!out.defined()) Py_RETURN_NONE;
  return wrap(out);
}

// paged_attn(desc, cache, q, out, ws) -> out
PyObject* paged_attn(PyObject* const* a) {
  const pf_paged_desc& d = *address<pf_paged_desc>(a[0]);
  const pf_paged_cache* cache = address<pf_paged_cache>(a[1]);
  const at::Tensor& q = tensor("q", a[2]);
  const c10::Device dev = cuda_device("q", q);
  const int64_t nq = (int64_t)d.n_heads * d.dh;
  const Rows qr = rows_of("q", q, d.batch, nq, at::kBFloat16, dev);
  const at::Tensor out = result(a[3], d.batch, nq, at::kBFloat16, dev);
  const Rows o = rows_of("out", out, d.batch, nq, at::kBFloat16, dev);
  size_t size;
  void* ws = bytes("ws", a[4], dev, &size);
  call(dev, [&](void* s) {
    return pf_paged_attn(&d, qr.p, qr.ld, cache, o.p, o.ld, ws, size, s);
  });
  return wrap(out);
}

// One of the functions above as Python calls it: N arguments, C++ exceptions turned into
// Python's.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments, not %zd", N, n);
    return nullptr;
  }
  try {
    return F(a);
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* init(PyObject*, PyObject* error) {
  Py_INCREF(error);
  Py_XDECREF(g_error);
  g_error = error;
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), int N>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<F, N>)), METH_FASTCALL,
          nullptr};
}

PyMethodDef kMethods[] = {
    {"init", init, METH_O, nullptr},
    method<rope_fwd, 9>("rope_fwd"),
    method<rope_bwd, 12>("rope_bwd"),
    method<window_fwd, 6>("window_fwd"),
    method<window_bwd, 11>("window_bwd"),
    method<paged_append, 12>("paged_append"),
    method<paged_attn, 5>("paged_attn"),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_local", nullptr, -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__local() {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddStringConstant(m, "built_for", PF_BUILT_FOR) < 0) {
    Py_DECREF(m);
    m = nullptr;
  }
  return m;
}
