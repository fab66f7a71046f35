// The matmul entry points' way from Python tensors to the C ABI: what binding.py does through ctypes, for plain calls.
//
// A small matmul takes 2 us on the device and 2 to launch; reading the tensors' attributes one by one from Python and marshalling eight
// arguments through ctypes took as long again (1 x 1024 x 1024, host-bound: 4.9 us a call, 2.8 with this and the plans remembered).
// matmul() and gemv_host() take the address of the library's function and the type that a descriptor must have, and return the
// library's return code, or None for anything that is not a plain call; binding.py then takes its own way, which also raises what there
// is to raise.  Nothing is kept between calls.  The 8-bit calls (quant_i8, gemm_i8, kv8_append, attn_kv8) return their tensors where the
// library returns 0, and allocate those that the caller did not bring.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAStream.h>
#include <cmath>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/razer.h"

namespace {

typedef int (*MatmulFn)(const razer_desc*, const void*, const void*, int, void*, void*, size_t, void*);
typedef int (*HostFn)(const razer_desc*, const void*, const void*, int, void*, void*, void*, void*, size_t, void*);

// The descriptor behind binding.RazerDesc (a ctypes structure: its memory through the buffer protocol).
struct Desc {
  Py_buffer view;
  bool held = false;
  const razer_desc* get(PyObject* type, PyObject* o) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != type) return nullptr;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
      PyErr_Clear();
      return nullptr;
    }
    held = true;
    return view.len == (Py_ssize_t)sizeof(razer_desc) ? static_cast<const razer_desc*>(view.buf) : nullptr;
  }
  ~Desc() {
    if (held) PyBuffer_Release(&view);
  }
};

// Plain torch.Tensor or Parameter objects only: a subclass may have attributes of its own.
bool plain(PyObject* o) { return THPVariable_CheckExact(o); }
const at::Tensor& tensor(PyObject* o) { return THPVariable_Unpack(o); }
bool dense(const at::Tensor& t) { return t.has_storage() && t.layout() == at::kStrided; }

void* address(PyObject* o) {
  void* p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
  if (PyErr_Occurred()) PyErr_Clear();
  return p;
}

// matmul(function, descriptor type, desc, packed, x, y, workspace)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7 || !plain(a[3]) || !plain(a[4]) || !plain(a[5]) || !plain(a[6])) Py_RETURN_NONE;
  const MatmulFn fn = reinterpret_cast<MatmulFn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    const at::Tensor &packed = tensor(a[3]), &x = tensor(a[4]), &y = tensor(a[5]), &ws = tensor(a[6]);
    Desc d;
    const razer_desc* desc = d.get(a[1], a[2]);
    if (!desc || !dense(packed) || !dense(x) || !dense(y) || !dense(ws) || !x.is_cuda() || x.scalar_type() != at::kBFloat16 || x.dim() < 2 ||
        !x.is_contiguous() || x.size(1) != desc->K || x.size(0) > INT32_MAX)
      Py_RETURN_NONE;
    const int M = (int)x.size(0);
    void *p = packed.data_ptr(), *px = x.data_ptr(), *py = y.data_ptr(), *pw = ws.data_ptr(), *st = c10::cuda::getCurrentCUDAStream().stream();
    const size_t bytes = (size_t)ws.numel();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(desc, p, px, M, py, pw, bytes, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

// gemv_host(function, descriptor type, desc, packed, x_host, y_host, x_stage, y_stage, workspace)
PyObject* gemv_host(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) Py_RETURN_NONE;
  for (int i = 3; i < 9; ++i)
    if (!plain(a[i])) Py_RETURN_NONE;
  const HostFn fn = reinterpret_cast<HostFn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    Desc d;
    const razer_desc* desc = d.get(a[1], a[2]);
    if (!desc) Py_RETURN_NONE;
    void* p[6];
    for (int i = 0; i < 6; ++i) {
      const at::Tensor& t = tensor(a[i + 3]);
      if (!dense(t) || ((i == 1 || i == 2) && t.is_cuda())) Py_RETURN_NONE;
      p[i] = t.data_ptr();
    }
    const at::Tensor& x = tensor(a[4]);
    if (x.dim() < 1 || x.size(0) > INT32_MAX) Py_RETURN_NONE;
    const int M = (int)x.size(0);
    const size_t bytes = (size_t)tensor(a[8]).numel();
    void* st = c10::cuda::getCurrentCUDAStream().stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = fn(desc, p[0], p[1], M, p[2], p[3], p[4], p[5], bytes, st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

// ---- 8-bit integers
typedef int (*QuantI8Fn)(const void*, int, int, int, long long, int8_t*, float*, void*);
typedef int (*GemmI8Fn)(const int8_t*, const float*, const int8_t*, const float*, int, int, int, void*, void*);
typedef int (*AppendFn)(const razer_kv8*, const void*, long long, const void*, long long, const int32_t*, int, const int32_t*, const int32_t*, int, int, void*);
typedef int (*AttnFn)(const razer_kv8*, const void*, long long, int, const int32_t*, int, const int32_t*, const int32_t*, int, int, float, void*, float*, void*, size_t,
                      void*);

// On the current device, with memory of its own.
bool here(const at::Tensor& t, at::ScalarType type, c10::DeviceIndex dev) { return dense(t) && t.is_cuda() && t.get_device() == dev && t.scalar_type() == type; }
bool whole(const at::Tensor& t, at::ScalarType type, c10::DeviceIndex dev, at::IntArrayRef shape) { return here(t, type, dev) && t.sizes() == shape && t.is_contiguous(); }
bool counts(const at::Tensor& t) {
  for (int64_t n : t.sizes())
    if (n > INT32_MAX) return false;
  return true;
}
// The library's function without the interpreter's lock: a launch may wait for room in its queue, and the device for a Python callback.  Arguments
// are read before.
template <class Fn, class... A>
int unlocked(Fn fn, A... a) {
  int rc;
  Py_BEGIN_ALLOW_THREADS
  rc = fn(a...);
  Py_END_ALLOW_THREADS
  return rc;
}
// The caller's tensor, or a new one where `o` is None; false where it is neither.
bool given(PyObject* o, at::Tensor& t, const at::Tensor& like, at::ScalarType type, at::IntArrayRef shape) {
  if (o == Py_None) {
    t = at::Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt));   // from the allocator, not through the dispatcher
    return true;
  }
  if (!plain(o)) return false;
  t = tensor(o);
  return true;
}
PyObject* pair_of(const at::Tensor& a, const at::Tensor& b) {
  PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b);
  PyObject* t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
  Py_XDECREF(x);
  Py_XDECREF(y);
  return t;
}

// quant_i8(function, x, codes or None, scales or None)
PyObject* quant_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4 || !plain(a[1])) Py_RETURN_NONE;
  const QuantI8Fn fn = reinterpret_cast<QuantI8Fn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream();
    const at::Tensor& x = tensor(a[1]);
    const bool fp32 = x.scalar_type() == at::kFloat;
    if (!here(x, fp32 ? at::kFloat : at::kBFloat16, st.device_index()) || x.dim() != 2 || x.stride(1) != 1 || !counts(x)) Py_RETURN_NONE;
    const int64_t M = x.size(0), K = x.size(1);
    at::Tensor codes, scales;
    if (!given(a[2], codes, x, at::kChar, {M, K}) || !given(a[3], scales, x, at::kFloat, {M}) || !whole(codes, at::kChar, st.device_index(), {M, K}) ||
        !whole(scales, at::kFloat, st.device_index(), {M}))
      Py_RETURN_NONE;
    const int rc = unlocked(fn, x.data_ptr(), (int)fp32, (int)M, (int)K, M == 1 ? K : x.stride(0), static_cast<int8_t*>(codes.data_ptr()), static_cast<float*>(scales.data_ptr()), st.stream());
    return rc == 0 ? pair_of(codes, scales) : PyLong_FromLong(rc);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

// gemm_i8(function, x codes, x scales, w codes, w scales, y or None)
PyObject* gemm_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 6 || !plain(a[1]) || !plain(a[2]) || !plain(a[3]) || !plain(a[4])) Py_RETURN_NONE;
  const GemmI8Fn fn = reinterpret_cast<GemmI8Fn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream();
    const c10::DeviceIndex dev = st.device_index();
    const at::Tensor &x = tensor(a[1]), &sx = tensor(a[2]), &w = tensor(a[3]), &sw = tensor(a[4]);
    if (!dense(x) || !dense(w) || x.dim() != 2 || w.dim() != 2 || !counts(x) || !counts(w)) Py_RETURN_NONE;
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
    at::Tensor y;
    if (!whole(x, at::kChar, dev, {M, K}) || !whole(w, at::kChar, dev, {N, K}) || !whole(sx, at::kFloat, dev, {M}) || !whole(sw, at::kFloat, dev, {N}) ||
        !given(a[5], y, x, at::kBFloat16, {M, N}) || !whole(y, at::kBFloat16, dev, {M, N}))
      Py_RETURN_NONE;
    const int rc = unlocked(fn, static_cast<const int8_t*>(x.data_ptr()), static_cast<const float*>(sx.data_ptr()), static_cast<const int8_t*>(w.data_ptr()),
                            static_cast<const float*>(sw.data_ptr()), (int)M, (int)N, (int)K, y.data_ptr(), st.stream());
    return rc == 0 ? THPVariable_Wrap(y) : PyLong_FromLong(rc);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

// The cache behind binding.RazerKv8, on the current device.
struct Cache {
  Py_buffer view;
  bool held = false;
  const razer_kv8* get(PyObject* type, PyObject* o, c10::DeviceIndex dev) {
    if (reinterpret_cast<PyObject*>(Py_TYPE(o)) != type) return nullptr;
    PyObject* pools = PyObject_GetAttrString(o, "tensors");
    const bool good = pools && PyTuple_Check(pools) && PyTuple_GET_SIZE(pools) == 4 && plain(PyTuple_GET_ITEM(pools, 0)) &&
                      tensor(PyTuple_GET_ITEM(pools, 0)).is_cuda() && tensor(PyTuple_GET_ITEM(pools, 0)).get_device() == dev;
    Py_XDECREF(pools);
    if (!good || PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
      PyErr_Clear();
      return nullptr;
    }
    held = true;
    return view.len == (Py_ssize_t)sizeof(razer_kv8) ? static_cast<const razer_kv8*>(view.buf) : nullptr;
  }
  ~Cache() {
    if (held) PyBuffer_Release(&view);
  }
};
// block table, q_start, kv_len of a batch
bool batch(PyObject* const* a, c10::DeviceIndex dev) {
  for (int i = 0; i < 3; ++i)
    if (!plain(a[i]) || !here(tensor(a[i]), at::kInt, dev) || !tensor(a[i]).is_contiguous() || !counts(tensor(a[i]))) return false;
  const at::Tensor &table = tensor(a[0]), &starts = tensor(a[1]), &lens = tensor(a[2]);
  return table.dim() == 2 && starts.dim() == 1 && lens.dim() == 1 && table.size(0) == lens.size(0) && starts.size(0) == lens.size(0) + 1;
}
// bf16 [T, heads, head_dim], a token's values side by side
bool rows(const at::Tensor& x, int64_t heads, int64_t D, c10::DeviceIndex dev) {
  return here(x, at::kBFloat16, dev) && x.dim() == 3 && x.size(1) == heads && x.size(2) == D && x.stride(2) == 1 && (heads == 1 || x.stride(1) == D) && counts(x);
}
long long stride_of(const at::Tensor& x) { return x.size(0) > 1 ? x.stride(0) : x.size(1) * x.size(2); }
const int32_t* ints(PyObject* o) { return static_cast<const int32_t*>(tensor(o).data_ptr()); }

// kv8_append(function, cache type, cache, k, v, block table, q_start, kv_len): the library's code, or None
PyObject* kv8_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8 || !plain(a[3]) || !plain(a[4])) Py_RETURN_NONE;
  const AppendFn fn = reinterpret_cast<AppendFn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream();
    const c10::DeviceIndex dev = st.device_index();
    Cache cache;
    const razer_kv8* c = cache.get(a[1], a[2], dev);
    const at::Tensor &k = tensor(a[3]), &v = tensor(a[4]);
    if (!c || !rows(k, c->heads, c->head_dim, dev) || !rows(v, c->heads, c->head_dim, dev) || k.size(0) != v.size(0) || !batch(a + 5, dev)) Py_RETURN_NONE;
    return PyLong_FromLong(unlocked(fn, c, k.data_ptr(), stride_of(k), v.data_ptr(), stride_of(v), ints(a[5]), (int)tensor(a[5]).size(1), ints(a[6]), ints(a[7]),
                                    (int)tensor(a[7]).size(0), (int)k.size(0), st.stream()));
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

// attn_kv8(function, cache type, cache, q, block table, q_start, kv_len, scale or None, out or None, lse or None, workspace)
PyObject* attn_kv8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 11 || !plain(a[3]) || !plain(a[10]) || (a[7] != Py_None && !PyFloat_CheckExact(a[7]))) Py_RETURN_NONE;
  const AttnFn fn = reinterpret_cast<AttnFn>(address(a[0]));
  if (!fn) Py_RETURN_NONE;
  try {
    const c10::cuda::CUDAStream st = c10::cuda::getCurrentCUDAStream();
    const c10::DeviceIndex dev = st.device_index();
    Cache cache;
    const razer_kv8* c = cache.get(a[1], a[2], dev);
    const at::Tensor &q = tensor(a[3]), &ws = tensor(a[10]);
    if (!c || !dense(q) || q.dim() != 3 || !rows(q, q.size(1), c->head_dim, dev) || !batch(a + 4, dev) || !here(ws, ws.scalar_type(), dev) ||
        ws.scalar_type() != at::kByte || !ws.is_contiguous())
      Py_RETURN_NONE;
    const int64_t T = q.size(0), H = q.size(1), D = q.size(2);
    at::Tensor out, lse;
    if (!given(a[8], out, q, at::kBFloat16, {T, H, D}) || !given(a[9], lse, q, at::kFloat, {T, H}) || !whole(out, at::kBFloat16, dev, {T, H, D}) ||
        !whole(lse, at::kFloat, dev, {T, H}))
      Py_RETURN_NONE;
    const float scale = a[7] == Py_None ? (float)(1.0 / std::sqrt((double)D)) : (float)PyFloat_AS_DOUBLE(a[7]);
    const int rc = unlocked(fn, c, q.data_ptr(), stride_of(q), (int)H, ints(a[4]), (int)tensor(a[4]).size(1), ints(a[5]), ints(a[6]), (int)tensor(a[6]).size(0), (int)T, scale,
                            out.data_ptr(), static_cast<float*>(lse.data_ptr()), ws.data_ptr(), (size_t)ws.numel(), st.stream());
    return rc == 0 ? pair_of(out, lse) : PyLong_FromLong(rc);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(quant_i8), CALL(gemm_i8), CALL(kv8_append), CALL(attn_kv8),
                         {"matmul", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(matmul)), METH_FASTCALL, nullptr},
                         {"gemv_host", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemv_host)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "razer_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_razer_call() { return PyModule_Create(&module); }
