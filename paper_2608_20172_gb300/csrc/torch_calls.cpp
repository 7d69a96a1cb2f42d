// torch_calls.cpp -- the serving calls of the Python binding in native code.
//
// A step's kernels take a few microseconds each, the binding's checks and allocations in Python 15 to
// 25.  These functions do the same for the common call (outputs to be allocated, the current stream):
// they check the tensors, allocate, call the C ABI and return the outputs.  Whatever they do not take
// as it is -- an argument of another kind, a check that fails, a status other than RELATION_OK -- they
// answer with None, and the binding goes its own way, which says what is wrong.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "relation.h"

namespace {

decltype(&relation_page_plan) g_page_plan;
decltype(&relation_cache_append) g_cache_append;
decltype(&relation_paged_decode) g_paged_decode;
decltype(&relation_paged_decode_workspace_size) g_workspace_size;
decltype(&relation_sample) g_sample;

struct Decline {};  // the binding's own way

// The current stream; the library launches on the current device, which has to be the operands'
relation_stream_t current_stream(c10::DeviceIndex device) {
  const c10::cuda::CUDAStream s = c10::cuda::getCurrentCUDAStream();
  if (s.device_index() != device) throw Decline();
  return reinterpret_cast<relation_stream_t>(s.stream());
}

const at::Tensor& tensor(PyObject* x) {
  if (!THPVariable_CheckExact(x)) throw Decline();
  return THPVariable_Unpack(x);
}
// A contiguous tensor of n entries on the device
const at::Tensor& dense(PyObject* x, at::ScalarType type, int64_t n, c10::DeviceIndex device) {
  const at::Tensor& t = tensor(x);
  if (t.scalar_type() != type || !t.is_contiguous() || t.numel() != n || !t.is_cuda() ||
      t.get_device() != device)
    throw Decline();
  return t;
}
template <typename T>
T* data(const at::Tensor& t) {
  return static_cast<T*>(t.data_ptr());
}
// None or such a tensor
template <typename T>
T* optional(PyObject* x, at::ScalarType type, int64_t n, c10::DeviceIndex device) {
  return x == Py_None ? nullptr : data<T>(dense(x, type, n, device));
}
// None or what the kernels may write: an int of the device
int* status_of(PyObject* x, c10::DeviceIndex device) {
  if (x == Py_None) return nullptr;
  const at::Tensor& t = tensor(x);
  if (t.scalar_type() != at::kInt || t.numel() < 1 || !t.is_cuda() || t.get_device() != device) throw Decline();
  return data<int>(t);
}
int integer(PyObject* x) {
  if (!PyLong_CheckExact(x)) throw Decline();
  const long v = PyLong_AsLong(x);  // (-1 and an error past 64 bits)
  if (v < -0x7fffffffL || v > 0x7fffffffL || (v == -1 && PyErr_Occurred())) throw Decline();
  return (int)v;
}
float real(PyObject* x) {
  if (PyFloat_CheckExact(x)) return (float)PyFloat_AS_DOUBLE(x);
  return (float)integer(x);
}
relation_dtype type_of(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return RELATION_F32;
  if (t.scalar_type() == at::kBFloat16) return RELATION_BF16;
  throw Decline();
}
// Rows of the table, contiguous each
const at::Tensor& table(PyObject* x, int64_t B, c10::DeviceIndex device) {
  const at::Tensor& t = tensor(x);
  if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) != B || t.stride(1) != 1 || !t.is_cuda() ||
      t.get_device() != device || t.size(1) > 0x7fffffff)
    throw Decline();
  return t;
}
bool same_layout(const at::Tensor& a, const at::Tensor& b) {
  return a.sizes() == b.sizes() && a.strides() == b.strides() && a.scalar_type() == b.scalar_type() &&
         a.is_cuda() && b.is_cuda() && a.get_device() == b.get_device();
}
relation_pages pages(const at::Tensor& k, const at::Tensor& v) {
  if (!same_layout(k, v) || k.dim() != 4 || k.stride(3) != 1) throw Decline();
  for (int64_t n : k.sizes())
    if (n > 0x7fffffff) throw Decline();
  return {(int)k.size(0), (int)k.size(1), (int)k.size(2), (int)k.size(3),
          k.stride(0),    k.stride(1),    k.stride(2)};
}

PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
// A tuple of tensors, or null with the error set
template <typename... T>
PyObject* tuple(T... t) {
  PyObject* all[] = {wrap(std::move(t))...};
  PyObject* r = PyTuple_New(sizeof...(T));
  bool ok = r != nullptr;
  for (size_t i = 0; i < sizeof...(T); ++i) {
    ok = ok && all[i];
    if (r && all[i]) PyTuple_SET_ITEM(r, i, all[i]);
    else Py_XDECREF(all[i]);
  }
  if (!ok) Py_CLEAR(r);
  return r;
}

// lengths, counts, block_table, free_pages, free_state, page_size, n_tokens, dev_status
PyObject* page_plan(PyObject* const* a) {
  const at::Tensor& lengths = tensor(a[0]);
  const int64_t B = lengths.numel();
  if (!lengths.is_cuda() || B > 0x7fffffff) throw Decline();
  const c10::DeviceIndex dev = lengths.get_device();
  dense(a[0], at::kInt, B, dev);
  const at::Tensor& counts = dense(a[1], at::kInt, B, dev);
  const at::Tensor& tab = table(a[2], B, dev);
  const at::Tensor& ring = dense(a[3], at::kInt, tensor(a[3]).numel(), dev);
  const at::Tensor& state = dense(a[4], at::kInt, 2, dev);
  const int page = integer(a[5]), n = integer(a[6]);
  if (n < 0 || ring.numel() > 0x7fffffff) throw Decline();
  const auto i32 = lengths.options();
  at::Tensor slots = at::empty({n}, i32.dtype(at::kLong)), positions = at::empty({n}, i32),
             starts = at::empty({B + 1}, i32), next = at::empty({B}, i32), after = at::empty({2}, i32);
  if (g_page_plan(data<int>(lengths), data<int>(counts), (int)B, page, data<int>(tab), (int)tab.size(1),
                  tab.stride(0), data<int>(ring), (int)ring.numel(), data<int>(state), data<int>(after),
                  data<int>(next), data<int>(starts), reinterpret_cast<long long*>(data<int64_t>(slots)),
                  data<int>(positions), n, status_of(a[7], dev), current_stream(dev)) != RELATION_OK)
    throw Decline();
  return tuple(slots, positions, starts, next, after);
}

// p1, p2, info, theta, positions, slots, k_pages, v_pages, pairing, rope_base, dev_status; p1's outputs
// are dense: a view that is not goes the binding's way
PyObject* cache_append(PyObject* const* a) {
  const at::Tensor &p1 = tensor(a[0]), &p2 = tensor(a[1]), &info = tensor(a[2]);
  const at::Tensor &k = tensor(a[6]), &v = tensor(a[7]);
  const relation_pages c = pages(k, v);
  const c10::DeviceIndex dev = k.get_device();
  if (!same_layout(p1, p2) || !same_layout(p1, info) || !p1.is_contiguous() || p1.dim() != 3 ||
      p1.size(1) != c.H || p1.size(2) != c.d_h || p1.scalar_type() != k.scalar_type() ||
      p1.get_device() != dev || p1.size(0) > 0x7fffffff)
    throw Decline();
  const int64_t N = p1.size(0);
  const float* theta = optional<float>(a[3], at::kFloat, p1.size(1) / 2, dev);
  const int* positions = optional<int>(a[4], at::kInt, N, dev);
  const at::Tensor& slots = dense(a[5], at::kLong, N, dev);
  const int pairing = integer(a[8]);
  at::Tensor q = at::empty_like(p1);
  if (g_cache_append(p1.data_ptr(), p2.data_ptr(), info.data_ptr(), theta, pairing, real(a[9]), positions,
                     reinterpret_cast<const long long*>(data<int64_t>(slots)), q.data_ptr(), (int)N,
                     p1.stride(0), p1.stride(1), k.data_ptr(), v.data_ptr(), c, type_of(p1),
                     status_of(a[10], dev), current_stream(dev)) != RELATION_OK)
    throw Decline();
  return wrap(std::move(q));
}

// q, k_pages, v_pages, block_table, lengths, lam, tau_s, dev_status
PyObject* paged_decode(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
  const relation_pages c = pages(k, v);
  const c10::DeviceIndex dev = k.get_device();
  if (q.dim() != 3 || !q.is_contiguous() || q.size(2) != c.d_h || q.scalar_type() != k.scalar_type() ||
      !q.is_cuda() || q.get_device() != dev || q.size(0) > 0x7fffffff || q.size(1) > 0x7fffffff)
    throw Decline();
  const int64_t B = q.size(0), H = q.size(1);
  const at::Tensor& lengths = dense(a[4], at::kInt, B, dev);
  const at::Tensor& tab = table(a[3], B, dev);
  const relation_dtype dt = type_of(q);
  const size_t bytes = g_workspace_size((int)H, c, dt);
  if (bytes == 0) throw Decline();
  at::Tensor y = at::empty_like(q), logz = at::empty({B, H}, q.options().dtype(at::kFloat)),
             ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
  if (g_paged_decode(q.data_ptr(), k.data_ptr(), v.data_ptr(), data<int>(tab), (int)tab.size(1),
                     tab.stride(0), data<int>(lengths), y.data_ptr(), data<float>(logz), real(a[5]),
                     real(a[6]), (int)B, (int)H, c, q.stride(0), q.stride(1), dt, ws.data_ptr(), bytes,
                     status_of(a[7], dev), current_stream(dev)) != RELATION_OK)
    throw Decline();
  return tuple(y, logz);
}

// logits, u, temperature, top_k, top_p, min_p, dev_status
PyObject* sample(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  if (x.dim() != 2 || x.stride(1) != 1 || !x.is_cuda() || x.size(0) > 0x7fffffff || x.size(1) > 0x7fffffff)
    throw Decline();
  const relation_dtype dt = type_of(x);
  const int64_t R = x.size(0);
  const c10::DeviceIndex dev = x.get_device();
  const at::Tensor& u = dense(a[1], at::kFloat, R, dev);
  const float* temperature = optional<float>(a[2], at::kFloat, R, dev);
  const int* top_k = optional<int>(a[3], at::kInt, R, dev);
  const float* top_p = optional<float>(a[4], at::kFloat, R, dev);
  const float* min_p = optional<float>(a[5], at::kFloat, R, dev);
  at::Tensor token = at::empty({R}, u.options().dtype(at::kInt)), logprob = at::empty({R}, u.options()),
             logz = at::empty({R}, u.options());
  if (g_sample(x.data_ptr(), (int)R, (int)x.size(1), x.stride(0), dt, data<float>(u), temperature, top_k,
               top_p, min_p, data<int>(token), data<float>(logprob), data<float>(logz), status_of(a[6], dev),
               current_stream(dev)) != RELATION_OK)
    throw Decline();
  return tuple(token, logprob, logz);
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
  try {
    if (n == N) return F(args);
  } catch (...) {  // (an allocation that failed, too, is tried again and reported there)
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}

// The addresses of the library's functions
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* f[5];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "five addresses");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i)
    if (!(f[i] = PyLong_AsVoidPtr(args[i]))) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
      return nullptr;
    }
  g_page_plan = reinterpret_cast<decltype(g_page_plan)>(f[0]);
  g_cache_append = reinterpret_cast<decltype(g_cache_append)>(f[1]);
  g_paged_decode = reinterpret_cast<decltype(g_paged_decode)>(f[2]);
  g_workspace_size = reinterpret_cast<decltype(g_workspace_size)>(f[3]);
  g_sample = reinterpret_cast<decltype(g_sample)>(f[4]);
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(bind), METH_FASTCALL, nullptr},
    {"page_plan", reinterpret_cast<PyCFunction>(entry<page_plan, 8>), METH_FASTCALL, nullptr},
    {"cache_append", reinterpret_cast<PyCFunction>(entry<cache_append, 11>), METH_FASTCALL, nullptr},
    {"paged_decode", reinterpret_cast<PyCFunction>(entry<paged_decode, 8>), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(entry<sample, 7>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "relation_calls", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit_relation_calls() { return PyModule_Create(&module); }
