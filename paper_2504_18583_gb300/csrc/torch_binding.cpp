// The tree operators on torch tensors, as a CPython module: checks, outputs and
// the call of the C ABI in one step.  (Through ctypes the same work, a dozen
// attribute reads, three allocations and a foreign call from Python, took 15 us
// beside kernels of 3.)  It holds no operator code: everything goes through
// libpard's exported functions, and without the module the operators raise.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>
#include <map>
#include <string>
#include <utility>

#include "pard.h"

namespace {

constexpr int64_t kPage = 16;
PyObject* g_error = nullptr;  // pard.PardError

struct Refuse {  // becomes a ValueError
  std::string why;
};
struct Raised {};  // a Python exception is set

const at::Tensor& tensor_of(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refuse{std::string(name) + ": want a tensor, got " + Py_TYPE(o)->tp_name};
  return THPVariable_Unpack(o);
}
std::string text(at::IntArrayRef s) {
  std::string r = "(";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
  return r + ")";
}

// The current device and its current stream, which t must lie on.
struct Where {
  c10::DeviceIndex dev;
  void* stream;
  explicit Where(const at::Tensor& t, const char* name) {
    dev = t.is_cuda() ? c10::cuda::current_device() : -1;
    if (!t.is_cuda() || t.get_device() != dev) throw Refuse{std::string(name) + ": tensors must lie on the current CUDA device"};
    stream = c10::cuda::getCurrentCUDAStream(dev).stream();
  }
  at::TensorOptions options(at::ScalarType type) const { return at::TensorOptions().dtype(type).device(at::kCUDA, dev); }
  // data of a contiguous tensor of this type and shape
  template <typename T = void>
  T* want(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    const at::Tensor& t = tensor_of(o, name);
    if (t.scalar_type() != type || t.sizes() != shape || !t.is_cuda() || t.get_device() != dev || !t.is_contiguous())
      throw Refuse{std::string(name) + ": want a contiguous " + c10::toString(type) + " tensor of shape " + text(shape) +
                   " on the same device, got " + c10::toString(t.scalar_type()) + " " + text(t.sizes()) + " on " + t.device().str()};
    return static_cast<T*>(t.data_ptr());
  }
  template <typename T = void>
  T* want_or_none(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) const {
    return o == Py_None ? nullptr : want<T>(o, name, type, shape);
  }
};

int type_code(at::ScalarType t, bool with_fp32, const char* name) {
  if (t == at::kBFloat16) return PARD_BF16;
  if (t == at::kHalf) return PARD_F16;
  if (with_fp32 && t == at::kFloat) return PARD_F32;
  throw Refuse{std::string(name) + (with_fp32 ? ": want fp32, bf16 or fp16" : ": want bf16 or fp16")};
}

// [pages, kv_heads, 16, head_dim] whose pages may lie apart: entries from one to the next
int64_t cache_stride(const at::Tensor& t, const char* name, at::ScalarType type, const Where& w) {
  if (t.dim() != 4 || t.scalar_type() != type || !t.is_cuda() || t.get_device() != w.dev || t.size(2) != kPage)
    throw Refuse{std::string(name) + ": want [pages, kv_heads, 16, head_dim] of " + c10::toString(type) + " on the same device"};
  const int64_t h = t.size(1), d = t.size(3);
  if (t.stride(3) != 1 || t.stride(2) != d || (h > 1 && t.stride(1) != kPage * d))
    throw Refuse{std::string(name) + ": each page must be a contiguous [kv_heads, 16, head_dim] block"};
  return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), h * kPage * d);
}

long whole(PyObject* o, const char* name) {
  const long v = PyLong_AsLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  if (v < INT32_MIN || v > INT32_MAX) throw Refuse{std::string(name) + ": out of range"};
  return v;
}
double real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Raised{};
  return v;
}
void done(pard_status code, const char* where) {
  if (code == PARD_OK) return;
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", (int)code, where) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, pard_last_error());
  }
  throw Raised{};
}
void count_is(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return;
  PyErr_Format(PyExc_TypeError, "want %zd arguments, got %zd", want, n);
  throw Raised{};
}
int64_t dim_of(const at::Tensor& t, int64_t dims, const char* name) {
  if (t.dim() != dims) throw Refuse{std::string(name) + ": want " + std::to_string(dims) + " dimensions, got " + text(t.sizes())};
  return dims;
}
PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject* tuple3(at::Tensor a, at::Tensor b, at::Tensor c) {
  return Py_BuildValue("(NNN)", wrap(std::move(a)), wrap(std::move(b)), wrap(std::move(c)));
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return F(a, n);
  } catch (const Refuse& r) {
    PyErr_SetString(PyExc_ValueError, r.why.c_str());
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

PyObject* tree_plan(PyObject* const* a, Py_ssize_t n) {
  count_is(n, 5);
  const at::Tensor& parents = tensor_of(a[0], "parents");
  const Where w(parents, "parents");
  dim_of(parents, 2, "parents");
  const int64_t B = parents.size(0), N = parents.size(1), P = tensor_of(a[3], "page_table").size(-1);
  const auto* d_parents = w.want<int32_t>(a[0], "parents", at::kInt, {B, N});
  const auto* d_nodes = w.want<int32_t>(a[1], "n_nodes", at::kInt, {B});
  const auto* d_ctx = w.want<int32_t>(a[2], "ctx_len", at::kInt, {B});
  const auto* d_table = w.want<int32_t>(a[3], "page_table", at::kInt, {B, P});
  const long pages = whole(a[4], "n_pages");
  at::Tensor mask = at::empty({B, N, (N + 63) / 64}, w.options(at::kLong)), pos = at::empty({B, N}, w.options(at::kInt)),
             slots = at::empty({B, N}, w.options(at::kLong));
  done(pard_tree_plan(d_parents, d_nodes, d_ctx, d_table, B, N, P, pages, static_cast<uint64_t*>(mask.data_ptr()),
                      pos.mutable_data_ptr<int32_t>(), slots.mutable_data_ptr<int64_t>(), w.stream),
       "pard_tree_plan");
  return tuple3(std::move(mask), std::move(pos), std::move(slots));
}

PyObject* qk_norm_rope(PyObject* const* a, Py_ssize_t n) {
  count_is(n, 13);
  const at::Tensor& qkv = tensor_of(a[0], "qkv");
  const Where w(qkv, "qkv");
  const at::ScalarType type = qkv.scalar_type();
  const int code = type_code(type, false, "qkv");
  if (qkv.dim() != 2 || qkv.stride(1) != 1) throw Refuse{"qkv: want [tokens, (Hq + 2 Hkv) * hd] rows of contiguous entries"};
  const int64_t T = qkv.size(0), width = qkv.size(1);
  const long Hq = whole(a[1], "n_q_heads"), Hkv = whole(a[2], "n_kv_heads");
  const at::Tensor &kc = tensor_of(a[5], "k_cache"), &vc = tensor_of(a[6], "v_cache");
  const int64_t stride = cache_stride(kc, "k_cache", type, w);
  const int64_t hd = kc.size(3);
  if (cache_stride(vc, "v_cache", type, w) != stride || vc.sizes() != kc.sizes() || kc.size(1) != Hkv ||
      width != (Hq + 2 * Hkv) * hd)
    throw Refuse{"qkv and caches disagree on heads, head_dim, pages or page stride"};
  int64_t half = 0;
  if (a[7] != Py_None) {
    dim_of(tensor_of(a[7], "inv_freq"), 1, "inv_freq");
    half = THPVariable_Unpack(a[7]).size(0);
  }
  const auto* d_pos = w.want<int32_t>(a[3], "pos", at::kInt, {T});
  const auto* d_slots = w.want<int64_t>(a[4], "slots", at::kLong, {T});
  const auto* d_freq = half ? w.want<float>(a[7], "inv_freq", at::kFloat, {half}) : nullptr;
  const void* d_qg = w.want_or_none(a[8], "q_gain", type, {hd});
  const void* d_kg = w.want_or_none(a[9], "k_gain", type, {hd});
  const double eps = real(a[10]), amplitude = real(a[12]);
  const int interleaved = PyObject_IsTrue(a[11]);
  if (interleaved < 0) throw Raised{};
  at::Tensor q = at::empty({T, Hq, hd}, w.options(type));
  done(pard_qk_norm_rope(qkv.data_ptr(), T > 1 ? qkv.stride(0) : std::max(width, qkv.stride(0)), code, T, Hq, Hkv, hd, d_qg,
                         d_kg, (float)eps, d_pos, d_slots, d_freq, 2 * half, interleaved, (float)amplitude, q.data_ptr(),
                         Hq * hd, kc.data_ptr(), vc.data_ptr(), stride, kc.size(0), w.stream),
       "pard_qk_norm_rope");
  return wrap(std::move(q));
}

// what attention calls without a workspace of their own use, one after the other on a stream
at::Tensor& workspace_of(int dev, void* stream) {
  static auto* all = new std::map<std::pair<int, void*>, at::Tensor>;  // never torn down: CUDA may be gone before it
  return (*all)[{dev, stream}];
}
PyObject* shared_workspace(PyObject* const*, Py_ssize_t n) {
  count_is(n, 0);
  const auto dev = c10::cuda::current_device();
  const at::Tensor& t = workspace_of(dev, c10::cuda::getCurrentCUDAStream(dev).stream());
  if (!t.defined()) Py_RETURN_NONE;
  return wrap(t);
}

PyObject* tree_attention(PyObject* const* a, Py_ssize_t n) {
  count_is(n, 11);
  const at::Tensor& q = tensor_of(a[0], "q");
  const Where w(q, "q");
  const at::ScalarType type = q.scalar_type();
  const int code = type_code(type, false, "q");
  dim_of(q, 4, "q");
  const int64_t B = q.size(0), N = q.size(1), Hq = q.size(2), hd = q.size(3);
  const int64_t node = N > 1 ? q.stride(1) : (B > 1 ? q.stride(0) : Hq * hd);
  if (q.stride(3) != 1 || (Hq > 1 && q.stride(2) != hd) || (B > 1 && q.stride(0) != N * node))
    throw Refuse{"q: a node's heads must be contiguous and nodes evenly spaced"};
  const at::Tensor &kc = tensor_of(a[1], "k_cache"), &vc = tensor_of(a[2], "v_cache");
  const int64_t stride = cache_stride(kc, "k_cache", type, w);
  if (cache_stride(vc, "v_cache", type, w) != stride || vc.sizes() != kc.sizes() || kc.size(3) != hd)
    throw Refuse{"q and caches disagree on head_dim, pages or page stride"};
  const int64_t P = tensor_of(a[3], "page_table").size(-1), Hkv = kc.size(1);
  const auto* d_table = w.want<int32_t>(a[3], "page_table", at::kInt, {B, P});
  const auto* d_ctx = w.want<int32_t>(a[4], "ctx_len", at::kInt, {B});
  const auto* d_nodes = w.want<int32_t>(a[5], "n_nodes", at::kInt, {B});
  const auto* d_mask = w.want<int64_t>(a[6], "mask", at::kLong, {B, N, (N + 63) / 64});
  const double scale = a[7] == Py_None ? 1.0 / std::sqrt((double)hd) : real(a[7]);
  at::Tensor out, workspace;
  if (a[8] == Py_None) out = at::empty({B, N, Hq, hd}, w.options(type));
  else { w.want(a[8], "out", type, {B, N, Hq, hd}); out = THPVariable_Unpack(a[8]); }
  const int64_t need = (int64_t)pard_tree_attention_workspace_bytes(B, N, Hq, Hkv, hd);
  const int capturing = PyObject_IsTrue(a[10]);
  if (a[9] != Py_None) {
    workspace = tensor_of(a[9], "workspace");
    if (!workspace.is_cuda() || workspace.get_device() != w.dev || !workspace.is_contiguous())
      throw Refuse{"workspace: want a contiguous tensor on the same device"};
  } else if (capturing) {  // a graph may run beside later calls: its calls have their own
    workspace = at::zeros({std::max<int64_t>(need, 16)}, w.options(at::kByte));
  } else {
    at::Tensor& shared = workspace_of(w.dev, w.stream);
    if (!shared.defined() || shared.numel() < need) shared = at::zeros({std::max<int64_t>(need, 16)}, w.options(at::kByte));
    workspace = shared;
  }
  done(pard_tree_attention(q.data_ptr(), node, code, B, N, Hq, Hkv, hd, kc.data_ptr(), vc.data_ptr(), stride, kc.size(0),
                           d_table, P, d_ctx, d_nodes, reinterpret_cast<const uint64_t*>(d_mask), (float)scale,
                           out.data_ptr(), workspace.data_ptr(), workspace.nbytes(), w.stream),
       "pard_tree_attention");
  return wrap(std::move(out));
}

PyObject* sample(PyObject* const* a, Py_ssize_t n) {
  count_is(n, 6);
  const at::Tensor& z = tensor_of(a[0], "logits");
  const Where w(z, "logits");
  const int code = type_code(z.scalar_type(), true, "logits");
  if (z.dim() != 2 || z.stride(1) != 1) throw Refuse{"logits: want [rows, vocab] with contiguous rows"};
  const int64_t R = z.size(0), V = z.size(1);
  const auto* d_u = w.want<float>(a[1], "u", at::kFloat, {R});
  const auto* d_t = w.want_or_none<float>(a[2], "temperature", at::kFloat, {R});
  const auto* d_k = w.want_or_none<int32_t>(a[3], "top_k", at::kInt, {R});
  const auto* d_p = w.want_or_none<float>(a[4], "top_p", at::kFloat, {R});
  const auto* d_m = w.want_or_none<float>(a[5], "min_p", at::kFloat, {R});
  at::Tensor token = at::empty({R}, w.options(at::kInt)), logprob = at::empty({R}, w.options(at::kFloat));
  done(pard_sample(z.data_ptr(), R > 1 ? z.stride(0) : std::max(V, z.stride(0)), code, R, V, d_u, d_t, d_k, d_p, d_m,
                   token.mutable_data_ptr<int32_t>(), logprob.mutable_data_ptr<float>(), w.stream),
       "pard_sample");
  return Py_BuildValue("(NN)", wrap(std::move(token)), wrap(std::move(logprob)));
}

PyObject* tree_commit(PyObject* const* a, Py_ssize_t n) {
  count_is(n, 7);
  const at::Tensor& sampled = tensor_of(a[0], "sampled");
  const Where w(sampled, "sampled");
  dim_of(sampled, 2, "sampled");
  const int64_t B = sampled.size(0), N = sampled.size(1), P = tensor_of(a[5], "page_table").size(-1);
  const at::Tensor& pool = tensor_of(a[6], "pool");
  if (pool.dim() != 6 || pool.size(1) != 2 || pool.size(4) != kPage || !pool.is_cuda() || pool.get_device() != w.dev ||
      (pool.scalar_type() != at::kBFloat16 && pool.scalar_type() != at::kHalf))
    throw Refuse{"pool: want [layers, 2, pages, kv_heads, 16, head_dim] of bf16 or fp16 on the same device"};
  const int64_t L = pool.size(0), pages = pool.size(2), Hkv = pool.size(3), hd = pool.size(5);
  if (pool.stride(5) != 1 || pool.stride(4) != hd || (Hkv > 1 && pool.stride(3) != kPage * hd))
    throw Refuse{"pool: each page must be a contiguous [kv_heads, 16, head_dim] block"};
  const auto* d_sampled = w.want<int32_t>(a[0], "sampled", at::kInt, {B, N});
  const auto* d_tokens = w.want<int32_t>(a[1], "tokens", at::kInt, {B, N});
  const auto* d_parents = w.want<int32_t>(a[2], "parents", at::kInt, {B, N});
  const auto* d_nodes = w.want<int32_t>(a[3], "n_nodes", at::kInt, {B});
  const auto* d_ctx = w.want<int32_t>(a[4], "ctx_len", at::kInt, {B});
  const auto* d_table = w.want<int32_t>(a[5], "page_table", at::kInt, {B, P});
  at::Tensor accept = at::empty({B}, w.options(at::kInt)), emitted = at::empty({B, N}, w.options(at::kInt)),
             length = at::empty({B}, w.options(at::kInt));
  done(pard_tree_commit(d_sampled, d_tokens, d_parents, d_nodes, d_ctx, d_table, B, N, P, pool.data_ptr(), pool.stride(0),
                        pool.stride(1), pages > 1 ? pool.stride(2) : Hkv * kPage * hd, L, Hkv, hd, pages,
                        accept.mutable_data_ptr<int32_t>(), emitted.mutable_data_ptr<int32_t>(),
                        length.mutable_data_ptr<int32_t>(), w.stream),
       "pard_tree_commit");
  return tuple3(std::move(accept), std::move(emitted), std::move(length));
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(g_error);
  g_error = cls;
  Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<F>)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {method<tree_plan>("tree_plan"),
                           method<qk_norm_rope>("qk_norm_rope"),
                           method<tree_attention>("tree_attention"),
                           method<shared_workspace>("shared_workspace"),
                           method<sample>("sample"),
                           method<tree_commit>("tree_commit"),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_tree_ops", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tree_ops(void) { return PyModule_Create(&g_module); }
