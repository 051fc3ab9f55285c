// Calls whose way through Python takes longer than the kernel behind them, as a Python extension on torch's own tensors.
//
// tsd_accept_commit_static is one launch of some 4 us.  Through ctypes, with its outputs allocated by torch.empty, a call took 10.5 us: three
// allocations and a view 5.4, the arguments' conversion and the launch 3.5.  From here 8 series of 4 x 16 take 6.2 us, 1024 of
// 6 x 96 6.5, the kernel's own time; on inputs that were not read just before 10.7 -> 6.9 and 10.2 -> 8.8.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>
#include <stdexcept>
#include <string>

#include "tsd.h"

namespace {

// tsd_accept_commit_static (tsd.h), handed over by the binding that loaded the library
using AcceptFn = int (*)(const float*, const float*, const float*, const int32_t*, int32_t, int32_t, int32_t, float, float, float, uint64_t,
                         uint32_t, int32_t*, float*, float*, float*, void*);
AcceptFn accept_fn = nullptr;

// A contiguous tensor of its own over `whole`'s memory from element `offset` on.
at::Tensor over(const at::Tensor& whole, at::IntArrayRef sizes, int64_t offset) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(whole.storage()), whole.key_set(), whole.dtype());
  t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
  t.unsafeGetTensorImpl()->set_storage_offset(offset);
  return t;
}

const at::Tensor* tensor(PyObject* o, const char* name) {
  if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
  PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
  return nullptr;
}

// (lib's function address)
PyObject* bind(PyObject*, PyObject* address) {
  void* p = PyLong_AsVoidPtr(address);
  if (!p && PyErr_Occurred()) return nullptr;
  accept_fn = reinterpret_cast<AcceptFn>(p);
  Py_RETURN_NONE;
}

// X, mu_q, mu_p, rounds or None, sigma_p, sigma_q, fallback_r, seed, flags, want_taps -> (status, n_acc, commit, ell, logu)
PyObject* accept_commit_static(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 10 || !accept_fn) {
    PyErr_SetString(PyExc_TypeError, "accept_commit_static takes ten arguments, after bind()");
    return nullptr;
  }
  const at::Tensor *X = tensor(args[0], "X"), *mu_q = X ? tensor(args[1], "mu_q") : nullptr, *mu_p = mu_q ? tensor(args[2], "mu_p") : nullptr;
  if (!mu_p) return nullptr;
  const at::Tensor* rounds = nullptr;
  if (args[3] != Py_None && !(rounds = tensor(args[3], "rounds"))) return nullptr;
  const double sigma_p = PyFloat_AsDouble(args[4]), sigma_q = PyFloat_AsDouble(args[5]), fallback_r = PyFloat_AsDouble(args[6]);
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(args[7]);
  const uint32_t flags = (uint32_t)PyLong_AsUnsignedLongMask(args[8]);
  const int taps = PyObject_IsTrue(args[9]);
  if (PyErr_Occurred()) return nullptr;
  try {
    if (X->dim() != 3) {
      PyErr_Format(PyExc_ValueError, "X must be [B, K, P], has %d dimensions", (int)X->dim());
      return nullptr;
    }
    if (!X->device().has_index()) {  // (a tensor that is not on a GPU, whose pointer must not reach a kernel)
      PyErr_Format(PyExc_ValueError, "Expected a cuda device, but got: %s", X->device().str().c_str());
      return nullptr;
    }
    const int64_t B = X->size(0), K = X->size(1), P = X->size(2);
    const auto f32 = at::TensorOptions().dtype(at::kFloat).device(X->device());
    // (the kernel writes every entry: nothing to fill beforehand)
    // (the two taps in one allocation.  Not the counts with them: torch.save refuses tensors of two types over one memory, and a kept count
    // would keep the taps.)
    at::Tensor n_acc = at::empty({B}, f32.dtype(at::kInt)), commit = at::empty({B, K + 1, P}, f32), ell, logu;
    if (taps) {
      const at::Tensor both = at::empty({2, B, K}, f32);
      ell = over(both, {B, K}, 0);
      logu = over(both, {B, K}, B * K);
    }
    auto at_of = [](const at::Tensor& t) { return static_cast<float*>(t.data_ptr()); };
    const float *x = at_of(*X), *q = at_of(*mu_q), *p = at_of(*mu_p);
    const int32_t* r = rounds ? static_cast<int32_t*>(rounds->data_ptr()) : nullptr;
    void* stream = c10::hip::getCurrentHIPStream(X->device().index()).stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = accept_fn(x, q, p, r, (int32_t)B, (int32_t)K, (int32_t)P, (float)sigma_p, (float)sigma_q, (float)fallback_r, seed, flags,
                   static_cast<int32_t*>(n_acc.data_ptr()), at_of(commit), taps ? at_of(ell) : nullptr, taps ? at_of(logu) : nullptr, stream);
    Py_END_ALLOW_THREADS
    PyObject* out = PyTuple_New(5);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(rc));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(n_acc));
    PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(commit));
    for (int i = 0; i < 2; ++i) {
      PyObject* o = taps ? THPVariable_Wrap(i ? logu : ell) : Py_None;
      if (!taps) Py_INCREF(Py_None);
      PyTuple_SET_ITEM(out, 3 + i, o);
    }
    return out;
  } catch (const std::exception&) {
    torch::translate_exception_to_python(std::current_exception());  // (torch.OutOfMemoryError among them)
    return nullptr;
  }
}

// ---- a round of the caller's own models: tsd_rope_append_static, tsd_paged_attn_static, tsd_verify_tokens_static -------------------
decltype(&tsd_rope_append_static) append_fn = nullptr;
decltype(&tsd_paged_attn_workspace) attn_bytes_fn = nullptr;
decltype(&tsd_paged_attn_static) attn_fn = nullptr;
decltype(&tsd_verify_tokens_workspace) verify_bytes_fn = nullptr;
decltype(&tsd_verify_tokens_static) verify_fn = nullptr;

// (the five functions' addresses, in the order above)
PyObject* bind_round(PyObject*, PyObject* const* args, Py_ssize_t n) {
  void* p[5];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "bind_round takes five addresses");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i) {
    p[i] = PyLong_AsVoidPtr(args[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_round: an address is 0");
      return nullptr;
    }
  }
  append_fn = reinterpret_cast<decltype(append_fn)>(p[0]);
  attn_bytes_fn = reinterpret_cast<decltype(attn_bytes_fn)>(p[1]);
  attn_fn = reinterpret_cast<decltype(attn_fn)>(p[2]);
  verify_bytes_fn = reinterpret_cast<decltype(verify_bytes_fn)>(p[3]);
  verify_fn = reinterpret_cast<decltype(verify_fn)>(p[4]);
  Py_RETURN_NONE;
}

struct Wrong : std::invalid_argument {  // becomes a ValueError
  using std::invalid_argument::invalid_argument;
};
struct WrongType : std::invalid_argument {  // becomes a TypeError
  using std::invalid_argument::invalid_argument;
};
// (the message is put together only where the check fails: some twenty of them took 1 us of a call)
#define NEED(ok, what)                       \
  do {                                       \
    if (!(ok)) throw Wrong(std::string(what)); \
  } while (0)

const at::Tensor& the(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw WrongType(std::string(name) + " must be a tensor");
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &the(o, name); }

int32_t whole(int64_t v, const char* name) {
  NEED(v >= 0 && v <= INT32_MAX, std::string(name) + " is out of range");
  return (int32_t)v;
}

void on_gpu(const at::Tensor& t, const char* name) {
  NEED(t.is_cuda(), std::string(name) + ": expected a cuda device, but got: " + t.device().str());
}
void like(const at::Tensor& t, const at::Tensor& first, const char* name) {
  NEED(t.device() == first.device(), std::string(name) + " is on " + t.device().str() + ", not on " + first.device().str());
  NEED(t.scalar_type() == first.scalar_type(), std::string(name) + " is of another type");
}
// A dense tensor of indices (or of other plain values) with these sizes, on the device of `first`.
void plain(const at::Tensor& t, const at::Tensor& first, at::ScalarType type, at::IntArrayRef sizes, const char* name) {
  NEED(t.device() == first.device(), std::string(name) + " is on " + t.device().str() + ", not on " + first.device().str());
  NEED(t.scalar_type() == type, std::string(name) + " must be of type " + c10::toString(type));
  NEED(t.sizes() == sizes, std::string(name) + " has another shape than its call's");
  NEED(t.is_contiguous(), std::string(name) + " must be contiguous");
}
int dtype_of(const at::Tensor& t, const char* name) {
  NEED(t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16, std::string(name) + " must be float32 or bfloat16");
  return t.scalar_type() == at::kFloat ? TSD_F32 : TSD_BF16;
}

// Nothing here has a gradient, and none is to be lost unsaid.
void no_gradient(const at::Tensor& t, const char* name) {
  NEED(!t.requires_grad(), std::string(name) + " wants a gradient, which this call does not have: call it under torch.no_grad(), or with detached tensors");
}
// A tensor that a call wrote counts as changed in place (those of inference mode have no count).
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// [B, T, heads, head_dim] with dense heads (dimensions of one step have no stride that matters)
tsd_rows rows_of(const at::Tensor& t, at::IntArrayRef sizes, const char* name) {
  NEED(t.sizes() == sizes, std::string(name) + " has another shape than its call's");
  NEED(t.stride(3) == 1, std::string(name) + ": the last dimension must be dense");
  tsd_rows r;
  r.data_dev = t.data_ptr();
  r.stride_b = sizes[0] > 1 ? t.stride(0) : 0;
  r.stride_t = sizes[1] > 1 ? t.stride(1) : 0;
  r.stride_h = sizes[2] > 1 ? t.stride(2) : 0;
  return r;
}
// (an output's rows must not lie over one another)
void apart(const at::Tensor& t, const char* name) {
  for (int i = 0; i < t.dim(); ++i) NEED(t.size(i) < 2 || t.stride(i) != 0, std::string(name) + ": an output must not be expanded");
}

tsd_paged_cache cache_of(const at::Tensor& k, const at::Tensor& v, const at::Tensor& table, int64_t B) {
  tsd_paged_cache c;
  c.dtype = dtype_of(k, "k_pool");
  on_gpu(k, "k_pool");
  NEED(k.dim() == 4, "k_pool must be [pages, page_tokens, kv_heads, head_dim]");
  like(v, k, "v_pool");
  NEED(v.sizes() == k.sizes() && v.strides() == k.strides(), "k_pool and v_pool must have the same shape and strides");
  NEED(k.numel() > 0 && k.stride(3) == 1, "k_pool: needs a page, and heads that are dense");
  NEED(table.device() == k.device() && table.scalar_type() == at::kInt, "page_table must be int32, on the pools' device");
  NEED(table.dim() == 2 && table.size(0) == B && table.size(1) > 0 && (table.stride(1) == 1 || table.size(1) == 1),
       "page_table must be [B, pages per sequence], rows dense");
  c.k_dev = k.data_ptr();
  c.v_dev = v.data_ptr();
  c.page_stride = k.size(0) > 1 ? k.stride(0) : 0;
  c.token_stride = k.size(1) > 1 ? k.stride(1) : 0;
  c.head_stride = k.size(2) > 1 ? k.stride(2) : 0;
  c.page_table_dev = static_cast<const int32_t*>(table.data_ptr());
  c.pages_per_seq = whole(table.size(1), "page_table");
  NEED(B < 2 || table.stride(0) >= table.size(1), "page_table: rows must not overlap");
  c.table_stride = B > 1 ? whole(table.stride(0), "page_table") : c.pages_per_seq;
  c.n_pages = whole(k.size(0), "k_pool");
  c.page_tokens = whole(k.size(1), "k_pool");
  c.n_kv_heads = whole(k.size(2), "k_pool");
  c.head_dim = whole(k.size(3), "k_pool");
  return c;
}

// A call's body, with what it throws as Python's own errors.
template <typename F>
PyObject* guarded(const F& body) {
  try {
    return body();
  } catch (const WrongType& e) {
    PyErr_SetString(PyExc_TypeError, e.what());
  } catch (const Wrong& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception&) {
    torch::translate_exception_to_python(std::current_exception());
  }
  return nullptr;
}

// q, k, v, k_pool, v_pool, page_table, base, freq, positions, n_new, interleaved, amplitude, out -> (status, out)
PyObject* rope_append_static(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 13 || !append_fn) throw WrongType("rope_append_static takes thirteen arguments, after bind_round()");
    const at::Tensor &q = the(args[0], "q"), &k = the(args[1], "k"), &v = the(args[2], "v"), &k_pool = the(args[3], "k_pool"),
                     &v_pool = the(args[4], "v_pool"), &table = the(args[5], "page_table"), &base = the(args[6], "base"), &freq = the(args[7], "freq");
    const at::Tensor *positions = maybe(args[8], "positions"), *n_new = maybe(args[9], "n_new"), *to = maybe(args[12], "out");
    const int inter = PyObject_IsTrue(args[10]);
    const double amplitude = PyFloat_AsDouble(args[11]);
    if (PyErr_Occurred()) return nullptr;
    if (c10::GradMode::is_enabled()) {
      no_gradient(q, "q");
      no_gradient(k, "k");
      no_gradient(v, "v");
      no_gradient(k_pool, "k_pool");
      no_gradient(v_pool, "v_pool");
      no_gradient(freq, "freq");
      if (to) no_gradient(*to, "out");
    }
    NEED(q.dim() == 4, "q must be [B, T, heads, head_dim]");
    const int64_t B = q.size(0), T = q.size(1);
    tsd_paged_cache cache = cache_of(k_pool, v_pool, table, B);
    like(q, k_pool, "q");
    like(k, k_pool, "k");
    like(v, k_pool, "v");
    apart(k_pool, "k_pool");
    const tsd_rows rq = rows_of(q, {B, T, q.size(2), cache.head_dim}, "q"), rk = rows_of(k, {B, T, cache.n_kv_heads, cache.head_dim}, "k"),
                   rv = rows_of(v, {B, T, cache.n_kv_heads, cache.head_dim}, "v");
    plain(base, q, at::kInt, {B}, "base");
    if (positions) plain(*positions, q, at::kInt, {B, T}, "positions");
    if (n_new) plain(*n_new, q, at::kInt, {B}, "n_new");
    NEED(freq.dim() == 1, "freq must be [rotary_dim / 2]");
    plain(freq, q, at::kDouble, {freq.size(0)}, "freq");
    const c10::DeviceGuard guard(q.device());
    at::Tensor out = to ? *to : at::empty({B, T, q.size(2), cache.head_dim}, q.options());
    if (to) {
      like(out, q, "out");
      apart(out, "out");
    }
    const tsd_rows ro = rows_of(out, q.sizes(), "out");
    void* stream = c10::hip::getCurrentHIPStream(q.device().index()).stream();
    const int32_t b = whole(B, "B"), t = whole(T, "T"), hq = whole(q.size(2), "heads"), r = whole(2 * freq.size(0), "freq");
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = append_fn(&cache, b, t, hq, &rq, &ro, &rk, &rv, static_cast<const int32_t*>(base.data_ptr()),
                   n_new ? static_cast<const int32_t*>(n_new->data_ptr()) : nullptr, positions ? static_cast<const int32_t*>(positions->data_ptr()) : nullptr,
                   static_cast<const double*>(freq.data_ptr()), r, (float)amplitude, inter ? TSD_FLAG_ROPE_INTERLEAVED : 0, stream);
    Py_END_ALLOW_THREADS
    if (rc == TSD_OK) {
      written(k_pool);
      written(v_pool);
      if (to) written(out);
    }
    return Py_BuildValue("iN", rc, THPVariable_Wrap(out));
  });
}

// q, k_pool, v_pool, page_table, lens, max_len or 0, scale or NaN (head_dim ^ -1/2), n_new, out, want_lse -> (status, out, lse)
PyObject* paged_attn_static(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 10 || !attn_fn) throw WrongType("paged_attn_static takes ten arguments, after bind_round()");
    const at::Tensor &q = the(args[0], "q"), &k_pool = the(args[1], "k_pool"), &v_pool = the(args[2], "v_pool"), &table = the(args[3], "page_table"),
                     &lens = the(args[4], "lens");
    const long long asked = PyLong_AsLongLong(args[5]);
    double scale = PyFloat_AsDouble(args[6]);
    const at::Tensor *n_new = maybe(args[7], "n_new"), *to = maybe(args[8], "out");
    const int want_lse = PyObject_IsTrue(args[9]);
    if (PyErr_Occurred()) return nullptr;
    if (c10::GradMode::is_enabled()) {
      no_gradient(q, "q");
      no_gradient(k_pool, "k_pool");
      no_gradient(v_pool, "v_pool");
      if (to) no_gradient(*to, "out");
    }
    NEED(q.dim() == 4, "q must be [B, T, heads, head_dim]");
    const int64_t B = q.size(0), T = q.size(1), H = q.size(2);
    tsd_paged_cache cache = cache_of(k_pool, v_pool, table, B);
    like(q, k_pool, "q");
    const tsd_rows rq = rows_of(q, {B, T, H, cache.head_dim}, "q");
    plain(lens, q, at::kInt, {B}, "lens");
    if (n_new) plain(*n_new, q, at::kInt, {B}, "n_new");
    const int32_t b = whole(B, "B"), t = whole(T, "T"), h = whole(H, "heads"),
                  max_len = whole(asked ? asked : (int64_t)cache.pages_per_seq * cache.page_tokens, "max_len");
    if (std::isnan(scale)) scale = 1.0 / std::sqrt((double)cache.head_dim);
    const c10::DeviceGuard guard(q.device());
    size_t bytes = 0;
    int rc = attn_bytes_fn(&cache, b, t, h, max_len, &bytes);
    at::Tensor out = to ? *to : at::empty({B, T, H, cache.head_dim}, q.options()), lse, work;
    if (to) {
      like(out, q, "out");
      apart(out, "out");
    }
    const tsd_rows ro = rows_of(out, q.sizes(), "out");
    if (want_lse) lse = at::empty({B, T, H}, q.options().dtype(at::kFloat));
    if (rc == TSD_OK) {
      if (bytes) work = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
      void* stream = c10::hip::getCurrentHIPStream(q.device().index()).stream();
      Py_BEGIN_ALLOW_THREADS
      rc = attn_fn(&cache, b, t, h, &rq, &ro, want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, static_cast<const int32_t*>(lens.data_ptr()),
                   n_new ? static_cast<const int32_t*>(n_new->data_ptr()) : nullptr, max_len, (float)scale, bytes ? work.data_ptr() : nullptr, bytes, stream);
      Py_END_ALLOW_THREADS
      if (rc == TSD_OK && to) written(out);
    }
    PyObject* l = want_lse ? THPVariable_Wrap(lse) : Py_None;
    if (!want_lse) Py_INCREF(Py_None);
    return Py_BuildValue("iNN", rc, THPVariable_Wrap(out), l);
  });
}

// draft, q or None, p, uniforms, n_draft -> (status, n_acc, tokens)
PyObject* verify_tokens_static(PyObject*, PyObject* const* args, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    if (n != 5 || !verify_fn) throw WrongType("verify_tokens_static takes five arguments, after bind_round()");
    const at::Tensor& draft = the(args[0], "draft");
    const at::Tensor *q = maybe(args[1], "q"), &p = the(args[2], "p"), &uniforms = the(args[3], "uniforms");
    const at::Tensor* n_draft = maybe(args[4], "n_draft");
    on_gpu(p, "p");
    const int dtype = dtype_of(p, "p");
    NEED(draft.dim() == 2 && p.dim() == 3, "draft must be [B, K], p [B, K + 1, V]");
    NEED(draft.scalar_type() == at::kInt || draft.scalar_type() == at::kLong, "draft must be int32 or int64");
    const int64_t B = draft.size(0), K = draft.size(1), V = p.size(2);
    plain(draft, p, draft.scalar_type(), {B, K}, "draft");
    NEED(p.size(0) == B && p.size(1) == K + 1 && (V == 1 || p.stride(2) == 1), "p must be [B, K + 1, V], rows dense");
    if (q) {
      like(*q, p, "q");
      NEED(q->dim() == 3 && q->size(0) == B && q->size(1) == K && q->size(2) == V && (V == 1 || q->stride(2) == 1), "q must be [B, K, V], rows dense");
    }
    plain(uniforms, p, at::kFloat, {B, K + 1}, "uniforms");
    if (n_draft) plain(*n_draft, p, at::kInt, {B}, "n_draft");
    const int32_t b = whole(B, "B"), k = whole(K, "K"), vv = whole(V, "V");
    const c10::DeviceGuard guard(p.device());
    size_t bytes = 0;
    int rc = verify_bytes_fn(b, k, vv, dtype, &bytes);
    at::Tensor n_acc, tokens, work;
    if (rc == TSD_OK) {
      n_acc = at::empty({B}, p.options().dtype(at::kInt));
      tokens = at::empty({B, K + 1}, draft.options());
      work = at::empty({(int64_t)bytes}, p.options().dtype(at::kByte));
      void* stream = c10::hip::getCurrentHIPStream(p.device().index()).stream();
      Py_BEGIN_ALLOW_THREADS
      rc = verify_fn(draft.data_ptr(), q ? q->data_ptr() : nullptr, p.data_ptr(), dtype, (int)draft.element_size(), b, k, vv, q ? q->stride(0) : 0,
                     q ? q->stride(1) : 0, p.stride(0), p.stride(1), static_cast<const float*>(uniforms.data_ptr()),
                     n_draft ? static_cast<const int32_t*>(n_draft->data_ptr()) : nullptr, static_cast<int32_t*>(n_acc.data_ptr()), tokens.data_ptr(),
                     work.data_ptr(), bytes, stream);
      Py_END_ALLOW_THREADS
    }
    if (rc != TSD_OK) return Py_BuildValue("iOO", rc, Py_None, Py_None);
    return Py_BuildValue("iNN", rc, THPVariable_Wrap(n_acc), THPVariable_Wrap(tokens));
  });
}

template <typename F>
PyCFunction fast(F* f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}

PyMethodDef methods[] = {{"bind", bind, METH_O, "the address of tsd_accept_commit_static"},
                         {"accept_commit_static", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(accept_commit_static)), METH_FASTCALL,
                          "see binding.accept_commit_static"},
                         {"bind_round", fast(bind_round), METH_FASTCALL, "the addresses of the calls of a round"},
                         {"rope_append_static", fast(rope_append_static), METH_FASTCALL, "see binding.rope_append_static"},
                         {"paged_attn_static", fast(paged_attn_static), METH_FASTCALL, "see binding.paged_attn_static"},
                         {"verify_tokens_static", fast(verify_tokens_static), METH_FASTCALL, "see binding.verify_tokens_static"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
