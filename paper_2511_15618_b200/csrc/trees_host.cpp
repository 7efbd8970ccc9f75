// The calls on trees, pages and scores for torch tensors: checks, outputs and workspaces, and the C call on torch's current
// stream, in one native function each.  (A pass of a decode loop makes a handful of these calls, each a few microseconds of
// the device; checked and allocated from Python they took 14 to 17 us of the host each, 4 of them the launches.)
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <limits>

#include "../../include/flashmesh.h"

namespace {

PyObject* error_class = nullptr;         // FmError(code, where)

struct Refused { int code; const char* where; };
inline void need(bool ok, const char* what) { if (!ok) throw Refused{FM_ERR_INVALID_ARG, what}; }
inline void check(int rc, const char* where) { if (rc != FM_OK) throw Refused{rc, where}; }

inline const at::Tensor& tensor(PyObject* o, const char* what) {
  need(THPVariable_Check(o), what);
  return THPVariable_Unpack(o);
}
inline int32_t number(PyObject* o, const char* what) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); need(false, what); }
  need(v >= std::numeric_limits<int32_t>::min() && v <= std::numeric_limits<int32_t>::max(), what);
  return (int32_t)v;
}
template <typename T> inline T* address(PyObject* o, const char* what) {
  void* p = PyLong_AsVoidPtr(o);
  if (p == nullptr) { PyErr_Clear(); need(false, what); }
  return static_cast<T*>(p);
}
inline bool lies_on(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }
inline int32_t* ids(const at::Tensor& t, int device, const char* what) {
  need(t.scalar_type() == at::kInt && lies_on(t, device) && t.is_contiguous(), what);
  return static_cast<int32_t*>(t.data_ptr());
}
inline bool shaped(const at::Tensor& t, std::initializer_list<int64_t> s) { return t.sizes().equals(at::IntArrayRef(s.begin(), s.size())); }
// (the stride of a dimension of size 1 means nothing, and differs between views of the same contents)
inline int64_t step(const at::Tensor& t, int64_t d, int64_t otherwise) { return t.size(d) > 1 ? t.stride(d) : otherwise; }
inline bool alike(const at::Tensor& x, const at::Tensor& y) {
  if (!x.sizes().equals(y.sizes())) return false;
  for (int64_t d = 0; d < x.dim(); ++d)
    if (step(x, d, 0) != step(y, d, 0)) return false;
  return true;
}
inline bool fits(int64_t n) { return n <= std::numeric_limits<int32_t>::max(); }
inline at::Tensor fresh(std::initializer_list<int64_t> s, const at::Tensor& like, at::ScalarType type) {
  return at::empty(at::IntArrayRef(s.begin(), s.size()), like.options().dtype(type).requires_grad(false));
}
// There is no backward pass: a result without a gradient for an input that asks for one would lose it without a word
inline void no_gradient(const at::Tensor& t) {
  need(!(t.requires_grad() && at::GradMode::is_enabled()), "an input requires a gradient, and this call has none: call it under torch.no_grad(), or detach the input");
}
// in place: what autograd has kept of the tensor for a backward pass is no longer that
inline void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
inline void all_written(PyObject* const* a, Py_ssize_t first, Py_ssize_t end, const char* what) {
  for (Py_ssize_t i = first; i < end; ++i) written(tensor(a[i], what));
}
inline PyObject* given(PyObject* o) { return o == Py_None ? nullptr : o; }

// f(), with refusals as FmError and torch's errors as torch raises them
template <typename F>
PyObject* run(F f) {
  HANDLE_TH_ERRORS
  try {
    at::AutoDispatchBelowADInplaceOrView no_grad;
    return f();
  } catch (const Refused& r) {
    PyObject* e = PyObject_CallFunction(error_class, "is", r.code, r.where);
    if (e != nullptr) { PyErr_SetObject(error_class, e); Py_DECREF(e); }
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}
PyObject* tuple_of(std::initializer_list<at::Tensor> t) {
  PyObject* r = PyTuple_New((Py_ssize_t)t.size());
  if (r == nullptr) return nullptr;
  Py_ssize_t i = 0;
  for (const at::Tensor& x : t) {
    PyObject* o = THPVariable_Wrap(x);
    if (o == nullptr) { Py_DECREF(r); return nullptr; }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// (cache, pages, device, layer, q, k_new, v_new, row_off, parent, seqs, window, n_prefix, scale, max_nodes, max_len, want_lse, out)
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    need(n_args == 17, "attention: 17 arguments");
    const fm_cache& c = *address<fm_cache>(a[0], "attention: cache");
    const fm_pages& p = *address<fm_pages>(a[1], "attention: pages");
    const int device = number(a[2], "attention: device"), layer = number(a[3], "attention: a number out of range");
    const at::Tensor &q = tensor(a[4], "attention: q"), &k = tensor(a[5], "attention: k_new"), &v = tensor(a[6], "attention: v_new"),
                     &off = tensor(a[7], "attention: row_off"), &parent = tensor(a[8], "attention: parent");
    for (const at::Tensor* t : {&q, &k, &v}) no_gradient(*t);
    const at::ScalarType type = c.dtype == FM_BF16 ? at::kBFloat16 : at::kHalf;
    const int64_t dh = c.head_dim;
    need(q.dim() == 3 && q.size(2) == dh && q.stride(2) == 1 && step(q, 1, dh) == dh && q.scalar_type() == type && lies_on(q, device),
         "attention: q [rows, heads, head_dim] of the cache's type");
    const int64_t rows = q.size(0), heads = q.size(1), n = off.numel() - 1;
    need(shaped(k, {rows, c.n_kv_heads, dh}) && alike(k, v) && k.stride(2) == 1 && step(k, 1, dh) == dh &&
             k.scalar_type() == type && v.scalar_type() == type && lies_on(k, device) && lies_on(v, device),
         "attention: k_new and v_new [rows, kv heads, head_dim] of the cache's type, with the same strides");
    PyObject* const listed = given(a[9]);
    const int32_t* seqs = nullptr;
    if (listed != nullptr) {
      const at::Tensor& s = tensor(listed, "attention: seqs");
      need(shaped(s, {n}), "attention: seqs [n]");
      seqs = ids(s, device, "seqs: a contiguous int32 tensor on the cache's device");
    }
    need((n >= 1 || (n == 0 && rows == 0)) && shaped(parent, {rows}) && (seqs != nullptr || n <= p.max_seqs) && fits(n) && fits(rows) && fits(heads),
         "attention: row_off [n + 1], parent [rows], seqs [n]");
    const char* const range = "attention: a number out of range";
    fm_tree_args t{};
    t.window = number(a[10], range);
    t.n_prefix = number(a[11], range);
    if (given(a[12]) == nullptr) {
      t.scale = (float)(1.0 / std::sqrt((double)dh));
    } else {
      const double s = PyFloat_AsDouble(a[12]);
      if (s == -1.0 && PyErr_Occurred()) { PyErr_Clear(); need(false, range); }
      t.scale = (float)s;
    }
    t.max_nodes = given(a[13]) != nullptr ? number(a[13], range) : (int32_t)std::min<int64_t>(rows, FM_MAX_TREE_NODES);
    t.max_len = given(a[14]) != nullptr ? number(a[14], range) : (int32_t)std::min<int64_t>((int64_t)p.max_pages * p.page_slots, std::numeric_limits<int32_t>::max());
    t.batch = (int32_t)n; t.n_heads = (int32_t)heads; t.max_pages = p.max_pages; t.max_seqs = p.max_seqs;
    t.table = p.table; t.lens = p.lens; t.status = p.status; t.seqs = seqs;
    t.row_off = ids(off, device, "row_off: a contiguous int32 tensor on the cache's device");
    t.parent = ids(parent, device, "parent: a contiguous int32 tensor on the cache's device");
    t.q_row_stride = step(q, 0, heads * dh);
    t.new_row_stride = step(k, 0, c.n_kv_heads * dh);
    at::Tensor out;
    if (given(a[16]) == nullptr) {
      out = fresh({rows, heads, dh}, q, type);
    } else {
      out = tensor(a[16], "attention: out");
      no_gradient(out);
      need(out.sizes() == q.sizes() && out.scalar_type() == type && lies_on(out, device) && out.stride(2) == 1 && step(out, 1, dh) == dh, "attention: out like q");
    }
    t.out_row_stride = step(out, 0, heads * dh);
    const int want_lse = PyObject_IsTrue(a[15]);
    if (want_lse < 0) return nullptr;
    at::Tensor lse;
    if (want_lse) lse = fresh({rows, heads}, q, at::kFloat);
    if (rows == 0) {                                         // (no tree has a node)
      if (want_lse) return tuple_of({out, lse});
      return THPVariable_Wrap(out);
    }
    t.n_rows = (int32_t)rows;
    t.fill = (given(a[16]) == nullptr ? FM_FILL_OUT : 0) | (want_lse ? FM_FILL_LSE : 0);       // (what is allocated here holds no stale values)
    t.q = q.data_ptr(); t.k_new = k.data_ptr(); t.v_new = v.data_ptr(); t.out = out.data_ptr();
    t.lse = want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr;
    const size_t bytes = fm_tree_attention_bytes(&c, &t);    // (0: the call itself refuses)
    at::Tensor work;
    if (bytes > 0) work = fresh({(int64_t)bytes}, q, at::kByte);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    check(fm_tree_attention(&c, layer, &t, bytes > 0 ? work.data_ptr() : nullptr, bytes, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()),
          "fm_tree_attention");
    if (given(a[16]) != nullptr) written(out);
    if (want_lse) return tuple_of({out, lse});
    return THPVariable_Wrap(out);
  });
}

// (cache, pages, device, seqs, k_new, v_new, row_off, path, n_acc, max_rows, tensors that it writes ...)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    need(n_args >= 10, "append: 10 arguments");
    const fm_cache& c = *address<fm_cache>(a[0], "append: cache");
    const fm_pages& p = *address<fm_pages>(a[1], "append: pages");
    const int device = number(a[2], "append: device");
    const at::Tensor &seqs = tensor(a[3], "append: seqs"), &k = tensor(a[4], "append: k_new"), &v = tensor(a[5], "append: v_new"), &off = tensor(a[6], "append: row_off");
    no_gradient(k);
    no_gradient(v);
    const int64_t n = seqs.numel();
    need(seqs.dim() == 1 && shaped(off, {n + 1}) && fits(n), "append: seqs [n], row_off [n + 1]");
    const at::ScalarType type = c.dtype == FM_BF16 ? at::kBFloat16 : at::kHalf;
    need(k.dim() == 4 && k.size(0) == c.n_layers && k.size(2) == c.n_kv_heads && k.size(3) == c.head_dim && alike(k, v) &&
             k.stride(3) == 1 && k.scalar_type() == type && v.scalar_type() == type && lies_on(k, device) && lies_on(v, device) && fits(k.size(1)),
         "append: k_new and v_new [layers, rows, kv heads, head_dim] of the cache's type, with the same strides");
    need((given(a[7]) == nullptr) == (given(a[8]) == nullptr), "append: path and n_acc go together");
    const int32_t *path = nullptr, *n_acc = nullptr;
    int64_t stride = 0;
    if (given(a[7]) != nullptr) {
      const at::Tensor &pt = tensor(a[7], "append: path"), &at_ = tensor(a[8], "append: n_acc");
      need(pt.dim() == 2 && pt.size(0) == n && shaped(at_, {n}) && fits(pt.size(1)), "append: path [n, stride], n_acc [n]");
      stride = pt.size(1);
      path = ids(pt, device, "path: a contiguous int32 tensor on the cache's device");
      n_acc = ids(at_, device, "n_acc: a contiguous int32 tensor on the cache's device");
    }
    int32_t most = given(a[9]) != nullptr ? number(a[9], "append: max_rows") : (int32_t)(path != nullptr ? stride : k.size(1));
    const bool none = k.size(1) == 0;                        // no rows, and tensors without an address: entries may append nothing
    if (none) most = std::min(most, 0);
    const fm_new_rows rows{none ? c.k : k.data_ptr(), none ? c.v : v.data_ptr(), step(k, 0, 0), step(k, 1, 0), step(k, 2, 0), (int32_t)k.size(1)};
    const int32_t* s = ids(seqs, device, "seqs: a contiguous int32 tensor on the cache's device");
    const int32_t* o = ids(off, device, "row_off: a contiguous int32 tensor on the cache's device");
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    check(fm_pages_append(&p, &c, &rows, s, o, path, (int32_t)stride, n_acc, (int32_t)n, most,
                          c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()), "fm_pages_append");
    all_written(a, 10, n_args, "append: a tensor of the cache");
    Py_RETURN_NONE;
  });
}

// (cache, pages, device, first, second, tensors that it writes ...): fork (src, dst), reserve (seqs, grow), truncate (seqs, lens)
enum class Lists { fork, reserve, truncate };
template <Lists WHICH>
PyObject* lists(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    constexpr const char* name = WHICH == Lists::fork ? "fm_pages_fork" : WHICH == Lists::reserve ? "fm_pages_reserve" : "fm_pages_truncate";
    need(n_args >= 5, name);
    const fm_cache& c = *address<fm_cache>(a[0], name);
    const fm_pages& p = *address<fm_pages>(a[1], name);
    const int device = number(a[2], name);
    const at::Tensor &x = tensor(a[3], name), &y = tensor(a[4], name);
    need(x.dim() == 1 && x.sizes() == y.sizes() && fits(x.numel()), "two lists of the same length");
    const int32_t *u = ids(x, device, "a list: a contiguous int32 tensor on the cache's device"), *v = ids(y, device, "a list: a contiguous int32 tensor on the cache's device");
    const int32_t n = (int32_t)x.numel();
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    check(WHICH == Lists::fork ? fm_pages_fork(&p, u, v, n, stream) : WHICH == Lists::reserve ? fm_pages_reserve(&p, &c, u, v, n, stream)
                                                                                               : fm_pages_truncate(&p, u, v, n, stream), name);
    all_written(a, 5, n_args, name);
    Py_RETURN_NONE;
  });
}

// (cache, pages, device, table, tensors that it writes ...): the pages in use
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    need(n_args >= 4, "compact: 4 arguments");
    const fm_cache& c = *address<fm_cache>(a[0], "compact: cache");
    const fm_pages& p = *address<fm_pages>(a[1], "compact: pages");
    const int device = number(a[2], "compact: device");
    const at::Tensor used = fresh({1}, tensor(a[3], "compact: table"), at::kInt);
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    check(fm_pages_compact(&p, &c, static_cast<int32_t*>(used.data_ptr()), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()), "fm_pages_compact");
    all_written(a, 4, n_args, "compact: a tensor of the cache");
    return THPVariable_Wrap(used);
  });
}

// (tokens, parent, row_off, predicted, max_nodes)
PyObject* accept(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    need(n_args == 5, "tree_accept: 5 arguments");
    const char* const what = "tree_accept: tokens, parent, predicted [rows]; row_off [n + 1]";
    const at::Tensor &tokens = tensor(a[0], what), &parent = tensor(a[1], what), &off = tensor(a[2], what), &predicted = tensor(a[3], what);
    const int64_t rows = tokens.numel(), n = off.numel() - 1;
    need(tokens.is_cuda() && tokens.dim() == 1 && fits(rows) && parent.sizes() == tokens.sizes() && predicted.sizes() == tokens.sizes() && n >= 0 && fits(n), what);
    const int device = tokens.get_device();
    const int32_t stride = given(a[4]) != nullptr ? number(a[4], "tree_accept: max_nodes") : (int32_t)std::min<int64_t>(std::max<int64_t>(rows, 1), FM_MAX_TREE_NODES);
    const int32_t *t = ids(tokens, device, "tokens: a contiguous int32 tensor on one device"), *p = ids(parent, device, "parent: a contiguous int32 tensor on one device"),
                  *o = ids(off, device, "row_off: a contiguous int32 tensor on one device"), *w = ids(predicted, device, "predicted: a contiguous int32 tensor on one device");
    if (rows == 0) t = p = w = o;                            // (tensors without an address; no tree has a node to read)
    const at::Tensor path = fresh({n, std::max(stride, 0)}, tokens, at::kInt), n_acc = fresh({n}, tokens, at::kInt), next = fresh({n}, tokens, at::kInt);
    if (n == 0) return tuple_of({path, n_acc, next});
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
    check(fm_tree_accept_rows(t, p, o, w, (int32_t)rows, (int32_t)n, static_cast<int32_t*>(path.data_ptr()), stride, static_cast<int32_t*>(n_acc.data_ptr()),
                         static_cast<int32_t*>(next.data_ptr()), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()), "fm_tree_accept");
    return tuple_of({path, n_acc, next});
  });
}

// (logits, tokens, top)
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return run([&]() -> PyObject* {
    need(n_args == 3, "logprobs: 3 arguments");
    const char* const what = "logprobs: logits [rows, vocab] in float32, bfloat16 or float16 on a CUDA device";
    const at::Tensor& x = tensor(a[0], what);
    no_gradient(x);
    const at::ScalarType type = x.scalar_type();
    const int kind = type == at::kFloat ? FM_FP32 : type == at::kBFloat16 ? FM_BF16 : type == at::kHalf ? FM_FP16 : -1;
    need(kind >= 0 && x.dim() == 2 && x.is_cuda() && x.size(1) >= 1 && (x.stride(1) == 1 || x.size(1) == 1) && fits(x.size(0)) && fits(x.size(1)), what);
    const int64_t rows = x.size(0), vocab = x.size(1);
    const int device = x.get_device(), top = number(a[2], "logprobs: top");
    need(top >= 0 && top <= vocab, "logprobs: tokens [rows], top");
    const int32_t* tokens = nullptr;
    if (given(a[1]) != nullptr) {
      const at::Tensor& t = tensor(a[1], "logprobs: tokens [rows], top");
      need(shaped(t, {rows}), "logprobs: tokens [rows], top");
      tokens = ids(t, device, "tokens: a contiguous int32 tensor on the logits' device");
    }
    const at::Tensor lp = fresh({rows}, x, at::kFloat), ent = fresh({rows}, x, at::kFloat), rank = fresh({rows}, x, at::kInt), ids_ = fresh({rows, top}, x, at::kInt),
                     tops = fresh({rows, top}, x, at::kFloat);
    if (rows > 0) {
      const c10::cuda::CUDAGuard guard((c10::DeviceIndex)device);
      check(fm_logprobs(x.data_ptr(), kind, (int32_t)rows, (int32_t)vocab, rows > 1 ? x.stride(0) : vocab, tokens, static_cast<float*>(lp.data_ptr()),
                        static_cast<float*>(ent.data_ptr()), static_cast<int32_t*>(rank.data_ptr()), top, static_cast<int32_t*>(ids_.data_ptr()),
                        static_cast<float*>(tops.data_ptr()), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream()), "fm_logprobs");
    }
    return tuple_of({lp, ent, rank, ids_, tops});
  });
}

PyObject* set_error(PyObject*, PyObject* o) {
  Py_INCREF(o);
  Py_XSETREF(error_class, o);
  Py_RETURN_NONE;
}

PyMethodDef fast(const char* name, PyObject* (*f)(PyObject*, PyObject* const*, Py_ssize_t)) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {
    fast("attention", attention), fast("append", append), fast("fork", lists<Lists::fork>), fast("reserve", lists<Lists::reserve>),
    fast("truncate", lists<Lists::truncate>), fast("compact", compact), fast("accept", accept), fast("logprobs", logprobs),
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};
#ifndef FM_BUILT_FOR
#define FM_BUILT_FOR "fm built for: not said"
#endif
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_trees", FM_BUILT_FOR, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__trees() { return PyModule_Create(&module); }
