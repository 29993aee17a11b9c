// Python entry of the decode-side calls: takes torch tensors, checks type, device, layout and shape, and calls the C ABI.
// A decoding step makes a handful of calls per layer whose kernels take a few microseconds each; checking ten tensors and
// marshalling them in Python takes 10 to 15.  The C functions come in as addresses (set_functions), so that this module
// serves whichever build of the library the binding has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "shareprefill.h"

namespace {

// Read from the file before it is loaded: an entry that was compiled for another torch or Python is not.
__attribute__((used)) const char kBuiltAgainst[] = SP_BUILT_AGAINST;

struct Functions {
  decltype(&sp_page_tables) page_tables;
  decltype(&sp_qk_norm_rope) qk_norm_rope;
  decltype(&sp_tree_attn) tree_attn;
  decltype(&sp_cache_keep) cache_keep;
} fn{};

struct Refused {};      // a Python exception has been set

[[noreturn]] void refuse(const char* what, const char* expected, int device) {
  PyErr_Format(PyExc_ValueError, "%s: expected %s on cuda:%d", what, expected, device);
  throw Refused();
}

const at::Tensor& tensor(PyObject* o, const char* what, const char* expected, int device, at::ScalarType type) {
  if (!THPVariable_Check(o)) refuse(what, expected, device);
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != device) refuse(what, expected, device);
  return t;
}

int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused();
  return v;
}
int small(PyObject* o) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) { PyErr_SetString(PyExc_OverflowError, "an integer argument does not fit 32 bits"); throw Refused(); }
  return (int)v;
}

// A contiguous int32 tensor of `dims` dimensions; n0 / n1 < 0: any size.
struct Ints {
  int32_t* p = nullptr;
  int n0 = 0, n1 = 0;
};
Ints ints(PyObject* o, const char* what, int device, int dims, int64_t n0, int64_t n1 = -1) {
  const at::Tensor& t = tensor(o, what, "a contiguous int32 tensor", device, at::kInt);
  if (!t.is_contiguous()) refuse(what, "a contiguous int32 tensor", device);
  if (t.dim() != dims || (n0 >= 0 && t.size(0) != n0) || (dims > 1 && n1 >= 0 && t.size(1) != n1)) {
    if (dims == 1 && n0 < 0) PyErr_Format(PyExc_ValueError, "%s: expected one dimension", what);
    else if (dims == 1) PyErr_Format(PyExc_ValueError, "%s: expected %lld elements in one dimension", what, (long long)n0);
    else PyErr_Format(PyExc_ValueError, "%s: expected a two-dimensional tensor of %lld rows", what, (long long)n0);
    throw Refused();
  }
  if (t.numel() > INT32_MAX) { PyErr_Format(PyExc_ValueError, "%s: too large", what); throw Refused(); }
  return {static_cast<int32_t*>(t.data_ptr()), (int)t.size(0), dims > 1 ? (int)t.size(1) : 1};
}
Ints maybe_ints(PyObject* o, const char* what, int device, int dims, int64_t n0, int64_t n1 = -1) {
  return o == Py_None ? Ints{} : ints(o, what, device, dims, n0, n1);
}

// [heads, rows, dim] or [1, heads, rows, dim]; caches [pages, heads, page, dim].
sp_tensor view(PyObject* o, const char* what, int device, bool cache) {
  const at::Tensor& t = tensor(o, what, "a bf16 tensor", device, at::kBFloat16);
  const auto shape = t.sizes(), stride = t.strides();
  const int lead = 4 - (int)shape.size();
  if (lead < 0 || lead > (cache ? 0 : 1)) {
    PyErr_Format(PyExc_ValueError, "%s: expected %s", what, cache ? "[pages, heads, page, dim]" : "[heads, rows, dim]");
    throw Refused();
  }
  sp_tensor v;
  v.data = t.data_ptr();
  v.shape[0] = 1;
  v.stride[0] = 0;
  for (int x = lead; x < 4; ++x) { v.shape[x] = shape[x - lead]; v.stride[x] = stride[x - lead]; }
  return v;
}

void* stream_of(PyObject* o, int device) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
  return reinterpret_cast<void*>(integer(o));
}
sp_ctx* context(PyObject* o) { return reinterpret_cast<sp_ctx*>(integer(o)); }

template <typename Body>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, Body body) {
  if (given != wanted) return PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", wanted, given);
  if (!fn.page_tables) return PyErr_Format(PyExc_RuntimeError, "set_functions has not been called");
  try {
    return PyLong_FromLong(body());
  } catch (const Refused&) {
    return nullptr;
  } catch (const std::exception& e) {
    return PyErr_Format(PyExc_RuntimeError, "%s", e.what());
  }
}

PyObject* set_functions(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "expected 4 addresses");
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "a null address");
  }
  fn = {reinterpret_cast<decltype(fn.page_tables)>(p[0]), reinterpret_cast<decltype(fn.qk_norm_rope)>(p[1]),
        reinterpret_cast<decltype(fn.tree_attn)>(p[2]), reinterpret_cast<decltype(fn.cache_keep)>(p[3])};
  Py_RETURN_NONE;
}

// ctx, device, past_lens, new_lens, page, free_pages, block_table, seq_lens, row_start, positions, slots, info, parents, tree_mask, stream
PyObject* page_tables(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 15, [&] {
    const int dev = small(a[1]);
    const Ints past = ints(a[2], "past_lens", dev, 1, -1);
    const int n = past.n0;
    const Ints fresh = ints(a[3], "new_lens", dev, 1, n), free_pages = ints(a[5], "free_pages", dev, 1, -1), table = ints(a[6], "block_table", dev, 2, n);
    const Ints lens = ints(a[7], "seq_lens", dev, 1, n), start = ints(a[8], "row_start", dev, 1, (int64_t)n + 1), slots = ints(a[10], "slots", dev, 1, -1);
    const Ints pos = ints(a[9], "positions", dev, 1, slots.n0), info = ints(a[11], "info", dev, 1, 4);
    const Ints parents = maybe_ints(a[12], "parents", dev, 1, slots.n0), bits = maybe_ints(a[13], "tree_mask", dev, 2, slots.n0);
    return fn.page_tables(context(a[0]), past.p, fresh.p, n, small(a[4]), free_pages.p, free_pages.n0, table.p, table.n1, parents.p, lens.p, start.p, pos.p,
                          slots.p, reinterpret_cast<uint32_t*>(bits.p), bits.n1, slots.n0, info.p, stream_of(a[14], dev));
  });
}

// ctx, device, q, k, v, positions, inv_freq, q_out, k_out, v_out, k_cache, v_cache, slots, q_weight, k_weight, eps, interleaved, stream
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 18, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), k = view(a[3], "k", dev, false), v = view(a[4], "v", dev, false), q_out = view(a[7], "q_out", dev, false);
    const int64_t rows = q.shape[2], d = q.shape[3];
    sp_tensor opt[4];
    const sp_tensor* given[4];
    const char* names[4] = {"k_out", "v_out", "k_cache", "v_cache"};
    for (int i = 0; i < 4; ++i) {
      given[i] = nullptr;
      if (a[8 + i] == Py_None) continue;
      opt[i] = view(a[8 + i], names[i], dev, i >= 2);
      given[i] = &opt[i];
    }
    if (!THPVariable_Check(a[6]) || THPVariable_Unpack(a[6]).is_cuda() || THPVariable_Unpack(a[6]).scalar_type() != at::kDouble ||
        THPVariable_Unpack(a[6]).dim() != 1 || !THPVariable_Unpack(a[6]).is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "inv_freq: expected a contiguous one-dimensional float64 tensor on the host");
      throw Refused();
    }
    const at::Tensor& freq = THPVariable_Unpack(a[6]);
    const void* weight[2];
    for (int i = 0; i < 2; ++i) {
      weight[i] = nullptr;
      if (a[13 + i] == Py_None) continue;
      const at::Tensor& w = tensor(a[13 + i], i ? "k_weight" : "q_weight", "a contiguous bf16 tensor of one head's size", dev, at::kBFloat16);
      if (w.dim() != 1 || w.size(0) != d || !w.is_contiguous()) refuse(i ? "k_weight" : "q_weight", "a contiguous bf16 tensor of one head's size", dev);
      weight[i] = w.data_ptr();
    }
    const double eps = PyFloat_AsDouble(a[15]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused();
    const int interleaved = PyObject_IsTrue(a[16]);
    if (interleaved < 0) throw Refused();
    return fn.qk_norm_rope(context(a[0]), &q, &k, &v, weight[0], weight[1], (float)eps, static_cast<const double*>(freq.data_ptr()),
                           (int)std::min<int64_t>(freq.size(0), INT32_MAX), interleaved, ints(a[5], "positions", dev, 1, rows).p, &q_out, given[0], given[1],
                           given[2], given[3], maybe_ints(a[12], "slots", dev, 1, rows).p, stream_of(a[17], dev));
  });
}

// ctx, device, q, k_cache, v_cache, block_table, seq_lens, row_start, out, tree_mask, lse_out, stream
PyObject* tree_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 12, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), k = view(a[3], "k_cache", dev, true), v = view(a[4], "v_cache", dev, true), out = view(a[8], "out", dev, false);
    const Ints lens = ints(a[6], "seq_lens", dev, 1, -1);
    const int n = lens.n0;
    const Ints table = ints(a[5], "block_table", dev, 2, n), start = ints(a[7], "row_start", dev, 1, (int64_t)n + 1);
    const Ints bits = maybe_ints(a[9], "tree_mask", dev, 2, q.shape[2]);
    if (a[9] != Py_None && bits.n1 < 1) { PyErr_SetString(PyExc_ValueError, "tree_mask: expected at least one word a row"); throw Refused(); }   // its address would be null: a chain
    float* lse = nullptr;
    if (a[10] != Py_None) {
      const at::Tensor& t = tensor(a[10], "lse_out", "a contiguous fp32 tensor [heads, rows]", dev, at::kFloat);
      if (t.dim() != 2 || t.size(0) != q.shape[1] || t.size(1) != q.shape[2] || !t.is_contiguous()) refuse("lse_out", "a contiguous fp32 tensor [heads, rows]", dev);
      lse = static_cast<float*>(t.data_ptr());
    }
    return fn.tree_attn(context(a[0]), &q, &k, &v, table.p, table.n1, lens.p, start.p, n, reinterpret_cast<uint32_t*>(bits.p), bits.n1, &out, lse,
                        stream_of(a[11], dev));
  });
}

// ctx, device, k_cache, v_cache, block_table, past_lens, kept, n_kept, lens_out, stream
PyObject* cache_keep(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 10, [&] {
    const int dev = small(a[1]);
    const sp_tensor k = view(a[2], "k_cache", dev, true), v = view(a[3], "v_cache", dev, true);
    const Ints past = ints(a[5], "past_lens", dev, 1, -1);
    const int n = past.n0;
    const Ints table = ints(a[4], "block_table", dev, 2, n), kept = ints(a[6], "kept", dev, 2, n), n_kept = ints(a[7], "n_kept", dev, 1, n);
    const Ints lens = ints(a[8], "lens_out", dev, 1, n);
    return fn.cache_keep(context(a[0]), &k, &v, table.p, table.n1, past.p, n, kept.p, n_kept.p, kept.n1, lens.p, stream_of(a[9], dev));
  });
}

template <typename F>
PyCFunction method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef methods[] = {
    {"set_functions", method(set_functions), METH_FASTCALL, "addresses of sp_page_tables, sp_qk_norm_rope, sp_tree_attn, sp_cache_keep"},
    {"page_tables", method(page_tables), METH_FASTCALL, "status code of sp_page_tables"},
    {"qk_norm_rope", method(qk_norm_rope), METH_FASTCALL, "status code of sp_qk_norm_rope"},
    {"tree_attn", method(tree_attn), METH_FASTCALL, "status code of sp_tree_attn"},
    {"cache_keep", method(cache_keep), METH_FASTCALL, "status code of sp_cache_keep"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_decode_calls", "Decode-side calls of the SharePrefill library on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decode_calls() { return PyModule_Create(&module); }
