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
  decltype(&sp_qk_norm_rope_q4) qk_norm_rope_q4;
  decltype(&sp_tree_attn_q4) tree_attn_q4;
  decltype(&sp_cache_keep_q4) cache_keep_q4;
  decltype(&sp_cache_read_q4) cache_read_q4;
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
  if (n != 8) return PyErr_Format(PyExc_TypeError, "expected 8 addresses");
  void* p[8];
  for (int i = 0; i < 8; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "a null address");
  }
  fn = {reinterpret_cast<decltype(fn.page_tables)>(p[0]), reinterpret_cast<decltype(fn.qk_norm_rope)>(p[1]),
        reinterpret_cast<decltype(fn.tree_attn)>(p[2]), reinterpret_cast<decltype(fn.cache_keep)>(p[3]),
        reinterpret_cast<decltype(fn.qk_norm_rope_q4)>(p[4]), reinterpret_cast<decltype(fn.tree_attn_q4)>(p[5]),
        reinterpret_cast<decltype(fn.cache_keep_q4)>(p[6]), reinterpret_cast<decltype(fn.cache_read_q4)>(p[7])};
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

// The 4-bit cache: uint8 [pages, heads, bytes of a page]; the page's size follows from the head's.
sp_q4_cache q4_view(PyObject* o, int device, int64_t head_dim) {
  const at::Tensor& t = tensor(o, "cache", "a uint8 tensor", device, at::kByte);
  const int64_t block = 17 * head_dim;               // 16 tokens
  if (t.dim() != 3 || (t.size(2) != 1 && t.stride(2) != 1)) {
    PyErr_SetString(PyExc_ValueError, "cache: expected [pages, heads, bytes of a page], the bytes contiguous");
    throw Refused();
  }
  if (head_dim <= 0 || head_dim > 1024 || t.size(2) % block != 0) {
    PyErr_Format(PyExc_ValueError, "cache: pages of %lld bytes do not hold heads of %lld elements", (long long)t.size(2), (long long)head_dim);
    throw Refused();
  }
  return sp_q4_cache{t.data_ptr(), t.size(0), t.size(1), t.size(2) / block * 16, head_dim, t.stride(0), t.stride(1)};
}

// What the two forms of the norm and rotation share of their arguments.
struct Turning {
  const double* freq;
  int n_freq;
  const void* weight[2];
  float eps;
  int interleaved;
};
Turning turning(PyObject* inv_freq, PyObject* const* weights, PyObject* eps, PyObject* interleaved, int dev, int64_t d) {
  Turning r;
  if (!THPVariable_Check(inv_freq) || THPVariable_Unpack(inv_freq).is_cuda() || THPVariable_Unpack(inv_freq).scalar_type() != at::kDouble ||
      THPVariable_Unpack(inv_freq).dim() != 1 || !THPVariable_Unpack(inv_freq).is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "inv_freq: expected a contiguous one-dimensional float64 tensor on the host");
    throw Refused();
  }
  const at::Tensor& freq = THPVariable_Unpack(inv_freq);
  r.freq = static_cast<const double*>(freq.data_ptr());
  r.n_freq = (int)std::min<int64_t>(freq.size(0), INT32_MAX);
  for (int i = 0; i < 2; ++i) {
    r.weight[i] = nullptr;
    if (weights[i] == Py_None) continue;
    const at::Tensor& w = tensor(weights[i], i ? "k_weight" : "q_weight", "a contiguous bf16 tensor of one head's size", dev, at::kBFloat16);
    if (w.dim() != 1 || w.size(0) != d || !w.is_contiguous()) refuse(i ? "k_weight" : "q_weight", "a contiguous bf16 tensor of one head's size", dev);
    r.weight[i] = w.data_ptr();
  }
  const double e = PyFloat_AsDouble(eps);
  if (e == -1.0 && PyErr_Occurred()) throw Refused();
  r.eps = (float)e;
  r.interleaved = PyObject_IsTrue(interleaved);
  if (r.interleaved < 0) throw Refused();
  return r;
}
// Views of up to N arguments, some of them None.
template <int N>
struct Views {
  sp_tensor t[N];
  const sp_tensor* p[N];
  Views(PyObject* const* a, const char* const* names, int dev, int first_cache) {
    for (int i = 0; i < N; ++i) {
      p[i] = nullptr;
      if (a[i] == Py_None) continue;
      t[i] = view(a[i], names[i], dev, i >= first_cache);
      p[i] = &t[i];
    }
  }
};
const char* const kOutNames[4] = {"k_out", "v_out", "k_cache", "v_cache"};

// ctx, device, q, k, v, positions, inv_freq, q_out, k_out, v_out, k_cache, v_cache, slots, q_weight, k_weight, eps, interleaved, stream
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 18, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), k = view(a[3], "k", dev, false), v = view(a[4], "v", dev, false), q_out = view(a[7], "q_out", dev, false);
    const int64_t rows = q.shape[2];
    const Views<4> to(a + 8, kOutNames, dev, 2);
    const Turning r = turning(a[6], a + 13, a[15], a[16], dev, q.shape[3]);
    return fn.qk_norm_rope(context(a[0]), &q, &k, &v, r.weight[0], r.weight[1], r.eps, r.freq, r.n_freq, r.interleaved, ints(a[5], "positions", dev, 1, rows).p,
                           &q_out, to.p[0], to.p[1], to.p[2], to.p[3], maybe_ints(a[12], "slots", dev, 1, rows).p, stream_of(a[17], dev));
  });
}

// ctx, device, q, k, v, positions, inv_freq, q_out, k_out, v_out, cache, slots, q_weight, k_weight, eps, interleaved, stream
PyObject* qk_norm_rope_q4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 17, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), k = view(a[3], "k", dev, false), v = view(a[4], "v", dev, false), q_out = view(a[7], "q_out", dev, false);
    const int64_t rows = q.shape[2];
    const Views<2> to(a + 8, kOutNames, dev, 2);
    const sp_q4_cache cache = q4_view(a[10], dev, q.shape[3]);
    const Turning r = turning(a[6], a + 12, a[14], a[15], dev, q.shape[3]);
    return fn.qk_norm_rope_q4(context(a[0]), &q, &k, &v, r.weight[0], r.weight[1], r.eps, r.freq, r.n_freq, r.interleaved,
                              ints(a[5], "positions", dev, 1, rows).p, &q_out, to.p[0], to.p[1], &cache, ints(a[11], "slots", dev, 1, rows).p, stream_of(a[16], dev));
  });
}

float* lse_of(PyObject* o, const sp_tensor& q, int dev) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o, "lse_out", "a contiguous fp32 tensor [heads, rows]", dev, at::kFloat);
  if (t.dim() != 2 || t.size(0) != q.shape[1] || t.size(1) != q.shape[2] || !t.is_contiguous()) refuse("lse_out", "a contiguous fp32 tensor [heads, rows]", dev);
  return static_cast<float*>(t.data_ptr());
}
Ints tree_bits(PyObject* o, const sp_tensor& q, int dev) {
  const Ints bits = maybe_ints(o, "tree_mask", dev, 2, q.shape[2]);
  if (o != Py_None && bits.n1 < 1) { PyErr_SetString(PyExc_ValueError, "tree_mask: expected at least one word a row"); throw Refused(); }   // its address would be null: a chain
  return bits;
}

// ctx, device, q, k_cache, v_cache, block_table, seq_lens, row_start, out, tree_mask, lse_out, stream
PyObject* tree_attn(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 12, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), k = view(a[3], "k_cache", dev, true), v = view(a[4], "v_cache", dev, true), out = view(a[8], "out", dev, false);
    const Ints lens = ints(a[6], "seq_lens", dev, 1, -1);
    const int n = lens.n0;
    const Ints table = ints(a[5], "block_table", dev, 2, n), start = ints(a[7], "row_start", dev, 1, (int64_t)n + 1);
    const Ints bits = tree_bits(a[9], q, dev);
    float* lse = lse_of(a[10], q, dev);
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

// ctx, device, q, cache, block_table, seq_lens, row_start, out, tree_mask, lse_out, stream
PyObject* tree_attn_q4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 11, [&] {
    const int dev = small(a[1]);
    const sp_tensor q = view(a[2], "q", dev, false), out = view(a[7], "out", dev, false);
    const sp_q4_cache cache = q4_view(a[3], dev, q.shape[3]);
    const Ints lens = ints(a[5], "seq_lens", dev, 1, -1);
    const int n = lens.n0;
    const Ints table = ints(a[4], "block_table", dev, 2, n), start = ints(a[6], "row_start", dev, 1, (int64_t)n + 1);
    const Ints bits = tree_bits(a[8], q, dev);
    float* lse = lse_of(a[9], q, dev);
    return fn.tree_attn_q4(context(a[0]), &q, &cache, table.p, table.n1, lens.p, start.p, n, reinterpret_cast<uint32_t*>(bits.p), bits.n1, &out, lse,
                           stream_of(a[10], dev));
  });
}

// ctx, device, cache, block_table, past_lens, kept, n_kept, lens_out, head_dim, stream
PyObject* cache_keep_q4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 10, [&] {
    const int dev = small(a[1]);
    const sp_q4_cache cache = q4_view(a[2], dev, integer(a[8]));
    const Ints past = ints(a[4], "past_lens", dev, 1, -1);
    const int n = past.n0;
    const Ints table = ints(a[3], "block_table", dev, 2, n), kept = ints(a[5], "kept", dev, 2, n), n_kept = ints(a[6], "n_kept", dev, 1, n);
    const Ints lens = ints(a[7], "lens_out", dev, 1, n);
    return fn.cache_keep_q4(context(a[0]), &cache, table.p, table.n1, past.p, n, kept.p, n_kept.p, kept.n1, lens.p, stream_of(a[9], dev));
  });
}

// ctx, device, cache, block_table, seq_lens, row_start, k_out, v_out, stream
PyObject* cache_read_q4(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded(n_args, 9, [&] {
    const int dev = small(a[1]);
    const sp_tensor k = view(a[6], "k_out", dev, false), v = view(a[7], "v_out", dev, false);
    const sp_q4_cache cache = q4_view(a[2], dev, k.shape[3]);
    const Ints lens = ints(a[4], "seq_lens", dev, 1, -1);
    const int n = lens.n0;
    const Ints table = ints(a[3], "block_table", dev, 2, n), start = ints(a[5], "row_start", dev, 1, (int64_t)n + 1);
    return fn.cache_read_q4(context(a[0]), &cache, table.p, table.n1, lens.p, start.p, n, &k, &v, stream_of(a[8], dev));
  });
}

template <typename F>
PyCFunction method(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f)); }

PyMethodDef methods[] = {
    {"set_functions", method(set_functions), METH_FASTCALL, "addresses of sp_page_tables, sp_qk_norm_rope, sp_tree_attn, sp_cache_keep, and of the last three's _q4 forms and sp_cache_read_q4"},
    {"page_tables", method(page_tables), METH_FASTCALL, "status code of sp_page_tables"},
    {"qk_norm_rope", method(qk_norm_rope), METH_FASTCALL, "status code of sp_qk_norm_rope"},
    {"tree_attn", method(tree_attn), METH_FASTCALL, "status code of sp_tree_attn"},
    {"cache_keep", method(cache_keep), METH_FASTCALL, "status code of sp_cache_keep"},
    {"qk_norm_rope_q4", method(qk_norm_rope_q4), METH_FASTCALL, "status code of sp_qk_norm_rope_q4"},
    {"tree_attn_q4", method(tree_attn_q4), METH_FASTCALL, "status code of sp_tree_attn_q4"},
    {"cache_keep_q4", method(cache_keep_q4), METH_FASTCALL, "status code of sp_cache_keep_q4"},
    {"cache_read_q4", method(cache_read_q4), METH_FASTCALL, "status code of sp_cache_read_q4"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_decode_calls", "Decode-side calls of the SharePrefill library on torch tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__decode_calls() { return PyModule_Create(&module); }
