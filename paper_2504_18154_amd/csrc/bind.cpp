// The marshalling of the hot calls' arguments (binding.py) in C++: tensors to addresses, sizes and row strides, the current
// stream's handle, and the call of the C ABI without the interpreter's lock.  Every function returns the call's status, or -1 for
// arguments that it does not take (anything but tensors or None, and integers of 32 bits): binding.py then goes the way through ctypes, which
// decides what such arguments mean and raises what is to be raised.
//
// Why: a call on a small batch keeps the GPU busy for 4 to 8 us, and the way through ctypes took the host 5.3 to 5.9 before the
// launch, of which 2 to 3 were a method call into the tensor per address and dimension; here it is 0.8 to 1.  Launches included, the
// host takes 64 us for 16 decode calls on one sequence (111 before; the device 131), 134 us for 16 times append and prefill of one short
// prompt (185 before), about as long as the device (132 replayed from a graph): 188 -> 132 to 147 us back to back.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <limits>

#include "../../include/ecoserve.h"

namespace {

// The entry points, as the library that binding.py has loaded holds them.
struct Entries {
  decltype(&ecoserve_kv_append_strided) append;
  decltype(&ecoserve_attn_prefill_strided) prefill;
  decltype(&ecoserve_attn_decode_strided) decode;
  decltype(&ecoserve_attn_decode_append) decode_append;
  decltype(&ecoserve_attn_decode_noalloc) noalloc;
} entry;
struct SparseEntries {
  decltype(&ecoserve_kv_append_rope) rope;
  decltype(&ecoserve_kv_summary) summary;
  decltype(&ecoserve_select_workspace_bytes) select_bytes;
  decltype(&ecoserve_block_select) select;
  decltype(&ecoserve_sparse_workspace_bytes) sparse_bytes;
  decltype(&ecoserve_attn_sparse) sparse;
} more;

// Reads the arguments of a call.  What is binding.py's business is noted, and not thrown: an exception takes 2.5 us, half of what the
// other way takes for such a call.
struct Arguments {
  PyObject* const* a;
  bool taken = true;

  const at::Tensor* tensor(int i) {
    if (THPVariable_CheckExact(a[i])) return &THPVariable_Unpack(a[i]);
    taken = false;
    return nullptr;
  }
  void* address(int i) {
    if (a[i] == Py_None) return nullptr;
    const at::Tensor* const t = tensor(i);
    return t ? t->data_ptr() : nullptr;
  }
  template <typename T>
  T* as(int i) {
    return static_cast<T*>(address(i));
  }
  int32_t narrow(int64_t n) {
    if (n < std::numeric_limits<int32_t>::min() || n > std::numeric_limits<int32_t>::max()) taken = false;
    return (int32_t)n;
  }
  int64_t integer(int i) {
    if (!PyLong_CheckExact(a[i])) return taken = false;
    int overflow = 0;
    const long long n = PyLong_AsLongLongAndOverflow(a[i], &overflow);
    if (overflow) taken = false;
    return n;
  }
  int32_t narrow_integer(int i) { return narrow(integer(i)); }
  void* handle(int i) { return reinterpret_cast<void*>((uintptr_t)integer(i)); }
  int32_t size(int i, int64_t d) {
    const at::Tensor* const t = tensor(i);
    if (t && t->dim() > d) return narrow(t->size(d));
    return taken = false;
  }
  int32_t numel(int i) {
    const at::Tensor* const t = tensor(i);
    return t ? narrow(t->numel()) : 0;
  }
  // Elements between consecutive tokens of a [tokens, heads, D] tensor or view whose heads are contiguous.
  int64_t row_stride(int i) {
    const at::Tensor* const t = tensor(i);
    if (!t || t->dim() != 3 || t->stride(2) != 1 || t->stride(1) != t->size(2)) return taken = false;
    return t->size(0) > 1 ? t->stride(0) : t->size(1) * t->size(2);
  }
  int32_t or_all(int i, int32_t all) { return a[i] == Py_None ? all : narrow_integer(i); }
};

// Runs f on `want` arguments; -1: not taken.
template <typename F>
PyObject* guarded(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F f) {
  int status = -1;
  try {
    Arguments in{a};
    if (n == want) status = f(in);
  } catch (...) {  // (what torch throws for a tensor without storage: the other way raises it again, for the caller)
    status = -1;
  }
  return PyLong_FromLong(status);
}
// The call itself on the current stream, without the interpreter's lock, if all its arguments are taken.
template <typename F>
int unlocked(const Arguments& in, F f) {
  if (!in.taken) return -1;
  void* const s = c10::hip::getCurrentHIPStream().stream();
  struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
  } scope;
  return f(s);
}

// (handle, k_cache, v_cache, k_new, v_new, cu_q, ctx_before, block_table, max_new_len, row stride of a packed array or 0: the tensors')
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 10, [](Arguments& in) {
    auto* const c = static_cast<ecoserve_ctx*>(in.handle(0));
    void *const kc = in.address(1), *const vc = in.address(2), *const kn = in.address(3), *const vn = in.address(4);
    const auto *cu = in.as<const int32_t>(5), *before = in.as<const int32_t>(6), *table = in.as<const int32_t>(7);
    const int32_t B = in.numel(6), T = in.size(3, 0), width = in.size(7, 1), most = in.or_all(8, T);
    int64_t stride = in.integer(9);
    if (stride == 0) {
      stride = in.row_stride(3);
      if (stride != in.row_stride(4)) in.taken = false;
    }
    return unlocked(in, [&](void* s) { return entry.append(c, kc, vc, kn, vn, stride, cu, before, table, width, B, T, most, s); });
  });
}

// (handle, q, k_cache, v_cache, cu_q, ctx_before, block_table, out, lse, max_q_len, row stride of a packed array or 0: the tensor's)
PyObject* attn_prefill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 11, [](Arguments& in) {
    auto* const c = static_cast<ecoserve_ctx*>(in.handle(0));
    void *const q = in.address(1), *const kc = in.address(2), *const vc = in.address(3), *const out = in.address(7);
    const auto *cu = in.as<const int32_t>(4), *before = in.as<const int32_t>(5), *table = in.as<const int32_t>(6);
    auto* const lse = in.as<float>(8);
    const int32_t B = in.numel(5), T = in.size(1, 0), width = in.size(6, 1), most = in.or_all(9, T);
    const int64_t packed = in.integer(10), stride = packed ? packed : in.row_stride(1);
    return unlocked(in, [&](void* s) { return entry.prefill(c, q, stride, kc, vc, cu, before, table, width, out, lse, B, T, most, s); });
  });
}

// (handle, q, k_cache, v_cache, block_table, ctx_len, out, max_ctx_len, lse, row stride of a packed array or 0: the tensor's)
PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 10, [](Arguments& in) {
    auto* const c = static_cast<ecoserve_ctx*>(in.handle(0));
    void *const q = in.address(1), *const kc = in.address(2), *const vc = in.address(3), *const out = in.address(6);
    const auto *table = in.as<const int32_t>(4), *len = in.as<const int32_t>(5);
    auto* const lse = in.as<float>(8);
    const int32_t B = in.numel(5), width = in.size(4, 1), most = in.narrow_integer(7);
    const int64_t packed = in.integer(9), stride = packed ? packed : in.row_stride(1);
    return unlocked(in, [&](void* s) { return entry.decode(c, q, stride, kc, vc, table, width, len, out, lse, B, most, s); });
  });
}

// (handle, q, k_new, v_new, k_cache, v_cache, block_table, ctx_len, out, max_ctx_len, lse)
PyObject* attn_decode_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 11, [](Arguments& in) {
    auto* const c = static_cast<ecoserve_ctx*>(in.handle(0));
    const int64_t stride = in.row_stride(1), fresh = in.row_stride(2);
    if (fresh != in.row_stride(3)) in.taken = false;
    void *const q = in.address(1), *const kn = in.address(2), *const vn = in.address(3), *const kc = in.address(4), *const vc = in.address(5), *const out = in.address(8);
    const auto *table = in.as<const int32_t>(6), *len = in.as<const int32_t>(7);
    auto* const lse = in.as<float>(10);
    const int32_t B = in.numel(7), width = in.size(6, 1), most = in.narrow_integer(9);
    return unlocked(in, [&](void* s) { return entry.decode_append(c, q, stride, kn, vn, fresh, kc, vc, table, width, len, out, lse, B, most, s); });
  });
}

// (device, address of the layout, q, k_cache, v_cache, block_table, ctx_len, out, max_ctx_len, lse)
PyObject* attn_decode_noalloc(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(a, n, 10, [](Arguments& in) {
    const int32_t device = in.narrow_integer(0);
    const auto* const layout = static_cast<const ecoserve_layout*>(in.handle(1));
    void *const q = in.address(2), *const kc = in.address(3), *const vc = in.address(4), *const out = in.address(7);
    const auto *table = in.as<const int32_t>(5), *len = in.as<const int32_t>(6);
    auto* const lse = in.as<float>(9);
    const int32_t B = in.numel(6), width = in.size(5, 1), most = in.narrow_integer(8);
    return unlocked(in, [&](void* s) { return entry.noalloc(device, layout, q, kc, vc, table, width, len, out, lse, B, most, s); });
  });
}

// The calls below look at what they are given (binding.py raises for what is not taken): tensors of the context's GPU, of its types and
// sizes.  `l`: the context's layout, `device` its GPU.
struct LayerArguments : Arguments {
  const ecoserve_layout* l;
  int device;
  const at::Tensor* here(int i, at::ScalarType type) {
    const at::Tensor* const t = tensor(i);
    if (t && t->is_cuda() && t->get_device() == device && t->scalar_type() == type) return t;
    taken = false;
    return nullptr;
  }
  at::ScalarType element() const { return l->dtype == ECOSERVE_BF16 ? at::kBFloat16 : at::kFloat; }
  // [tokens, heads, D], heads contiguous: address, and the distance of the tokens
  struct Rows {
    void* at = nullptr;
    int64_t stride = 0;
  };
  Rows rows(int i, int64_t tokens, int32_t heads) {
    const at::Tensor* const t = here(i, element());
    if (!t || t->dim() != 3 || t->size(0) != tokens || t->size(1) != heads || t->size(2) != l->head_dim) return taken = false, Rows();
    return {t->data_ptr(), row_stride(i)};
  }
  // contiguous and at least so long
  void* whole(int i, at::ScalarType type, int64_t least) {
    const at::Tensor* const t = here(i, type);
    if (!t || !t->is_contiguous() || t->numel() < least) return taken = false, nullptr;
    return t->data_ptr();
  }
  const int32_t* ints(int i, int64_t least) { return static_cast<const int32_t*>(whole(i, at::kInt, least)); }
  const int32_t* table(int i, int64_t sequences) {
    const at::Tensor* const t = here(i, at::kInt);
    if (!t || t->dim() != 2 || t->size(0) < sequences) taken = false;
    return ints(i, 0);
  }
  int64_t side(int sides) const { return (int64_t)l->num_blocks * l->num_kv_heads * sides; }
  void* pool(int i) { return whole(i, element(), side(16) * l->head_dim); }
  void* summaries(int i) { return whole(i, at::kChar, side(2 * ((l->head_dim + 31) / 32 * 32) + 1)); }
  // [tokens, K/V heads, entries]
  int32_t* lists(int i, int64_t tokens, int32_t& entries) {
    const at::Tensor* const t = here(i, at::kInt);
    if (!t || t->dim() != 3 || t->size(0) != tokens || t->size(1) != l->num_kv_heads || !t->is_contiguous()) return taken = false, nullptr;
    entries = narrow(t->size(2));
    return static_cast<int32_t*>(t->data_ptr());
  }
  // the caller's workspace, or one of torch's allocator, which gives it to nobody else on this stream before the call's kernels are through
  struct Space {
    void* at;
    size_t bytes;
    at::Tensor held;
  };
  Space space(int i, size_t need) {
    if (a[i] == Py_None) {
      if (!need || !taken) return {nullptr, 0, {}};
      at::Tensor t = at::empty({(int64_t)need}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, device));
      return {t.data_ptr(), need, t};
    }
    const at::Tensor* const t = tensor(i);
    if (!t || !t->is_cuda() || t->get_device() != device || !t->is_contiguous()) return taken = false, Space{nullptr, 0, {}};
    return {t->data_ptr(), (size_t)t->nbytes(), {}};
  }
  template <typename F>
  int call(F f) {
    if (!taken) return -1;
    void* const s = c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream();
    struct Unlocked {
      PyThreadState* const state = PyEval_SaveThread();
      ~Unlocked() { PyEval_RestoreThread(state); }
    } scope;
    return f(s);
  }
};
template <typename F>
PyObject* guarded_layer(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F f) {
  return guarded(a, n, want, [&](Arguments& plain) {
    LayerArguments in{plain};
    auto* const c = static_cast<ecoserve_ctx*>(in.handle(0));
    in.l = static_cast<const ecoserve_layout*>(in.handle(1));
    in.device = in.narrow_integer(2);
    return in.taken && in.l ? f(in, c) : -1;
  });
}

// (handle, address of the layout, device, address of the rope, inv_freq, k_cache, v_cache, k_new, v_new, cu_q, ctx_before, block_table, positions, q, q_out, max_new_len)
PyObject* kv_append_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_layer(a, n, 16, [](LayerArguments& in, ecoserve_ctx* c) {
    const auto* const rope = static_cast<const ecoserve_rope*>(in.handle(3));
    if (!in.taken || !rope) return -1;
    const int32_t T = in.size(7, 0), B = in.numel(10), width = in.size(11, 1), most = in.or_all(15, T);
    const auto* const freq = static_cast<const double*>(in.whole(4, at::kDouble, rope->rotary_dim / 2));
    void *const kc = in.pool(5), *const vc = in.pool(6);
    const auto kn = in.rows(7, T, in.l->num_kv_heads), vn = in.rows(8, T, in.l->num_kv_heads);
    if (kn.stride != vn.stride) in.taken = false;
    const int32_t *const cu = in.ints(9, (int64_t)B + 1), *const before = in.ints(10, B), *const table = in.table(11, B);
    const int32_t* positions = nullptr;
    if (in.a[12] != Py_None) {
      positions = in.ints(12, (int64_t)rope->num_axes * T);
      if (in.size(12, 0) != rope->num_axes || in.size(12, 1) != T) in.taken = false;
    }
    LayerArguments::Rows q, qo;
    if ((in.a[13] == Py_None) != (in.a[14] == Py_None)) in.taken = false;
    if (in.taken && in.a[13] != Py_None) q = in.rows(13, T, in.l->num_q_heads), qo = in.rows(14, T, in.l->num_q_heads);
    return in.call([&](void* s) { return more.rope(c, rope, freq, positions, q.at, q.stride, qo.at, qo.stride, kc, vc, kn.at, vn.at, kn.stride, cu, before, table, width, B, T, most, s); });
  });
}

// (handle, address of the layout, device, k_cache, summary, cu_q, ctx_before, block_table, T, max_new_len)
PyObject* kv_summary(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_layer(a, n, 10, [](LayerArguments& in, ecoserve_ctx* c) {
    void *const kc = in.pool(3), *const summary = in.summaries(4);
    const int32_t B = in.numel(6), width = in.size(7, 1), T = in.narrow_integer(8), most = in.or_all(9, T);
    const int32_t *const cu = in.ints(5, (int64_t)B + 1), *const before = in.ints(6, B), *const table = in.table(7, B);
    return in.call([&](void* s) { return more.summary(c, kc, summary, cu, before, table, width, B, T, most, s); });
  });
}

// (handle, address of the layout, device, q, summary, ctx_before, block_table, blocks, max_ctx_len, keep_first, keep_last, cu_q, workspace)
PyObject* block_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_layer(a, n, 13, [](LayerArguments& in, ecoserve_ctx* c) {
    const int32_t T = in.size(3, 0), B = in.numel(5), width = in.size(6, 1), most = in.narrow_integer(8), first = in.narrow_integer(9), last = in.narrow_integer(10);
    const auto q = in.rows(3, T, in.l->num_q_heads);
    const void* const summary = in.summaries(4);
    const int32_t *const before = in.ints(5, B), *const table = in.table(6, B), *const cu = in.a[11] == Py_None ? nullptr : in.ints(11, (int64_t)B + 1);
    int32_t entries = 0;
    int32_t* const lists = in.lists(7, T, entries);
    const auto ws = in.space(12, in.taken ? more.select_bytes(in.l, T, most) : 0);
    return in.call([&](void* s) { return more.select(c, q.at, q.stride, summary, cu, before, table, width, lists, entries, first, last, B, T, most, ws.at, ws.bytes, s); });
  });
}

// (handle, address of the layout, device, q, k_cache, v_cache, ctx_before, block_table, blocks, out, lse, cu_q, workspace)
PyObject* attn_sparse(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded_layer(a, n, 13, [](LayerArguments& in, ecoserve_ctx* c) {
    const int32_t T = in.size(3, 0), B = in.numel(6), width = in.size(7, 1);
    const auto q = in.rows(3, T, in.l->num_q_heads);
    void *const kc = in.pool(4), *const vc = in.pool(5);
    const int32_t *const before = in.ints(6, B), *const table = in.table(7, B), *const cu = in.a[11] == Py_None ? nullptr : in.ints(11, (int64_t)B + 1);
    int32_t entries = 0;
    const int32_t* const lists = in.lists(8, T, entries);
    const int64_t heads = (int64_t)T * in.l->num_q_heads;
    void* const out = in.whole(9, in.element(), heads * in.l->head_dim);
    float* const lse = in.a[10] == Py_None ? nullptr : static_cast<float*>(in.whole(10, at::kFloat, heads));
    const auto ws = in.space(12, in.taken ? more.sparse_bytes(c, T, entries) : 0);
    return in.call([&](void* s) { return more.sparse(c, q.at, q.stride, kc, vc, cu, before, table, width, lists, entries, out, lse, B, T, ws.at, ws.bytes, s); });
  });
}

// (addresses of the entry points, in the order of SparseEntries)
PyObject* bind_sparse(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* at[6];
  if (n != 6) {
    PyErr_SetString(PyExc_TypeError, "bind_sparse() takes six addresses");
    return nullptr;
  }
  for (int i = 0; i < 6; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (!at[i] && PyErr_Occurred()) return nullptr;
  }
  more.rope = reinterpret_cast<decltype(more.rope)>(at[0]);
  more.summary = reinterpret_cast<decltype(more.summary)>(at[1]);
  more.select_bytes = reinterpret_cast<decltype(more.select_bytes)>(at[2]);
  more.select = reinterpret_cast<decltype(more.select)>(at[3]);
  more.sparse_bytes = reinterpret_cast<decltype(more.sparse_bytes)>(at[4]);
  more.sparse = reinterpret_cast<decltype(more.sparse)>(at[5]);
  Py_RETURN_NONE;
}

// (addresses of the entry points, in the order of Entries)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* at[5];
  if (n != 5) {
    PyErr_SetString(PyExc_TypeError, "bind() takes five addresses");
    return nullptr;
  }
  for (int i = 0; i < 5; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (!at[i] && PyErr_Occurred()) return nullptr;
  }
  entry.append = reinterpret_cast<decltype(entry.append)>(at[0]);
  entry.prefill = reinterpret_cast<decltype(entry.prefill)>(at[1]);
  entry.decode = reinterpret_cast<decltype(entry.decode)>(at[2]);
  entry.decode_append = reinterpret_cast<decltype(entry.decode_append)>(at[3]);
  entry.noalloc = reinterpret_cast<decltype(entry.noalloc)>(at[4]);
  Py_RETURN_NONE;
}

#define ECO_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ECO_FAST(bind), ECO_FAST(kv_append), ECO_FAST(attn_prefill), ECO_FAST(attn_decode), ECO_FAST(attn_decode_append),
                         ECO_FAST(attn_decode_noalloc),
                         ECO_FAST(bind_sparse), ECO_FAST(kv_append_rope), ECO_FAST(kv_summary), ECO_FAST(block_select), ECO_FAST(attn_sparse), {nullptr, nullptr, 0, nullptr}};
// (ECO_BIND_FITS: the interpreter and the torch that this is compiled for; build.py looks for it in the built file)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", "Marshalling of the hot calls' arguments, " ECO_BIND_FITS, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind() { return PyModule_Create(&module); }
