// The calls of binding.py that a serving loop makes for every step, as a CPython module: the
// arguments are read from the tensors, results and workspaces allocated and the C ABI called
// without going through Python objects for each of them. Marshalling a small call in Python
// (ctypes, torch.empty, torch.cuda.current_stream) took 6 to 13 us, two to four times as long
// as issuing its kernels; here it is about 1 us.
//
// The library itself is loaded by binding.py, which hands over the addresses of its functions.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cp_attn.h"

namespace {

struct Functions {
  decltype(&cp_workspace_bytes) workspace_bytes;
  decltype(&cp_attn_partial) partial;
  decltype(&cp_attn_decode) decode;
  decltype(&cp_attn_decode_static) decode_static;
  decltype(&cp_attn_merge) merge;
  decltype(&cp_kv_append) append;
  decltype(&cp_ring_passkv) ring[3];  // pass-KV, pass-Q, pass-Q decode
} fn = {};

struct CacheFunctions {
  decltype(&cp_tree_attn) tree_attn;
  decltype(&cp_tree_accept) tree_accept;
  decltype(&cp_kv_attn_weight) weight;
  decltype(&cp_kv_evict) evict;
} cache_fn = {};

PyObject* get_device = nullptr;      // torch._C._cuda_getDevice
PyObject* get_raw_stream = nullptr;  // torch._C._cuda_getCurrentRawStream

struct Raised {};  // a Python error is set

[[noreturn]] void raise(PyObject* type, const char* what) {
  PyErr_SetString(type, what);
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch tensor");
  return THPVariable_Unpack(o);
}
void* pointer(const at::Tensor& t) {
  if (!t.is_contiguous())
    raise(PyExc_AssertionError, "tensors handed to the C ABI must be contiguous");
  return const_cast<void*>(t.const_data_ptr());
}
void* pointer(PyObject* o) { return o == Py_None ? nullptr : pointer(tensor(o)); }

int32_t dtype_code(at::ScalarType t) {
  if (t == at::kBFloat16) return CP_BF16;
  if (t == at::kFloat) return CP_FP32;
  PyErr_Format(PyExc_TypeError, "unsupported dtype %s", at::toString(t));
  throw Raised{};
}
at::ScalarType dtype_or(PyObject* o, at::ScalarType other) {
  if (o == Py_None) return other;
  if (!THPDtype_Check(o)) raise(PyExc_TypeError, "out_dtype must be a torch dtype");
  return reinterpret_cast<THPDtype*>(o)->scalar_type;
}
float number(PyObject* o) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Raised{};
  return (float)x;
}

// A raw stream given as a number, or torch's current one.
void* stream_of(PyObject* o) {
  if (o != Py_None) {
    void* const s = PyLong_AsVoidPtr(o);
    if (s == nullptr && PyErr_Occurred()) throw Raised{};
    return s;
  }
  PyObject* const dev = PyObject_CallNoArgs(get_device);
  if (dev == nullptr) throw Raised{};
  PyObject* const raw = PyObject_CallOneArg(get_raw_stream, dev);
  Py_DECREF(dev);
  if (raw == nullptr) throw Raised{};
  void* const s = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  if (s == nullptr && PyErr_Occurred()) throw Raised{};
  return s;
}

struct Workspace {
  at::Tensor own;
  void* ptr = nullptr;
  size_t bytes = 0;
  void set(const at::Tensor& t) {
    const uintptr_t p = (uintptr_t)t.const_data_ptr(), a = (p + 255) & ~(uintptr_t)255;
    const int64_t left = t.numel() - (int64_t)(a - p);
    ptr = (void*)a;
    bytes = left > 0 ? (size_t)left : 0;   // (one that ends in front of its first aligned byte holds nothing)
  }
};
void use_workspace(Workspace& w, PyObject* given, const cp_shape& s, int32_t kind,
                   const at::Tensor& like) {
  if (given != Py_None) {
    w.set(tensor(given));
    return;
  }
  const size_t need = fn.workspace_bytes(&s, kind);
  if (need == 0) return;
  w.own = at::empty({(int64_t)need + 256}, like.options().dtype(at::kByte));
  w.set(w.own);
}

cp_shape rows_shape(const at::Tensor& q, const at::Tensor& k, int64_t batch, float scale,
                    int32_t flags) {
  if (q.dim() != 3 || k.dim() != 3) raise(PyExc_ValueError, "q and k must have three dimensions");
  cp_shape s = {};
  s.dtype = dtype_code(q.scalar_type());
  s.head_dim = (int32_t)q.size(2);
  s.n_q_heads = (int32_t)q.size(1);
  s.n_kv_heads = (int32_t)k.size(1);
  s.batch = (int32_t)batch;
  s.flags = flags;
  s.total_q = q.size(0);
  s.total_kv = k.size(0);
  s.softmax_scale = scale;
  return s;
}

// `given`, or a new tensor.
at::Tensor result(PyObject* given, at::IntArrayRef sizes, const at::Tensor& like,
                  at::ScalarType dtype) {
  return given != Py_None ? tensor(given) : at::empty(sizes, like.options().dtype(dtype));
}
PyObject* object(PyObject* given, const at::Tensor& t) {
  if (given == Py_None) return THPVariable_Wrap(t);
  Py_INCREF(given);
  return given;
}
PyObject* pair(PyObject* a, PyObject* b) {
  if (a == nullptr || b == nullptr) {
    Py_XDECREF(a);
    Py_XDECREF(b);
    return nullptr;
  }
  PyObject* const t = PyTuple_Pack(2, a, b);
  Py_DECREF(a);
  Py_DECREF(b);
  return t;
}
PyObject* status(int rc) { return PyLong_FromLong(rc); }

// Other threads run while the library is called, as they do in a ctypes call: a launch blocks
// once the stream's queue is full. The tensors are the caller's arguments or held on the stack.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F, typename... A>
int call(F f, A... args) {
  const Unlocked u;
  return f(args...);
}

void arguments(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) raise(PyExc_TypeError, "wrong number of arguments");
  if (fn.decode == nullptr) raise(PyExc_RuntimeError, "the library is not loaded");
}

// Every function returns its result, or the (nonzero) status of the C call as a number.
template <typename F>
PyObject* guarded(F f) {
  try {
    return f();
  } catch (const Raised&) {
    return nullptr;
  } catch (const std::exception& e) {   // of torch: out of memory, no device
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// q, k, v, q_pos, kv_pos, cu_seqlens_q, cu_seqlens_kv, out_dtype, scale, out, lse, workspace, stream
PyObject* partial(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    arguments(n, 13);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
    const int64_t batch = a[5] == Py_None ? 1 : tensor(a[5]).numel() - 1;
    const cp_shape s = rows_shape(q, k, batch, number(a[8]), 0);
    const at::Tensor out = result(a[9], q.sizes(), q, dtype_or(a[7], q.scalar_type()));
    const at::Tensor lse = result(a[10], {q.size(0), q.size(1)}, q, at::kFloat);
    Workspace w;
    use_workspace(w, a[11], s, CP_WS_PARTIAL, q);
    const int rc = call(fn.partial, &s, pointer(q), pointer(k), pointer(a[2]), (int32_t*)pointer(a[3]),
                              (int32_t*)pointer(a[4]), (int32_t*)pointer(a[5]),
                              (int32_t*)pointer(a[6]), pointer(out), (float*)pointer(lse),
                              dtype_code(out.scalar_type()), w.ptr, w.bytes, stream_of(a[12]));
    return rc != CP_OK ? status(rc) : pair(object(a[9], out), object(a[10], lse));
  });
}

// q, k, v, q_pos, kv_pos, cu_seqlens_kv, bid, out_dtype, scale, out, lse, workspace, stream, unique
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    arguments(n, 14);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
    const int unique = PyObject_IsTrue(a[13]);
    if (unique < 0) throw Raised{};
    const cp_shape s = rows_shape(q, k, tensor(a[5]).numel() - 1, number(a[8]),
                                  unique ? CP_SHAPE_UNIQUE_BID : 0);
    const at::Tensor out = result(a[9], q.sizes(), q, dtype_or(a[7], q.scalar_type()));
    const at::Tensor lse = result(a[10], {q.size(0), q.size(1)}, q, at::kFloat);
    Workspace w;
    use_workspace(w, a[11], s, CP_WS_DECODE, q);
    const int rc = call(fn.decode, &s, pointer(q), pointer(k), pointer(a[2]), (int32_t*)pointer(a[3]),
                             (int32_t*)pointer(a[4]), (int32_t*)pointer(a[5]),
                             (int32_t*)pointer(a[6]), pointer(out), (float*)pointer(lse),
                             dtype_code(out.scalar_type()), w.ptr, w.bytes, stream_of(a[12]));
    return rc != CP_OK ? status(rc) : pair(object(a[9], out), object(a[10], lse));
  });
}

// q, k, v, q_pos, kv_pos, cu_seqlens_kv, bid, out, lse, scale, stream, unique
PyObject* decode_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    arguments(n, 12);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &out = tensor(a[7]);
    const int unique = PyObject_IsTrue(a[11]);
    if (unique < 0) throw Raised{};
    const cp_shape s = rows_shape(q, k, tensor(a[5]).numel() - 1, number(a[9]),
                                  unique ? CP_SHAPE_UNIQUE_BID : 0);
    return status(call(fn.decode_static, &s, pointer(q), pointer(k), pointer(a[2]),
                                   (int32_t*)pointer(a[3]), (int32_t*)pointer(a[4]),
                                   (int32_t*)pointer(a[5]), (int32_t*)pointer(a[6]), pointer(out),
                                   (float*)pointer(a[8]), dtype_code(out.scalar_type()),
                                   stream_of(a[10])));
  });
}

// outs, lses (sequences), out_dtype, out, lse_out, want_lse, stream
PyObject* merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
  PyObject *outs = nullptr, *lses = nullptr;
  PyObject* const r = guarded([&]() -> PyObject* {
    arguments(n, 7);
    outs = PySequence_Fast(a[0], "outs must be a sequence of tensors");
    if (outs == nullptr) throw Raised{};
    lses = PySequence_Fast(a[1], "lses must be a sequence of tensors");
    if (lses == nullptr) throw Raised{};
    const Py_ssize_t parts = PySequence_Fast_GET_SIZE(outs);
    if (parts == 0) raise(PyExc_IndexError, "list index out of range");
    if (PySequence_Fast_GET_SIZE(lses) != parts)
      raise(PyExc_IndexError, "outs and lses differ in length");
    const at::Tensor& o0 = tensor(PySequence_Fast_GET_ITEM(outs, 0));
    if (o0.dim() < 1) raise(PyExc_IndexError, "partial outputs need a channel dimension");
    const int64_t d = o0.size(-1), rows = d > 0 ? o0.numel() / d : 0;
    const at::Tensor out = result(a[3], o0.sizes(), o0, dtype_or(a[2], o0.scalar_type()));
    const int want = PyObject_IsTrue(a[5]);
    if (want < 0) throw Raised{};
    at::Tensor lse;
    if (a[4] != Py_None) lse = tensor(a[4]);
    else if (want) lse = at::empty(o0.sizes().slice(0, o0.dim() - 1), o0.options().dtype(at::kFloat));
    // (the C call rejects more than CP_MAX_PARTS before it reads the arrays)
    const void* op[CP_MAX_PARTS];
    const float* lp[CP_MAX_PARTS];
    for (Py_ssize_t i = 0; i < parts && i < CP_MAX_PARTS; ++i) {
      op[i] = pointer(PySequence_Fast_GET_ITEM(outs, i));
      lp[i] = (const float*)pointer(PySequence_Fast_GET_ITEM(lses, i));
    }
    const int rc = call(fn.merge, rows, (int32_t)d, (int32_t)parts, op, lp,
                            dtype_code(o0.scalar_type()), pointer(out),
                            dtype_code(out.scalar_type()),
                            lse.defined() ? (float*)pointer(lse) : nullptr, stream_of(a[6]));
    if (rc != CP_OK) return status(rc);
    PyObject* l;
    if (lse.defined()) {
      l = object(a[4], lse);
    } else {
      l = Py_None;
      Py_INCREF(l);
    }
    return pair(object(a[3], out), l);
  });
  Py_XDECREF(outs);
  Py_XDECREF(lses);
  return r;
}

// k_new, v_new, pos_new, cu_seqlens_new, k, v, kv_pos, cu, used, dropped (of the cache), slots,
// batch, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    arguments(n, 13);
    const at::Tensor &k = tensor(a[0]), &cache = tensor(a[4]);
    const int64_t slots = PyLong_AsLongLong(a[10]), batch = PyLong_AsLongLong(a[11]);
    if (PyErr_Occurred()) throw Raised{};
    if (k.dim() != 3) raise(PyExc_ValueError, "k_new must have three dimensions");
    if (k.scalar_type() != cache.scalar_type() || cache.size(1) != k.size(1) ||
        cache.size(2) != k.size(2))
      raise(PyExc_ValueError, "new K/V rows do not match the cache's row shape or dtype");
    if (tensor(a[3]).numel() != batch + 1 || tensor(a[2]).numel() != k.size(0))
      raise(PyExc_ValueError, "cu_seqlens_new / pos_new sizes do not match");
    cp_shape s = {};
    s.dtype = dtype_code(k.scalar_type());
    s.head_dim = (int32_t)k.size(2);
    s.n_q_heads = s.n_kv_heads = (int32_t)k.size(1);
    s.batch = (int32_t)batch;
    s.total_q = k.size(0);
    s.total_kv = slots;
    return status(call(fn.append, &s, pointer(k), pointer(a[1]), (int32_t*)pointer(a[2]),
                            (int32_t*)pointer(a[3]), pointer(cache), pointer(a[5]),
                            (int32_t*)pointer(a[6]), (int32_t*)pointer(a[7]),
                            (int32_t*)pointer(a[8]), (int32_t*)pointer(a[9]), stream_of(a[12])));
  });
}

// ---- calls on the KV cache: trees of drafted tokens, attention weight, eviction ----

void cache_arguments(Py_ssize_t n, Py_ssize_t want) {
  arguments(n, want);
  if (cache_fn.tree_attn == nullptr) raise(PyExc_RuntimeError, "the library is not loaded");
}
// What a tensor has to be; `numel` < 0: any number of elements.
const at::Tensor& checked(PyObject* o, at::ScalarType type, int64_t numel, const char* name) {
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != type) {
    PyErr_Format(PyExc_TypeError, "%s must be %s", name, at::toString(type));
    throw Raised{};
  }
  if (numel >= 0 && t.numel() != numel) {
    PyErr_Format(PyExc_ValueError, "%s has the wrong number of elements", name);
    throw Raised{};
  }
  return t;
}
int32_t* ints(PyObject* o, int64_t numel, const char* name) {
  return (int32_t*)pointer(checked(o, at::kInt, numel, name));
}
// All tensors of a call lie on the current GPU, whose stream the call is made on.
void on_current_device(PyObject* const* a, std::initializer_list<int> which) {
  PyObject* const dev = PyObject_CallNoArgs(get_device);
  if (dev == nullptr) throw Raised{};
  const long current = PyLong_AsLong(dev);
  Py_DECREF(dev);
  if (current == -1 && PyErr_Occurred()) throw Raised{};
  for (const int i : which) {
    if (a[i] == Py_None) continue;
    const at::Tensor& t = tensor(a[i]);
    if (!t.is_cuda() || t.get_device() != current)
      raise(PyExc_ValueError, "tensors must be on the current GPU");
  }
}
void same_rows(const at::Tensor& x, const at::Tensor& cache, const char* what) {
  if (x.dim() != 3) raise(PyExc_ValueError, what);
  if (x.scalar_type() != cache.scalar_type() || x.size(1) != cache.size(1) ||
      x.size(2) != cache.size(2))
    raise(PyExc_ValueError, what);
}
// K rows of a cache in a[i], V, positions, boundaries and counts behind it; the shape of a call on it.
cp_shape cache_shape(PyObject* const* a, int i) {
  const at::Tensor &k = tensor(a[i]), &cu = checked(a[i + 3], at::kInt, -1, "cu_seqlens_kv");
  if (k.dim() != 3) raise(PyExc_ValueError, "a cache's K must have three dimensions");
  same_rows(tensor(a[i + 1]), k, "K and V of the cache differ in shape or dtype");
  if (tensor(a[i + 1]).size(0) != k.size(0)) raise(PyExc_ValueError, "K and V of the cache differ in length");
  checked(a[i + 2], at::kInt, k.size(0), "kv_pos of the cache");
  checked(a[i + 4], at::kInt, cu.numel(), "used of the cache");
  cp_shape s = {};
  s.dtype = dtype_code(k.scalar_type());
  s.head_dim = (int32_t)k.size(2);
  s.n_q_heads = s.n_kv_heads = (int32_t)k.size(1);
  s.batch = (int32_t)cu.numel() - 1;
  s.total_kv = k.size(0);
  return s;
}
void queries(cp_shape& s, const at::Tensor& q, const at::Tensor& cache, float scale) {
  if (q.dim() != 3) raise(PyExc_ValueError, "q must have three dimensions");
  if (q.scalar_type() != cache.scalar_type() || q.size(2) != cache.size(2))
    raise(PyExc_ValueError, "q does not match the cache's head_dim or dtype");
  s.n_q_heads = (int32_t)q.size(1);
  s.total_q = q.size(0);
  s.softmax_scale = scale;
}
// Words of a node's mask.
int32_t mask_words(PyObject* o, int64_t nodes) {
  const at::Tensor& m = checked(o, at::kLong, -1, "tree_mask");
  if (m.dim() != 2 || m.size(0) != nodes)
    raise(PyExc_ValueError, "tree_mask must be [nodes, words] of int64");
  return (int32_t)m.size(1);
}

// q, q_pos, cu_seqlens_q, k_new, v_new, tree_mask, k, v, kv_pos, cu, used (of the cache), out_dtype,
// scale, out, lse, workspace, stream
PyObject* tree_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    cache_arguments(n, 17);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[6]);
    cp_shape s = cache_shape(a, 6);
    queries(s, q, k, number(a[12]));
    int32_t words = 0;
    if ((a[3] == Py_None) != (a[4] == Py_None) || (a[3] == Py_None) != (a[5] == Py_None))
      raise(PyExc_ValueError, "k_new, v_new and tree_mask come together");
    if (a[3] != Py_None) {
      for (int i = 3; i < 5; ++i) {
        same_rows(tensor(a[i]), k, "k_new / v_new do not match the cache's row shape or dtype");
        if (tensor(a[i]).size(0) != s.total_q) raise(PyExc_ValueError, "a row of k_new and v_new per node");
      }
      words = mask_words(a[5], s.total_q);
    }
    int32_t* const q_pos = ints(a[1], s.total_q, "q_pos");
    int32_t* const cu_q = ints(a[2], s.batch + 1, "cu_seqlens_q");
    if (a[13] != Py_None && tensor(a[13]).numel() != q.numel())
      raise(PyExc_ValueError, "out has the wrong number of elements");
    if (a[14] != Py_None) checked(a[14], at::kFloat, s.total_q * s.n_q_heads, "lse");
    on_current_device(a, {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 13, 14, 15});
    const at::Tensor out = result(a[13], q.sizes(), q, dtype_or(a[11], q.scalar_type()));
    const at::Tensor lse = result(a[14], {q.size(0), q.size(1)}, q, at::kFloat);
    Workspace w;
    use_workspace(w, a[15], s, CP_WS_TREE, q);
    const int rc = call(cache_fn.tree_attn, &s, pointer(q), q_pos, cu_q, pointer(a[3]), pointer(a[4]),
                        (const uint64_t*)pointer(a[5]), words, pointer(k), pointer(a[7]),
                        (int32_t*)pointer(a[8]), (int32_t*)pointer(a[9]), (int32_t*)pointer(a[10]),
                        pointer(out), (float*)pointer(lse), dtype_code(out.scalar_type()), w.ptr,
                        w.bytes, stream_of(a[16]));
    return rc != CP_OK ? status(rc) : pair(object(a[13], out), object(a[14], lse));
  });
}

// k_new, v_new, pos_new, cu_seqlens_new, tree_mask, accepted, k, v, kv_pos, cu, used, dropped (of the
// cache), stream
PyObject* tree_accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    cache_arguments(n, 13);
    const at::Tensor &k_new = tensor(a[0]), &k = tensor(a[6]);
    cp_shape s = cache_shape(a, 6);
    for (int i = 0; i < 2; ++i)
      same_rows(tensor(a[i]), k, "k_new / v_new do not match the cache's row shape or dtype");
    s.total_q = k_new.size(0);
    if (tensor(a[1]).size(0) != s.total_q) raise(PyExc_ValueError, "a row of k_new and v_new per node");
    const int32_t words = mask_words(a[4], s.total_q);
    int32_t* const pos = ints(a[2], s.total_q, "pos_new");
    int32_t* const cu = ints(a[3], s.batch + 1, "cu_seqlens_new");
    int32_t* const accepted = ints(a[5], s.batch, "accepted");
    int32_t* const dropped = ints(a[11], 1, "dropped");
    on_current_device(a, {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11});
    return status(call(cache_fn.tree_accept, &s, pointer(k_new), pointer(a[1]), pos, cu,
                       (const uint64_t*)pointer(a[4]), words, accepted, pointer(k), pointer(a[7]),
                       (int32_t*)pointer(a[8]), (int32_t*)pointer(a[9]), (int32_t*)pointer(a[10]),
                       dropped, stream_of(a[12])));
  });
}

// q, q_pos, cu_seqlens_q, lse, weight, k, v, kv_pos, cu, used (of the cache), decay, scale, workspace,
// stream
PyObject* kv_weight(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    cache_arguments(n, 14);
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[5]);
    cp_shape s = cache_shape(a, 5);
    queries(s, q, k, number(a[11]));
    const float decay = number(a[10]);
    int32_t* const q_pos = ints(a[1], s.total_q, "q_pos");
    int32_t* const cu_q = ints(a[2], s.batch + 1, "cu_seqlens_q");
    const at::Tensor& lse = checked(a[3], at::kFloat, s.total_q * s.n_q_heads, "lse");
    const at::Tensor& weight = checked(a[4], at::kFloat, s.total_kv, "weight");
    on_current_device(a, {0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 12});
    Workspace w;
    use_workspace(w, a[12], s, CP_WS_WEIGHT, q);
    return status(call(cache_fn.weight, &s, pointer(q), q_pos, cu_q, (float*)pointer(lse), pointer(k),
                       (int32_t*)pointer(a[7]), (int32_t*)pointer(a[8]), (int32_t*)pointer(a[9]), decay,
                       (float*)pointer(weight), w.ptr, w.bytes, stream_of(a[13])));
  });
}

// k, v, kv_pos, cu, used (of the cache), weight, budget, protect_from, sinks, the same six of the
// destination or None, workspace, stream
PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    cache_arguments(n, 17);
    const at::Tensor& k = tensor(a[0]);
    const cp_shape s = cache_shape(a, 0);
    const at::Tensor& weight = checked(a[5], at::kFloat, s.total_kv, "weight");
    int32_t* const budget = ints(a[6], s.batch, "budget");
    int32_t* const protect = a[7] == Py_None ? nullptr : ints(a[7], s.batch, "protect_from");
    const long sinks = PyLong_AsLong(a[8]);
    if (sinks == -1 && PyErr_Occurred()) throw Raised{};
    if (sinks < 0 || sinks > INT32_MAX) raise(PyExc_ValueError, "sinks must be a count of positions");
    int64_t slots_to = 0;
    if (a[9] != Py_None) {
      const cp_shape d = cache_shape(a, 9);
      same_rows(tensor(a[9]), k, "the caches differ in row shape or dtype");
      if (d.batch != s.batch) raise(PyExc_ValueError, "the caches differ in their number of sequences");
      checked(a[14], at::kFloat, d.total_kv, "into_weight");
      slots_to = d.total_kv;
    }
    on_current_device(a, {0, 1, 2, 3, 4, 5, 6, 7, 9, 10, 11, 12, 13, 14, 15});
    Workspace w;
    use_workspace(w, a[15], s, CP_WS_EVICT, k);
    return status(call(cache_fn.evict, &s, pointer(k), pointer(a[1]), (int32_t*)pointer(a[2]),
                       (float*)pointer(weight), (int32_t*)pointer(a[3]), (int32_t*)pointer(a[4]), budget,
                       protect, (int32_t)sinks, pointer(a[9]), pointer(a[10]), (int32_t*)pointer(a[11]),
                       (float*)pointer(a[14]), (int32_t*)pointer(a[12]), (int32_t*)pointer(a[13]),
                       slots_to, w.ptr, w.bytes, stream_of(a[16])));
  });
}

// which driver, address of a cp_ring_desc, stream
PyObject* ring(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> PyObject* {
    arguments(n, 3);
    const long which = PyLong_AsLong(a[0]);
    if (which < 0 || which > 2) raise(PyExc_ValueError, "no such ring driver");
    void* const desc = PyLong_AsVoidPtr(a[1]);
    if (PyErr_Occurred()) throw Raised{};
    return status(call(fn.ring[which], (const cp_ring_desc*)desc, stream_of(a[2])));
  });
}

// addresses of cp_workspace_bytes, cp_attn_partial, cp_attn_decode, cp_attn_decode_static,
// cp_attn_merge, cp_kv_append, cp_ring_passkv, cp_ring_passq, cp_ring_passq_decode
PyObject* connect(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 9) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  void* p[9];
  for (int i = 0; i < 9; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a function is missing");
      return nullptr;
    }
  }
  if (get_device == nullptr) {
    PyObject* const m = PyImport_ImportModule("torch._C");
    if (m == nullptr) return nullptr;
    get_device = PyObject_GetAttrString(m, "_cuda_getDevice");
    get_raw_stream = PyObject_GetAttrString(m, "_cuda_getCurrentRawStream");
    Py_DECREF(m);
    if (get_device == nullptr || get_raw_stream == nullptr) {
      Py_CLEAR(get_device);
      Py_CLEAR(get_raw_stream);
      return nullptr;
    }
  }
  fn.workspace_bytes = (decltype(fn.workspace_bytes))p[0];
  fn.partial = (decltype(fn.partial))p[1];
  fn.decode = (decltype(fn.decode))p[2];
  fn.decode_static = (decltype(fn.decode_static))p[3];
  fn.merge = (decltype(fn.merge))p[4];
  fn.append = (decltype(fn.append))p[5];
  for (int i = 0; i < 3; ++i) fn.ring[i] = (decltype(fn.ring[0]))p[6 + i];
  Py_RETURN_NONE;
}

// addresses of cp_tree_attn, cp_tree_accept, cp_kv_attn_weight, cp_kv_evict
PyObject* connect_cache(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  void* p[4];
  for (int i = 0; i < 4; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (p[i] == nullptr) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a function is missing");
      return nullptr;
    }
  }
  cache_fn.tree_attn = (decltype(cache_fn.tree_attn))p[0];
  cache_fn.tree_accept = (decltype(cache_fn.tree_accept))p[1];
  cache_fn.weight = (decltype(cache_fn.weight))p[2];
  cache_fn.evict = (decltype(cache_fn.evict))p[3];
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"connect", (PyCFunction)(void*)connect, METH_FASTCALL, nullptr},
    {"connect_cache", (PyCFunction)(void*)connect_cache, METH_FASTCALL, nullptr},
    {"tree_attn", (PyCFunction)(void*)tree_attn, METH_FASTCALL, nullptr},
    {"tree_accept", (PyCFunction)(void*)tree_accept, METH_FASTCALL, nullptr},
    {"kv_weight", (PyCFunction)(void*)kv_weight, METH_FASTCALL, nullptr},
    {"kv_evict", (PyCFunction)(void*)kv_evict, METH_FASTCALL, nullptr},
    {"partial", (PyCFunction)(void*)partial, METH_FASTCALL, nullptr},
    {"decode", (PyCFunction)(void*)decode, METH_FASTCALL, nullptr},
    {"decode_static", (PyCFunction)(void*)decode_static, METH_FASTCALL, nullptr},
    {"merge", (PyCFunction)(void*)merge, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void*)append, METH_FASTCALL, nullptr},
    {"ring", (PyCFunction)(void*)ring, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_py_calls", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__py_calls(void) { return PyModule_Create(&module); }
