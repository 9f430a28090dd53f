// torch_calls.cpp — the device-driven calls on torch tensors: checks of types, devices, shapes and strides, and the argument
// structs of the C ABI, filled in from the tensors. A Python extension module, because on a small batch the host's part of a
// call takes longer than the kernel: reading seven tensors and packing a struct in Python took 3 to 4 us of a call of 11.
// The library's entry points are handed over by the binding (bind), which has loaded it.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <sstream>
#include <stdexcept>

#include "../../include/emaslice.h"

namespace {

int (*build_tables)(const paged_build_tables_t*, void*);
int (*write_kv)(const paged_write_kv_t*, void*);
int (*decode_tables)(const paged_decode_t*, void*);
int (*decode_diff)(const paged_decode_t*, void*);
int (*tree_attention)(const paged_tree_t*, void*);
int (*keep_rows)(const paged_keep_rows_t*, void*);
int (*copy_blocks)(const paged_copy_blocks_t*, void*);
int (*fork_requests)(const paged_fork_t*, void*);
int (*free_blocks)(const paged_free_t*, void*);
int (*compact)(const paged_compact_t*, void*);

struct PythonError {};  // the exception is set already

[[noreturn]] void refuse(const std::string& what) { throw std::invalid_argument(what); }

// A tensor with memory and strides of its own.
const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) refuse(std::string(name) + ": expected a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.layout() != at::kStrided || !(t.is_cuda() || t.is_cpu()) || !t.has_storage())
    refuse(std::string(name) + ": expected a dense tensor in GPU or host memory");
  return t;
}

std::string seen(const at::Tensor& t) {
  std::ostringstream s;
  s << "got " << t.sizes() << " of " << t.scalar_type() << " on " << t.device() << ", strides " << t.strides();
  return s.str();
}

uint64_t address(const at::Tensor& t) { return reinterpret_cast<uint64_t>(t.data_ptr()); }

uint32_t count(int64_t n, const char* name) {
  if (n > 0xffffffffll) refuse(std::string(name) + ": more than 2^32 - 1");
  return static_cast<uint32_t>(n);
}

// A dense array of one type on device number `dev` (-1: host memory); of a shape, if one is given.
template <typename T>
T* words(PyObject* o, const char* name, int64_t dev, at::ScalarType type, c10::IntArrayRef shape = {}) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.get_device() != dev || !t.is_contiguous() || (!shape.empty() && t.sizes() != shape)) {
    std::ostringstream s;
    s << name << ": expected a contiguous tensor of " << type << " on device " << dev;
    if (!shape.empty()) s << " of shape " << shape;
    refuse(s.str() + ", " + seen(t));
  }
  return reinterpret_cast<T*>(address(t));
}

int32_t* status_of(PyObject* o, int64_t dev) { return o == Py_None ? nullptr : words<int32_t>(o, "status", dev, at::kInt, {1}); }

// Address of an [n][rows][cols] tensor of 16-bit elements whose inner two dimensions are dense, and the bytes between its entries.
void* rows_of(PyObject* o, const char* name, int64_t dev, at::ScalarType type, int64_t n, int64_t rows, int64_t cols, uint64_t* stride) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.get_device() != dev || t.dim() != 3 || t.size(0) != n || t.size(1) != rows || t.size(2) != cols) {
    std::ostringstream s;
    s << name << ": expected [" << n << ", " << rows << ", " << cols << "] of " << type << " on device " << dev << ", ";
    refuse(s.str() + seen(t));
  }
  if ((t.stride(2) != 1 && cols > 1) || (t.stride(1) != cols && rows > 1))
    refuse(std::string(name) + ": the inner two dimensions have to be contiguous, " + seen(t));
  *stride = static_cast<uint64_t>(n > 1 ? t.stride(0) : rows * cols) * 2;
  return reinterpret_cast<void*>(address(t));
}

// Tables: address, entries from a row to the next, width.
int32_t* table_of(PyObject* o, int64_t dev, int64_t n, uint64_t* stride, uint32_t* width) {
  const at::Tensor& t = tensor(o, "tables");
  if (t.scalar_type() != at::kInt || t.get_device() != dev || t.dim() != 2 || t.size(0) != n || (t.stride(1) != 1 && t.size(1) > 1)) {
    std::ostringstream s;
    s << "tables: expected int32 [" << n << ", max_blocks] on device " << dev << ", rows contiguous, ";
    refuse(s.str() + seen(t));
  }
  *width = count(t.size(1), "tables");
  *stride = static_cast<uint64_t>(n > 1 ? t.stride(0) : t.size(1));
  return reinterpret_cast<int32_t*>(address(t));
}

int64_t number(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError();
  return v;
}

uint32_t natural(PyObject* o, const char* name) {
  const int64_t v = number(o);
  if (v < 0) refuse(std::string(name) + ": 0 or more");
  return count(v, name);
}

float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PythonError();
  return static_cast<float>(v);
}

// None, a number or a torch stream.
void* stream_of(PyObject* o) {
  if (o == Py_None) return nullptr;
  if (PyLong_Check(o)) return reinterpret_cast<void*>(static_cast<uintptr_t>(number(o)));
  PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
  if (!v) throw PythonError();
  const long long s = PyLong_AsLongLong(v);
  Py_DECREF(v);
  if (s == -1 && PyErr_Occurred()) throw PythonError();
  return reinterpret_cast<void*>(static_cast<uintptr_t>(s));
}

template <typename Args>
int call(int (*entry)(const Args*, void*), const Args& a, void* stream) {
  if (!entry) refuse("the library is not loaded");
  int rc;
  Py_BEGIN_ALLOW_THREADS rc = entry(&a, stream);
  Py_END_ALLOW_THREADS return rc;
}

template <typename Body>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, Body body) {
  try {
    if (given != wanted) refuse("wrong number of arguments");
    return PyLong_FromLong(body());
  } catch (const PythonError&) {
  } catch (const std::invalid_argument& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  }
  return nullptr;
}

const paged_cache_t* cache_of(PyObject* o) { return reinterpret_cast<const paged_cache_t*>(static_cast<uintptr_t>(number(o))); }

at::ScalarType type_of(const paged_cache_t* c) { return c->dtype ? at::kHalf : at::kBFloat16; }

// pool, device, lens, new_lens, block_tokens, tables, offsets, slots, positions, status, stream
PyObject* py_build(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    const int64_t dev = number(v[1]), nseq = tensor(v[2], "lens").numel(), room = tensor(v[7], "slots").numel();
    paged_build_tables_t a{};
    a.pool = reinterpret_cast<const paged_pool_t*>(static_cast<uintptr_t>(number(v[0])));
    a.nseq = count(nseq, "lens");
    a.max_tokens = count(room, "slots");
    a.block_tokens = natural(v[4], "block_tokens");
    a.lens = words<int32_t>(v[2], "lens", dev, at::kInt);
    a.new_lens = words<int32_t>(v[3], "new_lens", dev, at::kInt, {nseq});
    a.tables = table_of(v[5], dev, nseq, &a.table_stride, &a.max_blocks);
    a.offsets = words<int32_t>(v[6], "offsets", dev, at::kInt, {nseq + 1});
    a.slots = words<int64_t>(v[7], "slots", dev, at::kLong);
    a.positions = words<int32_t>(v[8], "positions", dev, at::kInt, {room});
    a.status = status_of(v[9], dev);
    return call(build_tables, a, stream_of(v[10]));
  });
}

// cache, device, k, v, slots, status, stream
PyObject* py_write(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 7, [&] {
    const paged_cache_t* c = cache_of(v[0]);
    const int64_t dev = number(v[1]), ntok = tensor(v[4], "slots").numel();
    paged_write_kv_t a{};
    a.cache = c;
    a.ntok = count(ntok, "slots");
    a.k = rows_of(v[2], "k", dev, type_of(c), ntok, c->num_kv_heads, c->head_dim, &a.k_stride);
    a.v = rows_of(v[3], "v", dev, type_of(c), ntok, c->num_kv_heads, c->head_dim, &a.v_stride);
    a.slots = words<int64_t>(v[4], "slots", dev, at::kLong);
    a.status = status_of(v[5], dev);
    return call(write_kv, a, stream_of(v[6]));
  });
}

// cache, device, tables, lens, q, sm_scale, out, workspace, window, status, stream, and lse (plain) or lam, norm_weight, eps, out_scale
int decode(PyObject* const* v, bool diff) {
  const paged_cache_t* c = cache_of(v[0]);
  const int64_t dev = number(v[1]), nseq = tensor(v[3], "lens").numel(), d = c->head_dim;
  const at::Tensor& rows = tensor(v[diff ? 6 : 4], diff ? "out" : "q");
  const int64_t heads = rows.dim() == 3 ? rows.size(1) : -1;
  paged_decode_t a{};
  a.cache = c;
  a.nseq = count(nseq, "lens");
  a.tables = table_of(v[2], dev, nseq, &a.table_stride, &a.max_blocks);
  a.lens = words<int32_t>(v[3], "lens", dev, at::kInt);
  a.q = diff ? rows_of(v[4], "q", dev, type_of(c), nseq, 2 * heads, d / 2, &a.q_stride)
             : rows_of(v[4], "q", dev, type_of(c), nseq, heads, d, &a.q_stride);
  a.out = rows_of(v[6], "out", dev, type_of(c), nseq, heads, d, &a.out_stride);
  a.num_heads = count(heads, "heads");
  a.sm_scale = real(v[5]);
  const at::Tensor& work = tensor(v[7], "workspace");
  if (!work.is_contiguous() || work.get_device() != dev) refuse("workspace: a contiguous tensor on the cache's device, " + seen(work));
  a.workspace = reinterpret_cast<void*>(address(work));
  a.workspace_bytes = work.nbytes();
  a.window = natural(v[8], "window");
  a.status = status_of(v[9], dev);
  a.out_scale = 1.f;
  if (diff) {
    a.lam = words<float>(v[11], "lam", dev, at::kFloat, {heads});
    if (v[12] != Py_None) a.norm_weight = words<float>(v[12], "norm_weight", dev, at::kFloat, {d});
    a.eps = real(v[13]);
    a.out_scale = real(v[14]);
  } else if (v[11] != Py_None) {
    a.lse = words<float>(v[11], "lse", dev, at::kFloat, {nseq, heads});
  }
  return call(diff ? decode_diff : decode_tables, a, stream_of(v[10]));
}

PyObject* py_decode(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 12, [&] { return decode(v, false); });
}

PyObject* py_diff(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 15, [&] { return decode(v, true); });
}

// A [n][width] tensor of one type with dense rows: address, elements from a row to the next, width.
template <typename T>
T* matrix(PyObject* o, const char* name, int64_t dev, at::ScalarType type, int64_t n, uint64_t* stride, uint32_t* width) {
  const at::Tensor& t = tensor(o, name);
  if (t.scalar_type() != type || t.get_device() != dev || t.dim() != 2 || t.size(0) != n || (t.stride(1) != 1 && t.size(1) > 1)) {
    std::ostringstream s;
    s << name << ": expected " << type << " [" << n << ", ..] on device " << dev << ", rows contiguous, ";
    refuse(s.str() + seen(t));
  }
  *width = count(t.size(1), name);
  *stride = static_cast<uint64_t>(n > 1 ? t.stride(0) : t.size(1));
  return reinterpret_cast<T*>(address(t));
}

// cache, device, tables, lens, offsets, q, sm_scale, out, workspace, mask, lse, window, positions, status, stream
PyObject* py_tree(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 15, [&] {
    const paged_cache_t* c = cache_of(v[0]);
    const int64_t dev = number(v[1]), nseq = tensor(v[3], "lens").numel(), d = c->head_dim;
    const at::Tensor& q = tensor(v[5], "q");
    const int64_t ntok = q.dim() == 3 ? q.size(0) : -1, heads = q.dim() == 3 ? q.size(1) : -1;
    paged_tree_t a{};
    a.cache = c;
    a.nseq = count(nseq, "lens");
    a.tables = table_of(v[2], dev, nseq, &a.table_stride, &a.max_blocks);
    a.lens = words<int32_t>(v[3], "lens", dev, at::kInt);
    a.offsets = words<int32_t>(v[4], "offsets", dev, at::kInt, {nseq + 1});
    a.q = rows_of(v[5], "q", dev, type_of(c), ntok, heads, d, &a.q_stride);
    a.out = rows_of(v[7], "out", dev, type_of(c), ntok, heads, d, &a.out_stride);
    a.ntok = count(ntok, "q");
    a.num_heads = count(heads, "heads");
    a.sm_scale = real(v[6]);
    const at::Tensor& work = tensor(v[8], "workspace");
    if (!work.is_contiguous() || work.get_device() != dev) refuse("workspace: a contiguous tensor on the cache's device, " + seen(work));
    a.workspace = reinterpret_cast<void*>(address(work));
    a.workspace_bytes = work.nbytes();
    if (v[9] != Py_None) {
      a.mask = matrix<uint64_t>(v[9], "mask", dev, at::kLong, ntok, &a.mask_stride, &a.mask_words);
      if (ntok && !a.mask_words) refuse("mask: at least one word for a token");
    }
    if (v[10] != Py_None) a.lse = words<float>(v[10], "lse", dev, at::kFloat, {ntok, heads});
    a.window = natural(v[11], "window");
    if (v[12] != Py_None) a.positions = words<int32_t>(v[12], "positions", dev, at::kInt, {ntok});
    a.status = status_of(v[13], dev);
    return call(tree_attention, a, stream_of(v[14]));
  });
}

// layers, their number, device, tables, lens, keep, counts, status, stream
PyObject* py_keep(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const int64_t dev = number(v[2]), nseq = tensor(v[4], "lens").numel();
    paged_keep_rows_t a{};
    a.layers = cache_of(v[0]);
    a.nlayers = natural(v[1], "layers");
    a.nseq = count(nseq, "lens");
    a.tables = table_of(v[3], dev, nseq, &a.table_stride, &a.max_blocks);
    a.lens = words<int32_t>(v[4], "lens", dev, at::kInt);
    a.keep = matrix<int32_t>(v[5], "keep", dev, at::kInt, nseq, &a.keep_stride, &a.max_keep);
    a.counts = words<int32_t>(v[6], "counts", dev, at::kInt, {nseq});
    a.status = status_of(v[7], dev);
    return call(keep_rows, a, stream_of(v[8]));
  });
}

int32_t* copies_of(PyObject* o, int64_t dev, uint32_t* n) {
  const at::Tensor& t = tensor(o, "copies");
  if (t.dim() != 2) refuse("copies: expected int32 [n, 3], " + seen(t));
  *n = count(t.size(0), "copies");
  return words<int32_t>(o, "copies", dev, at::kInt, {t.size(0), 3});
}

// layers, their number, device, copies, status, stream
PyObject* py_copy(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    const int64_t dev = number(v[2]);
    paged_copy_blocks_t a{};
    a.layers = cache_of(v[0]);
    a.nlayers = natural(v[1], "layers");
    a.copies = copies_of(v[3], dev, &a.ncopies);
    a.status = status_of(v[4], dev);
    return call(copy_blocks, a, stream_of(v[5]));
  });
}

// What the calls on shared blocks begin with: pool, shares, device, lens, block_tokens, tables.
template <typename Args>
int64_t begin(Args& a, PyObject* const* v) {
  const int64_t dev = number(v[2]), nseq = tensor(v[3], "lens").numel();
  a.pool = reinterpret_cast<const paged_pool_t*>(static_cast<uintptr_t>(number(v[0])));
  a.shares = reinterpret_cast<const paged_shares_t*>(static_cast<uintptr_t>(number(v[1])));
  a.nseq = count(nseq, "lens");
  a.lens = words<int32_t>(v[3], "lens", dev, at::kInt);
  a.block_tokens = natural(v[4], "block_tokens");
  a.tables = table_of(v[5], dev, nseq, &a.table_stride, &a.max_blocks);
  return dev;
}

// .., new_lens, src, dst, copies, status, stream
PyObject* py_fork(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    paged_fork_t a{};
    const int64_t dev = begin(a, v), nfork = tensor(v[7], "src").numel();
    a.new_lens = words<int32_t>(v[6], "new_lens", dev, at::kInt, {static_cast<int64_t>(a.nseq)});
    a.src = words<int32_t>(v[7], "src", dev, at::kInt);
    a.dst = words<int32_t>(v[8], "dst", dev, at::kInt, {nfork});
    a.copies = copies_of(v[9], dev, &a.nfork);
    if (a.nfork != nfork) refuse("copies: a row for every fork");
    a.status = status_of(v[10], dev);
    return call(fork_requests, a, stream_of(v[11]));
  });
}

// .., new_lens, status, stream
PyObject* py_free(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    paged_free_t a{};
    const int64_t dev = begin(a, v);
    a.new_lens = words<int32_t>(v[6], "new_lens", dev, at::kInt, {static_cast<int64_t>(a.nseq)});
    a.status = status_of(v[7], dev);
    return call(free_blocks, a, stream_of(v[8]));
  });
}

// .., limits, copies, status, stream
PyObject* py_compact(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    paged_compact_t a{};
    const int64_t dev = begin(a, v);
    a.limits = words<int32_t>(v[6], "limits", dev, at::kInt, {2});
    a.copies = copies_of(v[7], dev, &a.max_copies);
    a.status = status_of(v[8], dev);
    return call(compact, a, stream_of(v[9]));
  });
}

// Addresses of paged_tree_attention, paged_keep_rows, paged_copy_blocks, paged_fork, paged_free and paged_compact.
PyObject* py_bind_more(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    tree_attention = reinterpret_cast<decltype(tree_attention)>(static_cast<uintptr_t>(number(v[0])));
    keep_rows = reinterpret_cast<decltype(keep_rows)>(static_cast<uintptr_t>(number(v[1])));
    copy_blocks = reinterpret_cast<decltype(copy_blocks)>(static_cast<uintptr_t>(number(v[2])));
    fork_requests = reinterpret_cast<decltype(fork_requests)>(static_cast<uintptr_t>(number(v[3])));
    free_blocks = reinterpret_cast<decltype(free_blocks)>(static_cast<uintptr_t>(number(v[4])));
    compact = reinterpret_cast<decltype(compact)>(static_cast<uintptr_t>(number(v[5])));
    return 0;
  });
}

// Addresses of paged_build_tables, paged_write_kv, paged_decode_tables and paged_decode_diff.
PyObject* py_bind(PyObject*, PyObject* const* v, Py_ssize_t n) {
  return guarded(n, 4, [&] {
    build_tables = reinterpret_cast<decltype(build_tables)>(static_cast<uintptr_t>(number(v[0])));
    write_kv = reinterpret_cast<decltype(write_kv)>(static_cast<uintptr_t>(number(v[1])));
    decode_tables = reinterpret_cast<decltype(decode_tables)>(static_cast<uintptr_t>(number(v[2])));
    decode_diff = reinterpret_cast<decltype(decode_diff)>(static_cast<uintptr_t>(number(v[3])));
    return 0;
  });
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef methods[] = {{"bind", fast(py_bind), METH_FASTCALL, nullptr},     {"build", fast(py_build), METH_FASTCALL, nullptr},
                         {"write", fast(py_write), METH_FASTCALL, nullptr},   {"decode", fast(py_decode), METH_FASTCALL, nullptr},
                         {"diff", fast(py_diff), METH_FASTCALL, nullptr},     {"bind_more", fast(py_bind_more), METH_FASTCALL, nullptr},
                         {"tree", fast(py_tree), METH_FASTCALL, nullptr},     {"keep", fast(py_keep), METH_FASTCALL, nullptr},
                         {"copy", fast(py_copy), METH_FASTCALL, nullptr},     {"fork", fast(py_fork), METH_FASTCALL, nullptr},
                         {"free", fast(py_free), METH_FASTCALL, nullptr},     {"compact", fast(py_compact), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
