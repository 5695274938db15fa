// Calls of the key/value cache operators from torch tensors (scoot_kv_*).
//
// The operators take a few microseconds on the device, and a call made through
// ctypes from tensors' attributes took longer than that on the host: 9.1 us for
// slots, 6.8 for writes.  Here the tensors are looked at in C++, and the library's
// functions are called by the addresses that the loader has.  Each function tests
// its arguments in one expression and returns None if that fails: the Python side
// then finds out what is wrong and says so.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

namespace {

typedef int (*AssignFn)(const void*, const void*, int, int, void*, int, int64_t, const void*, int, int64_t, void*, void*, void*, void*,
                        void*, void*);
typedef int (*WriteFn)(const void*, const void*, int, int64_t, int, int, int64_t, int64_t, int64_t, int64_t, const void*, void*, void*,
                       int, int64_t, int, float, float, void*);
typedef int (*WorkspaceFn)(int64_t, int, int, int, int, int64_t, int64_t, int, uint64_t*);
typedef int (*AttentionFn)(const void*, int, int64_t, int, int, int, int64_t, int64_t, const void*, const void*, int, int64_t, int,
                           const void*, int, int64_t, const void*, const void*, int, int64_t, int64_t, float, int, float, float, void*,
                           int64_t, int64_t, void*, uint64_t, void*);
AssignFn assign_fn;
WriteFn write_fn;
WorkspaceFn workspace_fn;
AttentionFn attention_fn;
PyObject* raw_stream;  // torch's: device index -> stream

enum { kF16, kBF16, kF8, kNoType };

int type_of(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kHalf: return kF16;
    case at::kBFloat16: return kBF16;
    case at::kFloat8_e4m3fn: return kF8;
    default: return kNoType;
  }
}

bool is_list(const at::Tensor& t, at::ScalarType type) { return t.is_cuda() && t.scalar_type() == type && t.is_contiguous(); }

bool is_table(const at::Tensor& t, int64_t rows) {
  return t.is_cuda() && t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == rows &&
         (t.is_contiguous() || ((t.stride(1) == 1 || t.size(1) <= 1) && (rows <= 1 || t.stride(0) >= t.size(1))));
}

bool is_vectors(const at::Tensor& t, int64_t heads, int64_t dim) {
  return t.is_cuda() && t.dim() == 3 && t.size(2) == dim && t.size(1) == heads && t.stride(2) == 1;
}

bool are_caches(const at::Tensor& k, const at::Tensor& v) {
  return type_of(k) != kNoType && k.is_cuda() && v.is_cuda() && k.dim() == 4 && k.is_contiguous() && v.is_contiguous() &&
         v.scalar_type() == k.scalar_type() && v.sizes() == k.sizes();
}

bool with(const at::Tensor& t, std::initializer_list<const at::Tensor*> others) {
  for (const at::Tensor* o : others)
    if (o->get_device() != t.get_device()) return false;
  return true;
}

// The library launches on the current device: while one of these lives, that is the tensor's.
class OnDeviceOf {
 public:
  explicit OnDeviceOf(const at::Tensor& t) : impl_(t.device().type()), before_(impl_.getDevice()), other_(before_ != t.device()) {
    if (other_) impl_.setDevice(t.device());
  }
  ~OnDeviceOf() {
    if (other_) impl_.uncheckedSetDevice(before_);
  }
  OnDeviceOf(const OnDeviceOf&) = delete;
  OnDeviceOf& operator=(const OnDeviceOf&) = delete;

 private:
  const c10::impl::VirtualGuardImpl impl_;
  const c10::Device before_;
  const bool other_;
};

// What does not fit becomes what the library refuses.
int narrow(int64_t v) { return v > INT_MAX ? INT_MAX : v < INT_MIN ? INT_MIN : (int)v; }
int64_t stride_of(const at::Tensor& table) { return std::max<int64_t>(table.stride(0), table.size(1)); }

bool tensors(PyObject* const* args, std::initializer_list<int> at) {
  for (int i : at)
    if (!THPVariable_Check(args[i])) return false;
  return true;
}

// Whole numbers and floats out of arguments; a Python error if one is neither.
bool get(PyObject* o, int64_t& v) {
  v = PyLong_AsLongLong(o);
  return !(v == -1 && PyErr_Occurred());
}
bool get(PyObject* o, float& v) {
  v = (float)PyFloat_AsDouble(o);
  return !(v == -1.0f && PyErr_Occurred());
}
bool get_stream(PyObject* o, const at::Tensor& t, void*& stream) {
  int64_t v;
  if (o != Py_None) {
    if (!get(o, v)) return false;
  } else {
    PyObject* index = PyLong_FromLong(t.get_device());
    PyObject* r = index ? PyObject_CallOneArg(raw_stream, index) : nullptr;
    Py_XDECREF(index);
    if (!r) return false;
    const bool ok = get(r, v);
    Py_DECREF(r);
    if (!ok) return false;
  }
  stream = (void*)(intptr_t)v;
  return true;
}

at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like) {
  return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
}

// `size` elements from element `from` on of a tensor of bytes, as elements of `type`.
at::Tensor part(const at::Tensor& bytes, at::ScalarType type, int64_t from, int64_t size) {
  at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(bytes.storage()), bytes.key_set(),
                                                          c10::scalarTypeToTypeMeta(type));
  t.unsafeGetTensorImpl()->set_storage_offset(from);
  t.unsafeGetTensorImpl()->set_sizes_contiguous({size});
  return t;
}

// bind(assign, write, workspace, attention, raw_stream): addresses of the library's functions.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  int64_t at[4];
  if (n != 5) return PyErr_Format(PyExc_TypeError, "bind takes 5 arguments");
  for (int i = 0; i < 4; ++i)
    if (!get(args[i], at[i])) return nullptr;
  assign_fn = (AssignFn)at[0];
  write_fn = (WriteFn)at[1];
  workspace_fn = (WorkspaceFn)at[2];
  attention_fn = (AttentionFn)at[3];
  Py_INCREF(args[4]);
  Py_XDECREF(raw_stream);
  raw_stream = args[4];
  Py_RETURN_NONE;
}

// assign(context_len, new_len, block_table, free_blocks, block_size, max_tokens, stream[, query_start, seq_len, positions,
// slots, counts]) -> status and, if they were not given, the five results.
PyObject* assign(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 && n != 12) return PyErr_Format(PyExc_TypeError, "assign takes 7 or 12 arguments");
  if (!tensors(args, {0, 1, 2, 3}) || (n == 12 && !tensors(args, {7, 8, 9, 10, 11}))) Py_RETURN_NONE;
  const at::Tensor &ctx = THPVariable_Unpack(args[0]), &add = THPVariable_Unpack(args[1]), &table = THPVariable_Unpack(args[2]),
                   &free = THPVariable_Unpack(args[3]);
  const int64_t seqs = ctx.numel();
  if (!(is_list(ctx, at::kInt) && is_list(add, at::kInt) && add.numel() == seqs && is_list(free, at::kInt) && is_table(table, seqs) &&
        with(ctx, {&add, &table, &free})))
    Py_RETURN_NONE;
  int64_t block_size, max_tokens;
  void* stream;
  if (!get(args[4], block_size) || !get(args[5], max_tokens)) return nullptr;
  if (max_tokens < 0) Py_RETURN_NONE;
  at::Tensor r[5];
  if (n == 12) {
    const int64_t size[5] = {seqs + 1, seqs, max_tokens, max_tokens, 4};
    for (int i = 0; i < 5; ++i) {
      r[i] = THPVariable_Unpack(args[7 + i]);
      if (!is_list(r[i], i == 3 ? at::kLong : at::kInt) || r[i].numel() != size[i] || !with(ctx, {&r[i]})) Py_RETURN_NONE;
    }
  } else {
    const at::Tensor all = make({8 * max_tokens + 4 * (2 * seqs + 5 + max_tokens)}, at::kByte, ctx);
    r[3] = part(all, at::kLong, 0, max_tokens);
    int64_t from = 2 * max_tokens;
    for (int i : {0, 1, 4, 2}) {
      const int64_t size = i == 0 ? seqs + 1 : i == 1 ? seqs : i == 4 ? 4 : max_tokens;
      r[i] = part(all, at::kInt, from, size);
      from += size;
    }
  }
  if (!get_stream(args[6], ctx, stream)) return nullptr;
  const OnDeviceOf on(ctx);
  const int rc = assign_fn(ctx.data_ptr(), add.data_ptr(), narrow(seqs), narrow(block_size), table.data_ptr(), narrow(table.size(1)),
                           stride_of(table), free.data_ptr(), narrow(free.numel()), max_tokens, r[0].data_ptr(), r[1].data_ptr(),
                           r[2].data_ptr(), r[3].data_ptr(), r[4].data_ptr(), stream);
  if (n == 12) return PyLong_FromLong(rc);
  PyObject* got = PyTuple_New(6);
  if (!got) return nullptr;
  PyTuple_SET_ITEM(got, 0, PyLong_FromLong(rc));
  for (int i = 0; i < 5; ++i) PyTuple_SET_ITEM(got, i + 1, THPVariable_Wrap(std::move(r[i])));
  return got;
  END_HANDLE_TH_ERRORS
}

// write(k, v, slots, k_cache, v_cache, k_scale, v_scale, stream) -> status
PyObject* write(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 8) return PyErr_Format(PyExc_TypeError, "write takes 8 arguments");
  if (!tensors(args, {0, 1, 2, 3, 4})) Py_RETURN_NONE;
  const at::Tensor &k = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[1]), &slots = THPVariable_Unpack(args[2]),
                   &kc = THPVariable_Unpack(args[3]), &vc = THPVariable_Unpack(args[4]);
  if (!are_caches(kc, vc)) Py_RETURN_NONE;
  const int64_t heads = kc.size(1), dim = kc.size(3), tokens = slots.numel();
  if (!(type_of(k) < kF8 && v.scalar_type() == k.scalar_type() && is_vectors(k, heads, dim) && is_vectors(v, heads, dim) &&
        k.size(0) == tokens && v.size(0) == tokens && is_list(slots, at::kLong) && with(k, {&v, &slots, &kc, &vc})))
    Py_RETURN_NONE;
  float ks, vs;
  void* stream;
  if (!get(args[5], ks) || !get(args[6], vs) || !get_stream(args[7], k, stream)) return nullptr;
  const OnDeviceOf on(k);
  return PyLong_FromLong(write_fn(k.data_ptr(), v.data_ptr(), type_of(k), tokens, narrow(heads), narrow(dim), k.stride(0), k.stride(1),
                                  v.stride(0), v.stride(1), slots.data_ptr(), kc.data_ptr(), vc.data_ptr(), type_of(kc), kc.size(0),
                                  narrow(kc.size(2)), ks, vs, stream));
  END_HANDLE_TH_ERRORS
}

// attention(q, k_cache, v_cache, block_table, query_start, seq_len, max_new_len, max_seq_len, scale or None, window, k_scale,
// v_scale, out or None, workspace or None, stream) -> status, or out if it was made here
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15) return PyErr_Format(PyExc_TypeError, "attention takes 15 arguments");
  if (!tensors(args, {0, 1, 2, 3, 4, 5})) Py_RETURN_NONE;
  const at::Tensor &q = THPVariable_Unpack(args[0]), &kc = THPVariable_Unpack(args[1]), &vc = THPVariable_Unpack(args[2]),
                   &table = THPVariable_Unpack(args[3]), &start = THPVariable_Unpack(args[4]), &len = THPVariable_Unpack(args[5]);
  if (!are_caches(kc, vc)) Py_RETURN_NONE;
  const int64_t kv_heads = kc.size(1), dim = kc.size(3), seqs = len.numel();
  if (!(type_of(q) < kF8 && q.is_cuda() && q.dim() == 3 && q.size(2) == dim && q.stride(2) == 1 && is_list(len, at::kInt) &&
        is_list(start, at::kInt) && start.numel() == seqs + 1 && is_table(table, seqs) &&
        with(q, {&kc, &vc, &table, &start, &len})))
    Py_RETURN_NONE;
  const int64_t tokens = q.size(0), heads = q.size(1);
  at::Tensor out, space;
  const bool made = args[12] == Py_None;
  if (!made) {
    if (!THPVariable_Check(args[12])) Py_RETURN_NONE;
    out = THPVariable_Unpack(args[12]);
    if (!(out.scalar_type() == q.scalar_type() && is_vectors(out, heads, dim) && out.size(0) == tokens && with(q, {&out})))
      Py_RETURN_NONE;
  }
  int64_t max_new, max_seq, window;
  float scale = (float)(1.0 / std::sqrt((double)std::max<int64_t>(dim, 1))), ks, vs;
  void* stream;
  if (!get(args[6], max_new) || !get(args[7], max_seq) || (args[8] != Py_None && !get(args[8], scale)) || !get(args[9], window) ||
      !get(args[10], ks) || !get(args[11], vs) || !get_stream(args[14], q, stream))
    return nullptr;
  uint64_t need = 0;
  if (args[13] == Py_None) {
    const int rc = workspace_fn(tokens, narrow(heads), narrow(kv_heads), narrow(dim), narrow(seqs), max_new, max_seq, narrow(window), &need);
    if (rc != 0) return PyLong_FromLong(rc);
    if (need) space = make({(int64_t)need}, at::kByte, q);
  } else {
    if (!THPVariable_Check(args[13])) Py_RETURN_NONE;
    space = THPVariable_Unpack(args[13]);
    if (!is_list(space, at::kByte) || !with(q, {&space})) Py_RETURN_NONE;
    need = (uint64_t)space.numel();
  }
  if (made) out = make({tokens, heads, dim}, q.scalar_type(), q);
  const OnDeviceOf on(q);
  const int rc = attention_fn(q.data_ptr(), type_of(q), tokens, narrow(heads), narrow(kv_heads), narrow(dim), q.stride(0), q.stride(1),
                              kc.data_ptr(), vc.data_ptr(), type_of(kc), kc.size(0), narrow(kc.size(2)), table.data_ptr(),
                              narrow(table.size(1)), stride_of(table), start.data_ptr(), len.data_ptr(), narrow(seqs), max_new, max_seq,
                              scale, narrow(window), ks, vs, out.data_ptr(), out.stride(0), out.stride(1),
                              need ? space.data_ptr() : nullptr, need, stream);
  if (rc != 0 || !made) return PyLong_FromLong(rc);
  return THPVariable_Wrap(std::move(out));
  END_HANDLE_TH_ERRORS
}

PyMethodDef kMethods[] = {{"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr},
                          {"assign", (PyCFunction)(void (*)())assign, METH_FASTCALL, nullptr},
                          {"write", (PyCFunction)(void (*)())write, METH_FASTCALL, nullptr},
                          {"attention", (PyCFunction)(void (*)())attention, METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_kv_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_torch() { return PyModule_Create(&kModule); }
