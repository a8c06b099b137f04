// Python side of the hot calls: turns tensors into pointers and calls the C ABI.
//
// binding.py declares every call; the ones a training or serving loop makes each step come here.
// What bounds a small batch is the host: through ctypes a call with three tensors cost 2.6 us before
// it reached the library (two Python method calls per tensor, argument conversion), a grouped call
// over 64 tables 85 us.  Here a tensor is unpacked in a few nanoseconds.  No work of the table or of
// an operator is done in this file.
#include <Python.h>

#include <cstdint>
#include <exception>
#include <new>
#include <vector>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mono.h"

namespace {

using u32 = uint32_t;
using i64 = int64_t;
using ptr = void*;

// Addresses of the library's functions, set once by bind().
enum Fn {
  F_LOOKUP, F_LOOKUP_NOALLOC, F_LOOKUP_HOST, F_APPLY, F_APPLY_HOST, F_PREPARE, F_AHEAD, F_EXPIRE, F_EXPIRE_SLICE, F_FENCE,
  F_GROUP_PREPARE, F_GROUP_LOOKUP, F_GROUP_APPLY, F_TOKEN_ROWS, F_TOKEN_ROWS_GRAD, F_TOKEN_ROWS_GRAD_WORKSPACE, F_PACK_ROWS,
  F_PACKED_TOKEN_ROWS, F_PACKED_SCORES, F_COUNT
};
const char* const kNames[F_COUNT] = {
  "mono_lookup_pool", "mono_lookup_pool_noalloc", "mono_lookup_pool_host", "mono_apply_grads", "mono_apply_grads_host",
  "mono_prepare_push", "mono_group_ahead", "mono_expire", "mono_expire_slice", "mono_fence", "mono_group_prepare_push",
  "mono_group_lookup_pool", "mono_group_apply_grads", "mono_token_rows", "mono_token_rows_grad", "mono_token_rows_grad_workspace", "mono_pack_rows",
  "mono_packed_token_rows", "mono_packed_scores"
};
ptr g_fn[F_COUNT] = {};
PyObject* g_address_of = nullptr;      // binding._ptr, for what is neither a tensor, an int nor None

template <typename F>
F fn(Fn which) { return reinterpret_cast<F>(g_fn[which]); }

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2 || !PyDict_Check(args[0])) { PyErr_SetString(PyExc_TypeError, "bind(addresses, address_of)"); return nullptr; }
  for (int k = 0; k < F_COUNT; ++k) {
    PyObject* v = PyDict_GetItemString(args[0], kNames[k]);
    if (!v) { PyErr_SetString(PyExc_KeyError, kNames[k]); return nullptr; }
    g_fn[k] = PyLong_AsVoidPtr(v);
    if (PyErr_Occurred()) return nullptr;
  }
  Py_INCREF(args[1]);
  Py_XSETREF(g_address_of, args[1]);
  Py_RETURN_NONE;
}

bool expects(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, got);
  return false;
}

// A reference that is given back whichever way its scope is left.
struct Owned {
  PyObject* o;
  explicit Owned(PyObject* p) : o(p) {}
  Owned(const Owned&) = delete;
  Owned& operator=(const Owned&) = delete;
  ~Owned() { Py_XDECREF(o); }
};

// Whether x is a torch.Tensor (or Parameter) itself, with nobody listening to its methods: only then may its
// fields be read here.  A subclass may answer for itself, and so may a torch function mode.
bool plain_tensor(PyObject* x) { return THPVariable_CheckExact(x) && !at::impl::torch_function_mode_enabled(); }

// Raw address of a tensor / int / None / anything binding._ptr knows.  What a plain tensor refuses
// (one without storage: inside vmap, grad or jvp, sparse, opaque) is asked for again through Python, which says why.
bool address(PyObject* x, ptr* out) {
  if (plain_tensor(x)) {
    try {
      const at::Tensor& t = THPVariable_Unpack(x);
      if (t.is_contiguous()) { *out = t.data_ptr(); return true; }
    } catch (const std::exception&) {
    }
  }
  if (x == Py_None) { *out = nullptr; return true; }
  if (!PyLong_Check(x)) {
    const Owned r(PyObject_CallOneArg(g_address_of, x));
    if (!r.o) return false;
    *out = PyLong_AsVoidPtr(r.o);
    return !PyErr_Occurred();
  }
  *out = PyLong_AsVoidPtr(x);
  return !PyErr_Occurred();
}

bool integer(PyObject* x, i64* out) {
  *out = PyLong_AsLongLong(x);
  return !(*out == -1 && PyErr_Occurred());
}

template <typename C>
PyObject* without_gil(C&& call) {
  struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
  };
  int rc;
  { const Released released; rc = call(); }
  return PyLong_FromLong(rc);
}

// Every method is entered through this: a C++ exception that left one would end the process.
using Method = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
template <Method F>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) noexcept {
  try {
    return F(self, args, n);
  } catch (const std::bad_alloc&) {
    return PyErr_NoMemory();
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

// (t, ids, n_ids, offsets, n_bags)
struct Batch { ptr t, ids, off; i64 n_ids, n_bags; };
bool batch(PyObject* const* a, Batch* b) {
  return address(a[0], &b->t) && address(a[1], &b->ids) && integer(a[2], &b->n_ids) && address(a[3], &b->off) &&
         integer(a[4], &b->n_bags);
}

template <Fn W>
PyObject* announce(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Batch b;
  if (!expects(n, 5) || !batch(a, &b)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr, ptr, i64, ptr, i64)>(W)(b.t, b.ids, b.n_ids, b.off, b.n_bags); });
}

template <Fn W>
PyObject* pull(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Batch b;
  ptr out;
  if (!expects(n, 6) || !batch(a, &b) || !address(a[5], &out)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr, ptr, i64, ptr, i64, ptr)>(W)(b.t, b.ids, b.n_ids, b.off, b.n_bags, out); });
}

template <Fn W>
PyObject* push(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Batch b;
  ptr grad;
  i64 now;
  if (!expects(n, 7) || !batch(a, &b) || !address(a[5], &grad) || !integer(a[6], &now)) return nullptr;
  return without_gil([&] {
    return fn<int (*)(ptr, ptr, i64, ptr, i64, ptr, i64)>(W)(b.t, b.ids, b.n_ids, b.off, b.n_bags, grad, now);
  });
}

PyObject* expire(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ptr t;
  i64 now;
  if (!expects(n, 2) || !address(a[0], &t) || !integer(a[1], &now)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr, i64)>(F_EXPIRE)(t, now); });
}

PyObject* expire_slice(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ptr t;
  i64 now, slice, slices;
  if (!expects(n, 4) || !address(a[0], &t) || !integer(a[1], &now) || !integer(a[2], &slice) || !integer(a[3], &slices)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr, i64, u32, u32)>(F_EXPIRE_SLICE)(t, now, (u32)slice, (u32)slices); });
}

PyObject* fence(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ptr t;
  if (!expects(n, 1) || !address(a[0], &t)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr)>(F_FENCE)(t); });
}

// Pulls with the arguments of MonoTable.lookup_pool as they are: returns None, having done nothing,
// unless ids and offsets are contiguous 64-bit tensors on the table's device, and out a tensor, all of them plain.
// (handle, device, ids, offsets, out)
PyObject* table_pull(PyObject*, PyObject* const* a, Py_ssize_t n) {
  ptr t, out;
  i64 device;
  if (!expects(n, 5) || !address(a[0], &t) || !integer(a[1], &device)) return nullptr;
  if (!plain_tensor(a[2]) || !plain_tensor(a[3]) || !plain_tensor(a[4])) Py_RETURN_NONE;
  ptr pi, po;
  i64 n_ids, n_bags;
  try {
    const at::Tensor &ids = THPVariable_Unpack(a[2]), &off = THPVariable_Unpack(a[3]);
    for (const at::Tensor* x : {&ids, &off}) {
      const bool words = x->scalar_type() == at::kLong || x->scalar_type() == at::kUInt64;
      if (!words || !x->is_cuda() || x->get_device() != device || !x->is_contiguous()) Py_RETURN_NONE;
    }
    pi = ids.data_ptr(), po = off.data_ptr();
    n_ids = ids.numel(), n_bags = off.numel() - 1;
  } catch (const std::exception&) {
    Py_RETURN_NONE;                                          // (no storage: the Python way says why)
  }
  if (!address(a[4], &out)) return nullptr;
  return without_gil([&] { return fn<int (*)(ptr, ptr, i64, ptr, i64, ptr)>(F_LOOKUP)(t, pi, n_ids, po, n_bags, out); });
}

// Host arrays of the grouped calls: one entry per table.
struct Group {
  std::vector<ptr> t, ids, off, vec;
  std::vector<i64> n_ids, n_bags;
};

bool entries(PyObject* list, size_t n, std::vector<ptr>* p, std::vector<i64>* numel, i64 less) {
  const Owned own(PySequence_Fast(list, "grouped calls take lists, one entry per table"));
  PyObject* const seq = own.o;
  if (!seq) return false;
  bool ok = (size_t)PySequence_Fast_GET_SIZE(seq) == n;
  if (!ok) PyErr_SetString(PyExc_ValueError, "grouped calls take one batch per table");
  p->resize(n);
  if (numel) numel->resize(n);
  for (size_t i = 0; ok && i < n; ++i) {
    PyObject* x = PySequence_Fast_GET_ITEM(seq, i);
    ok = address(x, &(*p)[i]);
    if (!ok || !numel) continue;
    if (plain_tensor(x)) { (*numel)[i] = THPVariable_Unpack(x).numel() - less; continue; }
    const Owned r(PyObject_CallMethod(x, "numel", nullptr));
    ok = r.o && integer(r.o, &(*numel)[i]);
    (*numel)[i] -= less;
  }
  return ok;
}

bool group(PyObject* handles, PyObject* ids, PyObject* off, PyObject* vec, Group* g) {
  const Py_ssize_t n = PySequence_Size(handles);
  return n >= 0 && entries(handles, (size_t)n, &g->t, nullptr, 0) && entries(ids, (size_t)n, &g->ids, &g->n_ids, 0) &&
         entries(off, (size_t)n, &g->off, &g->n_bags, 1) && (!vec || entries(vec, (size_t)n, &g->vec, nullptr, 0));
}

// (handles, ids, offsets, stream)
PyObject* group_prepare(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Group g;
  ptr s;
  if (!expects(n, 4) || !group(a[0], a[1], a[2], nullptr, &g) || !address(a[3], &s)) return nullptr;
  return without_gil([&] {
    return fn<int (*)(int32_t, ptr*, ptr*, i64*, ptr*, i64*, ptr)>(F_GROUP_PREPARE)(
        (int32_t)g.t.size(), g.t.data(), g.ids.data(), g.n_ids.data(), g.off.data(), g.n_bags.data(), s);
  });
}

// (handles, ids, offsets, outs, stream)
PyObject* group_pull(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Group g;
  ptr s;
  if (!expects(n, 5) || !group(a[0], a[1], a[2], a[3], &g) || !address(a[4], &s)) return nullptr;
  return without_gil([&] {
    return fn<int (*)(int32_t, ptr*, ptr*, i64*, ptr*, i64*, ptr*, ptr)>(F_GROUP_LOOKUP)(
        (int32_t)g.t.size(), g.t.data(), g.ids.data(), g.n_ids.data(), g.off.data(), g.n_bags.data(), g.vec.data(), s);
  });
}

// (handles, ids, offsets, grads, now, stream)
PyObject* group_push(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Group g;
  ptr s;
  i64 now;
  if (!expects(n, 6) || !group(a[0], a[1], a[2], a[3], &g) || !integer(a[4], &now) || !address(a[5], &s)) return nullptr;
  return without_gil([&] {
    return fn<int (*)(int32_t, ptr*, ptr*, i64*, ptr*, i64*, ptr*, i64, ptr)>(F_GROUP_APPLY)(
        (int32_t)g.t.size(), g.t.data(), g.ids.data(), g.n_ids.data(), g.off.data(), g.n_bags.data(), g.vec.data(), now, s);
  });
}

// ---- operators on plain matrices: tensors as they are, on the current stream of their device ----

// The tensors of one call, in turn.  All of them have to be on one CUDA device; it is the current one while the call
// runs, and an output's version goes up, so that autograd sees that it was written (unless the call was refused).
struct Operands {
  const at::Device* device = nullptr;

  const at::Tensor* tensor(PyObject* x, const char* name) {
    if (!THPVariable_CheckExact(x)) { PyErr_Format(PyExc_TypeError, "%s: a torch.Tensor is expected, not %s", name, Py_TYPE(x)->tp_name); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(x);
    if (!t.is_cuda()) { PyErr_Format(PyExc_ValueError, "%s is not on a CUDA device (there is no CPU path)", name); return nullptr; }
    if (!device) { at_ = t.device(); device = &at_; }
    if (t.device() != at_) { PyErr_Format(PyExc_ValueError, "%s is on another device than the tensors before it", name); return nullptr; }
    if (t.is_neg()) { PyErr_Format(PyExc_ValueError, "%s is a view that negates what its memory holds: resolve_neg() it", name); return nullptr; }
    return &t;
  }

  // Rows of elements next to each other: a 2-d tensor with any distance between its rows, or a contiguous one of any shape.
  bool matrix(PyObject* x, const char* name, bool written, mono_matrix_t* m) {
    const at::Tensor* t = tensor(x, name);
    if (!t) return false;
    switch (t->scalar_type()) {
      case at::kFloat: m->type = MONO_F32; break;
      case at::kBFloat16: m->type = MONO_BF16; break;
      case at::kHalf: m->type = MONO_F16; break;
      default: PyErr_Format(PyExc_TypeError, "%s: float32, bfloat16 or float16 is expected", name); return false;
    }
    const i64 dims = t->dim();
    if (dims < 1) { PyErr_Format(PyExc_ValueError, "%s is a single number, not rows", name); return false; }
    m->cols = t->size(dims - 1);
    if (dims == 2 && (m->cols <= 1 || t->stride(1) == 1)) {
      m->rows = t->size(0);
      m->stride = m->rows > 1 ? t->stride(0) : m->cols;
    } else if (t->is_contiguous()) {
      m->rows = 1;                                         // (a single row even where it has no columns: scores of no packed rows)
      for (i64 d = 0; d + 1 < dims; ++d) m->rows *= t->size(d);
      m->stride = m->cols;
    } else {
      PyErr_Format(PyExc_ValueError, "%s: the columns of a row have to be next to each other", name);
      return false;
    }
    m->data = t->data_ptr();
    m->pad_ = 0;
    if (written) writes(*t);
    return true;
  }

  void writes(const at::Tensor& t) { written_[n_written_++] = &t; }

  bool tokens(PyObject* x, const void** data, int32_t* type, i64* n) {
    const at::Tensor* t = tensor(x, "tokens");
    if (!t) return false;
    if (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) { PyErr_SetString(PyExc_TypeError, "tokens: int32 or int64 is expected"); return false; }
    if (!t->is_contiguous()) { PyErr_SetString(PyExc_ValueError, "tokens have to be contiguous"); return false; }
    *type = t->scalar_type() == at::kInt ? MONO_I32 : MONO_I64;
    *data = t->data_ptr();
    *n = t->numel();
    return true;
  }

  // q and scales of rows that have `cols` columns
  bool packed(PyObject* q, PyObject* scales, PyObject* group, i64 cols, mono_packed_t* p) {
    i64 g;
    if (!integer(group, &g)) return false;
    if (g != 32 && g != 64 && g != 128) { PyErr_SetString(PyExc_ValueError, "group: 32, 64 or 128 is expected"); return false; }
    const at::Tensor* t = tensor(q, "q");
    mono_matrix_t s;
    if (!t || !matrix(scales, "scales", false, &s)) return false;
    const i64 bytes = (cols + 31) / 32 * 16, groups = (cols + g - 1) / g;
    if (t->scalar_type() != at::kByte) { PyErr_SetString(PyExc_TypeError, "q: uint8 is expected"); return false; }
    if (t->dim() != 2 || t->size(1) < bytes || t->stride(1) != 1) {
      PyErr_Format(PyExc_ValueError, "q: rows of at least %lld bytes next to each other are expected", (long long)bytes);
      return false;
    }
    if (s.rows != t->size(0) || s.cols < groups) {
      PyErr_Format(PyExc_ValueError, "scales: a row of at least %lld scales is expected for each row of q", (long long)groups);
      return false;
    }
    p->q = static_cast<uint8_t*>(t->data_ptr());
    p->scales = s.data;
    p->rows = t->size(0);
    p->cols = cols;
    p->q_stride = p->rows > 1 ? t->stride(0) : bytes;
    p->scale_stride = p->rows > 1 ? s.stride : groups;
    p->group = (int32_t)g;
    p->scale_type = s.type;
    return true;
  }

  template <typename C>
  PyObject* run(C&& call) {
    const c10::DeviceGuard guard(at_);
    // (through the device's interface: torch's CUDA library and headers need not be there to build this file)
    const c10::impl::VirtualGuardImpl device(at_.type());
    const ptr stream = device.getStreamNativeHandle(device.getStream(at_));
    int rc = MONO_OK;
    PyObject* const result = without_gil([&] { return rc = call(stream); });
    if (rc == MONO_OK || rc == MONO_ERR_CUDA)
      for (int k = 0; k < n_written_; ++k)
        if (!written_[k]->is_inference()) written_[k]->unsafeGetTensorImpl()->bump_version();
    return result;
  }

 private:
  at::Device at_ = at::kCPU;
  const at::Tensor* written_[2] = {};
  int n_written_ = 0;
};

bool number(PyObject* x, float* out) {
  *out = (float)PyFloat_AsDouble(x);
  return !PyErr_Occurred();
}

// (weight, tokens, out, scale, padding)
PyObject* token_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Operands o;
  mono_matrix_t weight, out;
  const void* tokens;
  int32_t type;
  i64 count, padding;
  float scale;
  if (!expects(n, 5) || !number(a[3], &scale) || !integer(a[4], &padding) || !o.matrix(a[0], "weight", false, &weight) ||
      !o.tokens(a[1], &tokens, &type, &count) || !o.matrix(a[2], "out", true, &out)) return nullptr;
  return o.run([&](ptr s) { return fn<decltype(&mono_token_rows)>(F_TOKEN_ROWS)(&weight, tokens, type, count, padding, scale, &out, s); });
}

// (grad_out, tokens, grad_weight, scale, padding, accumulate, workspace or None)
PyObject* token_rows_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Operands o;
  mono_matrix_t grad, out;
  const void* tokens;
  int32_t type;
  i64 count, padding, bytes = 0;
  float scale;
  if (!expects(n, 7) || !number(a[3], &scale) || !integer(a[4], &padding)) return nullptr;
  const int accumulate = PyObject_IsTrue(a[5]);
  if (accumulate < 0 || !o.matrix(a[0], "grad_out", false, &grad) || !o.tokens(a[1], &tokens, &type, &count) || !o.matrix(a[2], "grad_weight", true, &out)) return nullptr;
  at::Tensor made;
  ptr workspace;
  if (a[6] == Py_None) {
    const int rc = fn<decltype(&mono_token_rows_grad_workspace)>(F_TOKEN_ROWS_GRAD_WORKSPACE)(count, out.rows, out.cols, &bytes);
    if (rc) return PyLong_FromLong(rc);
    const c10::DeviceGuard guard(*o.device);
    made = at::empty({bytes}, at::TensorOptions().dtype(at::kByte).device(*o.device));
    workspace = made.data_ptr();
  } else {
    const at::Tensor* t = o.tensor(a[6], "workspace");
    if (!t) return nullptr;
    if (!t->is_contiguous()) { PyErr_SetString(PyExc_ValueError, "workspace has to be contiguous"); return nullptr; }
    workspace = t->data_ptr();
    bytes = (i64)t->nbytes();
  }
  return o.run([&](ptr s) {
    return fn<decltype(&mono_token_rows_grad)>(F_TOKEN_ROWS_GRAD)(&grad, tokens, type, count, padding, scale, accumulate, &out, workspace, bytes, s);
  });
}

// (rows, q, scales, group)
PyObject* pack_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Operands o;
  mono_matrix_t rows;
  mono_packed_t packed;
  if (!expects(n, 4) || !o.matrix(a[0], "rows", false, &rows) || !o.packed(a[1], a[2], a[3], rows.cols, &packed)) return nullptr;
  o.writes(THPVariable_Unpack(a[1]));
  o.writes(THPVariable_Unpack(a[2]));
  return o.run([&](ptr s) { return fn<decltype(&mono_pack_rows)>(F_PACK_ROWS)(&rows, &packed, s); });
}

// (q, scales, group, tokens, out, scale, padding)
PyObject* packed_token_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Operands o;
  mono_matrix_t out;
  mono_packed_t packed;
  const void* tokens;
  int32_t type;
  i64 count, padding;
  float scale;
  if (!expects(n, 7) || !number(a[5], &scale) || !integer(a[6], &padding) || !o.matrix(a[4], "out", true, &out) || !o.packed(a[0], a[1], a[2], out.cols, &packed) ||
      !o.tokens(a[3], &tokens, &type, &count)) return nullptr;
  return o.run([&](ptr s) { return fn<decltype(&mono_packed_token_rows)>(F_PACKED_TOKEN_ROWS)(&packed, tokens, type, count, padding, scale, &out, s); });
}

// (q, scales, group, x, out)
PyObject* packed_scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Operands o;
  mono_matrix_t x, out;
  mono_packed_t packed;
  if (!expects(n, 5) || !o.matrix(a[3], "x", false, &x) || !o.matrix(a[4], "out", true, &out) || !o.packed(a[0], a[1], a[2], x.cols, &packed)) return nullptr;
  return o.run([&](ptr s) { return fn<decltype(&mono_packed_scores)>(F_PACKED_SCORES)(&packed, &x, &out, s); });
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(static_cast<Method>(guarded<f>))), METH_FASTCALL, nullptr
PyMethodDef kMethods[] = {
  {"bind", FAST(bind)},
  {"lookup_pool", FAST(pull<F_LOOKUP>)},
  {"lookup_pool_noalloc", FAST(pull<F_LOOKUP_NOALLOC>)},
  {"lookup_pool_host", FAST(pull<F_LOOKUP_HOST>)},
  {"apply_grads", FAST(push<F_APPLY>)},
  {"apply_grads_host", FAST(push<F_APPLY_HOST>)},
  {"prepare_push", FAST(announce<F_PREPARE>)},
  {"group_ahead", FAST(announce<F_AHEAD>)},
  {"expire", FAST(expire)},
  {"expire_slice", FAST(expire_slice)},
  {"fence", FAST(fence)},
  {"table_pull", FAST(table_pull)},
  {"group_prepare_push", FAST(group_prepare)},
  {"group_lookup_pool", FAST(group_pull)},
  {"group_apply_grads", FAST(group_push)},
  {"token_rows", FAST(token_rows)},
  {"token_rows_grad", FAST(token_rows_grad)},
  {"pack_rows", FAST(pack_rows)},
  {"packed_token_rows", FAST(packed_token_rows)},
  {"packed_scores", FAST(packed_scores)},
  {nullptr, nullptr, 0, nullptr}
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding_native", "pointers of tensors handed to the C ABI of mono.h", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding_native() { return PyModule_Create(&kModule); }
