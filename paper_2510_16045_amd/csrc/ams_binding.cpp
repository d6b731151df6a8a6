// The calls of the Linear, and of the KV cache, from Python in one native function each: what `ams_linear` and its variants in __init__.py check of their
// tensors, the current stream and the call of libams.so, with the interpreter left out.  An eager call of 256 x 768 is bound
// by this (the kernel takes 2.3 us).  It takes plain tensors and integers and answers None to everything else, and to a call that the library
// refuses: the caller then goes the long way, which raises what there is to raise.
//
// It is not linked to libams.so but given the addresses of the entry points of the one that the package has loaded: a path or a
// name in the dynamic section could find another tree's.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>

#include <cxxabi.h>
#include <math.h>
#include <string.h>

#include "../../include/ams.h"

namespace {

// A plain strided tensor on the current GPU (the kernels run there, in the order of its stream): no subclass, no wrapper of a
// transformation, no view that needs resolving.
const at::Tensor* plain(PyObject* o, c10::ScalarType type, c10::DeviceIndex device, bool contiguous = true) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined()) return nullptr;
  constexpr auto ordinary =
      c10::DispatchKeySet({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
  if ((t.key_set().raw_repr() & ~ordinary.raw_repr()) != 0 || !t.is_cuda() || t.get_device() != device || t.scalar_type() != type || (contiguous && !t.is_contiguous())) return nullptr;
  return &t;
}

bool whole(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  int overflow = 0;
  *v = PyLong_AsLongLongAndOverflow(o, &overflow);
  return !overflow;
}

enum Entry { kPlain, kWorkspace, kStatic, kGrouped };

// The entry points that are called, in the order in which bind() takes them.
struct Library {
  decltype(&ams_packed_bytes) packed_bytes;
  decltype(&ams_group_scales_count) group_scales_count;
  decltype(&ams_linear) linear;
  decltype(&ams_linear_ws) linear_ws;
  decltype(&ams_linear_static_ws) linear_static_ws;
  decltype(&ams_linear_grouped) linear_grouped;
} lib;

// bind(address of each entry point of Library)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* at[6];
  if (n != 6) return PyErr_Format(PyExc_TypeError, "bind takes 6 addresses");
  for (int i = 0; i < 6; i++)
    if (!(at[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
  static_assert(sizeof lib == sizeof at, "one address for each");
  memcpy(&lib, at, sizeof lib);
  Py_RETURN_NONE;
}

// What a call of the library takes.
struct Call {
  int64_t entry, M, N, K, group;
  int fmt;
  const void* w;
  const uint16_t *s, *x;
  uint16_t* y;
  void* ws;
  size_t ws_bytes;
  void* st;
};

// linear's arguments, checked; false for those that are not taken.
bool arguments(PyObject* const* a, Py_ssize_t n, Call* c) try {
  int64_t entry = 0, N = 0, fmt = 0, group = 0;
  if (!lib.linear || n != 8 || !whole(a[0], &entry) || !whole(a[4], &N) || !whole(a[5], &fmt)) return false;
  if (at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) return false;
  const auto stream = c10::hip::getCurrentHIPStream();  // of the current device
  const c10::DeviceIndex dev = stream.device_index();
  const at::Tensor *W = plain(a[1], at::kByte, dev), *scales = plain(a[2], at::kHalf, dev), *X = plain(a[3], at::kHalf, dev), *out = plain(a[6], at::kHalf, dev);
  if (!W || !scales || !X || !out || X->dim() != 2 || fmt < 0 || fmt > 0x7FFF) return false;
  const int64_t M = X->size(0), K = X->size(1);
  if (M > AMS_MAX_M || N <= 0 || N > (1 << 24) || out->numel() < M * N) return false;
  size_t bytes = 0, count = 0;
  if (lib.packed_bytes((int)fmt, N, K, &bytes) != AMS_OK || (size_t)W->numel() != bytes) return false;
  const at::Tensor* workspace = nullptr;
  if (entry == kGrouped) {
    if (!whole(a[7], &group) || lib.group_scales_count((int)fmt, N, K, group, &count) != AMS_OK || (size_t)scales->numel() != count) return false;
  } else {
    if (scales->numel() != N) return false;
    if (entry == kWorkspace && a[7] != Py_None && !(workspace = plain(a[7], at::kByte, dev))) return false;
  }
  *c = {entry, M, N, K, group, (int)fmt, W->const_data_ptr(), (const uint16_t*)scales->const_data_ptr(), (const uint16_t*)X->const_data_ptr(), (uint16_t*)out->data_ptr(),
        workspace ? workspace->data_ptr() : nullptr, workspace ? (size_t)workspace->numel() : 0, (void*)stream.stream()};
  return true;
} catch (...) {  // torch's own checks; the long way meets them again
  return false;
}

int call(const Call& c) {
  switch (c.entry) {
    case kPlain: return lib.linear(c.w, c.s, c.x, c.y, (int)c.M, c.N, c.K, c.fmt, c.st);
    case kWorkspace: return lib.linear_ws(c.w, c.s, c.x, c.y, (int)c.M, c.N, c.K, c.fmt, c.ws, c.ws_bytes, c.st);
    case kStatic: return lib.linear_static_ws(c.w, c.s, c.x, c.y, (int)c.M, c.N, c.K, c.fmt, c.st);
    case kGrouped: return lib.linear_grouped(c.w, c.s, c.group, c.x, c.y, (int)c.M, c.N, c.K, c.fmt, c.st);
  }
  return -1;
}

// The call, with the interpreter's lock given up for it.  It is taken again outside of every try block and destructor: where the
// interpreter ends meanwhile, pthread_exit ends a daemon thread there by unwinding its stack, and a handler that stops that, or
// a destructor that it would leave, aborts the process.
template <typename C>
int call_unlocked(const C& c) {
  PyThreadState* const state = PyEval_SaveThread();
  int rc = -1;
  try {
    rc = call(c);
  } catch (const abi::__forced_unwind&) {
    throw;
  } catch (...) {
  }
  PyEval_RestoreThread(state);
  return rc;
}

// linear(entry, W_packed, scales, X, N, fmt, out, workspace or scale_group): out, or None.
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Call c;
  if (!arguments(a, n, &c) || call_unlocked(c) != AMS_OK) Py_RETURN_NONE;
  Py_INCREF(a[6]);
  return a[6];
}

// ---- the 4-bit KV cache -------------------------------------------------------------------------------
struct KvLibrary {
  decltype(&ams_kv_block_bytes) block_bytes;
  decltype(&ams_kv_write) write;
  decltype(&ams_kv_read) read;
  decltype(&ams_kv_attention) attention;
} kv_lib;

// bind_kv(address of each entry point of KvLibrary)
PyObject* bind_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  void* at[4];
  if (n != 4) return PyErr_Format(PyExc_TypeError, "bind_kv takes 4 addresses");
  for (int i = 0; i < 4; i++)
    if (!(at[i] = PyLong_AsVoidPtr(a[i]))) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "no address");
  static_assert(sizeof kv_lib == sizeof at, "one address for each");
  memcpy(&kv_lib, at, sizeof kv_lib);
  Py_RETURN_NONE;
}

enum KvEntry { kKvWrite, kKvRead, kKvAttention };

struct KvCall {
  int64_t entry;
  ams_kv_cache cache;
  void *first, *second;  // q and out, or k and v
  int64_t rows, strides[4];
  float* lse;
  int64_t lse_stride, window, most;
  int heads, causal;
  float scale;
  void* ws;
  size_t ws_bytes;
  void* st;
};

// [rows, heads, dim] in fp16 with the channels of a head side by side
const at::Tensor* rows_of(PyObject* o, int64_t heads, int64_t dim, c10::DeviceIndex device, int64_t* strides) {
  const at::Tensor* const t = plain(o, at::kHalf, device, false);
  if (!t || t->dim() != 3 || (heads && t->size(1) != heads) || (dim && t->size(2) != dim) || t->stride(2) != 1) return nullptr;
  strides[0] = t->stride(0), strides[1] = t->stride(1);
  return t;
}

// The arguments of the three calls, checked; false for those that are not taken.
//   kv(entry, cache, block_table, kv_lens, scale_group, q_starts or None, ...)
//     kKvWrite: k, v;  kKvRead: head_dim, out k, out v;  kKvAttention: q, out, max_q_len or None, softmax_scale or None, causal, window, workspace or None, lse or None
bool kv_arguments(PyObject* const* a, Py_ssize_t n, KvCall* c) try {
  *c = {};
  int64_t group = 0, dim = 0;
  if (!kv_lib.attention || n < 8 || !whole(a[0], &c->entry) || !whole(a[4], &group) || n != (c->entry == kKvWrite ? 8 : c->entry == kKvRead ? 9 : 14)) return false;
  if (at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) return false;
  const auto stream = c10::hip::getCurrentHIPStream();  // of the current device
  const c10::DeviceIndex dev = stream.device_index();
  const at::Tensor *cache = plain(a[1], at::kByte, dev), *table = plain(a[2], at::kInt, dev, false), *lens = plain(a[3], at::kInt, dev);
  if (!cache || !table || !lens || cache->dim() != 3 || table->dim() != 2 || lens->dim() != 1 || group <= 0 || group > 1024) return false;
  const int64_t batch = table->size(0), width = table->size(1), kv_heads = cache->size(1);
  if (lens->size(0) != batch || (width > 1 && table->stride(1) != 1) || width > 0x7FFFFFFF || batch > AMS_KV_MAX_BATCH || kv_heads > AMS_KV_MAX_HEADS) return false;
  const at::Tensor* starts = nullptr;
  if (a[5] != Py_None && (!(starts = plain(a[5], at::kInt, dev)) || starts->dim() != 1 || starts->size(0) != batch + 1)) return false;
  const at::Tensor *x = nullptr, *y = nullptr;
  if (c->entry == kKvAttention) {
    x = rows_of(a[6], 0, 0, dev, c->strides);
    if (!x || !(y = rows_of(a[7], x->size(1), x->size(2), dev, c->strides + 2))) return false;
    dim = x->size(2);
    c->heads = (int)x->size(1);
    double scale = 0;
    if (a[9] == Py_None)
      scale = 1.0 / sqrt((double)dim);
    else if (PyFloat_CheckExact(a[9]))
      scale = PyFloat_AS_DOUBLE(a[9]);
    else
      return false;
    c->scale = (float)scale;
    if ((a[8] != Py_None && !whole(a[8], &c->most)) || !PyBool_Check(a[10]) || !whole(a[11], &c->window)) return false;
    c->causal = a[10] == Py_True;
    if (a[12] != Py_None) {
      const at::Tensor* const ws = plain(a[12], at::kByte, dev);
      if (!ws) return false;
      c->ws = ws->data_ptr(), c->ws_bytes = (size_t)ws->numel();
    }
    if (a[13] != Py_None) {
      const at::Tensor* const lse = plain(a[13], at::kFloat, dev, false);
      if (!lse || lse->dim() != 2 || lse->size(0) != x->size(0) || lse->size(1) != x->size(1) || (lse->size(1) > 1 && lse->stride(1) != 1)) return false;
      c->lse = (float*)lse->data_ptr(), c->lse_stride = lse->stride(0);
    }
  } else {
    const int first = c->entry == kKvWrite ? 6 : 7;
    if (c->entry == kKvRead && !whole(a[6], &dim)) return false;
    x = rows_of(a[first], kv_heads, dim, dev, c->strides);
    if (!x || !(y = rows_of(a[first + 1], kv_heads, x->size(2), dev, c->strides + 2))) return false;
    dim = x->size(2);
  }
  if (x->size(0) != y->size(0) || dim > 1024) return false;
  size_t sixteen = 0;  // bytes of 16 tokens
  if (kv_lib.block_bytes((int)dim, 16, (int)group, &sixteen) != AMS_OK) return false;
  const int64_t token = (int64_t)sixteen / 16, page = cache->size(2) / token;
  if (page * token != cache->size(2) || page > AMS_KV_MAX_PAGE) return false;
  c->cache = {cache->data_ptr(), (const int32_t*)table->const_data_ptr(), (const int32_t*)lens->const_data_ptr(), starts ? (const int32_t*)starts->const_data_ptr() : nullptr, cache->size(0),
              batch > 1 ? table->stride(0) : width, (int32_t)width, (int32_t)batch, (int32_t)kv_heads, (int32_t)dim, (int32_t)page, (int32_t)group};
  c->first = x->data_ptr(), c->second = y->data_ptr(), c->rows = x->size(0), c->st = (void*)stream.stream();
  return true;
} catch (...) {  // torch's own checks; the long way meets them again
  return false;
}

int call(const KvCall& c) {
  switch (c.entry) {
    case kKvWrite: return kv_lib.write(&c.cache, (const uint16_t*)c.first, (const uint16_t*)c.second, c.rows, c.strides[0], c.strides[1], c.strides[2], c.strides[3], c.st);
    case kKvRead: return kv_lib.read(&c.cache, (uint16_t*)c.first, (uint16_t*)c.second, c.rows, c.strides[0], c.strides[1], c.strides[2], c.strides[3], c.st);
    case kKvAttention:
      return kv_lib.attention(&c.cache, (const uint16_t*)c.first, (uint16_t*)c.second, c.lse, c.rows, c.heads, c.strides[0], c.strides[1], c.strides[2], c.strides[3], c.lse_stride, c.scale, c.causal, c.window,
                              c.most, c.ws, c.ws_bytes, c.st);
  }
  return -1;
}

// kv(...): True, or None for a call that was not taken (nothing is done then).
PyObject* kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  KvCall c;
  if (!kv_arguments(a, n, &c) || call_unlocked(c) != AMS_OK) Py_RETURN_NONE;
  Py_RETURN_TRUE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
                         {"bind_kv", (PyCFunction)(void (*)(void))bind_kv, METH_FASTCALL, nullptr},
                         {"kv", (PyCFunction)(void (*)(void))kv, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  PyObject* const m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "BUILT_FOR", AMS_TORCH) != 0) {  // whose tensors it reads
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
