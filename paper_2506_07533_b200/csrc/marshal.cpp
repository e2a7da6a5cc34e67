// Argument marshalling of the calls that a serving loop makes per layer and token: torch tensors in, C ABI structs out.
// The same checks and the same C functions as through ctypes, without the three microseconds of building the structs in
// Python (norm and rotation of one token: 9.5 us per call through ctypes, 5.4 us through this).  Nothing else lives here.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include "moqae.h"

namespace {

decltype(&moqae_norm_rope) g_norm_rope = nullptr;
decltype(&moqae_paged_append) g_append = nullptr;
decltype(&moqae_paged_decode_attn) g_decode = nullptr;
decltype(&moqae_paged_prefill_attn) g_prefill = nullptr;

// What the tensors of a call have to agree on.
struct Kind {
  at::ScalarType dtype;
  int device;
};
at::ScalarType scalar_of(int dtype) { return dtype == MOQAE_DTYPE_BF16 ? at::kBFloat16 : at::kHalf; }

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// [n][heads][128] with contiguous rows.  None: no rows (*given = nullptr).  False: not such a tensor.
bool rows(PyObject* o, const Kind& kind, int64_t n, moqae_rows* out, const moqae_rows** given) {
  *given = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || !t->is_cuda() || t->get_device() != kind.device || t->scalar_type() != kind.dtype || t->dim() != 3 || t->size(2) != 128 ||
      t->size(0) != n || (t->stride(2) != 1 && t->numel() != 0) || t->size(1) > INT32_MAX)
    return false;
  out->data = t->data_ptr();
  out->token_stride = t->stride(0);
  out->head_stride = t->stride(1);
  out->n_heads = static_cast<int32_t>(t->size(1));
  *given = out;
  return true;
}

// contiguous int32 values; None: null
bool ints(PyObject* o, const Kind& kind, int64_t n, const int32_t** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || !t->is_cuda() || t->get_device() != kind.device || t->scalar_type() != at::kInt || t->numel() != n || !t->is_contiguous()) return false;
  *out = static_cast<const int32_t*>(t->data_ptr());
  return true;
}

bool space(PyObject* o, const Kind& kind, void** out, int64_t* bytes) {
  *out = nullptr;
  *bytes = 0;
  if (o == Py_None) return true;
  const at::Tensor* t = tensor(o);
  if (!t || !t->is_cuda() || t->get_device() != kind.device || !t->is_contiguous()) return false;
  *out = t->data_ptr();
  *bytes = static_cast<int64_t>(t->nbytes());
  return true;
}

int64_t tokens_of(PyObject* o) {
  const at::Tensor* t = o == Py_None ? nullptr : tensor(o);
  return t && t->dim() == 3 && t->size(0) <= INT32_MAX ? t->size(0) : -1;
}

// The interpreter is free while the library enqueues (as it is under ctypes), and held again however that ends.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  Unlocked() = default;
  Unlocked(const Unlocked&) = delete;
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F> int enqueue(F call) {
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  const Unlocked free;
  return call(stream);
}

template <typename T> T address(PyObject* o) { return static_cast<T>(PyLong_AsVoidPtr(o)); }

PyObject* answer(int rc) { return PyLong_FromLong(rc); }

// A torch exception (a tensor without storage, say) becomes an argument error; none crosses into Python.
template <typename F> PyObject* guarded(F call) {
  try {
    return answer(call());
  } catch (...) {
    return answer(MOQAE_ERR_INVALID_ARG);
  }
}

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "bind takes 4 addresses");
  g_norm_rope = reinterpret_cast<decltype(g_norm_rope)>(PyLong_AsVoidPtr(a[0]));
  g_append = reinterpret_cast<decltype(g_append)>(PyLong_AsVoidPtr(a[1]));
  g_decode = reinterpret_cast<decltype(g_decode)>(PyLong_AsVoidPtr(a[2]));
  g_prefill = reinterpret_cast<decltype(g_prefill)>(PyLong_AsVoidPtr(a[3]));
  Py_RETURN_NONE;
}

// norm_rope(rope, rope dtype or -1, rope device or -1, q, k, positions, q_out, k_out, status)
PyObject* norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 9) return PyErr_Format(PyExc_TypeError, "norm_rope takes 9 arguments");
  return guarded([&]() -> int {
    const at::Tensor* some = tensor(a[3] != Py_None ? a[3] : a[4]);
    if (!some || !some->is_cuda()) return MOQAE_ERR_INVALID_ARG;
    const int dtype = some->scalar_type() == at::kBFloat16 ? MOQAE_DTYPE_BF16 : some->scalar_type() == at::kHalf ? MOQAE_DTYPE_FP16 : -1;
    if (dtype < 0) return MOQAE_ERR_INVALID_ARG;
    const Kind kind{some->scalar_type(), some->get_device()};
    const long rope_dtype = PyLong_AsLong(a[1]), rope_device = PyLong_AsLong(a[2]);
    if ((rope_dtype >= 0 && rope_dtype != dtype) || (rope_device >= 0 && rope_device != kind.device)) return MOQAE_ERR_INVALID_ARG;
    const int64_t n = tokens_of(a[3] != Py_None ? a[3] : a[4]);
    moqae_rows r[4];
    const moqae_rows* p[4];
    const int32_t *positions, *status;
    if (n < 0 || !rows(a[3], kind, n, &r[0], &p[0]) || !rows(a[4], kind, n, &r[1], &p[1]) || !rows(a[6], kind, n, &r[2], &p[2]) ||
        !rows(a[7], kind, n, &r[3], &p[3]) || !ints(a[5], kind, n, &positions) || !ints(a[8], kind, 4, &status))
      return MOQAE_ERR_INVALID_ARG;
    const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(kind.device));
    const moqae_rope* rope = address<const moqae_rope*>(a[0]);
    return enqueue([&](void* stream) {
      return g_norm_rope(rope, dtype, p[0], p[1], p[2] ? p[2] : p[0], p[3] ? p[3] : p[1], positions, static_cast<int32_t>(n),
                         const_cast<int32_t*>(status), stream);
    });
  });
}

// append(cache, dtype, device, rope or 0, rope dtype or -1, rope device or -1, k, v, positions, seq, q, q_out)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 12) return PyErr_Format(PyExc_TypeError, "append takes 12 arguments");
  return guarded([&]() -> int {
    const int dtype = static_cast<int>(PyLong_AsLong(a[1]));
    const Kind kind{scalar_of(dtype), static_cast<int>(PyLong_AsLong(a[2]))};
    const long rope_dtype = PyLong_AsLong(a[4]), rope_device = PyLong_AsLong(a[5]);
    if ((rope_dtype >= 0 && rope_dtype != dtype) || (rope_device >= 0 && rope_device != kind.device)) return MOQAE_ERR_INVALID_ARG;
    const int64_t n = tokens_of(a[6]);
    moqae_rows r[4];
    const moqae_rows* p[4];
    const int32_t *positions, *seq;
    if (n < 0 || !rows(a[6], kind, n, &r[0], &p[0]) || !rows(a[7], kind, n, &r[1], &p[1]) || !rows(a[10], kind, n, &r[2], &p[2]) ||
        !rows(a[11], kind, n, &r[3], &p[3]) || !ints(a[8], kind, n, &positions) || !ints(a[9], kind, n, &seq) || (!p[2] && p[3]))
      return MOQAE_ERR_INVALID_ARG;
    const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(kind.device));
    const moqae_paged_cache* cache = address<const moqae_paged_cache*>(a[0]);
    const moqae_rope* rope = address<const moqae_rope*>(a[3]);
    return enqueue([&](void* stream) {
      return g_append(cache, rope, p[0], p[1], p[2], p[3] ? p[3] : p[2], positions, seq, static_cast<int32_t>(n), stream);
    });
  });
}

// decode(cache, dtype, device, batch, q, out, workspace, options or 0)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 8) return PyErr_Format(PyExc_TypeError, "decode takes 8 arguments");
  return guarded([&]() -> int {
    const Kind kind{scalar_of(static_cast<int>(PyLong_AsLong(a[1]))), static_cast<int>(PyLong_AsLong(a[2]))};
    const int64_t n = PyLong_AsLong(a[3]);
    moqae_rows r[2];
    const moqae_rows* p[2];
    void* ws;
    int64_t bytes;
    if (!rows(a[4], kind, n, &r[0], &p[0]) || !rows(a[5], kind, n, &r[1], &p[1]) || !space(a[6], kind, &ws, &bytes)) return MOQAE_ERR_INVALID_ARG;
    const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(kind.device));
    const moqae_paged_cache* cache = address<const moqae_paged_cache*>(a[0]);
    const moqae_attn_options* options = address<const moqae_attn_options*>(a[7]);
    return enqueue([&](void* stream) { return g_decode(cache, p[0], p[1], options, ws, bytes, stream); });
  });
}

// prefill(cache, dtype, device, batch, q, cu_q, out, workspace, options or 0)
PyObject* prefill(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  if (n_args != 9) return PyErr_Format(PyExc_TypeError, "prefill takes 9 arguments");
  return guarded([&]() -> int {
    const Kind kind{scalar_of(static_cast<int>(PyLong_AsLong(a[1]))), static_cast<int>(PyLong_AsLong(a[2]))};
    const int64_t batch = PyLong_AsLong(a[3]), n = tokens_of(a[4]);
    moqae_rows r[2];
    const moqae_rows* p[2];
    const int32_t* cu_q;
    void* ws;
    int64_t bytes;
    if (n < 0 || !rows(a[4], kind, n, &r[0], &p[0]) || !rows(a[6], kind, n, &r[1], &p[1]) || !ints(a[5], kind, batch + 1, &cu_q) ||
        !space(a[7], kind, &ws, &bytes))
      return MOQAE_ERR_INVALID_ARG;
    const c10::cuda::CUDAGuard guard(static_cast<c10::DeviceIndex>(kind.device));
    const moqae_paged_cache* cache = address<const moqae_paged_cache*>(a[0]);
    const moqae_attn_options* options = address<const moqae_attn_options*>(a[8]);
    return enqueue([&](void* stream) { return g_prefill(cache, p[0], cu_q, static_cast<int32_t>(n), p[1], options, ws, bytes, stream); });
  });
}

PyMethodDef kMethods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, "addresses of the C functions"},
    {"norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(norm_rope)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(append)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode)), METH_FASTCALL, nullptr},
    {"prefill", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(prefill)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python whose inlined accessors are in here (build.marshal_key()); binding.py compares it with its own.
PyMODINIT_FUNC PyInit__marshal() {
  PyObject* m = PyModule_Create(&kModule);
  if (m && PyModule_AddStringConstant(m, "built_for", MOQAE_BUILT_FOR) != 0) Py_CLEAR(m);
  return m;
}
