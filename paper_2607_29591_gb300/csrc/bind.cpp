// The small calls' way from torch tensors to the C ABI.  A single token's reskv_rope,
// reskv_paged_append or reskv_paged_gather is bound by the host: reading the tensors
// attribute by attribute from Python took 4 of a call's 6.7 us, here the whole call
// takes 2.2 (append 7.3 -> 2.3, gather 4.9 -> 2.0).  Each function looks its tensors
// over, fills the ABI's structs and calls.  It returns the call's status, or -1 without
// having called where an argument is not of the plain kind; the caller's general path
// then takes the call or says what is wrong with it.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <climits>

#include "reskv.h"

namespace {

struct {
  decltype(&reskv_rope) rope;
  decltype(&reskv_paged_append) append;
  decltype(&reskv_paged_gather) gather;
  PyObject* current_stream;       // torch's: device index -> address
} g{};

const at::Tensor* tensor(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() ? &t : nullptr;
}

bool dtype_of(const at::Tensor& t, int32_t* code) {
  switch (t.scalar_type()) {
    case at::kBFloat16: *code = RESKV_BF16; return true;
    case at::kHalf: *code = RESKV_F16; return true;
    case at::kFloat: *code = RESKV_F32; return true;
    default: return false;
  }
}

// [tokens, heads, dim] with neighbouring elements in a row; heads < 0: any
bool heads_of(PyObject* o, int64_t tokens, int64_t heads, int64_t dim, reskv_heads* h) {
  const at::Tensor* t = tensor(o);
  if (!t || t->dim() != 3 || t->stride(2) != 1 || t->size(0) != tokens || t->size(2) != dim || t->size(1) > INT_MAX ||
      (heads >= 0 && t->size(1) != heads) || !dtype_of(*t, &h->dtype))
    return false;
  h->data = t->data_ptr();
  h->token_stride = t->stride(0);
  h->head_stride = t->stride(1);
  h->n_heads = int32_t(t->size(1));
  return true;
}

bool ints_of(PyObject* o, int64_t n, const int32_t** out) {
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != at::kInt || t->numel() != n || !t->is_contiguous()) return false;
  *out = static_cast<const int32_t*>(t->data_ptr());
  return true;
}

bool rotation_of(PyObject* table, PyObject* interleaved, reskv_rotation* r) {
  const at::Tensor* t = tensor(table);
  if (!t || t->dim() != 3 || t->size(2) != 2 || t->scalar_type() != at::kFloat || !t->is_contiguous() ||
      t->size(1) > INT_MAX / 2)
    return false;
  const int yes = PyObject_IsTrue(interleaved);
  if (yes < 0) return false;
  r->table = static_cast<const float*>(t->data_ptr());
  r->n_positions = t->size(0);
  r->rot_dim = int32_t(2 * t->size(1));
  r->interleaved = yes;
  return true;
}

// rows [batch, n_kv_heads, n, head_dim]
bool rows_of(PyObject* o, const reskv_paged_kv& kv, int64_t n, reskv_rows* r) {
  const at::Tensor* t = tensor(o);
  if (!t || t->dim() != 4 || t->size(0) != kv.batch || t->size(1) != kv.n_kv_heads || t->size(2) != n ||
      t->size(3) != kv.head_dim || t->stride(3) != 1 || !dtype_of(*t, &r->dtype))
    return false;
  r->data = t->data_ptr();
  r->batch_stride = t->stride(0);
  r->head_stride = t->stride(1);
  r->token_stride = t->stride(2);
  return true;
}

// An address, None for torch's current stream of the device, or a stream object.
bool stream_of(PyObject* o, int device, void** out) {
  PyObject* address = nullptr;
  if (o == Py_None) {
    PyObject* index = PyLong_FromLong(device);
    if (!index) return false;
    address = PyObject_CallOneArg(g.current_stream, index);
    Py_DECREF(index);
  } else if (PyLong_Check(o)) {
    address = Py_NewRef(o);
  } else {
    address = PyObject_GetAttrString(o, "cuda_stream");
  }
  if (!address) return false;
  *out = PyLong_AsVoidPtr(address);
  Py_DECREF(address);
  return !PyErr_Occurred();
}

// `body` returns the status, -1 where the general path is to take the call.
template <typename F>
PyObject* guarded(F body) {
  int st = -1;
  try {
    st = body();
  } catch (...) {
  }
  PyErr_Clear();
  return PyLong_FromLong(st);
}

template <typename F>
int without_gil(F call) {
  PyThreadState* held = PyEval_SaveThread();
  const int st = call();
  PyEval_RestoreThread(held);
  return st;
}

// addresses of the three entries, torch's current-stream function
PyObject* setup(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) return PyErr_Format(PyExc_TypeError, "setup takes 4 arguments");
  void* f[3];
  for (int i = 0; i < 3; ++i) {
    f[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  g.rope = reinterpret_cast<decltype(g.rope)>(f[0]);
  g.append = reinterpret_cast<decltype(g.append)>(f[1]);
  g.gather = reinterpret_cast<decltype(g.gather)>(f[2]);
  g.current_stream = Py_NewRef(a[3]);
  Py_RETURN_NONE;
}

// q, q_out, positions, table, k, k_out, interleaved, backward, status, stream
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 10 || !g.rope) return -1;
    const at::Tensor* q = tensor(a[0]);
    if (!q || q->dim() != 3 || q->size(2) > INT_MAX) return -1;
    const int64_t tokens = q->size(0), dim = q->size(2);
    reskv_heads x[2], y[2];
    reskv_rotation rot;
    const int32_t *positions, *status = nullptr;
    void* stream;
    const bool two = a[4] != Py_None;
    const int backward = PyObject_IsTrue(a[7]);
    if (backward < 0 || two != (a[5] != Py_None) || !heads_of(a[0], tokens, -1, dim, &x[0]) ||
        !heads_of(a[1], tokens, x[0].n_heads, dim, &y[0]) ||
        (two && (!heads_of(a[4], tokens, -1, dim, &x[1]) || !heads_of(a[5], tokens, x[1].n_heads, dim, &y[1]))) ||
        !ints_of(a[2], tokens, &positions) || !rotation_of(a[3], a[6], &rot) ||
        (a[8] != Py_None && !ints_of(a[8], 1, &status)) || !stream_of(a[9], q->get_device(), &stream))
      return -1;
    return without_gil([&] {
      return int(g.rope(&rot, positions, tokens, int32_t(dim), two ? 2 : 1, x, y, backward,
                        reinterpret_cast<uint32_t*>(const_cast<int32_t*>(status)), stream));
    });
  });
}

// address of a reskv_paged_kv, k, v, seqs, positions, table, interleaved, q, q_out, stream
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 10 || !g.append) return -1;
    const auto* kv = static_cast<const reskv_paged_kv*>(PyLong_AsVoidPtr(a[0]));
    const at::Tensor* k = tensor(a[1]);
    if (!kv || !k || k->dim() != 3) return -1;
    const int64_t tokens = k->size(0);
    reskv_heads kh, vh, qh, oh;
    reskv_rotation rot;
    const int32_t *seqs, *positions;
    void* stream;
    const bool turns = a[5] != Py_None, with_q = a[7] != Py_None;
    if (with_q != (a[8] != Py_None) || !heads_of(a[1], tokens, kv->n_kv_heads, kv->head_dim, &kh) ||
        !heads_of(a[2], tokens, kv->n_kv_heads, kv->head_dim, &vh) || !ints_of(a[3], tokens, &seqs) ||
        !ints_of(a[4], tokens, &positions) || (turns && !rotation_of(a[5], a[6], &rot)) ||
        (with_q && (!heads_of(a[7], tokens, -1, kv->head_dim, &qh) || !heads_of(a[8], tokens, qh.n_heads, kv->head_dim, &oh))) ||
        !stream_of(a[9], k->get_device(), &stream))
      return -1;
    return without_gil([&] {
      return int(g.append(kv, tokens, seqs, positions, turns ? &rot : nullptr, &kh, &vh, with_q ? &qh : nullptr,
                          with_q ? &oh : nullptr, stream));
    });
  });
}

// address of a reskv_paged_kv, lens, k_out, v_out, starts, stream, a tensor of the cache's device
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded([&]() -> int {
    if (n != 7 || !g.gather) return -1;
    const auto* kv = static_cast<const reskv_paged_kv*>(PyLong_AsVoidPtr(a[0]));
    const bool with_k = a[2] != Py_None, with_v = a[3] != Py_None;
    const at::Tensor *first = tensor(with_k ? a[2] : a[3]), *pages = tensor(a[6]);
    if (!kv || !first || !pages || first->dim() != 4) return -1;
    const int64_t rows = first->size(2);
    reskv_rows k, v;
    const int32_t *lens, *starts = nullptr;
    void* stream;
    if (!ints_of(a[1], kv->batch, &lens) || (with_k && !rows_of(a[2], *kv, rows, &k)) ||
        (with_v && !rows_of(a[3], *kv, rows, &v)) || (a[4] != Py_None && !ints_of(a[4], kv->batch, &starts)) ||
        !stream_of(a[5], pages->get_device(), &stream))
      return -1;
    return without_gil([&] {
      return int(g.gather(kv, starts, lens, rows, with_k ? &k : nullptr, with_v ? &v : nullptr, stream));
    });
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {method<setup>("setup"), method<rope>("rope"), method<append>("append"), method<gather>("gather"), {}};
PyModuleDef module{PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind() { return PyModule_Create(&module); }
