// The paged cache's calls for torch tensors: what binding.py does for the other calls in Python -- is this an int32 array, is it
// long enough, is it on the cache's device -- and the call itself.  Decoding makes these calls once a layer and token; asked from
// Python the questions take 3 us a call, as long as the launch behind them (6.4 us in all), asked here 0.3.
// No device work of its own, nothing kept between calls.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/lightkv.h"

#include <stdexcept>
#include <string>

namespace {

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };

// The descriptor of a Pages object (its address) and the index of its device.
struct Cache {
  const lightkv_pages *p;
  int64_t device;
};

Cache cache_of(PyObject *address, PyObject *device) {
  Cache c{static_cast<const lightkv_pages *>(PyLong_AsVoidPtr(address)), PyLong_AsLongLong(device)};
  if (PyErr_Occurred()) throw Refused("descriptor");
  return c;
}

const at::Tensor &tensor_of(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": a tensor expected");
  return THPVariable_Unpack(o);
}

bool on_device(const at::Tensor &t, const Cache &c) { return t.is_cuda() && t.get_device() == c.device; }

// An int32 array of at least n entries on the cache's device; None is NULL where it may be.
int32_t *ints(PyObject *o, int64_t n, const Cache &c, const char *what, bool optional = false) {
  if (optional && o == Py_None) return nullptr;
  const at::Tensor &t = tensor_of(o, what);
  if (t.scalar_type() != at::kInt || !on_device(t, c) || t.numel() < n || !t.is_contiguous())
    throw Refused(std::string(what) + ": contiguous int32 of at least " + std::to_string(n) + " entries on the table's device");
  return static_cast<int32_t *>(t.data_ptr());
}

struct Rows { void *at = nullptr; int64_t tok = 0, head = 0, n = 0; };

// Rows [n or more, heads, head_dim] (or [.., heads * head_dim]).
Rows rows(PyObject *o, int64_t heads, int64_t n, const Cache &c, const char *what, bool optional = false) {
  if (optional && o == Py_None) return Rows{};
  const at::Tensor &t = tensor_of(o, what);
  const int64_t d = c.p->head_dim;
  const bool flat = t.dim() == 2 && t.size(1) == heads * d, split = t.dim() == 3 && t.size(1) == heads && t.size(2) == d;
  if (t.scalar_type() != (c.p->dtype == LIGHTKV_BF16 ? at::kBFloat16 : at::kFloat) || !on_device(t, c) || !(flat || split) || t.size(0) < n || t.stride(-1) != 1)
    throw Refused(std::string(what) + ": " + (c.p->dtype == LIGHTKV_BF16 ? "bfloat16" : "float32") + " [" + std::to_string(n) + " or more, " + std::to_string(heads) + ", " + std::to_string(d) +
                  "] with contiguous elements on the table's device");
  return Rows{t.data_ptr(), t.stride(0), flat ? d : t.stride(1), t.size(0)};
}

void *stream_of(PyObject *o) {
  void *s = PyLong_AsVoidPtr(o);
  if (PyErr_Occurred()) throw Refused("stream");
  return s;
}

// Runs `body` (which returns a lightkv_status) with every C++ exception turned into a ValueError.
template <typename Body> PyObject *guarded(Py_ssize_t have, Py_ssize_t want, Body body) {
  try {
    if (have != want) throw Refused("number of arguments");
    return PyLong_FromLong(body());
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    return nullptr;
  }
}

template <typename Call> long without_lock(Call call) {
  int st;
  Py_BEGIN_ALLOW_THREADS
  st = call();
  Py_END_ALLOW_THREADS
  return st;
}

// (pages, device, cu_new, seq_lens, free_pages, free_count, seq_lens_out, free_count_out, slots, status, stream)
PyObject *page_alloc(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 11, [&] {
    const Cache c = cache_of(a[0], a[1]);
    const int64_t n = c.p->batch;
    const int32_t *cu = ints(a[2], n + 1, c, "cu_new"), *lens = ints(a[3], n, c, "seq_lens"), *pages = ints(a[4], c.p->n_pages, c, "free_pages"), *count = ints(a[5], 1, c, "free_count");
    int32_t *lens_out = ints(a[6], n, c, "seq_lens_out"), *count_out = ints(a[7], 1, c, "free_count_out"), *slots = ints(a[8], 0, c, "slots"), *status = ints(a[9], n, c, "status", true);
    const int64_t slot_rows = tensor_of(a[8], "slots").numel();
    void *s = stream_of(a[10]);
    return without_lock([&] { return lightkv_page_alloc(c.p, cu, lens, pages, count, lens_out, count_out, slots, slot_rows, status, s); });
  });
}

// (pages, device, done, seq_lens, free_pages, free_count, seq_lens_out, free_count_out, stream)
PyObject *page_free(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 9, [&] {
    const Cache c = cache_of(a[0], a[1]);
    const int64_t n = c.p->batch;
    const int32_t *done = ints(a[2], n, c, "done"), *lens = ints(a[3], n, c, "seq_lens"), *count = ints(a[5], 1, c, "free_count");
    int32_t *pages = ints(a[4], c.p->n_pages, c, "free_pages"), *lens_out = ints(a[6], n, c, "seq_lens_out"), *count_out = ints(a[7], 1, c, "free_count_out");
    void *s = stream_of(a[8]);
    return without_lock([&] { return lightkv_page_free(c.p, done, lens, pages, count, lens_out, count_out, s); });
  });
}

// (pages, device, slots, K, V, cu_new, stream): as many rows as the shortest of slots, K and V has
PyObject *page_write(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 7, [&] {
    const Cache c = cache_of(a[0], a[1]);
    const int32_t *slots = ints(a[2], 0, c, "slots"), *cu = ints(a[5], (int64_t)c.p->batch + 1, c, "cu_new", true);
    const Rows k = rows(a[3], c.p->kv_heads, 0, c, "K", true), v = rows(a[4], c.p->kv_heads, 0, c, "V", true);
    int64_t n = tensor_of(a[2], "slots").numel();
    if (a[3] != Py_None && k.n < n) n = k.n;
    if (a[4] != Py_None && v.n < n) n = v.n;
    if (n == 0) return (long)LIGHTKV_OK;
    void *s = stream_of(a[6]);
    return without_lock([&] { return lightkv_page_write(c.p, cu, slots, n, k.at, k.tok, k.head, v.at, v.tok, v.head, s); });
  });
}

// (pages, device, seq_lens, Q, out, ws, lse, softmax_scale, max_seq_tokens, stream)
PyObject *page_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args) {
  return guarded(n_args, 10, [&] {
    const Cache c = cache_of(a[0], a[1]);
    const int64_t n = c.p->batch, heads = c.p->heads;
    const double scale = PyFloat_AsDouble(a[7]);
    const long bound = PyLong_AsLong(a[8]);
    if (PyErr_Occurred()) throw Refused("softmax_scale, max_seq_tokens: numbers expected");
    if (bound < INT32_MIN || bound > INT32_MAX) throw Refused("max_seq_tokens: beyond 32 bits");
    // (zero stands for 1 / sqrt(head_dim))
    if (scale != 0 && (float)scale == 0) throw Refused("softmax_scale: too small for 32 bits");
    const int32_t *lens = ints(a[2], n, c, "seq_lens");
    const Rows q = rows(a[3], heads, n, c, "Q"), out = rows(a[4], heads, n, c, "out");
    const at::Tensor &ws = tensor_of(a[5], "ws");
    if (!on_device(ws, c) || !ws.is_contiguous()) throw Refused("ws: contiguous memory on the table's device");
    float *lse = nullptr;
    if (a[6] != Py_None) {
      const at::Tensor &t = tensor_of(a[6], "lse");
      if (t.scalar_type() != at::kFloat || !on_device(t, c) || t.numel() < heads * n || !t.is_contiguous()) throw Refused("lse: contiguous float32 [heads, batch] on the table's device");
      lse = static_cast<float *>(t.data_ptr());
    }
    void *s = stream_of(a[9]), *ws_at = ws.data_ptr();
    const size_t ws_bytes = ws.nbytes();
    return without_lock([&] {
      return lightkv_page_attention(c.p, lens, (int32_t)bound, q.at, q.tok, q.head, (float)scale, out.at, out.tok, out.head, lse, ws_at, ws_bytes, s);
    });
  });
}

template <typename F> PyCFunction as_c(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef METHODS[] = {
    {"page_alloc", as_c(page_alloc), METH_FASTCALL, nullptr},
    {"page_free", as_c(page_free), METH_FASTCALL, nullptr},
    {"page_write", as_c(page_write), METH_FASTCALL, nullptr},
    {"page_attention", as_c(page_attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_lk_pages", "Calls of the paged cache on torch tensors; each returns a lightkv_status.", -1, METHODS};

}  // namespace

PyMODINIT_FUNC PyInit__lk_pages() { return PyModule_Create(&MODULE); }
