// The binding's calls on tensors (grid.py): what they are given is looked at and
// put into the C interface's structures here, a tensor's type, device, shape and
// address in a few nanoseconds each.  The same in Python, with 50 ns for each of
// them and a call by ctypes, took 1.1 to 5.3 us of a call, as much as the launch.
//
// A tensor that does not fit is an AssertionError, as in grid.py; what the
// library itself refuses comes back as its code.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>

#include "../../include/grid.h"

namespace {

// The library's entry points, given by grid.py: the library that it has loaded.
struct Library {
  decltype(&grid_kv_append) kv_append;
  decltype(&grid_kv_append_tree) kv_append_tree;
  decltype(&grid_kv_attend) kv_attend;
  decltype(&grid_kv_attend_tree) kv_attend_tree;
  decltype(&grid_kv_compact) kv_compact;
  decltype(&grid_kv_copy) kv_copy;
  decltype(&grid_tree_plan) tree_plan;
  decltype(&grid_tree_accept) tree_accept;
  decltype(&grid_sample) sample;
  decltype(&grid_pages_update) pages_update;
} lib;

// What grid.py packs of a PagedKV ("Piiiii").
struct Cache {
  const grid_kv* kv;
  int heads, kv_heads, D, f16, device;
};

// The arguments of one call.  The first that does not fit sets the error; all later looks are then in vain.
struct Look {
  bool ok = true;
  int device = -1;

  void* no(const char* why) {
    if (ok) PyErr_SetString(PyExc_AssertionError, why);
    ok = false;
    return nullptr;
  }
  const at::Tensor* tensor(PyObject* o) {
    if (!ok) return nullptr;
    if (!THPVariable_Check(o)) return no("a tensor expected"), nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device) return no("a tensor on the current device (the handle's) expected"), nullptr;
    return &t;
  }
  // A tensor [n], or [n, m] where m is given, in one piece; None gives NULL where `some` is false
  void* dense(PyObject* o, at::ScalarType type, int64_t n, int64_t m, bool some) {
    if (!ok || (o == Py_None && !some)) return nullptr;
    const at::Tensor* t = tensor(o);
    if (!t) return nullptr;
    if (t->scalar_type() != type) return no(type == at::kInt ? "an int32 tensor expected" : "a tensor of another type expected");
    if (t->dim() != (m < 0 ? 1 : 2) || t->size(0) != n || (m >= 0 && t->size(1) != m) || !t->is_contiguous()) {
      if (m < 0)
        PyErr_Format(PyExc_AssertionError, "a contiguous tensor [%lld] expected", (long long)n);
      else
        PyErr_Format(PyExc_AssertionError, "a contiguous tensor [%lld, %lld] expected", (long long)n, (long long)m);
      ok = false;
      return nullptr;
    }
    return t->data_ptr();
  }
  int32_t* ints(PyObject* o, int64_t n, bool some = true) { return (int32_t*)dense(o, at::kInt, n, -1, some); }
  float* floats(PyObject* o, int64_t n, bool some = true) { return (float*)dense(o, at::kFloat, n, -1, some); }
  int32_t* ints2(PyObject* o, int64_t n, int64_t m) { return (int32_t*)dense(o, at::kInt, n, m, true); }
  float* floats2(PyObject* o, int64_t n, int64_t m, bool some = true) { return (float*)dense(o, at::kFloat, n, m, some); }
  // Rows of n contiguous values; their distance
  void* rows(PyObject* o, at::ScalarType type, int64_t B, int64_t n, int64_t* stride) {
    const at::Tensor* t = tensor(o);
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->dim() != 2 || t->size(0) != B || t->size(1) != n || (t->stride(1) != 1 && n != 1)) {
      if (ok) PyErr_Format(PyExc_AssertionError, "a tensor [%lld, %lld] of another type or shape expected, its rows contiguous", (long long)B, (long long)n);
      ok = false;
      return nullptr;
    }
    *stride = t->stride(0);
    return t->data_ptr();
  }
  // Sizes of the first axes, which the others are looked at by
  int64_t size(PyObject* o, int axis, int dims) {
    const at::Tensor* t = tensor(o);
    if (!t) return 0;
    if (t->dim() != dims) return no(dims == 1 ? "a tensor of one axis expected" : dims == 2 ? "a tensor of two axes expected" : "a tensor of three axes expected"), 0;
    return t->size(axis);
  }
  void int32(int64_t x) {
    if (x > INT32_MAX) no("sizes of up to 2^31 - 1 expected");
  }
  void on(int dev) {
    device = dev;
    if (ok && c10::cuda::current_device() != dev) no("the handle is on another device than the current one");
  }
  void on_current() { device = c10::cuda::current_device(); }
  void* stream(PyObject* o) {
    if (!ok) return nullptr;
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    PyObject* x = PyLong_Check(o) ? (Py_INCREF(o), o) : PyObject_GetAttrString(o, "cuda_stream");
    void* s = x ? PyLong_AsVoidPtr(x) : nullptr;
    Py_XDECREF(x);
    if (PyErr_Occurred()) ok = false;
    return s;
  }
  int whole(PyObject* o) {
    const long x = ok ? PyLong_AsLong(o) : 0;
    if (ok && (PyErr_Occurred() || x < INT32_MIN || x > INT32_MAX)) {
      PyErr_Clear();
      no("an int32 number expected");
    }
    return (int)x;
  }
  float number(PyObject* o) {
    const double x = ok ? PyFloat_AsDouble(o) : 0.;
    if (ok && PyErr_Occurred()) ok = false;
    return (float)x;
  }

  const Cache* cache(PyObject* o) {
    if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != sizeof(Cache)) return no("a PagedKV expected"), nullptr;
    const Cache* c = (const Cache*)PyBytes_AS_STRING(o);
    on(c->device);
    return c;
  }
  grid_heads heads(PyObject* o, const Cache* c, int64_t N, int H) {
    grid_heads h = {};
    const at::Tensor* t = tensor(o);
    if (!t) return h;
    if (t->scalar_type() != (c->f16 ? at::kHalf : at::kBFloat16) || t->dim() != 3 || t->size(0) != N || t->size(1) != H ||
        t->size(2) != c->D || t->stride(2) != 1)
      return no("a tensor [tokens, heads, D] of the cache's type expected, D contiguous"), h;
    return grid_heads{t->data_ptr(), t->stride(0), t->stride(1)};
  }
  grid_kv_chunk chunk(PyObject* table, PyObject* lens, PyObject* start, int64_t N) {
    grid_kv_chunk c = {};
    const int64_t B = size(lens, 0, 1);
    const int64_t pages = ok ? size(table, 1, 2) : 0;
    int64_t stride = 0;
    c.d_table = (const int32_t*)rows(table, at::kInt, B, pages, &stride);
    c.table_stride = B > 1 ? stride : pages;
    c.d_len = ints(lens, B);
    c.d_start = ints(start, B + 1, false);
    int32(N), int32(pages), int32(B);
    c.max_pages = (int)pages, c.B = (int)B, c.n_tokens = (int)N;
    return c;
  }
  grid_tree tree(PyObject* parent, PyObject* start, int64_t B) {
    const int64_t N = size(parent, 0, 1);
    int32(N), int32(B);
    return grid_tree{ints(parent, N), ints(start, B + 1, false), (int)B, (int)N};
  }
};

// The call itself.  Other threads may run meanwhile (the caller's arguments keep the tensors): a launch waits where the
// stream's queue is full, for a function of the host's that is written in Python, say.
template <typename F>
PyObject* go(F call) {
  struct Others {
    PyThreadState* mine = PyEval_SaveThread();
    ~Others() { PyEval_RestoreThread(mine); }
  };
  int code;
  {
    Others run;
    code = call();
  }
  return PyLong_FromLong(code);
}
#define NEEDS(n) \
  if (count != (n)) return PyErr_SetString(PyExc_TypeError, "wrong number of arguments"), nullptr

// kv table lens k v status start q q_out cos sin pairs q_norm k_norm eps depth stream
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(17);
  Look l;
  const Cache* c = l.cache(a[0]);
  if (!c) return nullptr;
  const int64_t N = l.size(a[3], 0, 3);
  const grid_kv_chunk chunk = l.chunk(a[1], a[2], a[6], N);
  const grid_heads k = l.heads(a[3], c, N, c->kv_heads), v = l.heads(a[4], c, N, c->kv_heads);
  int32_t* status = l.ints(a[5], chunk.B);
  grid_heads q = {}, out = {};
  const bool some_q = a[7] != Py_None, turned = a[9] != Py_None, normed = a[12] != Py_None || a[13] != Py_None;
  if (some_q != (a[8] != Py_None)) l.no("q and q_out go together");
  if (some_q) q = l.heads(a[7], c, N, c->heads), out = l.heads(a[8], c, N, c->heads);
  grid_rotation rot = {};
  if (turned != (a[10] != Py_None)) l.no("cos and sin go together");
  if (turned) {
    const int64_t n = l.size(a[9], 0, 2), half = l.ok ? l.size(a[9], 1, 2) : 0;
    rot.d_cos = l.floats2(a[9], n, half), rot.d_sin = l.floats2(a[10], n, half);
    l.int32(n), l.int32(2 * half);
    rot.n_pos = (int)n, rot.rot = (int)(2 * half);
    const int pairs = PyObject_IsTrue(a[11]);
    if (pairs < 0) l.ok = false;
    rot.pairs = pairs;
  }
  grid_head_norm norm = {};
  if (normed) {
    const at::ScalarType type = c->f16 ? at::kHalf : at::kBFloat16;
    norm.d_q = l.dense(a[12], type, c->D, -1, false), norm.d_k = l.dense(a[13], type, c->D, -1, false);
    norm.eps = l.number(a[14]);
  }
  const int32_t* depth = l.ints(a[15], N, false);
  void* stream = l.stream(a[16]);
  if (!l.ok) return nullptr;
  const grid_heads *qh = some_q ? &q : nullptr, *oh = some_q ? &out : nullptr;
  const grid_rotation* r = turned ? &rot : nullptr;
  const grid_head_norm* w = normed ? &norm : nullptr;
  const bool tree = a[15] != Py_None;
  return go([&] {
    return tree ? lib.kv_append_tree(c->kv, &chunk, &k, &v, qh, oh, r, w, depth, status, stream)
                : lib.kv_append(c->kv, &chunk, &k, &v, qh, oh, r, w, status, stream);
  });
}

// kv table lens q out status lse start scale sees stream
PyObject* kv_attend(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(11);
  Look l;
  const Cache* c = l.cache(a[0]);
  if (!c) return nullptr;
  const int64_t N = l.size(a[3], 0, 3);
  const grid_kv_chunk chunk = l.chunk(a[1], a[2], a[7], N);
  grid_kv_query query = {l.heads(a[3], c, N, c->heads), l.heads(a[4], c, N, c->heads), l.floats2(a[6], N, c->heads, false),
                         l.number(a[8]), 0};
  int32_t* status = l.ints(a[5], chunk.B);
  const uint32_t* sees = nullptr;
  int64_t words = 0;
  if (a[9] != Py_None) {
    words = l.size(a[9], 1, 2);
    if (words <= 0) l.no("sees [tokens, words] expected");
    sees = (const uint32_t*)l.ints2(a[9], N, words);
    l.int32(words);
  }
  void* stream = l.stream(a[10]);
  if (!l.ok) return nullptr;
  const bool tree = a[9] != Py_None;
  return go([&] {
    return tree ? lib.kv_attend_tree(c->kv, &chunk, &query, sees, (int)words, status, stream)
                : lib.kv_attend(c->kv, &chunk, &query, status, stream);
  });
}

// kv table lens path count status n_tokens start stream
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(9);
  Look l;
  const Cache* c = l.cache(a[0]);
  if (!c) return nullptr;
  const grid_kv_chunk chunk = l.chunk(a[1], a[2], a[7], l.whole(a[6]));
  const int64_t most = l.size(a[3], 1, 2);
  const int32_t *path = l.ints2(a[3], chunk.B, most), *taken = l.ints(a[4], chunk.B);
  int32_t* status = l.ints(a[5], chunk.B);
  l.int32(most);
  void* stream = l.stream(a[8]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.kv_compact(c->kv, &chunk, path, taken, (int)most, status, stream); });
}

// kv copies status stream
PyObject* kv_copy(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(4);
  Look l;
  const Cache* c = l.cache(a[0]);
  if (!c) return nullptr;
  const int64_t n = l.size(a[2], 0, 1);
  const int32_t* copies = l.ints2(a[1], 3, n);
  int32_t* status = l.ints(a[2], n);
  l.int32(n);
  void* stream = l.stream(a[3]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.kv_copy(c->kv, copies, (int)n, status, stream); });
}

// parent depth sees status start stream
PyObject* tree_plan(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(6);
  Look l;
  l.on_current();
  const int64_t B = l.size(a[3], 0, 1);
  const grid_tree tree = l.tree(a[0], a[4], B);
  const int64_t words = l.size(a[2], 1, 2);
  int32_t *depth = l.ints(a[1], tree.n_tokens), *sees = l.ints2(a[2], tree.n_tokens, words), *status = l.ints(a[3], B);
  l.int32(words);
  void* stream = l.stream(a[5]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.tree_plan(&tree, depth, (uint32_t*)sees, (int)words, status, stream); });
}

// parent tokens sampled path count out status start eos stream
PyObject* tree_accept(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(10);
  Look l;
  l.on_current();
  const int64_t B = l.size(a[6], 0, 1);
  const grid_tree tree = l.tree(a[0], a[7], B);
  const int64_t most = l.size(a[3], 1, 2);
  const int32_t *tokens = l.ints(a[1], tree.n_tokens), *sampled = l.ints(a[2], tree.n_tokens);
  int32_t *path = l.ints2(a[3], B, most), *taken = l.ints(a[4], B), *out = l.ints2(a[5], B, most), *status = l.ints(a[6], B);
  const int eos = l.whole(a[8]);
  l.int32(most);
  void* stream = l.stream(a[9]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.tree_accept(&tree, tokens, sampled, eos, (int)most, path, taken, out, status, stream); });
}

// logits noise tokens status mask temperature top_k top_p min_p logprob eos stream
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(12);
  Look l;
  l.on_current();
  const int64_t B = l.size(a[0], 0, 2), V = l.ok ? l.size(a[0], 1, 2) : 0;
  if (!l.ok) return nullptr;
  const at::ScalarType type = THPVariable_Unpack(a[0]).scalar_type();
  if (type != at::kFloat && type != at::kBFloat16) l.no("float32 or bfloat16 logits expected");
  grid_sample_step s = {};
  s.d_logits = l.rows(a[0], type, B, V, &s.logit_stride);
  s.d_noise = (const float*)l.rows(a[1], at::kFloat, B, V, &s.noise_stride);
  if (a[4] != Py_None) s.d_mask = (const uint32_t*)l.rows(a[4], at::kInt, B, (V + 31) / 32, &s.mask_stride);
  s.d_temperature = l.floats(a[5], B, false);
  s.d_top_k = l.ints(a[6], B, false);
  s.d_top_p = l.floats(a[7], B, false), s.d_min_p = l.floats(a[8], B, false);
  l.int32(B), l.int32(V);
  s.dtype = type == at::kFloat ? GRID_DTYPE_F32 : GRID_DTYPE_BF16, s.B = (int)B, s.V = (int)V, s.eos = l.whole(a[10]);
  s.d_tokens = l.ints(a[2], B), s.d_logprob = l.floats(a[9], B, false), s.d_status = l.ints(a[3], B);
  void* stream = l.stream(a[11]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.sample(&s, stream); });
}

// handle device n_pages table held want table_out held_out copies refs status parent keep pinned stream
PyObject* pages_update(PyObject*, PyObject* const* a, Py_ssize_t count) {
  NEEDS(15);
  Look l;
  const grid_pages* p = (const grid_pages*)PyLong_AsVoidPtr(a[0]);
  if (PyErr_Occurred()) return nullptr;
  l.on(l.whole(a[1]));
  const int n_pages = l.whole(a[2]);
  const int64_t A = l.size(a[4], 0, 1), B = l.ok ? l.size(a[5], 0, 1) : 0, width = l.ok ? l.size(a[3], 1, 2) : 0,
                width_out = l.ok ? l.size(a[6], 1, 2) : 0;
  grid_pages_step s = {};
  int64_t by = 0, by_out = 0;
  s.d_table = (const int32_t*)l.rows(a[3], at::kInt, A, width, &by);
  s.d_table_out = (int32_t*)l.rows(a[6], at::kInt, B, width_out, &by_out);
  s.table_stride = A > 1 ? by : width, s.table_out_stride = B > 1 ? by_out : width_out;
  s.d_held = l.ints(a[4], A), s.d_want = l.ints(a[5], B), s.d_held_out = l.ints(a[7], B);
  s.d_copies = l.ints2(a[8], 3, B), s.d_refs = l.ints(a[9], n_pages), s.d_status = l.ints(a[10], B);
  s.d_parent = l.ints(a[11], B, false), s.d_keep = l.ints(a[12], B, false), s.d_pinned = l.ints(a[13], n_pages, false);
  if (l.ok && (s.d_table == s.d_table_out || s.d_held == s.d_held_out)) l.no("the new table and lengths need tensors of their own");
  l.int32(A), l.int32(B), l.int32(width), l.int32(width_out);
  s.A = (int)A, s.B = (int)B, s.width = (int)width, s.width_out = (int)width_out;
  void* stream = l.stream(a[14]);
  if (!l.ok) return nullptr;
  return go([&] { return lib.pages_update(p, &s, stream); });
}

// The entry points' addresses, in the order of Library.
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
  constexpr int n = sizeof(Library) / sizeof(void*);
  NEEDS(n);
  void* at[n];
  for (int i = 0; i < n; ++i) {
    at[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred()) return nullptr;
  }
  static_assert(sizeof(at) == sizeof(lib));
  memcpy(&lib, at, sizeof lib);
  Py_RETURN_NONE;
}

// (torch's own checks throw)
template <PyObject* (*kCall)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* a, Py_ssize_t count) {
  try {
    return kCall(self, a, count);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}
#define CALL(name) {#name, (PyCFunction)(void*)guarded<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(bind), CALL(kv_append), CALL(kv_attend), CALL(kv_compact), CALL(kv_copy), CALL(tree_plan),
                         CALL(tree_accept), CALL(sample), CALL(pages_update), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "grid_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_grid_binding() { return PyModule_Create(&module); }
