// Native side of the Python binding: turns the arguments of one compute call (torch tensors, integers, a stream) into
// the arguments of its C entry point and makes the call. Nothing of the method happens here.
//
// A decoding step is some forty calls of 5 to 15 us of device time each, so what a call costs the host decides
// whether the device waits for it. Through ctypes, with a Python-level pointer extraction per tensor and
// torch.cuda.current_stream(), a call of cast_tree_attention took 15 to 18 us (19 arguments) and one of
// cast_tree_expand 11 to 13 us; here the tensors are unpacked through torch's own C++ interface.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cast.h"

namespace {

// Arguments are taken in order; the first one that does not fit sets a Python exception and ends the call.
struct Args {
  PyObject* const* a;
  Py_ssize_t n;
  Py_ssize_t at = 0;
  bool ok = true;
  bool known_dtype = true;

  PyObject* next() {
    if (!ok) return nullptr;
    if (at >= n) {
      PyErr_SetString(PyExc_TypeError, "too few arguments");
      ok = false;
      return nullptr;
    }
    return a[at++];
  }
  int integer() {
    PyObject* o = next();
    if (!o) return 0;
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) ok = false;
    return (int)v;
  }
  size_t size() {
    PyObject* o = next();
    if (!o) return 0;
    const size_t v = PyLong_AsSize_t(o);
    if (v == (size_t)-1 && PyErr_Occurred()) ok = false;
    return v;
  }
  double real() {
    PyObject* o = next();
    if (!o) return 0.0;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) ok = false;
    return v;
  }
  cast_ctx* context() {
    PyObject* o = next();
    if (!o) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (p == nullptr && PyErr_Occurred()) ok = false;
    return static_cast<cast_ctx*>(p);
  }
  // device address of a tensor argument, null for None; `dtype`, where given, receives the logits / cache type
  template <typename T = void>
  T* tensor(cast_dtype* dtype = nullptr) {
    PyObject* o = next();
    if (!o || (o == Py_None && dtype == nullptr)) return nullptr;
    if (!THPVariable_Check(o)) {
      PyErr_SetString(PyExc_TypeError, "torch tensor expected");
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) {
      PyErr_SetString(PyExc_AssertionError, "device-resident contiguous tensor expected");
      ok = false;
      return nullptr;
    }
    if (dtype != nullptr) {
      if (t.scalar_type() == at::kFloat) *dtype = CAST_F32;
      else if (t.scalar_type() == at::kBFloat16) *dtype = CAST_BF16;
      else known_dtype = false;
    }
    return static_cast<T*>(t.data_ptr());
  }
  // the same for an argument of one type
  void* tensor_of(at::ScalarType type) {
    PyObject* o = ok && at < n ? a[at] : nullptr;
    if (o != nullptr && THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() != type) {
      PyErr_Format(PyExc_TypeError, "%s tensor expected", c10::toString(type));
      ok = false;
      return nullptr;
    }
    return tensor();
  }
  // rows [.., heads, D] that may lie apart (a view of a fused projection's output): dense heads, `stride` bytes from row to row,
  // which is the next argument; null for None
  void* strided(cast_dtype* dtype, bool* given, size_t* stride) {
    PyObject* o = next();
    *given = o != nullptr && o != Py_None;
    if (!o) return nullptr;
    if (o == Py_None) {
      *stride = size();
      return nullptr;
    }
    if (!THPVariable_Check(o)) {
      PyErr_SetString(PyExc_TypeError, "torch tensor expected");
      ok = false;
      return nullptr;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    *stride = size();
    if (!ok) return nullptr;
    const int64_t nd = t.dim();
    bool fits = t.is_cuda() && nd >= 2 && t.stride(nd - 1) == 1 && (t.size(nd - 2) == 1 || t.stride(nd - 2) == t.size(nd - 1));
    int64_t step = (int64_t)(*stride / t.element_size());
    for (int64_t d = nd - 3; fits && d >= 0; --d) {
      fits = t.size(d) == 1 || t.stride(d) == step;
      step *= t.size(d);
    }
    if (!fits || *stride % t.element_size() != 0) {
      PyErr_SetString(PyExc_AssertionError, "device-resident tensor of dense heads, rows one given stride apart, expected");
      ok = false;
      return nullptr;
    }
    if (t.scalar_type() == at::kFloat) *dtype = CAST_F32;
    else if (t.scalar_type() == at::kBFloat16) *dtype = CAST_BF16;
    else known_dtype = false;
    return t.data_ptr();
  }
  // codes and pairs of a 4-bit cache
  void* codes() { return tensor_of(at::kByte); }
  void* range() { return tensor_of(at::kBFloat16); }
  int32_t* ints() { return static_cast<int32_t*>(tensor_of(at::kInt)); }
  // the last argument: a torch stream, or None for the current one
  void* stream() {
    PyObject* o = next();
    if (!o) return nullptr;
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (h == nullptr) {
      ok = false;
      return nullptr;
    }
    void* s = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (s == nullptr && PyErr_Occurred()) ok = false;
    return s;
  }
  bool ready() {
    if (ok && at != n) {
      PyErr_SetString(PyExc_TypeError, "too many arguments");
      ok = false;
    }
    return ok;
  }
};

// Every wrapper returns the entry point's status as a Python integer. The call itself runs without the interpreter
// lock: a launch can block while the device's queue is full.
#define CALL(expr)                                            \
  if (!g.ready()) return nullptr;                             \
  if (!g.known_dtype) return PyLong_FromLong(CAST_ERR_DTYPE); \
  cast_status status;                                         \
  Py_BEGIN_ALLOW_THREADS                                      \
  status = (expr);                                            \
  Py_END_ALLOW_THREADS                                        \
  return PyLong_FromLong((long)status)

PyObject* step_begin(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_ctx* c = g.context();
  const int B = g.integer();
  auto* root = g.tensor<int32_t>();
  auto* kv_len = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_step_begin(c, B, root, kv_len, s));
}

PyObject* tree_expand(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  const int layer = g.integer();
  auto* logits = g.tensor(&dt);
  auto* tokens = g.tensor<int32_t>();
  auto* rows = g.tensor<int32_t>();
  auto* count = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_tree_expand(c, layer, logits, dt, tokens, rows, count, s));
}

PyObject* select_nodes(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_ctx* c = g.context();
  auto* tokens = g.tensor<int32_t>();
  auto* parent = g.tensor<int32_t>();
  auto* depth = g.tensor<int32_t>();
  auto* anc = g.tensor<uint32_t>();
  auto* pool = g.tensor<int32_t>();
  auto* scores = g.tensor<double>();
  auto* n_tree = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_select_nodes(c, tokens, parent, depth, anc, pool, scores, n_tree, s));
}

// cast_tree_attention and, with `rows`, cast_tree_attention_rows
template <bool kRows>
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  auto* q = g.tensor(&dt);
  auto* k = g.tensor();
  auto* v = g.tensor();
  const int B = g.integer(), Hq = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.tensor<int32_t>();
  const int cap = g.integer(), pages = g.integer();
  auto* kv_len = g.tensor<int32_t>();
  auto* anc = g.tensor<uint32_t>();
  auto* n_tree = g.tensor<int32_t>();
  int32_t* first = kRows ? g.tensor<int32_t>() : nullptr;
  const float scale = (float)g.real();
  auto* out = g.tensor();
  void* s = g.stream();
  CALL(cast_tree_attention_rows(c, q, k, v, dt, B, Hq, Hkv, D, page, table, cap, pages, kv_len, anc, n_tree, first, scale,
                                out, s));
}

PyObject* accept(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  auto* logits = g.tensor(&dt);
  const int B = g.integer();
  auto* tokens = g.tensor<int32_t>();
  auto* parent = g.tensor<int32_t>();
  auto* depth = g.tensor<int32_t>();
  auto* anc = g.tensor<uint32_t>();
  auto* n_tree = g.tensor<int32_t>();
  auto* len = g.tensor<int32_t>();
  auto* path = g.tensor<int32_t>();
  auto* bonus = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_accept(c, logits, dt, B, tokens, parent, depth, anc, n_tree, len, path, bonus, s));
}

PyObject* accept_stochastic(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  auto* target = g.tensor(&dt);
  auto* draft = g.tensor();
  const int B = g.integer();
  const double temperature = g.real();
  auto* tokens = g.tensor<int32_t>();
  auto* parent = g.tensor<int32_t>();
  auto* n_tree = g.tensor<int32_t>();
  auto* u_accept = g.tensor<double>();
  auto* u_bonus = g.tensor<double>();
  auto* len = g.tensor<int32_t>();
  auto* path = g.tensor<int32_t>();
  auto* bonus = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_accept_stochastic(c, target, draft, dt, B, temperature, tokens, parent, n_tree, u_accept, u_bonus, len, path,
                              bonus, s));
}

PyObject* accept_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  auto* logits = g.tensor(&dt);
  const int B = g.integer(), n_cap = g.integer(), vocab = g.integer(), max_depth = g.integer();
  auto* tokens = g.tensor<int32_t>();
  auto* parent = g.tensor<int32_t>();
  auto* n_tree = g.tensor<int32_t>();
  auto* len = g.tensor<int32_t>();
  auto* path = g.tensor<int32_t>();
  auto* bonus = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_accept_static(logits, dt, B, n_cap, vocab, max_depth, tokens, parent, n_tree, len, path, bonus, s));
}

PyObject* compact_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  auto* k = g.tensor(&dt);
  auto* v = g.tensor();
  const int B = g.integer(), layers = g.integer();
  const size_t stride = g.size();
  const int Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.tensor<int32_t>();
  const int cap = g.integer(), pages = g.integer();
  auto* path = g.tensor<int32_t>();
  auto* len = g.tensor<int32_t>();
  auto* kv_len = g.tensor<int32_t>();
  void* s = g.stream();
  CALL(cast_compact_kv(c, k, v, dt, B, layers, stride, Hkv, D, page, table, cap, pages, path, len, kv_len, s));
}

// Values `k` and `v` of a store or a load, of one type.
void both(Args& g, cast_dtype* dtype, void** k, void** v) {
  cast_dtype other = CAST_F32;
  *k = g.tensor(dtype);
  *v = g.tensor(&other);
  if (g.ok && other != *dtype) g.known_dtype = false;
}

PyObject* store_kv_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  void *k, *v;
  both(g, &dt, &k, &v);
  const int B = g.integer(), layers = g.integer(), rows = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* start = g.ints();
  auto* n_rows = g.ints();
  auto* kc = g.codes();
  auto* kr = g.range();
  auto* vc = g.codes();
  auto* vr = g.range();
  const size_t cs = g.size(), rs = g.size();
  void* s = g.stream();
  CALL(cast_store_kv_q4(c, k, v, dt, B, layers, rows, Hkv, D, page, table, cap, pages, start, n_rows, kc, kr, vc, vr, cs, rs, s));
}

PyObject* load_kv_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  auto* kc = g.codes();
  auto* kr = g.range();
  auto* vc = g.codes();
  auto* vr = g.range();
  const size_t cs = g.size(), rs = g.size();
  const int B = g.integer(), layers = g.integer(), rows = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* start = g.ints();
  auto* n_rows = g.ints();
  void *k, *v;
  both(g, &dt, &k, &v);
  void* s = g.stream();
  CALL(cast_load_kv_q4(c, kc, kr, vc, vr, cs, rs, dt, B, layers, rows, Hkv, D, page, table, cap, pages, start, n_rows, k, v, s));
}

PyObject* tree_attention_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32, dt_out = CAST_F32;
  cast_ctx* c = g.context();
  auto* q = g.tensor(&dt);
  auto* kc = g.codes();
  auto* kr = g.range();
  auto* vc = g.codes();
  auto* vr = g.range();
  const int B = g.integer(), Hq = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* kv_len = g.ints();
  auto* anc = g.tensor<uint32_t>();
  auto* n_tree = g.ints();
  auto* first = g.ints();
  const float scale = (float)g.real();
  auto* out = g.tensor(&dt_out);
  if (g.ok && dt_out != dt) g.known_dtype = false;
  void* s = g.stream();
  CALL(cast_tree_attention_q4(c, q, kc, kr, vc, vr, dt, B, Hq, Hkv, D, page, table, cap, pages, kv_len, anc, n_tree, first, scale,
                              out, s));
}

PyObject* compact_kv_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_ctx* c = g.context();
  auto* kc = g.codes();
  auto* kr = g.range();
  auto* vc = g.codes();
  auto* vr = g.range();
  const size_t cs = g.size(), rs = g.size();
  const int B = g.integer(), layers = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* path = g.ints();
  auto* len = g.ints();
  auto* kv_len = g.ints();
  void* s = g.stream();
  CALL(cast_compact_kv_q4(c, kc, kr, vc, vr, cs, rs, B, layers, Hkv, D, page, table, cap, pages, path, len, kv_len, s));
}

// cast_attention_mass and, with kQ4, cast_attention_mass_q4
template <bool kQ4>
PyObject* attention_mass(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32, dt_k = CAST_F32;
  cast_ctx* c = g.context();
  auto* q = g.tensor(&dt);
  void* k = kQ4 ? g.codes() : g.tensor(&dt_k);
  void* range = kQ4 ? g.range() : nullptr;
  if (!kQ4 && g.ok && dt_k != dt) g.known_dtype = false;
  const int B = g.integer(), layers = g.integer();
  const size_t qs = g.size(), ks = g.size(), rs = kQ4 ? g.size() : 0;
  const int Hq = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* path = g.ints();
  auto* len = g.ints();
  auto* kv_len = g.ints();
  const float scale = (float)g.real();
  auto* mass = static_cast<float*>(g.tensor_of(at::kFloat));
  void* s = g.stream();
  CALL(kQ4 ? cast_attention_mass_q4(c, q, k, range, dt, B, layers, qs, ks, rs, Hq, Hkv, D, page, table, cap, pages, path, len,
                                    kv_len, scale, mass, s)
           : cast_attention_mass(c, q, k, dt, B, layers, qs, ks, Hq, Hkv, D, page, table, cap, pages, path, len, kv_len, scale,
                                 mass, s));
}

PyObject* evict_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  void *k, *v;
  both(g, &dt, &k, &v);
  const int B = g.integer(), layers = g.integer();
  const size_t stride = g.size();
  const int Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer(), budget = g.integer(), recent = g.integer();
  auto* mass = static_cast<float*>(g.tensor_of(at::kFloat));
  auto* kept = g.ints();
  auto* kv_len = g.ints();
  void* s = g.stream();
  CALL(cast_evict_kv(c, k, v, dt, B, layers, stride, Hkv, D, page, table, cap, pages, budget, recent, mass, kept, kv_len, s));
}

PyObject* evict_kv_q4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_ctx* c = g.context();
  auto* kc = g.codes();
  auto* kr = g.range();
  auto* vc = g.codes();
  auto* vr = g.range();
  const size_t cs = g.size(), rs = g.size();
  const int B = g.integer(), layers = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer(), budget = g.integer(), recent = g.integer();
  auto* mass = static_cast<float*>(g.tensor_of(at::kFloat));
  auto* kept = g.ints();
  auto* kv_len = g.ints();
  void* s = g.stream();
  CALL(cast_evict_kv_q4(c, kc, kr, vc, vr, cs, rs, B, layers, Hkv, D, page, table, cap, pages, budget, recent, mass, kept, kv_len,
                        s));
}

PyObject* append_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_ctx* c = g.context();
  // every tensor of rows that is given has one type
  cast_dtype dt = CAST_F32, one = CAST_F32;
  bool any = false, given = false;
  auto same = [&] {
    if (g.ok && given && any && one != dt) g.known_dtype = false;
    if (given && !any) dt = one;
    any = any || given;
  };
  size_t qs = 0, ks = 0, vs = 0;
  void* q = g.strided(&one, &given, &qs);
  same();
  void* k = g.strided(&one, &given, &ks);
  same();
  void* v = g.strided(&one, &given, &vs);
  same();
  const int B = g.integer(), rows = g.integer(), Hq = g.integer(), Hkv = g.integer(), D = g.integer();
  auto* row_start = g.ints();
  auto* first = g.ints();
  auto* n_rows = g.ints();
  auto* depth = g.ints();
  auto* position = g.ints();
  auto* inv_freq = static_cast<double*>(g.tensor_of(at::kDouble));
  const int rot_dim = g.integer(), interleaved = g.integer();
  const float magnitude = (float)g.real();
  auto* q_weight = static_cast<float*>(g.tensor_of(at::kFloat));
  auto* k_weight = static_cast<float*>(g.tensor_of(at::kFloat));
  const float eps = (float)g.real();
  const int page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* start = g.ints();
  auto dense = [&]() -> void* {
    PyObject* o = g.ok && g.at < g.n ? g.a[g.at] : nullptr;
    given = o != nullptr && o != Py_None;
    void* t = given ? g.tensor(&one) : g.tensor();
    same();
    return t;
  };
  void* q_out = dense();
  void* kc = dense();
  void* vc = dense();
  void* s = g.stream();
  CALL(cast_append_kv(c, q, qs, k, ks, v, vs, dt, B, rows, Hq, Hkv, D, row_start, first, n_rows, depth, position, inv_freq, rot_dim,
                      interleaved, magnitude, q_weight, k_weight, eps, page, table, cap, pages, start, q_out, kc, vc, s));
}

// Queries and the two caches of an attention, of one type; the same of its output.
void attended(Args& g, cast_dtype* dt, void** q, void** k, void** v) {
  cast_dtype other = CAST_F32;
  *q = g.tensor(dt);
  both(g, &other, k, v);
  if (g.ok && other != *dt) g.known_dtype = false;
}
void* output(Args& g, cast_dtype dt) {
  cast_dtype other = CAST_F32;
  void* out = g.tensor(&other);
  if (g.ok && other != dt) g.known_dtype = false;
  return out;
}

PyObject* chunk_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  void *q, *k, *v;
  attended(g, &dt, &q, &k, &v);
  const int B = g.integer(), rows = g.integer();
  auto* row_start = g.ints();
  const int Hq = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* kv_len = g.ints();
  auto* n_new = g.ints();
  const int window = g.integer(), sinks = g.integer();
  const float scale = (float)g.real();
  void* out = output(g, dt);
  void* s = g.stream();
  CALL(cast_chunk_attention(c, q, k, v, dt, B, rows, row_start, Hq, Hkv, D, page, table, cap, pages, kv_len, n_new, window, sinks,
                            scale, out, s));
}

PyObject* tree_attention_window(PyObject*, PyObject* const* a, Py_ssize_t n) {
  Args g{a, n};
  cast_dtype dt = CAST_F32;
  cast_ctx* c = g.context();
  void *q, *k, *v;
  attended(g, &dt, &q, &k, &v);
  const int B = g.integer(), Hq = g.integer(), Hkv = g.integer(), D = g.integer(), page = g.integer();
  auto* table = g.ints();
  const int cap = g.integer(), pages = g.integer();
  auto* kv_len = g.ints();
  auto* anc = g.tensor<uint32_t>();
  auto* depth = g.ints();
  auto* n_tree = g.ints();
  auto* first = g.ints();
  const int window = g.integer(), sinks = g.integer();
  const float scale = (float)g.real();
  void* out = output(g, dt);
  void* s = g.stream();
  CALL(cast_tree_attention_window(c, q, k, v, dt, B, Hq, Hkv, D, page, table, cap, pages, kv_len, anc, depth, n_tree, first, window,
                                  sinks, scale, out, s));
}

#define METHOD(name, fn) {name, (PyCFunction)(void (*)())(fn), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD("step_begin", step_begin),
    METHOD("tree_expand", tree_expand),
    METHOD("select_nodes", select_nodes),
    METHOD("tree_attention", tree_attention<false>),
    METHOD("tree_attention_rows", tree_attention<true>),
    METHOD("accept", accept),
    METHOD("accept_stochastic", accept_stochastic),
    METHOD("accept_static", accept_static),
    METHOD("compact_kv", compact_kv),
    METHOD("store_kv_q4", store_kv_q4),
    METHOD("load_kv_q4", load_kv_q4),
    METHOD("tree_attention_q4", tree_attention_q4),
    METHOD("compact_kv_q4", compact_kv_q4),
    METHOD("attention_mass", attention_mass<false>),
    METHOD("attention_mass_q4", attention_mass<true>),
    METHOD("evict_kv", evict_kv),
    METHOD("evict_kv_q4", evict_kv_q4),
    METHOD("append_kv", append_kv),
    METHOD("chunk_attention", chunk_attention),
    METHOD("tree_attention_window", tree_attention_window),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cast_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cast_calls() { return PyModule_Create(&module); }
