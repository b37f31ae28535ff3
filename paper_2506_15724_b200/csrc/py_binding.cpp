// Python entry points of the library's asynchronous calls: pointers, strides and sizes are read from the tensors here, the
// status comes back as an int. What bounds a call on one layer is the host: with the arguments gathered in Python and handed
// over by ctypes a decode call took 5.4 us, here 3.1, nearly all of it the launch.
#define PY_SSIZE_T_CLEAN
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>

#include "madakv.h"

namespace {

// The arguments of one call, in order. A failed conversion throws; the Python error is set.
struct Args {
  PyObject* const* at;
  Py_ssize_t left;
  Py_buffer cfg_buf;
  bool has_cfg = false;

  Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : at(args), left(n) {
    if (n != want) fail(PyExc_TypeError, "wrong number of arguments");
  }
  ~Args() {
    if (has_cfg) PyBuffer_Release(&cfg_buf);
  }
  [[noreturn]] static void fail(PyObject* type, const char* what) {
    PyErr_SetString(type, what);
    throw python_error();
  }
  PyObject* next() {
    --left;
    return *at++;
  }
  const madakv_config* config() {
    PyObject* o = next();
    PyObject* inner = PyObject_CheckBuffer(o) ? nullptr : PyObject_GetAttrString(o, "_obj");  // (what ctypes.byref gives)
    if (!inner && PyErr_Occurred()) throw python_error();
    const int rc = PyObject_GetBuffer(inner ? inner : o, &cfg_buf, PyBUF_SIMPLE);
    Py_XDECREF(inner);
    if (rc) throw python_error();
    has_cfg = true;
    if (cfg_buf.len < (Py_ssize_t)sizeof(madakv_config)) fail(PyExc_TypeError, "expected a MadakvConfig");
    return static_cast<const madakv_config*>(cfg_buf.buf);
  }
  const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "expected a tensor");
    return THPVariable_Unpack(o);
  }
  template <typename T = void>
  T* ptr() {
    PyObject* o = next();
    return o == Py_None ? nullptr : static_cast<T*>(tensor(o).data_ptr());
  }
  const at::Tensor& tensor() { return tensor(next()); }
  int32_t integer() {
    const long v = PyLong_AsLong(next());
    if (v == -1 && PyErr_Occurred()) throw python_error();
    if (v != (int32_t)v) fail(PyExc_OverflowError, "expected an integer of 32 bits");
    return (int32_t)v;
  }
};

madakv_strides strides(const at::Tensor& t) {
  const auto st = t.strides();
  if (st.size() != 5 || st[4] != 1) Args::fail(PyExc_AssertionError, "expected [B, L, H, tokens, d] with contiguous d");
  return {st[0], st[1], st[2], st[3]};
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// The call itself runs without the interpreter's lock, as it does through ctypes: a launch may wait for room in the queue.
template <typename F>
PyObject* without_lock(F call) {
  int rc;
  Py_BEGIN_ALLOW_THREADS;
  rc = call();
  Py_END_ALLOW_THREADS;
  return PyLong_FromLong(rc);
}

template <bool kGiven>
PyObject* score(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 7);
  const madakv_config* cfg = a.config();
  const at::Tensor &q = a.tensor(), &k = a.tensor();
  const madakv_strides sq = strides(q), sk = strides(k);
  const int32_t* seq_len = a.ptr<int32_t>();
  float *lse = a.ptr<float>(), *psi = a.ptr<float>();
  const at::Tensor& ws = a.tensor();
  void *qp = q.data_ptr(), *kp = k.data_ptr(), *wp = ws.data_ptr(), *st = stream();
  const size_t bytes = (size_t)ws.numel();
  return without_lock([&] {
    return kGiven ? madakv_score_lse(cfg, qp, sq, kp, sk, seq_len, lse, psi, wp, bytes, st)
                  : madakv_score(cfg, qp, sq, kp, sk, seq_len, lse, psi, wp, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

PyObject* allocate(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 11);
  const madakv_config* cfg = a.config();
  const float* psi = a.ptr<float>();
  const uint8_t* mask = a.ptr<uint8_t>();
  const int32_t *seq_len = a.ptr<int32_t>(), *budget = a.ptr<int32_t>();
  double *mass = a.ptr<double>(), *pref = a.ptr<double>();
  int32_t* demand = a.ptr<int32_t>();
  double* phi = a.ptr<double>();
  int32_t* budgets = a.ptr<int32_t>();
  const at::Tensor& ws = a.tensor();
  void *wp = ws.data_ptr(), *st = stream();
  const size_t bytes = (size_t)ws.numel();
  return without_lock(
      [&] { return madakv_allocate(cfg, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, wp, bytes, st); });
  END_HANDLE_TH_ERRORS
}

PyObject* allocate_layer(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 12);
  const madakv_config* cfg = a.config();
  const int32_t layer = a.integer();
  const float* psi = a.ptr<float>();
  const uint8_t* mask = a.ptr<uint8_t>();
  const int32_t *seq_len = a.ptr<int32_t>(), *budget = a.ptr<int32_t>();
  double *mass = a.ptr<double>(), *pref = a.ptr<double>();
  int32_t* demand = a.ptr<int32_t>();
  double* phi = a.ptr<double>();
  int32_t* budgets = a.ptr<int32_t>();
  const at::Tensor& ws = a.tensor();
  void *wp = ws.data_ptr(), *st = stream();
  const size_t bytes = (size_t)ws.numel();
  return without_lock([&] {
    return madakv_allocate_layer(cfg, layer, psi, mask, seq_len, budget, mass, pref, demand, phi, budgets, wp, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

PyObject* demand_layer(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 8);
  const madakv_config* cfg = a.config();
  const float* psi = a.ptr<float>();
  const uint8_t* mask = a.ptr<uint8_t>();
  const int32_t* seq_len = a.ptr<int32_t>();
  double *mass = a.ptr<double>(), *pref = a.ptr<double>();
  int32_t* demand = a.ptr<int32_t>();
  const at::Tensor& ws = a.tensor();
  void *wp = ws.data_ptr(), *st = stream();
  const size_t bytes = (size_t)ws.numel();
  return without_lock([&] { return madakv_demand_layer(cfg, psi, mask, seq_len, mass, pref, demand, wp, bytes, st); });
  END_HANDLE_TH_ERRORS
}

PyObject* select(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 9);
  const madakv_config* cfg = a.config();
  const float* psi = a.ptr<float>();
  const uint8_t* mask = a.ptr<uint8_t>();
  const int32_t *seq_len = a.ptr<int32_t>(), *budgets = a.ptr<int32_t>();
  int32_t* kept_len = a.ptr<int32_t>();
  int64_t* seg_off = a.ptr<int64_t>();
  const at::Tensor &kept_idx = a.tensor(), &ws = a.tensor();
  int32_t* ip = static_cast<int32_t*>(kept_idx.data_ptr());
  const int64_t capacity = kept_idx.numel();
  void *wp = ws.data_ptr(), *st = stream();
  const size_t bytes = (size_t)ws.numel();
  return without_lock(
      [&] { return madakv_select(cfg, psi, mask, seq_len, budgets, kept_len, seg_off, ip, capacity, wp, bytes, st); });
  END_HANDLE_TH_ERRORS
}

PyObject* compact(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 9);
  const madakv_config* cfg = a.config();
  const at::Tensor &k = a.tensor(), &v = a.tensor();
  if (k.strides() != v.strides()) Args::fail(PyExc_AssertionError, "k and v must have the same strides");
  const madakv_strides skv = strides(k);
  const int32_t* kept_idx = a.ptr<int32_t>();
  const int64_t* seg_off = a.ptr<int64_t>();
  const int32_t* kept_len = a.ptr<int32_t>();
  const at::Tensor& k_c = a.tensor();
  void* v_c = a.ptr();
  const at::Tensor& ws = a.tensor();
  void *kp = k.data_ptr(), *vp = v.data_ptr(), *kc = k_c.data_ptr(), *wp = ws.data_ptr(), *st = stream();
  const int64_t capacity = k_c.size(0);
  const size_t bytes = (size_t)ws.numel();
  return without_lock(
      [&] { return madakv_compact(cfg, kp, vp, skv, kept_idx, seg_off, kept_len, kc, v_c, capacity, wp, bytes, st); });
  END_HANDLE_TH_ERRORS
}

PyObject* decode_attn(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Args a(args, n, 12);
  const madakv_config* cfg = a.config();
  const int32_t layer = a.integer();
  const void *q = a.ptr(), *k_new = a.ptr(), *v_new = a.ptr();
  const at::Tensor& k_c = a.tensor();
  void* v_c = a.ptr();
  const int64_t* seg_off = a.ptr<int64_t>();
  int32_t* kept_len = a.ptr<int32_t>();
  void* out = a.ptr();
  float* lse = a.ptr<float>();
  const at::Tensor& ws = a.tensor();
  void *kc = k_c.data_ptr(), *wp = ws.data_ptr(), *st = stream();
  const int64_t capacity = k_c.size(0);
  const size_t bytes = (size_t)ws.numel();
  return without_lock([&] {
    return madakv_decode_attn(cfg, layer, q, k_new, v_new, kc, v_c, seg_off, kept_len, capacity, out, lse, wp, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

// ---- the cache in 4 bits, tracking, eviction: tensors are checked against the config before their pointers are passed on
struct Checked : Args {
  const madakv_config* cfg;
  int64_t units, heads;  // (sequence, layer, KV head)s; (sequence, layer, query head)s
  int bad_config = MADAKV_OK;
  c10::DeviceIndex device;

  Checked(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : Args(args, n, want) {
    cfg = config();
    size_t bytes;
    bad_config = madakv_workspace_bytes(cfg, &bytes);  // (before its numbers are used)
    units = (int64_t)cfg->batch * cfg->n_layers * cfg->n_kv_heads;
    heads = (int64_t)cfg->batch * cfg->n_layers * cfg->n_q_heads;
    device = c10::cuda::current_device();
  }
  [[noreturn]] static void wrong(const char* name, const char* what) {
    PyErr_Format(PyExc_ValueError, "%s: %s", name, what);
    throw python_error();
  }
  at::ScalarType dtype() const { return cfg->dtype == MADAKV_F32 ? at::kFloat : at::kBFloat16; }
  const at::Tensor& on_device(PyObject* o, const char* name, at::ScalarType type) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.device().index() != device) wrong(name, "expected a tensor on the current CUDA device");
    if (t.scalar_type() != type) wrong(name, "wrong dtype");
    return t;
  }
  // A contiguous tensor of at least `least` elements (exactly so many with `exact`).
  template <typename P = void>
  P* array(const char* name, at::ScalarType type, int64_t least, bool optional = false, bool exact = false) {
    PyObject* o = next();
    if (optional && o == Py_None) return nullptr;
    const at::Tensor& t = on_device(o, name, type);
    if (!t.is_contiguous()) wrong(name, "expected a contiguous tensor");
    if (t.numel() < least || (exact && t.numel() != least)) wrong(name, "wrong size for this config and cache");
    return static_cast<P*>(t.data_ptr());
  }
  // [capacity, row] of a cache; its first array says the capacity
  template <typename P = void>
  P* cache(const char* name, at::ScalarType type, int64_t row, int64_t& capacity) {
    if (capacity < 0) {
      const at::Tensor& t = tensor(*at);
      if (t.dim() < 2) wrong(name, "expected [capacity, ...]");
      capacity = t.size(0);
    }
    return array<P>(name, type, capacity * row, false, true);
  }
  void* strided(const char* name, madakv_strides& st) {  // [B, L, H_kv, at least n_max, d]
    const at::Tensor& t = on_device(next(), name, dtype());
    st = strides(t);
    if (t.size(0) != cfg->batch || t.size(1) != cfg->n_layers || t.size(2) != cfg->n_kv_heads || t.size(3) < cfg->max_seq_len ||
        t.size(4) != cfg->head_dim)
      wrong(name, "wrong size for this config");
    return t.data_ptr();
  }
  void* workspace(size_t& bytes) {
    const at::Tensor& t = tensor();
    if (!t.is_cuda() || t.device().index() != device || !t.is_contiguous()) wrong("ws", "expected a contiguous tensor on the current CUDA device");
    bytes = t.nbytes();
    return t.data_ptr();
  }
  float real() {
    const double v = PyFloat_AsDouble(next());
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
  }
};

struct QuantCache {
  uint8_t *k_code, *v_code;
  void *k_par, *v_par;
  int64_t capacity = -1;
  explicit QuantCache(Checked& a) {
    const int64_t d = a.cfg->head_dim;
    k_code = a.cache<uint8_t>("k_code", at::kByte, d / 2, capacity);
    k_par = a.cache("k_par", at::kBFloat16, d / 16, capacity);
    v_code = a.cache<uint8_t>("v_code", at::kByte, d / 2, capacity);
    v_par = a.cache("v_par", at::kBFloat16, d / 16, capacity);
  }
};

PyObject* compact_quant(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Checked a(args, n, 11);
  if (a.bad_config) return PyLong_FromLong(a.bad_config);
  madakv_strides sk, sv;
  void *k = a.strided("k", sk), *v = a.strided("v", sv);
  if (sk.batch != sv.batch || sk.layer != sv.layer || sk.head != sv.head || sk.token != sv.token)
    Args::fail(PyExc_AssertionError, "k and v must have the same strides");
  const int32_t* kept_idx = a.array<int32_t>("kept_idx", at::kInt, 0);
  const int64_t listed = a.tensor(args[3]).numel();
  const int64_t* seg_off = a.array<int64_t>("seg_off", at::kLong, a.units + 1);
  const int32_t* kept_len = a.array<int32_t>("kept_len", at::kInt, a.units);
  const QuantCache c(a);
  if (listed < c.capacity) Checked::wrong("kept_idx", "shorter than the cache");
  size_t bytes;
  void *ws = a.workspace(bytes), *st = stream();
  return without_lock([&] {
    return madakv_compact_quant(a.cfg, k, v, sk, kept_idx, seg_off, kept_len, c.k_code, c.k_par, c.v_code, c.v_par, c.capacity,
                                ws, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

PyObject* expand_quant(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Checked a(args, n, 8);
  if (a.bad_config) return PyLong_FromLong(a.bad_config);
  const int64_t* rows = a.array<int64_t>("rows", at::kLong, 0, true);
  const int64_t given = rows || args[1] != Py_None ? a.tensor(args[1]).numel() : -1;
  const QuantCache c(a);
  const int64_t d = a.cfg->head_dim, n_rows = given >= 0 ? given : c.capacity;
  void *k = a.array("k_out", a.dtype(), n_rows * d, false, true), *v = a.array("v_out", a.dtype(), n_rows * d, false, true), *st = stream();
  if (n_rows == 0) return PyLong_FromLong(MADAKV_OK);  // (empty tensors have no pointers)
  return without_lock(
      [&] { return madakv_expand_quant(a.cfg, rows, n_rows, c.k_code, c.k_par, c.v_code, c.v_par, c.capacity, k, v, st); });
  END_HANDLE_TH_ERRORS
}

struct Track {
  float *acc, *scratch;
  int32_t* kept_idx;
  const int32_t* position;
  float decay;
  Track(Checked& a, int64_t capacity, bool optional) {
    acc = a.array<float>("acc", at::kFloat, capacity, optional);
    scratch = a.array<float>("scratch", at::kFloat, capacity * (a.cfg->n_q_heads / a.cfg->n_kv_heads), optional);
    kept_idx = a.array<int32_t>("kept_idx", at::kInt, capacity, true);
    position = a.array<int32_t>("position", at::kInt, a.cfg->batch, true);
    decay = a.real();
  }
};

template <bool kQuant>
PyObject* decode_more(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Checked a(args, n, kQuant ? 19 : 17);
  if (a.bad_config) return PyLong_FromLong(a.bad_config);
  const int64_t d = a.cfg->head_dim;
  const int32_t layer = a.integer();
  void* q = a.array("q", a.dtype(), a.heads * d, false, true);
  void *k_new = a.array("k_new", a.dtype(), a.units * d, true, true), *v_new = a.array("v_new", a.dtype(), a.units * d, true, true);
  int64_t capacity = -1;
  void *k_c, *v_c, *k_par = nullptr, *v_par = nullptr;
  if constexpr (kQuant) {
    const QuantCache c(a);
    k_c = c.k_code, k_par = c.k_par, v_c = c.v_code, v_par = c.v_par, capacity = c.capacity;
  } else {
    k_c = a.cache("k_c", a.dtype(), d, capacity);
    v_c = a.cache("v_c", a.dtype(), d, capacity);
  }
  const int64_t* seg_off = a.array<int64_t>("seg_off", at::kLong, a.units + 1);
  int32_t* kept_len = a.array<int32_t>("kept_len", at::kInt, a.units);
  void* out = a.array("out", a.dtype(), a.heads * d, false, true);
  float* lse = a.array<float>("lse_out", at::kFloat, a.heads, true, true);
  size_t bytes;
  void* ws = a.workspace(bytes);
  const Track t(a, capacity, kQuant);
  void* st = stream();
  return without_lock([&] {
    if constexpr (kQuant)
      return madakv_decode_attn_quant(a.cfg, layer, q, k_new, v_new, (uint8_t*)k_c, k_par, (uint8_t*)v_c, v_par, seg_off, kept_len,
                                      capacity, out, lse, t.acc, t.scratch, t.kept_idx, t.position, t.decay, ws, bytes, st);
    else
      return madakv_decode_attn_track(a.cfg, layer, q, k_new, v_new, k_c, v_c, seg_off, kept_len, capacity, out, lse, t.acc,
                                      t.scratch, t.kept_idx, t.position, t.decay, ws, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

template <bool kQuant>
PyObject* evict(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  Checked a(args, n, kQuant ? 13 : 11);
  if (a.bad_config) return PyLong_FromLong(a.bad_config);
  const int64_t d = a.cfg->head_dim;
  const int32_t layer = a.integer();
  const int32_t* limit = a.array<int32_t>("limit", at::kInt, a.units);
  const int32_t recent = a.integer();
  float* acc = a.array<float>("acc", at::kFloat, 0);
  int32_t* kept_idx = a.array<int32_t>("kept_idx", at::kInt, 0);
  const int64_t least = std::min(a.tensor(args[4]).numel(), a.tensor(args[5]).numel());
  const int64_t* seg_off = a.array<int64_t>("seg_off", at::kLong, a.units + 1);
  int32_t* kept_len = a.array<int32_t>("kept_len", at::kInt, a.units);
  int64_t capacity = -1;
  void *k_c, *v_c, *k_par = nullptr, *v_par = nullptr;
  if constexpr (kQuant) {
    const QuantCache c(a);
    k_c = c.k_code, k_par = c.k_par, v_c = c.v_code, v_par = c.v_par, capacity = c.capacity;
  } else {
    k_c = a.cache("k_c", a.dtype(), d, capacity);
    v_c = a.cache("v_c", a.dtype(), d, capacity);
  }
  if (least < capacity) Checked::wrong("acc, kept_idx", "shorter than the cache");
  size_t bytes;
  void *ws = a.workspace(bytes), *st = stream();
  return without_lock([&] {
    if constexpr (kQuant)
      return madakv_evict_quant(a.cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, capacity, (uint8_t*)k_c, k_par,
                                (uint8_t*)v_c, v_par, ws, bytes, st);
    else
      return madakv_evict(a.cfg, layer, limit, recent, acc, kept_idx, seg_off, kept_len, capacity, k_c, v_c, ws, bytes, st);
  });
  END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction as_method(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {
    {"score", as_method(score<false>), METH_FASTCALL, nullptr},
    {"score_lse", as_method(score<true>), METH_FASTCALL, nullptr},
    {"allocate", as_method(allocate), METH_FASTCALL, nullptr},
    {"allocate_layer", as_method(allocate_layer), METH_FASTCALL, nullptr},
    {"demand_layer", as_method(demand_layer), METH_FASTCALL, nullptr},
    {"select", as_method(select), METH_FASTCALL, nullptr},
    {"compact", as_method(compact), METH_FASTCALL, nullptr},
    {"decode_attn", as_method(decode_attn), METH_FASTCALL, nullptr},
    {"compact_quant", as_method(compact_quant), METH_FASTCALL, nullptr},
    {"expand_quant", as_method(expand_quant), METH_FASTCALL, nullptr},
    {"decode_attn_quant", as_method(decode_more<true>), METH_FASTCALL, nullptr},
    {"decode_attn_track", as_method(decode_more<false>), METH_FASTCALL, nullptr},
    {"evict", as_method(evict<false>), METH_FASTCALL, nullptr},
    {"evict_quant", as_method(evict<true>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&module); }
