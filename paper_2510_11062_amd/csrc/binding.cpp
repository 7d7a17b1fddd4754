// The calls whose kernels are short, as Python makes them: they check their tensors, make the outputs and enqueue the kernels.
//
// A grouping call of a training step is 7 to 17 us of kernels, so what the host does around it is what a program waits for: of 16.3
// us for 64 responses, seven outputs made one by one from Python were 9, the checks and pointers of the arguments 3.  A rollout's token
// takes 4 us of rotation, 4 of appending and 14 of attention a layer; made from Python, the first two took 18 and 24, now 6 and 6.5.  Everything else in
// api.py stays Python: those calls' kernels are longer than what the host does in front of them.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <cmath>
#include <utility>

#include "at_grpo.h"

namespace {

using GroupFn = decltype(&at_grpo_group_advantage);
using MixedFn = decltype(&at_grpo_group_advantage_mixed);

enum Key { REWARD, GROUP_ID, N_GROUPS, SEG_OFFSETS, PERM, ADV, MEAN, STD, BEST, KEYS };
const char* const kKeyNames[KEYS] = {"reward", "group_id", "n_groups", "seg_offsets", "perm", "adv", "group_mean", "group_std", "best"};
PyObject* g_keys[KEYS];

// a contiguous tensor of the dtype on a GPU, or null
const at::Tensor* tensor(PyObject* o, at::ScalarType dtype) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  return t.is_cuda() && t.scalar_type() == dtype && t.is_contiguous() ? &t : nullptr;
}

// Other Python threads run while it lives, as they do during torch.empty: an allocation may have to wait for the driver, or for a thread
// that holds the allocator's lock and waits for Python's.
struct WithoutPythonLock {
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutPythonLock() { PyEval_RestoreThread(state); }
};

// group_advantage(function's address, env_id, agent_id, turn_id, reward or r_team, r_loc or None, alpha, n_env, n_agent, n_turn,
//                 eps_std, ddof, norm, want_stats, want_best, workspace, its bytes, stream)
// Returns the outputs, or the call's status, or None where an argument is no contiguous GPU tensor of its dtype (the caller says which).
// With r_loc the function is at_grpo_group_advantage_mixed, else at_grpo_group_advantage.
PyObject* group_advantage(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  // From the first look at a tensor on: some cannot say whether they are contiguous, and what they throw must not leave C.  An
  // allocator's error keeps the Python type that torch.empty raises it with (torch.OutOfMemoryError).
  HANDLE_TH_ERRORS
  if (n_args != 18) {
    PyErr_SetString(PyExc_TypeError, "group_advantage takes 18 arguments");
    return nullptr;
  }
  const bool mixed = v[5] != Py_None;
  const at::Tensor* ids[3];
  for (int k = 0; k < 3; ++k)
    if (!(ids[k] = tensor(v[1 + k], at::kInt))) Py_RETURN_NONE;
  const at::Tensor* reward = tensor(v[4], at::kFloat);
  const at::Tensor* loc = mixed ? tensor(v[5], at::kFloat) : nullptr;
  if (!reward || (mixed && !loc)) Py_RETURN_NONE;
  void* fn = PyLong_AsVoidPtr(v[0]);
  const double alpha = PyFloat_AsDouble(v[6]), eps_std = PyFloat_AsDouble(v[10]);
  const int64_t n_env = PyLong_AsLongLong(v[7]), n_agent = PyLong_AsLongLong(v[8]), n_turn = PyLong_AsLongLong(v[9]);
  const int64_t ddof = PyLong_AsLongLong(v[11]), norm = PyLong_AsLongLong(v[12]);
  const bool want_stats = PyObject_IsTrue(v[13]) == 1, want_best = PyObject_IsTrue(v[14]) == 1;
  void* ws = PyLong_AsVoidPtr(v[15]);
  const size_t ws_bytes = PyLong_AsSize_t(v[16]);
  void* stream = PyLong_AsVoidPtr(v[17]);
  if (PyErr_Occurred()) return nullptr;

  const int64_t R = reward->numel(), keys = n_env * n_agent * n_turn, groups = R < keys ? R : keys;
  const at::TensorOptions f32 = reward->options(), i32 = f32.dtype(at::kInt);
  at::Tensor out[KEYS];
  int status;
  {
    const WithoutPythonLock others_run;
    auto make_f = [&](Key key, int64_t n) { return static_cast<float*>((out[key] = at::empty({n}, f32)).data_ptr()); };
    auto make_i = [&](Key key, int64_t n) { return static_cast<int32_t*>((out[key] = at::empty({n}, i32)).data_ptr()); };
    float* mix = mixed ? make_f(REWARD, R) : nullptr;
    int32_t* group_id = make_i(GROUP_ID, R);
    int32_t* n_groups = make_i(N_GROUPS, 1);
    int32_t* seg = make_i(SEG_OFFSETS, groups + 1);
    int32_t* perm = make_i(PERM, R);
    float* adv = make_f(ADV, R);
    float* mean = want_stats ? make_f(MEAN, groups) : nullptr;
    float* std = want_stats ? make_f(STD, groups) : nullptr;
    int32_t* best = mixed && want_best ? make_i(BEST, groups) : nullptr;
    const int32_t *env = static_cast<const int32_t*>(ids[0]->data_ptr()), *agent = static_cast<const int32_t*>(ids[1]->data_ptr()),
                  *turn = static_cast<const int32_t*>(ids[2]->data_ptr());
    const float *r = static_cast<const float*>(reward->data_ptr()), *l = loc ? static_cast<const float*>(loc->data_ptr()) : nullptr;
    const int32_t nR = static_cast<int32_t>(R), nE = static_cast<int32_t>(n_env), nA = static_cast<int32_t>(n_agent),
                  nT = static_cast<int32_t>(n_turn), dd = static_cast<int32_t>(ddof), nm = static_cast<int32_t>(norm);
    status = mixed ? reinterpret_cast<MixedFn>(fn)(nR, nE, nA, nT, env, agent, turn, r, l, static_cast<float>(alpha),
                                                   static_cast<float>(eps_std), dd, nm, mix, group_id, n_groups, seg, perm, adv, mean,
                                                   std, best, ws, ws_bytes, stream)
                   : reinterpret_cast<GroupFn>(fn)(nR, nE, nA, nT, env, agent, turn, r, static_cast<float>(eps_std), dd, nm, group_id,
                                                   n_groups, seg, perm, adv, mean, std, ws, ws_bytes, stream);
  }
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict) return nullptr;
  for (int k = mixed ? REWARD : GROUP_ID; k < (mixed ? KEYS : BEST); ++k) {
    THPObjectPtr o(THPVariable_Wrap(std::move(out[k])));      // None where there is no tensor
    if (!o || PyDict_SetItem(dict.get(), g_keys[k], o.get()) != 0) return nullptr;
  }
  return dict.release();
  END_HANDLE_TH_ERRORS
}

// ---- queries, keys and the rollout's cache ------------------------------------------------------------
// Each of the functions below returns a dict, the call's status, or None where an argument is not what it should be (the caller says which).

PyObject *g_names[8], *g_q, *g_k, *g_dq, *g_dk, *g_dqw, *g_dkw, *g_out, *g_lse;
const char* const kFields[8] = {"cache_k", "cache_v", "pages", "length", "cu_q", "group_seq", "prefix_len", "prefix_pages"};

const at::Tensor* as_tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

bool known(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
int32_t code(at::ScalarType t) { return t == at::kFloat ? AT_GRPO_F32 : AT_GRPO_BF16; }

// Rows of heads [tokens, heads, D], of `like`'s dtype, device, tokens and D where there is one, of `heads` heads where that is not 0.
bool rows(PyObject* o, const at::Tensor* like, int64_t heads, at_grpo_rows* out, const at::Tensor** tensor) {
  const at::Tensor* t = as_tensor(o);
  if (!t || t->dim() != 3 || !t->is_cuda() || !known(t->scalar_type())) return false;
  if (like && (t->scalar_type() != like->scalar_type() || t->device() != like->device() || t->size(0) != like->size(0) || t->size(2) != like->size(2)))
    return false;
  if (heads && t->size(1) != heads) return false;
  const int64_t step = 16 / static_cast<int64_t>(t->element_size());
  out->data = t->data_ptr();
  out->token_stride = t->stride(0);
  out->head_stride = t->stride(1);
  if (t->numel() && (t->stride(2) != 1 || out->token_stride % step || out->head_stride % step || reinterpret_cast<uintptr_t>(out->data) % 16)) return false;
  *tensor = t;
  return t->size(0) <= 0x7fffffff && t->size(1) <= 0x7fffffff && t->size(2) <= 0x7fffffff;
}

// A contiguous vector of n elements on the device, or None (then null).
bool vector(PyObject* o, int64_t n, at::ScalarType dtype, at::Device device, const void** out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor* t = as_tensor(o);
  if (!t || t->dim() != 1 || t->size(0) != n || t->scalar_type() != dtype || t->device() != device || !t->is_contiguous()) return false;
  *out = t->data_ptr();
  return true;
}

bool layer_of(const at::Tensor& x, PyObject* rope, PyObject* qw, PyObject* kw, double eps, bool interleaved, at_grpo_norm_rope* out) {
  *out = at_grpo_norm_rope{code(x.scalar_type()), static_cast<int32_t>(x.size(2)), 0, interleaved ? AT_GRPO_ROPE_INTERLEAVED : AT_GRPO_ROPE_HALF,
                           0, static_cast<float>(eps), nullptr, nullptr, nullptr};
  if (rope != Py_None) {
    const at::Tensor* t = as_tensor(rope);
    if (!t || t->dim() != 3 || t->size(2) != 2 || t->scalar_type() != at::kFloat || t->device() != x.device() || !t->is_contiguous()) return false;
    if (t->size(0) > 0x7fffffff || t->size(1) > 0x3fffffff) return false;
    out->n_pos = static_cast<int32_t>(t->size(0));
    out->rot_dim = static_cast<int32_t>(2 * t->size(1));
    out->table = static_cast<const float*>(t->data_ptr());
  }
  return vector(qw, x.size(2), x.scalar_type(), x.device(), &out->q_weight) && vector(kw, x.size(2), x.scalar_type(), x.device(), &out->k_weight);
}

// The fields of a KVBatch.  The references keep the tensors alive while the call is made.
struct Cache {
  THPObjectPtr held[8];
  at_grpo_kv c{};
  const at::Tensor* k = nullptr;
};

bool cache_of(PyObject* o, Cache* out) {
  const at::Tensor* t[8] = {};
  for (int i = 0; i < 8; ++i) {
    out->held[i] = THPObjectPtr(PyObject_GetAttr(o, g_names[i]));
    if (!out->held[i]) {
      PyErr_Clear();
      return false;
    }
    if (out->held[i].get() == Py_None) continue;
    t[i] = as_tensor(out->held[i].get());
    if (!t[i] || !t[i]->is_cuda() || !t[i]->is_contiguous() || (i >= 2 && t[i]->scalar_type() != at::kInt) || (i && t[0] && t[i]->device() != t[0]->device()))
      return false;
  }
  if (!t[0] || !t[1] || !t[2] || !t[3]) return false;
  const at::Tensor &k = *t[0], &pages = *t[2];
  if (k.dim() != 4 || !known(k.scalar_type()) || t[1]->sizes() != k.sizes() || t[1]->scalar_type() != k.scalar_type()) return false;
  const int64_t n_seq = t[3]->numel(), n_group = t[5] ? t[5]->numel() - 1 : 0;
  if (pages.dim() != 2 || pages.size(0) != n_seq || (t[4] && t[4]->numel() != n_seq + 1)) return false;
  if (t[5] && (n_group < 0 || !t[6] || !t[7] || t[6]->numel() != n_group || t[7]->dim() != 2 || t[7]->size(0) != n_group)) return false;
  for (int64_t x : {k.size(0), k.size(1), k.size(2), k.size(3), n_seq, n_group, pages.size(1), n_group ? t[7]->size(1) : 0})
    if (x > 0x7fffffff) return false;
  const auto ints = [](const at::Tensor* x) { return x ? static_cast<const int32_t*>(x->data_ptr()) : nullptr; };
  out->k = t[0];
  out->c = at_grpo_kv{code(k.scalar_type()), static_cast<int32_t>(k.size(1)), static_cast<int32_t>(k.size(3)), static_cast<int32_t>(k.size(2)),
                      static_cast<int32_t>(k.size(0)), static_cast<int32_t>(n_seq), static_cast<int32_t>(pages.size(1)), static_cast<int32_t>(n_group),
                      n_group ? static_cast<int32_t>(t[7]->size(1)) : 0, k.data_ptr(), t[1]->data_ptr(), ints(t[2]), ints(t[3]), ints(t[4]),
                      n_group ? ints(t[5]) : nullptr, n_group ? ints(t[6]) : nullptr, n_group ? ints(t[7]) : nullptr};
  return true;
}

// Rows of the cache's dtype, head size and device.
bool cache_rows(const Cache& kv, PyObject* o, const at::Tensor* like, int64_t heads, at_grpo_rows* out, const at::Tensor** tensor) {
  return rows(o, like, heads, out, tensor) && (*tensor)->scalar_type() == kv.k->scalar_type() && (*tensor)->size(2) == kv.k->size(3) &&
         (*tensor)->device() == kv.k->device();
}

// The output that the caller gave, or a new one of the input's shape.
bool output(PyObject* given, const at::Tensor& like, at::Tensor* made, at_grpo_rows* out) {
  if (given != Py_None) {
    const at::Tensor* t;
    if (!rows(given, &like, like.size(1), out, &t)) return false;
    *made = *t;
    return true;
  }
  {
    const WithoutPythonLock others_run;
    *made = at::empty(like.sizes(), like.options());
  }
  *out = at_grpo_rows{made->data_ptr(), like.size(1) * like.size(2), like.size(2)};
  return true;
}

bool put(PyObject* dict, PyObject* key, at::Tensor&& t) {
  THPObjectPtr o(THPVariable_Wrap(std::move(t)));      // None where there is no tensor
  return o && PyDict_SetItem(dict, key, o.get()) == 0;
}

// qk_norm_rope(function's address, q, k, rope, position, q_weight, k_weight, eps, interleaved, q_out, k_out, data_error, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 13) {
    PyErr_SetString(PyExc_TypeError, "qk_norm_rope takes 13 arguments");
    return nullptr;
  }
  const at::Tensor *q = nullptr, *k = nullptr;
  at_grpo_rows rq{}, rk{}, oq{}, ok{};
  if ((v[1] != Py_None && !rows(v[1], nullptr, 0, &rq, &q)) || (v[2] != Py_None && !rows(v[2], q, 0, &rk, &k)) || (!q && !k)) Py_RETURN_NONE;
  const at::Tensor& x = q ? *q : *k;
  const double eps = PyFloat_AsDouble(v[7]);
  const bool interleaved = PyObject_IsTrue(v[8]) == 1;
  void* stream = PyLong_AsVoidPtr(v[12]);
  if (PyErr_Occurred()) return nullptr;
  at_grpo_norm_rope layer;
  const void *position, *word;
  if (!layer_of(x, v[3], v[5], v[6], eps, interleaved, &layer) || !vector(v[4], x.size(0), at::kInt, x.device(), &position) ||
      !vector(v[11], 1, at::kInt, x.device(), &word))
    Py_RETURN_NONE;
  at::Tensor out[2];
  if ((q && !output(v[9], *q, &out[0], &oq)) || (k && !output(v[10], *k, &out[1], &ok))) Py_RETURN_NONE;
  const int status = reinterpret_cast<decltype(&at_grpo_qk_norm_rope)>(PyLong_AsVoidPtr(v[0]))(
      &layer, static_cast<int32_t>(x.size(0)), q ? static_cast<int32_t>(q->size(1)) : 0, k ? static_cast<int32_t>(k->size(1)) : 0, &rq, &rk,
      static_cast<const int32_t*>(position), &oq, &ok, static_cast<int32_t*>(const_cast<void*>(word)), stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict || !put(dict.get(), g_q, std::move(out[0])) || !put(dict.get(), g_k, std::move(out[1]))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

// qk_norm_rope_bwd(function's address, dq_out, dk_out, q, k, rope, position, q_weight, k_weight, eps, interleaved, dq, dk, data_error,
//                  workspace, its bytes, stream)
PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 17) {
    PyErr_SetString(PyExc_TypeError, "qk_norm_rope_bwd takes 17 arguments");
    return nullptr;
  }
  const at::Tensor *q = nullptr, *k = nullptr, *unused;
  at_grpo_rows rq{}, rk{}, gq{}, gk{}, oq{}, ok{};
  if ((v[3] != Py_None && !rows(v[3], nullptr, 0, &rq, &q)) || (v[4] != Py_None && !rows(v[4], q, 0, &rk, &k)) || (!q && !k)) Py_RETURN_NONE;
  if ((q && !rows(v[1], q, q->size(1), &gq, &unused)) || (k && !rows(v[2], k, k->size(1), &gk, &unused))) Py_RETURN_NONE;
  const at::Tensor& x = q ? *q : *k;
  const double eps = PyFloat_AsDouble(v[9]);
  const bool interleaved = PyObject_IsTrue(v[10]) == 1;
  void* ws = PyLong_AsVoidPtr(v[14]);
  const size_t ws_bytes = PyLong_AsSize_t(v[15]);
  void* stream = PyLong_AsVoidPtr(v[16]);
  if (PyErr_Occurred()) return nullptr;
  at_grpo_norm_rope layer;
  const void *position, *word;
  if (!layer_of(x, v[5], v[7], v[8], eps, interleaved, &layer) || !vector(v[6], x.size(0), at::kInt, x.device(), &position) ||
      !vector(v[13], 1, at::kInt, x.device(), &word))
    Py_RETURN_NONE;
  at::Tensor out[4];
  if ((q && !output(v[11], *q, &out[0], &oq)) || (k && !output(v[12], *k, &out[1], &ok))) Py_RETURN_NONE;
  float* dw[2] = {nullptr, nullptr};
  for (int i = 0; i < 2; ++i)
    if (i ? k && layer.k_weight : q && layer.q_weight) {
      const WithoutPythonLock others_run;
      out[2 + i] = at::empty({x.size(2)}, x.options().dtype(at::kFloat));
      dw[i] = static_cast<float*>(out[2 + i].data_ptr());
    }
  const int status = reinterpret_cast<decltype(&at_grpo_qk_norm_rope_bwd)>(PyLong_AsVoidPtr(v[0]))(
      &layer, static_cast<int32_t>(x.size(0)), q ? static_cast<int32_t>(q->size(1)) : 0, k ? static_cast<int32_t>(k->size(1)) : 0, &gq, &gk, &rq, &rk,
      static_cast<const int32_t*>(position), &oq, &ok, dw[0], dw[1], static_cast<int32_t*>(const_cast<void*>(word)), ws, ws_bytes, stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  PyObject* const keys[4] = {g_dq, g_dk, g_dqw, g_dkw};
  if (!dict) return nullptr;
  for (int i = 0; i < 4; ++i)
    if (!put(dict.get(), keys[i], std::move(out[i]))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

// check_kv(KVBatch): whether its tensors belong together
PyObject* check_kv(PyObject*, PyObject* kv) {
  HANDLE_TH_ERRORS
  Cache cache;
  return PyBool_FromLong(cache_of(kv, &cache));
  END_HANDLE_TH_ERRORS
}

// kv_append(function's address, KVBatch, q, k, v, rope, q_weight, k_weight, eps, interleaved, q_out, data_error, stream)
PyObject* kv_append(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 13) {
    PyErr_SetString(PyExc_TypeError, "kv_append takes 13 arguments");
    return nullptr;
  }
  Cache kv;
  const at::Tensor *q = nullptr, *k, *val;
  at_grpo_rows rq{}, rk, rv, oq{};
  if (!cache_of(v[1], &kv) || !cache_rows(kv, v[3], nullptr, kv.c.Hk, &rk, &k) || !cache_rows(kv, v[4], k, kv.c.Hk, &rv, &val) ||
      (v[2] != Py_None && !cache_rows(kv, v[2], k, 0, &rq, &q)))
    Py_RETURN_NONE;
  const double eps = PyFloat_AsDouble(v[8]);
  const bool interleaved = PyObject_IsTrue(v[9]) == 1;
  void* stream = PyLong_AsVoidPtr(v[12]);
  if (PyErr_Occurred()) return nullptr;
  at_grpo_norm_rope layer;
  const void* word;
  if (!layer_of(*k, v[5], v[6], v[7], eps, interleaved, &layer) || !vector(v[11], 1, at::kInt, k->device(), &word)) Py_RETURN_NONE;
  at::Tensor out;
  if (q && !output(v[10], *q, &out, &oq)) Py_RETURN_NONE;
  const int status = reinterpret_cast<decltype(&at_grpo_kv_append)>(PyLong_AsVoidPtr(v[0]))(
      &kv.c, &layer, static_cast<int32_t>(k->size(0)), q ? static_cast<int32_t>(q->size(1)) : 0, &rq, &rk, &rv, &oq,
      static_cast<int32_t*>(const_cast<void*>(word)), stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict || !put(dict.get(), g_q, std::move(out))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

// prefix_attention(function's address, its workspace query's address, KVBatch, q, scale or None, causal, max_q, out, want_lse, data_error,
//                  workspace or None, stream)
// Where the workspace is none or too small: (bytes,).
PyObject* prefix_attention(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "prefix_attention takes 12 arguments");
    return nullptr;
  }
  Cache kv;
  const at::Tensor* q;
  at_grpo_rows rq, ro;
  if (!cache_of(v[2], &kv) || !cache_rows(kv, v[3], nullptr, 0, &rq, &q)) Py_RETURN_NONE;
  const double scale = v[4] == Py_None ? 1.0 / std::sqrt(static_cast<double>(q->size(2))) : PyFloat_AsDouble(v[4]);
  const int causal = PyObject_IsTrue(v[5]) == 1;
  const long long max_q = PyLong_AsLongLong(v[6]);
  const bool want_lse = PyObject_IsTrue(v[8]) == 1;
  void* stream = PyLong_AsVoidPtr(v[11]);
  if (PyErr_Occurred()) return nullptr;
  const void* word;
  if (max_q < 1 || max_q > 0x7fffffff || !vector(v[9], 1, at::kInt, q->device(), &word)) Py_RETURN_NONE;
  const int32_t n = static_cast<int32_t>(q->size(0)), heads = static_cast<int32_t>(q->size(1)), most = static_cast<int32_t>(max_q);
  const size_t bytes = reinterpret_cast<decltype(&at_grpo_prefix_attention_workspace_bytes)>(PyLong_AsVoidPtr(v[1]))(&kv.c, n, heads, most);
  if (bytes == 0) Py_RETURN_NONE;
  const at::Tensor* ws = as_tensor(v[10]);
  if (!ws || static_cast<size_t>(ws->numel()) < bytes) return Py_BuildValue("(n)", static_cast<Py_ssize_t>(bytes));
  at::Tensor out, lse;
  if (!output(v[7], *q, &out, &ro)) Py_RETURN_NONE;
  if (want_lse) {
    const WithoutPythonLock others_run;
    lse = at::empty({q->size(0), q->size(1)}, q->options().dtype(at::kFloat));
  }
  const int status = reinterpret_cast<decltype(&at_grpo_prefix_attention)>(PyLong_AsVoidPtr(v[0]))(
      &kv.c, n, heads, &rq, static_cast<float>(scale), causal, most, &ro, want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr,
      static_cast<int32_t*>(const_cast<void*>(word)), ws->data_ptr(), static_cast<size_t>(ws->numel()), stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict || !put(dict.get(), g_out, std::move(out)) || !put(dict.get(), g_lse, std::move(lse))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction fast(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}

PyMethodDef g_methods[] = {{"group_advantage", fast(group_advantage), METH_FASTCALL, nullptr},
                           {"qk_norm_rope", fast(qk_norm_rope), METH_FASTCALL, nullptr},
                           {"qk_norm_rope_bwd", fast(qk_norm_rope_bwd), METH_FASTCALL, nullptr},
                           {"check_kv", check_kv, METH_O, nullptr},
                           {"kv_append", fast(kv_append), METH_FASTCALL, nullptr},
                           {"prefix_attention", fast(prefix_attention), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  for (int k = 0; k < KEYS; ++k)
    if (!(g_keys[k] = PyUnicode_InternFromString(kKeyNames[k]))) return nullptr;
  for (int k = 0; k < 8; ++k)
    if (!(g_names[k] = PyUnicode_InternFromString(kFields[k]))) return nullptr;
  const std::pair<PyObject**, const char*> more[] = {{&g_q, "q"}, {&g_k, "k"}, {&g_dq, "dq"}, {&g_dk, "dk"}, {&g_dqw, "dq_weight"},
                                                     {&g_dkw, "dk_weight"}, {&g_out, "out"}, {&g_lse, "lse"}};
  for (const auto& [name, text] : more)
    if (!(*name = PyUnicode_InternFromString(text))) return nullptr;
  return PyModule_Create(&g_module);
}
