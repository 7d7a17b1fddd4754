// The calls whose kernels are short, as Python makes them: they check their tensors, make the outputs and enqueue the kernels.
//
// A grouping call of a training step is 7 to 17 us of kernels, so what the host does around it is what a program waits for: of 16.3
// us for 64 responses, seven outputs made one by one from Python were 9, the checks and pointers of the arguments 3.  A rollout's token
// takes 4 us of rotation, 4 of appending and 14 of attention a layer; made from Python, the first two took 18 and 24, now 6 and 6.5.  The plan of
// a step is 4 us of kernel with up to seven outputs, rules on the logits of four candidates 12, and both go this way too.  Everything else in
// api.py stays Python: those calls' kernels are longer than what the host does in front of them.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
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
// tree_attention: the same with ancestors in place of causal
// Where the workspace is none or too small: (bytes,).
template <bool TREE>
PyObject* attention(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 12) {
    PyErr_SetString(PyExc_TypeError, "prefix_attention and tree_attention take 12 arguments");
    return nullptr;
  }
  Cache kv;
  const at::Tensor* q;
  at_grpo_rows rq, ro;
  if (!cache_of(v[2], &kv) || !cache_rows(kv, v[3], nullptr, 0, &rq, &q)) Py_RETURN_NONE;
  const double scale = v[4] == Py_None ? 1.0 / std::sqrt(static_cast<double>(q->size(2))) : PyFloat_AsDouble(v[4]);
  const int causal = !TREE && PyObject_IsTrue(v[5]) == 1;
  const long long max_q = PyLong_AsLongLong(v[6]);
  const bool want_lse = PyObject_IsTrue(v[8]) == 1;
  void* stream = PyLong_AsVoidPtr(v[11]);
  if (PyErr_Occurred()) return nullptr;
  const void *word, *ancestors = nullptr;
  if (max_q < 1 || max_q > 0x7fffffff || !vector(v[9], 1, at::kInt, q->device(), &word)) Py_RETURN_NONE;
  if (TREE && (v[5] == Py_None || !vector(v[5], q->size(0), at::kLong, q->device(), &ancestors))) Py_RETURN_NONE;
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
  float* const sums = want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr;
  int32_t* const flags = static_cast<int32_t*>(const_cast<void*>(word));
  void* const fn = PyLong_AsVoidPtr(v[0]);
  const size_t held = static_cast<size_t>(ws->numel());
  const int status = TREE ? reinterpret_cast<decltype(&at_grpo_tree_attention)>(fn)(&kv.c, n, heads, &rq, static_cast<const uint64_t*>(ancestors),
                                                                                  static_cast<float>(scale), most, &ro, sums, flags, ws->data_ptr(), held, stream)
                          : reinterpret_cast<decltype(&at_grpo_prefix_attention)>(fn)(&kv.c, n, heads, &rq, static_cast<float>(scale), causal, most, &ro, sums,
                                                                                    flags, ws->data_ptr(), held, stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict || !put(dict.get(), g_out, std::move(out)) || !put(dict.get(), g_lse, std::move(lse))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

// ---- drafted tokens -----------------------------------------------------------------------------------

enum Planned { LENGTH, STATE, CU_Q, SEQ, POSITION, SLOT, ANCESTORS, PLANNED };
const char* const kPlanned[PLANNED] = {"length", "state", "cu_q", "seq", "position", "slot", "ancestors"};
enum PoolField { POOL_PAGES, RING, PAGE_SIZE, GROUP_SEQ, PREFIX_LEN, POOL_FIELDS };
const char* const kPoolFields[POOL_FIELDS] = {"pages", "ring", "page_size", "group_seq", "prefix_len"};
PyObject *g_planned[PLANNED], *g_pool[POOL_FIELDS];

template <typename X>
X* data(const at::Tensor& t) { return t.defined() ? static_cast<X*>(t.data_ptr()) : nullptr; }

// The attributes `names` of an object, kept alive; false where one is missing.
template <int N>
bool fields_of(PyObject* o, PyObject* const (&names)[N], THPObjectPtr (&held)[N]) {
  for (int i = 0; i < N; ++i) {
    held[i] = THPObjectPtr(PyObject_GetAttr(o, names[i]));
    if (!held[i]) {
      PyErr_Clear();
      return false;
    }
  }
  return true;
}

// A contiguous int32 matrix of so many rows on the device.
const at::Tensor* matrix(PyObject* o, int64_t n_rows, at::ScalarType dtype, at::Device device) {
  const at::Tensor* t = as_tensor(o);
  return t && t->dim() == 2 && (n_rows < 0 || t->size(0) == n_rows) && t->size(0) <= 0x7fffffff && t->size(1) <= 0x7fffffff &&
                 t->scalar_type() == dtype && t->device() == device && t->is_contiguous()
             ? t
             : nullptr;
}

// group_seq and what stands beside it, [n_group]: both or none
bool groups_of(PyObject* group_seq, PyObject* beside, at::Device device, const void** seq, const void** len, int32_t* n_group) {
  *seq = *len = nullptr;
  *n_group = 0;
  if (group_seq == Py_None) return true;
  const at::Tensor* t = as_tensor(group_seq);
  if (!t || t->dim() != 1 || t->size(0) < 1 || t->size(0) > 0x7fffffff || beside == Py_None) return false;
  *n_group = static_cast<int32_t>(t->size(0) - 1);
  return vector(group_seq, t->size(0), at::kInt, device, seq) && vector(beside, *n_group, at::kInt, device, len);
}

// kv_plan(function's address, its workspace query's, PagePool, length, add, state, n_tok, keep, parent, length_out, state_out, data_error,
//         workspace or None, stream)
// Where the workspace is none or too small: (bytes,).
PyObject* kv_plan(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 14) {
    PyErr_SetString(PyExc_TypeError, "kv_plan takes 14 arguments");
    return nullptr;
  }
  THPObjectPtr held[POOL_FIELDS];
  if (!fields_of(v[2], g_pool, held)) Py_RETURN_NONE;
  const at::Tensor *length = as_tensor(v[3]), *ring = as_tensor(held[RING].get());
  if (!length || length->dim() != 1 || !length->is_cuda() || length->size(0) > 0x7fffffff || !ring || ring->dim() != 1 || ring->size(0) > 0x7fffffff)
    Py_RETURN_NONE;
  const int64_t n_seq = length->size(0), page_size = PyLong_AsLongLong(held[PAGE_SIZE].get()), n_tok = PyLong_AsLongLong(v[6]);
  void* stream = PyLong_AsVoidPtr(v[13]);
  if (PyErr_Occurred()) return nullptr;
  const at::Device device = length->device();
  const at::Tensor* pages = matrix(held[POOL_PAGES].get(), n_seq, at::kInt, device);
  const void *lengths, *free_pages, *adds, *states, *keeps, *parents, *group_seq, *prefix_len, *word;
  int32_t n_group;
  if (!pages || page_size < 0 || page_size > 0x7fffffff || n_tok < 0 || n_tok > 0x7fffffff || v[5] == Py_None || v[4] == Py_None ||
      !vector(v[3], n_seq, at::kInt, device, &lengths) || !vector(held[RING].get(), ring->size(0), at::kInt, device, &free_pages) ||
      !vector(v[4], n_seq, at::kInt, device, &adds) || !vector(v[5], 2, at::kInt, device, &states) || !vector(v[7], n_seq, at::kInt, device, &keeps) ||
      !vector(v[8], n_tok, at::kInt, device, &parents) || !vector(v[11], 1, at::kInt, device, &word) ||
      !groups_of(held[GROUP_SEQ].get(), held[PREFIX_LEN].get(), device, &group_seq, &prefix_len, &n_group))
    Py_RETURN_NONE;
  const at_grpo_page_pool pool{static_cast<int32_t>(page_size), static_cast<int32_t>(ring->size(0)), static_cast<int32_t>(n_seq),
                               static_cast<int32_t>(pages->size(1)), n_group, data<int32_t>(*pages),
                               static_cast<int32_t*>(const_cast<void*>(free_pages)), static_cast<const int32_t*>(group_seq),
                               static_cast<const int32_t*>(prefix_len)};
  const size_t bytes = reinterpret_cast<decltype(&at_grpo_kv_plan_workspace_bytes)>(PyLong_AsVoidPtr(v[1]))(pool.n_seq);
  const at::Tensor* ws = as_tensor(v[12]);
  if (!ws || static_cast<size_t>(ws->numel()) < bytes) return Py_BuildValue("(n)", static_cast<Py_ssize_t>(bytes));
  // New outputs are views of one buffer: seven made one by one take 4 of the call's 11 us.
  at::Tensor out[PLANNED];
  const int64_t sizes[PLANNED] = {n_seq, 2, n_seq + 1, n_tok, n_tok, n_tok, n_tok};
  int64_t place[PLANNED + 1] = {0};      // in bytes
  for (int i = 0; i < PLANNED; ++i) {
    PyObject* const given = i == LENGTH ? v[9] : i == STATE ? v[10] : Py_None;
    const void* at;
    place[i + 1] = place[i];
    if (given != Py_None) {
      if (!vector(given, sizes[i], at::kInt, device, &at)) Py_RETURN_NONE;
      out[i] = *as_tensor(given);
    } else if (i != ANCESTORS || v[8] != Py_None) {
      place[i + 1] += (sizes[i] * (i >= SLOT ? 8 : 4) + 15) / 16 * 16;
    }
  }
  {
    const WithoutPythonLock others_run;
    const at::Tensor buffer = at::empty({place[PLANNED]}, length->options().dtype(at::kByte));
    for (int i = 0; i < PLANNED; ++i) {
      if (out[i].defined() || (i == ANCESTORS && v[8] == Py_None)) continue;
      const at::ScalarType dtype = i >= SLOT ? at::kLong : at::kInt;
      out[i] = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buffer.storage()), buffer.key_set(), c10::scalarTypeToTypeMeta(dtype));
      out[i].unsafeGetTensorImpl()->set_storage_offset(place[i] / (i >= SLOT ? 8 : 4));
      out[i].unsafeGetTensorImpl()->set_sizes_contiguous(c10::IntArrayRef(&sizes[i], 1));
    }
  }
  const int status = reinterpret_cast<decltype(&at_grpo_kv_plan)>(PyLong_AsVoidPtr(v[0]))(
      &pool, static_cast<int32_t>(n_tok), static_cast<const int32_t*>(lengths), static_cast<const int32_t*>(keeps), static_cast<const int32_t*>(adds),
      static_cast<const int32_t*>(parents), static_cast<const int32_t*>(states), data<int32_t>(out[LENGTH]), data<int32_t>(out[STATE]),
      data<int32_t>(out[CU_Q]), data<int32_t>(out[SEQ]), data<int32_t>(out[POSITION]), data<int64_t>(out[SLOT]), data<uint64_t>(out[ANCESTORS]),
      static_cast<int32_t*>(const_cast<void*>(word)), ws->data_ptr(), static_cast<size_t>(ws->numel()), stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict) return nullptr;
  for (int i = 0; i < PLANNED; ++i)
    if (!put(dict.get(), g_planned[i], std::move(out[i]))) return nullptr;
  return dict.release();
  END_HANDLE_TH_ERRORS
}

enum RuleField {
  R_TOKENS, R_LENGTH, R_PROMPT, R_PROMPT_LEN, R_GROUP_SEQ, R_CU_Q, R_DRAFTED, R_ANCESTORS, R_REPETITION, R_PRESENCE, R_FREQUENCY, R_TEMPERATURE, R_BIAS_CU,
  R_BIAS_TOKEN, R_BIAS, R_ALLOWED, R_MASK_ROW, RULE_FIELDS
};
const char* const kRuleFields[RULE_FIELDS] = {"tokens", "length", "prompt", "prompt_len", "group_seq", "cu_q", "drafted", "ancestors", "repetition", "presence",
                                              "frequency", "temperature", "bias_cu", "bias_token", "bias", "allowed", "mask_row"};
PyObject *g_rule[RULE_FIELDS], *g_best;

// Rows [n, V] with contiguous elements, as far apart as they are long or farther.
const at::Tensor* logit_rows(PyObject* o) {
  const at::Tensor* t = as_tensor(o);
  return t && t->dim() == 2 && t->is_cuda() && known(t->scalar_type()) && t->size(0) <= 0x7fffffff && t->size(1) <= 0x7fffffff &&
                 (t->numel() == 0 || ((t->stride(1) == 1 || t->size(1) == 1) && (t->size(0) == 1 || t->stride(0) >= t->size(1))))
             ? t
             : nullptr;
}

// The fields of a LogitRules for n rows of V logits.
bool sampling_rules(THPObjectPtr (&held)[RULE_FIELDS], int64_t n, int64_t V, at::Device device, at_grpo_sampling_rules* r) {
  const auto field = [&](int i) { return held[i].get(); };
  const auto there = [&](int i) { return field(i) != Py_None; };
  int64_t n_seq = n;
  if (there(R_CU_Q)) {
    const at::Tensor* t = as_tensor(field(R_CU_Q));
    if (!t || t->dim() != 1 || t->size(0) < 1 || t->size(0) > 0x7fffffff) return false;
    n_seq = t->size(0) - 1;
  }
  r->n_seq = static_cast<int32_t>(n_seq);
  const void *cu, *len, *groups, *prompt_len, *drafted, *ancestors, *bias_cu, *bias_token, *bias, *mask_row;
  if (!vector(field(R_CU_Q), n_seq + 1, at::kInt, device, &cu) || !vector(field(R_DRAFTED), n, at::kInt, device, &drafted) ||
      !vector(field(R_ANCESTORS), n, at::kLong, device, &ancestors) || !vector(field(R_MASK_ROW), n, at::kInt, device, &mask_row))
    return false;
  r->cu_q = static_cast<const int32_t*>(cu);
  r->drafted = static_cast<const int32_t*>(drafted);
  r->ancestors = static_cast<const uint64_t*>(ancestors);
  r->mask_row = static_cast<const int32_t*>(mask_row);
  const float** const settings[4] = {&r->repetition, &r->presence, &r->frequency, &r->temperature};
  for (int i = 0; i < 4; ++i) {
    const void* p;
    if (!vector(field(R_REPETITION + i), n_seq, at::kFloat, device, &p)) return false;
    *settings[i] = static_cast<const float*>(p);
  }
  if (there(R_TOKENS)) {
    const at::Tensor* t = matrix(field(R_TOKENS), n_seq, at::kInt, device);
    if (!t || !there(R_LENGTH) || !vector(field(R_LENGTH), n_seq, at::kInt, device, &len)) return false;
    r->tokens = data<const int32_t>(*t);
    r->length = static_cast<const int32_t*>(len);
    r->max_tokens = static_cast<int32_t>(t->size(1));
  }
  if (there(R_PROMPT)) {
    if (!there(R_GROUP_SEQ) || !groups_of(field(R_GROUP_SEQ), field(R_PROMPT_LEN), device, &groups, &prompt_len, &r->n_group)) return false;
    const at::Tensor* t = matrix(field(R_PROMPT), r->n_group, at::kInt, device);
    if (!t) return false;
    r->group_seq = static_cast<const int32_t*>(groups);
    r->prompt_len = static_cast<const int32_t*>(prompt_len);
    r->prompt = r->n_group ? data<const int32_t>(*t) : nullptr;
    r->max_prompt = static_cast<int32_t>(t->size(1));
  }
  if (there(R_BIAS_CU)) {
    const at::Tensor* t = as_tensor(field(R_BIAS));
    const int64_t m = t && t->dim() == 1 ? t->size(0) : -1;
    if (m < 0 || m > 0x7fffffff || !there(R_BIAS_TOKEN) || !vector(field(R_BIAS_CU), n_seq + 1, at::kInt, device, &bias_cu) ||
        !vector(field(R_BIAS_TOKEN), m, at::kInt, device, &bias_token) || !vector(field(R_BIAS), m, at::kFloat, device, &bias))
      return false;
    r->bias_cu = static_cast<const int32_t*>(bias_cu);
    r->bias_token = static_cast<const int32_t*>(bias_token);
    r->bias = static_cast<const float*>(bias);
    r->n_bias = static_cast<int32_t>(m);
  }
  if (there(R_ALLOWED)) {
    const at::Tensor* t = matrix(field(R_ALLOWED), -1, at::kInt, device);
    if (!t || t->size(1) != (V + 31) / 32 || !there(R_MASK_ROW)) return false;
    r->allowed = t->size(0) ? data<const uint32_t>(*t) : nullptr;
    r->n_mask = static_cast<int32_t>(t->size(0));
  }
  return true;
}

// logit_rules(function's address, its workspace query's, LogitRules, logits, out or None, the dtype of a new one or None, want_lse, want_best,
//             data_error, workspace or None, stream)
// Where the workspace is none or too small: (bytes,).
PyObject* logit_rules(PyObject*, PyObject* const* v, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (n_args != 11) {
    PyErr_SetString(PyExc_TypeError, "logit_rules takes 11 arguments");
    return nullptr;
  }
  THPObjectPtr held[RULE_FIELDS];
  const at::Tensor *logits = logit_rows(v[3]), *given = v[4] == Py_None ? nullptr : logit_rows(v[4]);
  if (!logits || !fields_of(v[2], g_rule, held) || (v[4] != Py_None && !given)) Py_RETURN_NONE;
  const int64_t n = logits->size(0), V = logits->size(1);
  if (given && (given->sizes() != logits->sizes() || given->device() != logits->device())) Py_RETURN_NONE;
  const bool want_lse = PyObject_IsTrue(v[6]) == 1, want_best = PyObject_IsTrue(v[7]) == 1;
  void* stream = PyLong_AsVoidPtr(v[10]);
  if (PyErr_Occurred()) return nullptr;
  const void* word;
  at_grpo_sampling_rules r{};
  r.dtype = r.out_dtype = code(logits->scalar_type());
  r.V = static_cast<int32_t>(V);
  if (!vector(v[8], 1, at::kInt, logits->device(), &word) || !sampling_rules(held, n, V, logits->device(), &r)) Py_RETURN_NONE;
  at::Tensor out, lse, best;
  if (given) {
    out = *given;
  } else if (v[5] != Py_None) {
    if (!THPDtype_Check(v[5]) || !known(reinterpret_cast<THPDtype*>(v[5])->scalar_type)) Py_RETURN_NONE;
    const WithoutPythonLock others_run;
    out = at::empty({n, V}, logits->options().dtype(reinterpret_cast<THPDtype*>(v[5])->scalar_type));
  }
  if (out.defined()) r.out_dtype = code(out.scalar_type());
  const size_t bytes = reinterpret_cast<decltype(&at_grpo_logit_rules_workspace_bytes)>(PyLong_AsVoidPtr(v[1]))(&r, static_cast<int32_t>(n));
  if (bytes == 0) Py_RETURN_NONE;
  const at::Tensor* ws = as_tensor(v[9]);
  if (!ws || static_cast<size_t>(ws->numel()) < bytes) return Py_BuildValue("(n)", static_cast<Py_ssize_t>(bytes));
  {
    const WithoutPythonLock others_run;
    if (want_lse) lse = at::empty({n}, logits->options().dtype(at::kFloat));
    if (want_best) best = at::empty({n}, logits->options().dtype(at::kInt));
  }
  const int status = reinterpret_cast<decltype(&at_grpo_logit_rules)>(PyLong_AsVoidPtr(v[0]))(
      &r, static_cast<int32_t>(n), logits->data_ptr(), logits->stride(0), data<void>(out), out.defined() ? out.stride(0) : 0, data<float>(lse),
      data<int32_t>(best), static_cast<int32_t*>(const_cast<void*>(word)), ws->data_ptr(), static_cast<size_t>(ws->numel()), stream);
  if (status != AT_GRPO_OK) return PyLong_FromLong(status);
  THPObjectPtr dict(PyDict_New());
  if (!dict || !put(dict.get(), g_out, std::move(out)) || !put(dict.get(), g_lse, std::move(lse)) || !put(dict.get(), g_best, std::move(best))) return nullptr;
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
                           {"prefix_attention", fast(attention<false>), METH_FASTCALL, nullptr},
                           {"tree_attention", fast(attention<true>), METH_FASTCALL, nullptr},
                           {"kv_plan", fast(kv_plan), METH_FASTCALL, nullptr},
                           {"logit_rules", fast(logit_rules), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
  for (int k = 0; k < KEYS; ++k)
    if (!(g_keys[k] = PyUnicode_InternFromString(kKeyNames[k]))) return nullptr;
  for (int k = 0; k < 8; ++k)
    if (!(g_names[k] = PyUnicode_InternFromString(kFields[k]))) return nullptr;
  for (int k = 0; k < PLANNED; ++k)
    if (!(g_planned[k] = PyUnicode_InternFromString(kPlanned[k]))) return nullptr;
  for (int k = 0; k < POOL_FIELDS; ++k)
    if (!(g_pool[k] = PyUnicode_InternFromString(kPoolFields[k]))) return nullptr;
  for (int k = 0; k < RULE_FIELDS; ++k)
    if (!(g_rule[k] = PyUnicode_InternFromString(kRuleFields[k]))) return nullptr;
  const std::pair<PyObject**, const char*> more[] = {{&g_q, "q"}, {&g_k, "k"}, {&g_dq, "dq"}, {&g_dk, "dk"}, {&g_dqw, "dq_weight"},
                                                     {&g_dkw, "dk_weight"}, {&g_out, "out"}, {&g_lse, "lse"}, {&g_best, "best"}};
  for (const auto& [name, text] : more)
    if (!(*name = PyUnicode_InternFromString(text))) return nullptr;
  return PyModule_Create(&g_module);
}
