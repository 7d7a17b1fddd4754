"""Thin Python binding of libat_grpo.so: argument marshalling only (for the calls whose kernels are short in csrc/binding.cpp).

Every function has the name of the C entry point it calls (see include/at_grpo.h) and takes
torch tensors that already live on the GPU; outputs and the workspace are allocated here with
torch (device memory plumbing) and everything is enqueued on torch's current stream.  There is
no fallback: if the HIP library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence

import torch

# current stream of a device, as an integer (a torch without a GPU backend lacks it; there every call is refused before this)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libat_grpo.so")
_lib = None
_binding = None             # csrc/binding.cpp, loaded by the first call that goes through it
_group_fn = _mixed_fn = 0   # addresses of the library's grouping calls
_fn = {}                    # and of the others that go through it

AGG = {"token_mean": 0, "seq_mean_token_mean": 1}
NORM = {"std": 0, "none": 1}
NORM_FILL = 256      # or'ed into norm: the group buffers are filled behind the last group, so they need not be cleared
GROUP_BY = {"agent_turn": 0, "trajectory": 1, "parallel": 2}
CALL_GROUP_ADVANTAGE, CALL_TOKEN_LOGPROB, CALL_POLICY_LOSS_FWD, CALL_POLICY_LOSS_BWD, CALL_SURROGATE, \
    CALL_HEAD_UPDATE, CALL_DIAGNOSTICS, CALL_TOKEN_ENTROPY, CALL_POLICY_LOSS_FWD_BWD, CALL_QK_NORM_ROPE_BWD = range(10)
DTYPE = {torch.float32: 0, torch.bfloat16: 1}
ROPE_SCALING = {"plain": 0, "linear": 1, "base": 2, "parts": 3}

EXPORTS = [
    "at_grpo_group_advantage", "at_grpo_group_advantage_mixed", "at_grpo_group_advantage_static",
    "at_grpo_group_advantage_keyed", "at_grpo_group_advantage_keyed_workspace_bytes",
    "at_grpo_static_scratch_bytes", "at_grpo_token_logprob", "at_grpo_surrogate_from_logp",
    "at_grpo_surrogate_diagnostics", "at_grpo_token_entropy",
    "at_grpo_policy_loss_fwd", "at_grpo_policy_loss_bwd", "at_grpo_policy_loss_fwd_bwd", "at_grpo_head_update", "at_grpo_workspace_bytes",
    "at_grpo_status_string", "at_grpo_version", "at_grpo_profile_enable", "at_grpo_profile_classes",
    "at_grpo_profile_read", "at_grpo_rope_table", "at_grpo_qk_norm_rope", "at_grpo_qk_norm_rope_bwd", "at_grpo_kv_append",
    "at_grpo_prefix_attention", "at_grpo_prefix_attention_workspace_bytes",
]


class AtGrpoError(RuntimeError):
    pass


class _Adam(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("max_grad_norm", C.c_float), ("step", C.c_int32),
                ("decoupled", C.c_int32)]


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Rope(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("scaling", C.c_int32), ("base", C.c_double), ("factor", C.c_double), ("trained", C.c_double),
                ("slow", C.c_double), ("fast", C.c_double), ("magnitude", C.c_double)]


class _NormRope(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("D", C.c_int32), ("rot_dim", C.c_int32), ("layout", C.c_int32), ("n_pos", C.c_int32),
                ("eps", C.c_float), ("table", C.c_void_p), ("q_weight", C.c_void_p), ("k_weight", C.c_void_p)]


class _KV(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("Hk", C.c_int32), ("D", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32),
                ("n_seq", C.c_int32), ("max_pages", C.c_int32), ("n_group", C.c_int32), ("max_prefix_pages", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("pages", C.c_void_p), ("length", C.c_void_p), ("cu_q", C.c_void_p),
                ("group_seq", C.c_void_p), ("prefix_len", C.c_void_p), ("prefix_pages", C.c_void_p)]


class _Batch(C.Structure):
    _fields_ = [
        ("dtype", C.c_int32), ("H", C.c_int32), ("V", C.c_int32), ("n_heads", C.c_int32),
        ("n_tok", C.c_int64), ("n_resp", C.c_int32), ("n_agent", C.c_int32),
        ("cu_seqlens", C.c_void_p), ("hidden", C.c_void_p), ("W", C.POINTER(C.c_void_p)),
        ("token_id", C.c_void_p), ("mask", C.c_void_p), ("resp_agent", C.c_void_p),
        ("head_of_agent", C.c_void_p),
    ]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Loads libat_grpo.so (built in-tree by paper_2510_11062_amd.build); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise AtGrpoError(f"{_LIB_PATH} is missing: run `python -m paper_2510_11062_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(_LIB_PATH)
    vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
    lib.at_grpo_group_advantage.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, f32, i32, i32,
                                            vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.at_grpo_group_advantage.restype = C.c_int
    lib.at_grpo_group_advantage_mixed.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, vp, f32, f32, i32, i32,
                                                  vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.at_grpo_group_advantage_mixed.restype = C.c_int
    lib.at_grpo_group_advantage_keyed.argtypes = [i32, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, f32, i32, i32,
                                                  vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.at_grpo_group_advantage_keyed.restype = C.c_int
    lib.at_grpo_group_advantage_keyed_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.at_grpo_group_advantage_keyed_workspace_bytes.restype = sz
    lib.at_grpo_group_advantage_static.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, f32, i32, i32,
                                                   vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.at_grpo_group_advantage_static.restype = C.c_int
    lib.at_grpo_static_scratch_bytes.argtypes = []
    lib.at_grpo_static_scratch_bytes.restype = sz
    lib.at_grpo_token_logprob.argtypes = [C.POINTER(_Batch), vp, vp, vp, sz, vp]
    lib.at_grpo_token_logprob.restype = C.c_int
    lib.at_grpo_surrogate_from_logp.argtypes = [C.POINTER(_Batch), vp, vp, vp, f32, f32, i32, vp, vp, vp,
                                                vp, sz, vp]
    lib.at_grpo_surrogate_from_logp.restype = C.c_int
    lib.at_grpo_token_entropy.argtypes = [C.POINTER(_Batch), vp, vp, vp, vp, sz, vp]
    lib.at_grpo_token_entropy.restype = C.c_int
    lib.at_grpo_surrogate_diagnostics.argtypes = [C.POINTER(_Batch), vp, vp, vp, f32, f32, vp, vp, vp, sz, vp]
    lib.at_grpo_surrogate_diagnostics.restype = C.c_int
    lib.at_grpo_policy_loss_fwd.argtypes = [C.POINTER(_Batch), vp, vp, f32, f32, i32, vp, vp, vp, vp, vp,
                                            vp, sz, vp]
    lib.at_grpo_policy_loss_fwd.restype = C.c_int
    lib.at_grpo_head_update.argtypes = [i32, i32, i32, i32, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                        C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                        C.POINTER(_Adam), vp, vp, sz, vp]
    lib.at_grpo_head_update.restype = C.c_int
    lib.at_grpo_policy_loss_bwd.argtypes = [C.POINTER(_Batch), vp, vp, vp, vp, f32, f32, i32, vp, vp,
                                            C.POINTER(C.c_void_p), i32, vp, sz, vp]
    lib.at_grpo_policy_loss_bwd.restype = C.c_int
    lib.at_grpo_policy_loss_fwd_bwd.argtypes = [C.POINTER(_Batch), vp, vp, f32, f32, i32, vp, vp, vp, vp, vp, vp,
                                                vp, C.POINTER(C.c_void_p), i32, vp, sz, vp]
    lib.at_grpo_policy_loss_fwd_bwd.restype = C.c_int
    lib.at_grpo_workspace_bytes.argtypes = [i32, C.POINTER(_Batch), i32, i32, i32, i32]
    lib.at_grpo_workspace_bytes.restype = sz
    lib.at_grpo_status_string.argtypes = [i32]
    lib.at_grpo_status_string.restype = C.c_char_p
    lib.at_grpo_version.restype = i32
    lib.at_grpo_profile_enable.argtypes = [i32]
    lib.at_grpo_profile_classes.restype = i32
    lib.at_grpo_profile_read.argtypes = [i32, C.POINTER(C.c_char_p), C.POINTER(C.c_int64),
                                         C.POINTER(C.c_double)]
    rows, layer, kv = C.POINTER(_Rows), C.POINTER(_NormRope), C.POINTER(_KV)
    lib.at_grpo_rope_table.argtypes = [C.POINTER(_Rope), i32, vp, vp]
    lib.at_grpo_qk_norm_rope.argtypes = [layer, i32, i32, i32, rows, rows, vp, rows, rows, vp, vp]
    lib.at_grpo_qk_norm_rope_bwd.argtypes = [layer, i32, i32, i32, rows, rows, rows, rows, vp, rows, rows, vp, vp, vp, vp, sz, vp]
    lib.at_grpo_kv_append.argtypes = [kv, layer, i32, i32, rows, rows, rows, rows, vp, vp]
    lib.at_grpo_prefix_attention.argtypes = [kv, i32, i32, rows, f32, i32, i32, rows, vp, vp, vp, sz, vp]
    for name in ("at_grpo_rope_table", "at_grpo_qk_norm_rope", "at_grpo_qk_norm_rope_bwd", "at_grpo_kv_append", "at_grpo_prefix_attention"):
        getattr(lib, name).restype = C.c_int
    lib.at_grpo_prefix_attention_workspace_bytes.argtypes = [kv, i32, i32, i32]
    lib.at_grpo_prefix_attention_workspace_bytes.restype = sz
    _lib = lib
    return lib


def load_binding():
    """Loads _binding.so (built in-tree with the library) for the calls that go through it: two that group responses, and those on
    queries, keys and the rollout's cache; raises if it is missing or was built for another torch.  Every other call does without."""
    global _binding, _group_fn, _mixed_fn
    if _binding is None:
        lib = load_library()
        try:
            from . import _binding as binding
        except ImportError as e:
            raise AtGrpoError(f"_binding.so is missing or does not load ({e}): run `python -m paper_2510_11062_amd.build`") from e
        _group_fn = C.cast(lib.at_grpo_group_advantage, C.c_void_p).value
        _mixed_fn = C.cast(lib.at_grpo_group_advantage_mixed, C.c_void_p).value
        for name in ("at_grpo_qk_norm_rope", "at_grpo_qk_norm_rope_bwd", "at_grpo_kv_append", "at_grpo_prefix_attention",
                     "at_grpo_prefix_attention_workspace_bytes"):
            _fn[name] = C.cast(getattr(lib, name), C.c_void_p).value
        _binding = binding
    return _binding


def _check(status: int, what: str):
    if status != 0:
        msg = load_library().at_grpo_status_string(status).decode()
        raise AtGrpoError(f"{what} failed: {msg} (status {status})")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    return _raw_stream(torch.cuda.current_device())


def _dev_check(*tensors):
    for t in tensors:
        if t is not None and not (t.is_cuda and t.is_contiguous()):
            raise AtGrpoError("tensors must be contiguous CUDA/HIP tensors")


_workspace_cache = {}
_workspace_retired = []
_scratch_cache = {}      # (device, stream): (workspace, its part behind the error word)


def _workspace(nbytes: int, device) -> torch.Tensor:
    """A cached scratch tensor per (device, stream), grown on demand.

    Calls on different streams never share scratch (nothing orders them).  A workspace that is outgrown
    is kept alive until release_workspace(): a HIP graph captured earlier holds its raw pointer, and a
    replay must not find that memory handed to somebody else."""
    key = (device.index, _raw_stream(device.index))
    ws = _workspace_cache.get(key)
    if ws is None or ws.numel() < nbytes:
        if ws is not None:
            _workspace_retired.append(ws)
        ws = torch.empty(int(nbytes), dtype=torch.uint8, device=device)
        _workspace_cache[key] = ws
    return ws


def _scratch(nbytes: int, device) -> torch.Tensor:
    """The workspace behind its first 256 bytes, for calls that keep no error word: the last word of those that do stays there."""
    ws = _workspace(int(nbytes) + 256, device)
    scratch = ws[256:]
    scratch.keeps_no_error_word = True
    _scratch_cache[device.index, _raw_stream(device.index)] = ws, scratch
    return scratch


def _scratch_at_hand(key) -> Optional[torch.Tensor]:
    """What _scratch gave last for this (device, stream), if it is still part of the workspace."""
    held = _scratch_cache.get(key)
    return held[1] if held is not None and held[0] is _workspace_cache.get(key) else None


def release_workspace():
    """Drops every cached workspace (only when no captured graph that used the binding will be replayed)."""
    _workspace_cache.clear()
    _scratch_cache.clear()
    _workspace_retired.clear()


def _i32_check(**tensors):
    for name, t in tensors.items():
        if t is not None and t.dtype != torch.int32:
            raise AtGrpoError(f"{name} must be int32, got {t.dtype}")


def _f32_check(**tensors):
    for name, t in tensors.items():
        if t is not None and t.dtype != torch.float32:
            raise AtGrpoError(f"{name} must be float32, got {t.dtype}")


@dataclass
class Batch:
    """Python-side mirror of at_grpo_batch; keeps the tensors alive."""
    hidden: Optional[torch.Tensor]
    W: Optional[Sequence[torch.Tensor]]
    token_id: Optional[torch.Tensor]
    cu_seqlens: torch.Tensor
    mask: Optional[torch.Tensor] = None
    resp_agent: Optional[torch.Tensor] = None
    head_of_agent: Optional[torch.Tensor] = None
    n_tok: Optional[int] = None
    V: Optional[int] = None
    n_heads: Optional[int] = None

    def to_c(self):
        _dev_check(self.hidden, self.token_id, self.cu_seqlens, self.mask, self.resp_agent, self.head_of_agent)
        b = _Batch()
        if self.hidden is not None:
            if self.hidden.dtype == torch.float32:
                b.dtype = 0
            elif self.hidden.dtype == torch.bfloat16:
                b.dtype = 1
            else:
                raise AtGrpoError("hidden must be float32 or bfloat16")
            b.H = self.hidden.shape[1]
            n_tok = self.hidden.shape[0]
        else:
            b.dtype, b.H = 0, 0
            n_tok = self.n_tok
        heads = list(self.W) if self.W is not None else []
        for w in heads:
            _dev_check(w)
            if w.dtype != self.hidden.dtype or w.shape[1] != b.H:
                raise AtGrpoError("every head must have hidden's dtype and H columns")
        b.V = heads[0].shape[0] if heads else int(self.V)
        b.n_heads = len(heads) if heads else int(self.n_heads or 1)
        b.n_tok = int(n_tok)
        if self.cu_seqlens.dtype != torch.int64:
            raise AtGrpoError("cu_seqlens must be int64")
        b.n_resp = self.cu_seqlens.numel() - 1
        b.n_agent = 0 if self.head_of_agent is None else self.head_of_agent.numel()
        b.cu_seqlens = self.cu_seqlens.data_ptr()
        b.hidden = 0 if self.hidden is None else self.hidden.data_ptr()
        self._w_array = (C.c_void_p * max(len(heads), 1))(*[w.data_ptr() for w in heads])
        b.W = C.cast(self._w_array, C.POINTER(C.c_void_p)) if heads else None
        for name, dt in (("token_id", torch.int32), ("mask", torch.uint8), ("resp_agent", torch.int32),
                         ("head_of_agent", torch.int32)):
            t = getattr(self, name)
            if t is not None and t.dtype != dt:
                raise AtGrpoError(f"{name} must be {dt}")
            setattr(b, name, 0 if t is None else t.data_ptr())
        return b


def at_grpo_workspace_bytes(call: int, batch: Optional[Batch] = None, n_resp=0, n_env=0, n_agent=0, n_turn=0) -> int:
    lib = load_library()
    cb = batch.to_c() if batch is not None else None
    return int(lib.at_grpo_workspace_bytes(call, C.byref(cb) if cb is not None else None,
                                           n_resp, n_env, n_agent, n_turn))


def at_grpo_group_advantage(env_id, agent_id, turn_id, reward, n_env: int, n_agent: int, n_turn: int,
                            eps_std: float = 1e-6, ddof: int = 0, norm: str = "std", want_stats: bool = True):
    """Returns dict(group_id, n_groups, seg_offsets, perm, adv, group_mean, group_std, workspace)."""
    if _binding is None:
        load_binding()
    return _group_call("at_grpo_group_advantage", _group_fn, env_id, agent_id, turn_id, reward, None, 0.0, n_env, n_agent, n_turn,
                       eps_std, ddof, norm, want_stats, False)


def _group_call(what, fn, env_id, agent_id, turn_id, reward, r_loc, alpha, n_env, n_agent, n_turn, eps_std, ddof, norm, want_stats,
                want_best):
    out = None
    if reward.is_cuda:
        ws = _workspace(_group_workspace_bytes(0, reward.numel(), n_env, n_agent, n_turn, 1), reward.device)
        out = _binding.group_advantage(fn, env_id, agent_id, turn_id, reward, r_loc, alpha, n_env, n_agent, n_turn, eps_std, ddof,
                                       NORM[norm] | NORM_FILL, want_stats, want_best, ws.data_ptr(), ws.numel(), _stream())
    if type(out) is dict:
        out["workspace"] = ws
        return out
    if out is None:     # says which argument it was
        _dev_check(env_id, agent_id, turn_id, reward, r_loc)
        _f32_check(**(dict(reward=reward) if r_loc is None else dict(r_team=reward, r_loc=r_loc)))
        _i32_check(env_id=env_id, agent_id=agent_id, turn_id=turn_id)
        raise AtGrpoError(f"{what}: every argument must be a tensor")
    _check(out, what)


@functools.lru_cache(maxsize=256)
def _group_workspace_bytes(mode: int, R: int, n_env: int, n_agent: int, n_turn: int, n_sample: int) -> int:
    nbytes = load_library().at_grpo_group_advantage_keyed_workspace_bytes(mode, R, n_env, n_agent, n_turn, n_sample)
    if nbytes == 0:
        raise AtGrpoError("at_grpo_workspace_bytes rejected the id extents")
    return int(nbytes)


def _group_buffers(R: int, gmax: int, dev, want_stats: bool):
    """Uncleared outputs of a grouping call made with NORM_FILL (every entry is written)."""
    e = torch.empty
    i32, f32 = torch.int32, torch.float32
    return dict(group_id=e(R, dtype=i32, device=dev), n_groups=e(1, dtype=i32, device=dev),
                seg_offsets=e(gmax + 1, dtype=i32, device=dev), perm=e(R, dtype=i32, device=dev),
                adv=e(R, dtype=f32, device=dev), group_mean=e(gmax, dtype=f32, device=dev) if want_stats else None,
                group_std=e(gmax, dtype=f32, device=dev) if want_stats else None)


def group_advantage_outputs(R: int, n_keys: int, dev, want_stats: bool = True):
    """Output tensors of a grouping call (allocated by the caller, never by the library)."""
    gmax = min(R, n_keys)
    return dict(
        group_id=torch.empty(R, dtype=torch.int32, device=dev),
        n_groups=torch.zeros(1, dtype=torch.int32, device=dev),
        seg_offsets=torch.zeros(gmax + 1, dtype=torch.int32, device=dev),
        perm=torch.zeros(R, dtype=torch.int32, device=dev),
        adv=torch.empty(R, dtype=torch.float32, device=dev),
        group_mean=torch.zeros(gmax, dtype=torch.float32, device=dev) if want_stats else None,
        group_std=torch.zeros(gmax, dtype=torch.float32, device=dev) if want_stats else None,
        data_error=torch.zeros(1, dtype=torch.int32, device=dev),
    )


def at_grpo_group_advantage_keyed(group_by: str, env_id, agent_id, turn_id, reward, n_env: int, n_agent: int,
                                  n_turn: int, sample_id=None, n_sample: int = 1, eps_std: float = 1e-6,
                                  ddof: int = 0, norm: str = "std"):
    """at_grpo_group_advantage under the grouping `group_by` ("agent_turn", "trajectory", "parallel")."""
    lib = load_library()
    _dev_check(env_id, agent_id, turn_id, reward, sample_id)
    _f32_check(reward=reward)
    _i32_check(env_id=env_id, agent_id=agent_id, turn_id=turn_id, sample_id=sample_id)
    R = reward.numel()
    mode = GROUP_BY[group_by]
    n_keys = n_env if mode == 1 else n_env * n_agent * n_turn * (n_sample if mode == 2 else 1)
    out = _group_buffers(R, min(R, n_keys), reward.device, True)
    out["data_error"] = torch.zeros(1, dtype=torch.int32, device=reward.device)
    ws = _workspace(_group_workspace_bytes(mode, R, n_env, n_agent, n_turn, n_sample), reward.device)
    st = lib.at_grpo_group_advantage_keyed(mode, R, n_env, n_agent, n_turn, n_sample, _ptr(env_id), _ptr(agent_id),
                                           _ptr(turn_id), _ptr(sample_id), _ptr(reward), eps_std, ddof, NORM[norm] | NORM_FILL,
                                           _ptr(out["group_id"]), _ptr(out["n_groups"]), _ptr(out["seg_offsets"]),
                                           _ptr(out["perm"]), _ptr(out["adv"]), _ptr(out["group_mean"]),
                                           _ptr(out["group_std"]), _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_group_advantage_keyed")
    out["workspace"] = ws
    return out


def at_grpo_static_scratch_bytes() -> int:
    return int(load_library().at_grpo_static_scratch_bytes())


def at_grpo_group_advantage_static(env_id, agent_id, turn_id, reward, n_env: int, n_agent: int, n_turn: int,
                                   eps_std: float = 1e-6, ddof: int = 0, norm: str = "std",
                                   out: Optional[dict] = None):
    """at_grpo_group_advantage on the library's own fixed scratch array: no workspace is passed and the
    call allocates nothing (pass `out` from group_advantage_outputs to keep the binding from allocating
    either).  Returns the dict of outputs, data_error[1] holding the call's error word."""
    lib = load_library()
    _dev_check(env_id, agent_id, turn_id, reward)
    _f32_check(reward=reward)
    _i32_check(env_id=env_id, agent_id=agent_id, turn_id=turn_id)
    R = reward.numel()
    if out is None:
        out = group_advantage_outputs(R, n_env * n_agent * n_turn, reward.device)
    st = lib.at_grpo_group_advantage_static(R, n_env, n_agent, n_turn, _ptr(env_id), _ptr(agent_id), _ptr(turn_id),
                                            _ptr(reward), eps_std, ddof, NORM[norm], _ptr(out["group_id"]),
                                            _ptr(out["n_groups"]), _ptr(out["seg_offsets"]), _ptr(out["perm"]),
                                            _ptr(out["adv"]), _ptr(out.get("group_mean")), _ptr(out.get("group_std")),
                                            _ptr(out.get("data_error")), _stream())
    _check(st, "at_grpo_group_advantage_static")
    return out


def at_grpo_group_advantage_mixed(env_id, agent_id, turn_id, r_team, r_loc, alpha: float, n_env: int,
                                  n_agent: int, n_turn: int, eps_std: float = 1e-6, ddof: int = 0,
                                  norm: str = "std", want_stats: bool = True, want_best: bool = True):
    """Eq. (3) mixing in front of at_grpo_group_advantage, plus the per-group arg max.

    Returns the dict of at_grpo_group_advantage extended by reward[R] and best[min(R, keys)]."""
    if _binding is None:
        load_binding()
    if r_loc is None:
        raise AtGrpoError("at_grpo_group_advantage_mixed needs r_loc")
    return _group_call("at_grpo_group_advantage_mixed", _mixed_fn, env_id, agent_id, turn_id, r_team, r_loc, alpha, n_env, n_agent,
                       n_turn, eps_std, ddof, norm, want_stats, want_best)


def at_grpo_head_update(W, dW, m, v, step: int, W_master=None, lr: float = 1e-6, beta1: float = 0.9,
                        beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
                        max_grad_norm: float = 1.0, decoupled: bool = True):
    """Clip by the joint gradient norm, then one Adam step per head, in place on W / W_master / m / v.

    W, dW, m, v (and W_master for bf16 heads) are lists of [V, H] tensors.  Returns
    dict(grad_norm=tensor[2] (norm, factor), workspace)."""
    lib = load_library()
    n_heads = len(W)
    _dev_check(*W, *dW, *m, *v, *(W_master or []))
    V, H = W[0].shape
    dtype = DTYPE[W[0].dtype]
    dev = W[0].device

    def arr(ts):
        return (C.c_void_p * n_heads)(*[t.data_ptr() for t in ts])

    masters = arr(W_master) if W_master is not None else None
    opt = _Adam(lr, beta1, beta2, eps, weight_decay, max_grad_norm, step, 1 if decoupled else 0)
    grad_norm = torch.zeros(2, dtype=torch.float32, device=dev)
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_HEAD_UPDATE, None, 0, 0, 0, 0), dev)
    st = lib.at_grpo_head_update(dtype, H, V, n_heads, arr(W), masters, arr(dW), arr(m), arr(v), C.byref(opt),
                                 _ptr(grad_norm), _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_head_update")
    return dict(grad_norm=grad_norm, workspace=ws)


def at_grpo_token_logprob(batch: Batch, want_lse: bool = True):
    lib = load_library()
    cb = batch.to_c()
    dev = batch.hidden.device
    logp = torch.empty(cb.n_tok, dtype=torch.float32, device=dev)
    lse = torch.empty(cb.n_tok, dtype=torch.float32, device=dev) if want_lse else None
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_TOKEN_LOGPROB, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_token_logprob(C.byref(cb), _ptr(logp), _ptr(lse), _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_token_logprob")
    return dict(logp=logp, lse=lse, workspace=ws)


def at_grpo_token_entropy(batch: Batch):
    """logp, lse and the entropy of the next-token distribution at every participating row."""
    lib = load_library()
    cb = batch.to_c()
    dev = batch.hidden.device
    logp = torch.empty(cb.n_tok, dtype=torch.float32, device=dev)
    lse = torch.empty(cb.n_tok, dtype=torch.float32, device=dev)
    entropy = torch.empty(cb.n_tok, dtype=torch.float32, device=dev)
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_TOKEN_ENTROPY, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_token_entropy(C.byref(cb), _ptr(logp), _ptr(lse), _ptr(entropy), _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_token_entropy")
    return dict(logp=logp, lse=lse, entropy=entropy, workspace=ws)


def at_grpo_surrogate_from_logp(batch: Batch, logp, old_logp, adv, eps_low: float, eps_high: float,
                                agg: str = "token_mean"):
    lib = load_library()
    cb = batch.to_c()
    _dev_check(logp, old_logp, adv)
    _f32_check(logp=logp, old_logp=old_logp, adv=adv)
    dev = logp.device
    loss = torch.empty(cb.n_heads, dtype=torch.float32, device=dev)
    clip_mask = torch.empty(cb.n_tok, dtype=torch.uint8, device=dev)
    n_valid = torch.empty(cb.n_heads, dtype=torch.int32, device=dev)
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_SURROGATE, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_surrogate_from_logp(C.byref(cb), _ptr(logp), _ptr(old_logp), _ptr(adv), eps_low, eps_high,
                                         AGG[agg], _ptr(loss), _ptr(clip_mask), _ptr(n_valid), _ptr(ws),
                                         ws.numel(), _stream())
    _check(st, "at_grpo_surrogate_from_logp")
    return dict(loss=loss, clip_mask=clip_mask, n_valid=n_valid, workspace=ws)


def at_grpo_surrogate_diagnostics(batch: Batch, logp, old_logp, adv, eps_low: float, eps_high: float):
    """Returns dict(counts int32[n_heads, 4] (rows, below, above, zero-gradient),
    stats float32[n_heads, 2] (KL estimate, mean ratio), workspace)."""
    lib = load_library()
    cb = batch.to_c()
    _dev_check(logp, old_logp, adv)
    _f32_check(logp=logp, old_logp=old_logp, adv=adv)
    dev = logp.device
    counts = torch.empty((cb.n_heads, 4), dtype=torch.int32, device=dev)
    stats = torch.empty((cb.n_heads, 2), dtype=torch.float32, device=dev)
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_DIAGNOSTICS, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_surrogate_diagnostics(C.byref(cb), _ptr(logp), _ptr(old_logp), _ptr(adv), eps_low, eps_high,
                                           _ptr(counts), _ptr(stats), _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_surrogate_diagnostics")
    return dict(counts=counts, stats=stats, workspace=ws)


def at_grpo_policy_loss_fwd(batch: Batch, old_logp, adv, eps_low: float, eps_high: float,
                            agg: str = "token_mean", out: Optional[dict] = None):
    lib = load_library()
    cb = batch.to_c()
    _dev_check(old_logp, adv)
    _f32_check(old_logp=old_logp, adv=adv)
    dev = batch.hidden.device
    if out is None:
        out = dict(
            loss=torch.empty(cb.n_heads, dtype=torch.float32, device=dev),
            logp=torch.empty(cb.n_tok, dtype=torch.float32, device=dev),
            lse=torch.empty(cb.n_tok, dtype=torch.float32, device=dev),
            clip_mask=torch.empty(cb.n_tok, dtype=torch.uint8, device=dev),
            n_valid=torch.empty(cb.n_heads, dtype=torch.int32, device=dev),
        )
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_POLICY_LOSS_FWD, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_policy_loss_fwd(C.byref(cb), _ptr(old_logp), _ptr(adv), eps_low, eps_high, AGG[agg],
                                     _ptr(out["loss"]), _ptr(out["logp"]), _ptr(out["lse"]),
                                     _ptr(out["clip_mask"]), _ptr(out["n_valid"]), _ptr(ws), ws.numel(),
                                     _stream())
    _check(st, "at_grpo_policy_loss_fwd")
    out["workspace"] = ws
    return out


def at_grpo_policy_loss_bwd(batch: Batch, old_logp, adv, logp, lse, eps_low: float, eps_high: float,
                            agg: str = "token_mean", grad_loss=None, dW: Optional[List[torch.Tensor]] = None,
                            accumulate_dW: bool = False, d_hidden: Optional[torch.Tensor] = None):
    lib = load_library()
    cb = batch.to_c()
    _dev_check(old_logp, adv, logp, lse, grad_loss, d_hidden)
    _f32_check(old_logp=old_logp, adv=adv, logp=logp, lse=lse, grad_loss=grad_loss)
    if d_hidden is not None and (d_hidden.dtype != batch.hidden.dtype or d_hidden.shape != batch.hidden.shape):
        raise AtGrpoError("d_hidden must have hidden's dtype and shape")
    dev = batch.hidden.device
    if d_hidden is None:
        d_hidden = torch.empty_like(batch.hidden)
    if dW is None:
        if accumulate_dW:
            raise AtGrpoError("accumulate_dW needs dW tensors")
        dW = [torch.empty(w.shape, dtype=torch.float32, device=dev) for w in batch.W]
    for g in dW:
        _dev_check(g)
        if g.dtype != torch.float32:
            raise AtGrpoError("dW must be float32")
    dw_array = (C.c_void_p * len(dW))(*[g.data_ptr() for g in dW])
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_POLICY_LOSS_BWD, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_policy_loss_bwd(C.byref(cb), _ptr(old_logp), _ptr(adv), _ptr(logp), _ptr(lse), eps_low,
                                     eps_high, AGG[agg], _ptr(grad_loss), _ptr(d_hidden),
                                     C.cast(dw_array, C.POINTER(C.c_void_p)), 1 if accumulate_dW else 0,
                                     _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_policy_loss_bwd")
    return dict(d_hidden=d_hidden, dW=dW, workspace=ws)


def at_grpo_policy_loss_fwd_bwd(batch: Batch, old_logp, adv, eps_low: float, eps_high: float,
                                agg: str = "token_mean", grad_loss=None, dW: Optional[List[torch.Tensor]] = None,
                                accumulate_dW: bool = False, d_hidden: Optional[torch.Tensor] = None,
                                out: Optional[dict] = None):
    """Forward and backward of the policy loss from one pass over the logits; returns the outputs of both."""
    lib = load_library()
    cb = batch.to_c()
    _dev_check(old_logp, adv, grad_loss, d_hidden)
    _f32_check(old_logp=old_logp, adv=adv, grad_loss=grad_loss)
    if d_hidden is not None and (d_hidden.dtype != batch.hidden.dtype or d_hidden.shape != batch.hidden.shape):
        raise AtGrpoError("d_hidden must have hidden's dtype and shape")
    dev = batch.hidden.device
    if out is None:
        out = dict(
            loss=torch.empty(cb.n_heads, dtype=torch.float32, device=dev),
            logp=torch.empty(cb.n_tok, dtype=torch.float32, device=dev),
            lse=torch.empty(cb.n_tok, dtype=torch.float32, device=dev),
            clip_mask=torch.empty(cb.n_tok, dtype=torch.uint8, device=dev),
            n_valid=torch.empty(cb.n_heads, dtype=torch.int32, device=dev),
        )
    if d_hidden is None:
        d_hidden = torch.empty_like(batch.hidden)
    if dW is None:
        if accumulate_dW:
            raise AtGrpoError("accumulate_dW needs dW tensors")
        dW = [torch.empty(w.shape, dtype=torch.float32, device=dev) for w in batch.W]
    for g in dW:
        _dev_check(g)
        if g.dtype != torch.float32:
            raise AtGrpoError("dW must be float32")
    dw_array = (C.c_void_p * len(dW))(*[g.data_ptr() for g in dW])
    ws = _workspace(lib.at_grpo_workspace_bytes(CALL_POLICY_LOSS_FWD_BWD, C.byref(cb), 0, 0, 0, 0), dev)
    st = lib.at_grpo_policy_loss_fwd_bwd(C.byref(cb), _ptr(old_logp), _ptr(adv), eps_low, eps_high, AGG[agg],
                                         _ptr(grad_loss), _ptr(out["loss"]), _ptr(out["logp"]), _ptr(out["lse"]),
                                         _ptr(out["clip_mask"]), _ptr(out["n_valid"]), _ptr(d_hidden),
                                         C.cast(dw_array, C.POINTER(C.c_void_p)), 1 if accumulate_dW else 0,
                                         _ptr(ws), ws.numel(), _stream())
    _check(st, "at_grpo_policy_loss_fwd_bwd")
    out.update(d_hidden=d_hidden, dW=dW, workspace=ws)
    return out


def error_word(workspace: torch.Tensor) -> int:
    """Device error word of the last call that used this workspace (synchronises).  The calls on queries, keys and the cache keep none there."""
    if getattr(workspace, "keeps_no_error_word", False):
        raise AtGrpoError("this call keeps no error word in its workspace: it raises its bits in the data_error that it is given")
    return int(workspace[:4].view(torch.int32).item())


def at_grpo_profile_enable(on: bool):
    _check(load_library().at_grpo_profile_enable(1 if on else 0), "at_grpo_profile_enable")


def at_grpo_profile_read():
    """{kernel class: (launches, total_ms)} since profiling was enabled (synchronises)."""
    lib = load_library()
    out = {}
    for k in range(lib.at_grpo_profile_classes()):
        name = C.c_char_p()
        n = C.c_int64()
        ms = C.c_double()
        _check(lib.at_grpo_profile_read(k, C.byref(name), C.byref(n), C.byref(ms)), "at_grpo_profile_read")
        out[name.value.decode()] = (int(n.value), float(ms.value))
    return out


def at_grpo_version() -> int:
    return int(load_library().at_grpo_version())


# ---- queries, keys and the rollout's cache ------------------------------------------------------------
def at_grpo_rope_table(n_pos: int, rot_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, trained: float = 0.0,
                       slow: float = 1.0, fast: float = 32.0, magnitude: float = 1.0, device=None) -> torch.Tensor:
    """cos and sin of every position's angles, float32 [n_pos, rot_dim / 2, 2]; a program makes it once for all layers.

    `scaling` for contexts longer than the `trained` positions: "plain" (none), "linear" (frequencies / factor), "base" (a larger base),
    "parts" (pairs that turn more than `fast` times over the trained positions keep their frequency, those that turn less than `slow`
    times get frequency / factor, a ramp between)."""
    lib = load_library()
    if not 0 <= n_pos < 1 << 31 or not 0 < rot_dim <= 256 or rot_dim % 2:
        raise AtGrpoError("a rotation table has 0 to 2^31 - 1 positions and an even rot_dim of 2 to 256")
    table = torch.empty((n_pos, rot_dim // 2, 2), dtype=torch.float32, device="cuda" if device is None else device)
    _dev_check(table)
    c = _Rope(rot_dim, ROPE_SCALING[scaling], base, factor, trained, slow, fast, magnitude)
    _check(lib.at_grpo_rope_table(C.byref(c), n_pos, _ptr(table), _stream()), "at_grpo_rope_table")
    return table


def _rows(name: str, t: torch.Tensor, like: Optional[torch.Tensor], heads: Optional[int] = None):
    """Raises unless t is [tokens, heads, D] of the dtype, device, tokens and D of `like`, as at_grpo_rows can hold it."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3 or not t.is_cuda or t.dtype not in DTYPE:
        raise AtGrpoError(f"{name} must be a [tokens, heads, D] CUDA/HIP tensor of float32 or bfloat16")
    if like is not None and (t.dtype != like.dtype or t.device != like.device or t.shape[0] != like.shape[0] or t.shape[2] != like.shape[2]):
        raise AtGrpoError(f"{name} must have the dtype, device, tokens and head size of the other rows")
    if heads is not None and t.shape[1] != heads:
        raise AtGrpoError(f"{name} must have {heads} heads, got {t.shape[1]}")
    ts, hs, ds = t.stride()
    step = 16 // t.element_size()
    if t.numel() and (ds != 1 or ts % step or hs % step or t.data_ptr() % 16):
        raise AtGrpoError(f"{name}: the elements of a head must be contiguous, heads and tokens multiples of 16 bytes apart, and the data "
                          "16-byte aligned")


def _vector(name: str, t: Optional[torch.Tensor], n: int, dtype: torch.dtype, device):
    """Raises unless t is a contiguous 1-d tensor of n elements, or None."""
    if t is not None and (not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous()):
        raise AtGrpoError(f"{name} must be a contiguous {dtype} tensor of {n} elements on {device}")


def _layer(x: torch.Tensor, rope, q_weight, k_weight, eps: float, interleaved: bool):
    if rope is not None and (rope.dim() != 3 or rope.shape[2] != 2 or rope.dtype != torch.float32 or rope.device != x.device
                             or not rope.is_contiguous()):
        raise AtGrpoError("rope must be a contiguous float32 [positions, rot_dim / 2, 2] tensor on the rows' device")
    _vector("q_weight", q_weight, x.shape[2], x.dtype, x.device)
    _vector("k_weight", k_weight, x.shape[2], x.dtype, x.device)


def _word(data_error: Optional[torch.Tensor], device):
    return _vector("data_error", data_error, 1, torch.int32, device)


def at_grpo_qk_norm_rope(q, k, rope, position, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                         k_out=None, data_error=None):
    """Norm (where there is a weight) and rotation (where there is a table) of queries q [n, Hq, D] and keys k [n, Hk, D]; either may be
    None.  position int32 [n].  Outputs may be the inputs themselves.  Returns dict(q, k)."""
    if _binding is None:
        load_binding()
    x = q if q is not None else k
    out = None
    if x is not None and x.is_cuda:
        out = _binding.qk_norm_rope(_fn["at_grpo_qk_norm_rope"], q, k, rope, position, q_weight, k_weight, eps, interleaved, q_out, k_out,
                                    data_error, _stream())
    if type(out) is dict:
        return out
    x = _explain_qk(q, k, rope, position, q_weight, k_weight, eps, interleaved, dict(q_out=q_out), dict(k_out=k_out))
    _word(data_error, x.device)
    _refused(out, "at_grpo_qk_norm_rope")


def at_grpo_qk_norm_rope_bwd(dq_out, dk_out, q, k, rope, position, q_weight=None, k_weight=None, eps: float = 1e-6,
                             interleaved: bool = False, dq=None, dk=None, data_error=None):
    """Gradient of at_grpo_qk_norm_rope: from those of its outputs (and its inputs) to those of its inputs, in their dtype, and of the
    weights, float32 [D].  dq may be dq_out itself, dk dk_out.  Returns dict(dq, dk, dq_weight, dk_weight, workspace)."""
    if _binding is None:
        load_binding()
    x = q if q is not None else k
    out = None
    if x is not None and x.is_cuda:
        stream = _stream()
        ws = _scratch_at_hand((x.device.index, stream))
        if ws is None or ws.numel() < _rope_bwd_bytes():
            ws = _scratch(_rope_bwd_bytes(), x.device)
        out = _binding.qk_norm_rope_bwd(_fn["at_grpo_qk_norm_rope_bwd"], dq_out, dk_out, q, k, rope, position, q_weight, k_weight, eps, interleaved,
                                        dq, dk, data_error, ws.data_ptr(), ws.numel(), stream)
    if type(out) is dict:
        out["workspace"] = ws
        return out
    if q is not None and dq_out is None or k is not None and dk_out is None:
        raise AtGrpoError("the gradients of both outputs are needed")
    x = _explain_qk(q, k, rope, position, q_weight, k_weight, eps, interleaved, dict(dq_out=dq_out, dq=dq), dict(dk_out=dk_out, dk=dk))
    _word(data_error, x.device)
    _refused(out, "at_grpo_qk_norm_rope_bwd")


@functools.lru_cache(maxsize=1)
def _rope_bwd_bytes() -> int:
    return int(load_library().at_grpo_workspace_bytes(CALL_QK_NORM_ROPE_BWD, None, 0, 0, 0, 0))


def _explain_qk(q, k, rope, position, q_weight, k_weight, eps, interleaved, of_q, of_k):
    """Raises for the argument that the extension did not take, if there is one; returns the rows that the others go by."""
    x = q if q is not None else k
    if x is None:
        raise AtGrpoError("queries or keys are needed")
    if q is not None:
        _rows("q", q, None)
    if k is not None:
        _rows("k", k, q)
    _layer(x, rope, q_weight, k_weight, eps, interleaved)
    _vector("position", position, x.shape[0], torch.int32, x.device)
    for like, given in ((q, of_q), (k, of_k)):
        for name, t in given.items():
            if like is not None and t is not None:
                _rows(name, t, like, like.shape[1])
    return x


def _refused(out, what: str):
    if out is not None:
        _check(out, what)
    raise AtGrpoError(f"{what}: arguments that it does not take")


@dataclass
class KVBatch:
    """Python-side mirror of at_grpo_kv.  The tensors' contents may change between calls (lengths grow as tokens are appended)."""
    cache_k: torch.Tensor                       # [pages, Hk, page_size, D]
    cache_v: torch.Tensor
    pages: torch.Tensor                         # int32 [n_seq, max_pages]
    length: torch.Tensor                        # int32 [n_seq], new tokens counted
    cu_q: Optional[torch.Tensor] = None         # int32 [n_seq + 1]; None: one new token in every sequence
    group_seq: Optional[torch.Tensor] = None    # int32 [n_group + 1]; None: no prefixes
    prefix_len: Optional[torch.Tensor] = None   # int32 [n_group]
    prefix_pages: Optional[torch.Tensor] = None  # int32 [n_group, max_prefix_pages]

    def __post_init__(self):
        if _binding is None:
            load_binding()
        if not _binding.check_kv(self):
            self._explain()

    def _explain(self):
        """Raises for the tensor that does not belong with the others."""
        ck, cv = self.cache_k, self.cache_v
        _dev_check(ck, cv, self.pages, self.length, self.cu_q, self.group_seq, self.prefix_len, self.prefix_pages)
        _i32_check(pages=self.pages, length=self.length, cu_q=self.cu_q, group_seq=self.group_seq, prefix_len=self.prefix_len,
                   prefix_pages=self.prefix_pages)
        if ck.dim() != 4 or ck.dtype not in DTYPE or cv.shape != ck.shape or cv.dtype != ck.dtype:
            raise AtGrpoError("cache_k and cache_v must be [pages, heads, page_size, D] tensors of one shape, float32 or bfloat16")
        n_seq = self.length.numel()
        if self.pages.dim() != 2 or self.pages.shape[0] != n_seq:
            raise AtGrpoError("pages must be [n_seq, max_pages]")
        if self.cu_q is not None and self.cu_q.numel() != n_seq + 1:
            raise AtGrpoError("cu_q must have n_seq + 1 elements")
        if self.group_seq is not None:
            n_group = self.group_seq.numel() - 1
            if self.prefix_len is None or self.prefix_pages is None or n_group < 0 or self.prefix_len.numel() != n_group or \
                    self.prefix_pages.dim() != 2 or self.prefix_pages.shape[0] != n_group:
                raise AtGrpoError("groups need prefix_len [n_group] and prefix_pages [n_group, max_prefix_pages]")
        raise AtGrpoError("the tensors of a KVBatch must be on one device, with fewer than 2^31 rows and columns")

    def _rows(self, name: str, t: torch.Tensor, like: Optional[torch.Tensor], heads: Optional[int] = None):
        _rows(name, t, like, heads)
        if t.dtype != self.cache_k.dtype or t.shape[2] != self.cache_k.shape[3] or t.device != self.cache_k.device:
            raise AtGrpoError(f"{name} must have the cache's dtype, head size and device")


def at_grpo_kv_append(kv: KVBatch, q, k, v, rope, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                      data_error=None):
    """Normed and rotated keys k [n, Hk, D] and values v of the new tokens go into the cache; queries q [n, Hq, D] (or None), normed and
    rotated, to q_out, which may be q itself.  Returns dict(q)."""
    if _binding is None:
        load_binding()
    out = _binding.kv_append(_fn["at_grpo_kv_append"], kv, q, k, v, rope, q_weight, k_weight, eps, interleaved, q_out, data_error, _stream())
    if type(out) is dict:
        return out
    kv.__post_init__()
    heads = kv.cache_k.shape[1]
    kv._rows("k", k, None, heads)
    kv._rows("v", v, k, heads)
    if q is not None:
        kv._rows("q", q, k)
        if q_out is not None:
            kv._rows("q_out", q_out, q, q.shape[1])
    _layer(k, rope, q_weight, k_weight, eps, interleaved)
    _word(data_error, k.device)
    _refused(out, "at_grpo_kv_append")


def at_grpo_prefix_attention(kv: KVBatch, q, scale: Optional[float] = None, causal: bool = True, max_q: int = 1, out=None,
                             want_lse: bool = False, data_error=None):
    """Attention of the new tokens' queries q [n, Hq, D] over their sequences' tokens and their groups' prefixes (1 / sqrt(D) where no
    scale is given).  max_q: an upper bound of the new tokens of one sequence.  out may not share memory with q.
    Returns dict(out, lse, workspace)."""
    if _binding is None:
        load_binding()
    res = None
    if q.is_cuda:
        stream = _stream()
        ws = _scratch_at_hand((q.device.index, stream))
        call = lambda: _binding.prefix_attention(_fn["at_grpo_prefix_attention"], _fn["at_grpo_prefix_attention_workspace_bytes"], kv, q, scale,
                                                 causal, max_q, out, want_lse, data_error, ws, stream)
        res = call()
        if type(res) is tuple:
            ws = _scratch(res[0], q.device)
            res = call()
    if type(res) is dict:
        res["workspace"] = ws
        return res
    kv.__post_init__()
    kv._rows("q", q, None)
    if out is not None:
        kv._rows("out", out, q, q.shape[1])
    _word(data_error, q.device)
    if res is None:
        raise AtGrpoError("at_grpo_prefix_attention: heads, head size, page size, tokens or max_q that it does not cover")
    _refused(res, "at_grpo_prefix_attention")
