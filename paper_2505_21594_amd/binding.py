"""Thin ctypes binding over libeeverify.so: argument marshalling only.

Every step of the verification pass runs in the library's HIP kernels; this
module never computes anything itself and has no CPU fallback: if the shared
library is missing or does not load, importing the names below raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np

from . import build as _build

EE_MAX_M = 16
EE_MAX_EXITS = 40
EE_MAX_BATCH = 16
EE_MAX_ROWS = 48

EE_OK, EE_NOT_READY, EE_DONE = 0, 1, 2
EE_EINVAL, EE_ESTATE, EE_ECAPACITY, EE_EIO, EE_EFORMAT, EE_EDEVICE = -1, -2, -3, -4, -5, -6

HOLD_LAST, CONTINUE = 1, 2
KEEP_LOGITS = 1
NO_AUTOCOMMIT = 2
SAMPLING = 4
TIME_LAUNCHES = 16
FORM_AUTO, FORM_PLAIN, FORM_PACKED = 0, 1, 2
OPT_ATT_SPLITS, OPT_SCATTER_PAGES, OPT_HEAD_BATCH, OPT_PREFILL_GEMM, OPT_PREFILL_ATT_ROWS, OPT_SHARED_ATT = 1, 2, 3, 4, 5, 6
BF16, FP16, FP32 = 0, 1, 2
ACT_NONE, ACT_SILU, ACT_GELU = 0, 1, 2
EE_MAX_TOP, EE_NORM_MAX_DIM, EE_NORM_MAX_ROWS, EE_LINEAR_MAX = 64, 16384, 1 << 21, 1 << 22
LAUNCH_NAMES = ("qkv", "o", "gu", "dn", "head", "adapter_down", "adapter_up", "embed", "att", "sample")

EXPORTS = [
    "ee_last_error", "ee_model_load", "ee_model_load_ex", "ee_model_load_form", "ee_model_free", "ee_model_info", "ee_model_packed_bytes",
    "ee_session_create", "ee_session_free", "ee_session_fork", "ee_prefill", "ee_prefill_embeds", "ee_verify",
    "ee_verify_batch", "ee_verify_static", "ee_verify_sampled", "ee_wait_exit", "ee_query_exit", "ee_wait_final", "ee_query_final",
    "ee_pass_time_ms", "ee_kv_truncate", "ee_set_pending", "ee_kv_len", "ee_pending",
    "ee_verify_sampled_batch", "ee_debug_logits", "ee_debug_mfma_layout", "ee_debug_div_small", "ee_debug_linear_plan", "ee_tune_k_split", "ee_device_synchronize", "ee_session_option",
    "ee_launch_times", "ee_debug_copy", "ee_exit_pop", "ee_exit_order", "ee_latency_model",
    "ee_kv_append", "ee_attend", "ee_attend_workspace", "ee_accept_drafts", "ee_accept_workspace",
    "ee_score_tokens", "ee_score_workspace", "ee_distill", "ee_distill_workspace", "ee_norm", "ee_norm_grad", "ee_norm_grad_workspace",
    "ee_linear", "ee_linear_workspace", "ee_linear_grad", "ee_linear_grad_workspace",
]


class EEError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"[{code}] {msg}")
        self.code = code


class ModelConfigC(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("n_exits", ctypes.c_int32), ("exit_layers", ctypes.c_int32 * EE_MAX_EXITS),
                ("rope_base", ctypes.c_float), ("rms_eps", ctypes.c_float),
                ("n_adapters", ctypes.c_int32), ("adapter_width", ctypes.c_int32),
                ("max_rows", ctypes.c_int32), ("n_workgroups", ctypes.c_int32)]


class SamplingC(ctypes.Structure):
    _fields_ = [("draft_probs", ctypes.POINTER(ctypes.c_float)), ("u", ctypes.POINTER(ctypes.c_float)),
                ("v", ctypes.POINTER(ctypes.c_float)), ("temperature", ctypes.c_float)]


class VerifyResultC(ctypes.Structure):
    _fields_ = [("gamma", ctypes.c_int32), ("n_exits", ctypes.c_int32),
                ("accept_len", ctypes.c_int32), ("next_token", ctypes.c_int32),
                ("final_tokens", ctypes.c_int32 * EE_MAX_M),
                ("exit_accept_len", ctypes.c_int32 * EE_MAX_EXITS),
                ("exit_tokens", (ctypes.c_int32 * EE_MAX_M) * EE_MAX_EXITS),
                ("device_status", ctypes.c_int32), ("reserved", ctypes.c_int32 * 15),
                ("final_conf", ctypes.c_float * EE_MAX_M), ("exit_conf", (ctypes.c_float * EE_MAX_M) * EE_MAX_EXITS)]


class LatencyParamsC(ctypes.Structure):
    _fields_ = [("T_p", ctypes.c_double), ("T_q", ctypes.c_double), ("T_c", ctypes.c_double), ("T_r", ctypes.c_double),
                ("tau", ctypes.c_double), ("r", ctypes.c_double), ("gamma", ctypes.c_int32), ("n", ctypes.c_int32)]


class LatencyC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("ar_ms", "sd_ms", "fsd_ms", "ar_ms_per_token", "sd_ms_per_token", "fsd_ms_per_token",
                                                "speedup_ar_to_sd", "speedup_sd_to_fsd", "c", "projected_sd_to_fsd")]


class PagedCacheC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "n_kv_heads", "head_dim", "terms", "n_pages", "n_seqs", "table_stride", "reserved")] + [
        (k, ctypes.c_void_p) for k in ("k_pool", "v_pool", "page_table")]


class AppendArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("dtype", "q_out_dtype", "n_heads", "n_rows", "rope_len", "rope_pairs")] + [
        ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)] + [(k, ctypes.c_void_p) for k in ("row_start", "kv_len", "q", "k", "v", "q_out")] + [
        (k, ctypes.c_int64) for k in ("q_stride", "q_head_stride", "k_stride", "k_head_stride", "v_stride", "v_head_stride", "q_out_stride", "q_out_head_stride")] + [
        (k, ctypes.c_void_p) for k in ("q_gain", "k_gain", "rope")]


class AttendArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("dtype", "out_dtype", "n_heads", "n_rows", "n_groups", "max_kv", "max_shared")] + [("scale", ctypes.c_float)] + [
        (k, ctypes.c_void_p) for k in ("row_start", "kv_len", "group_start", "group_pages", "q", "out")] + [
        (k, ctypes.c_int64) for k in ("q_stride", "q_head_stride", "out_stride", "out_head_stride")]


class AcceptArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "n_seqs", "n_rows", "vocab", "reserved")] + [
        ("row_start", ctypes.c_void_p), ("logits", ctypes.c_void_p), ("logits_stride", ctypes.c_int64), ("drafts", ctypes.c_void_p), ("draft_probs", ctypes.c_void_p),
        ("probs_stride", ctypes.c_int64)] + [(k, ctypes.c_void_p) for k in ("u", "v", "temperature", "accept_len", "next_token")]


class ScoreArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "n_rows", "vocab", "top")] + [("temperature", ctypes.c_float), ("logits", ctypes.c_void_p),
                ("logits_stride", ctypes.c_int64)] + [(k, ctypes.c_void_p) for k in ("tokens", "logprob", "entropy", "top_ids", "top_logprobs")]


class DistillArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "grad_dtype", "n_rows", "vocab", "top", "rest")] + [("temperature", ctypes.c_float), ("logits", ctypes.c_void_p),
                ("logits_stride", ctypes.c_int64)] + [(k, ctypes.c_void_p) for k in ("ids", "logprobs", "loss", "d_loss", "d_logits")] + [("d_logits_stride", ctypes.c_int64)]


class NormArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "out_dtype", "n_rows", "dim", "center")] + [("eps", ctypes.c_float), ("reserved", ctypes.c_int32)] + [
        (k, ctypes.c_void_p) for k in ("x", "gain", "bias", "y")] + [(k, ctypes.c_int64) for k in ("x_stride", "y_stride")]


class NormGradArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "dy_dtype", "dx_dtype", "n_rows", "dim", "center")] + [("eps", ctypes.c_float)] + [
        (k, ctypes.c_void_p) for k in ("x", "dy", "gain", "dx", "d_gain", "d_bias")] + [(k, ctypes.c_int64) for k in ("x_stride", "dy_stride", "dx_stride")]


class LinearArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "out_dtype", "residual_dtype", "act", "n_rows", "n_in", "n_out")] + [
        (k, ctypes.c_void_p) for k in ("x", "weight", "bias", "residual", "y", "pre")] + [
        (k, ctypes.c_int64) for k in ("x_stride", "weight_stride", "residual_stride", "y_stride", "pre_stride")]


class LinearGradArgsC(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int32) for k in ("device", "dtype", "dx_dtype", "dw_dtype", "act", "n_rows", "n_in", "n_out")] + [
        (k, ctypes.c_void_p) for k in ("x", "weight", "dy", "pre", "dx", "d_weight", "d_bias")] + [
        (k, ctypes.c_int64) for k in ("x_stride", "weight_stride", "dy_stride", "pre_stride", "dx_stride", "dw_stride")]


_lib = None


def lib_path() -> str:
    return _build.LIB_PATH


def load_library():
    """Load libeeverify.so (building it first only if no built library exists)."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        _build.build()
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER
    vp, i32p, ci = ctypes.c_void_p, P(ctypes.c_int32), ctypes.c_int
    lib.ee_last_error.restype = ctypes.c_char_p
    lib.ee_last_error.argtypes = []
    lib.ee_model_load.argtypes = [ctypes.c_char_p, ci, P(vp)]
    lib.ee_model_load_ex.argtypes = [ctypes.c_char_p, ci, ci, P(vp)]
    lib.ee_model_load_form.argtypes = [ctypes.c_char_p, ci, ci, ci, P(vp)]
    lib.ee_model_packed_bytes.argtypes = [vp, P(ctypes.c_size_t)]
    lib.ee_model_free.argtypes = [vp]
    lib.ee_model_info.argtypes = [vp, P(ModelConfigC)]
    lib.ee_session_create.argtypes = [vp, ci, ci, ctypes.c_uint, P(vp)]
    lib.ee_session_free.argtypes = [vp]
    lib.ee_session_fork.argtypes = [vp, ci, vp]
    lib.ee_prefill.argtypes = [vp, i32p, ci, ctypes.c_uint, i32p]
    lib.ee_prefill_embeds.argtypes = [vp, vp, ci, i32p, ci, ctypes.c_uint, i32p]
    lib.ee_verify.argtypes = [vp, i32p, ci, i32p, ci, P(P(VerifyResultC))]
    lib.ee_verify_static.argtypes = [vp, i32p, ci, i32p, ci, P(P(VerifyResultC))]
    lib.ee_verify_sampled.argtypes = [vp, i32p, ci, i32p, ci, P(SamplingC), P(P(VerifyResultC))]
    lib.ee_verify_batch.argtypes = [P(vp), ci, P(i32p), ci, i32p, ci, P(P(VerifyResultC))]
    lib.ee_verify_sampled_batch.argtypes = [P(vp), ci, P(i32p), ci, i32p, ci, P(SamplingC), P(P(VerifyResultC))]
    lib.ee_wait_exit.argtypes = [vp, ci]
    lib.ee_query_exit.argtypes = [vp, ci]
    lib.ee_wait_final.argtypes = [vp]
    lib.ee_query_final.argtypes = [vp]
    lib.ee_pass_time_ms.argtypes = [vp, ci, P(ctypes.c_float)]
    lib.ee_kv_truncate.argtypes = [vp, ci]
    lib.ee_set_pending.argtypes = [vp, ctypes.c_int32]
    lib.ee_kv_len.argtypes = [vp, P(ci)]
    lib.ee_pending.argtypes = [vp, i32p]
    lib.ee_debug_logits.argtypes = [vp, ci, vp]
    lib.ee_debug_mfma_layout.argtypes = [ci]
    lib.ee_tune_k_split.argtypes = [ctypes.c_uint, ci]
    lib.ee_debug_div_small.argtypes = [ci, ctypes.POINTER(ctypes.c_int32), ci, ctypes.POINTER(ctypes.c_longlong)]
    lib.ee_debug_linear_plan.argtypes = [ctypes.c_int32] * 4 + [ctypes.POINTER(ctypes.c_int32)]
    lib.ee_device_synchronize.argtypes = [ci]
    lib.ee_session_option.argtypes = [vp, ci, ci]
    lib.ee_exit_pop.argtypes = [vp, ci, P(ci), P(ctypes.c_float)]
    lib.ee_exit_order.argtypes = [vp, P(ci), P(ctypes.c_float)]
    lib.ee_latency_model.argtypes = [P(LatencyParamsC), P(LatencyC)]
    lib.ee_debug_copy.argtypes = [ci, ctypes.c_size_t, ci]
    lib.ee_launch_times.argtypes = [vp, i32p, P(ctypes.c_float), ci, P(ci)]
    sz = ctypes.c_size_t
    lib.ee_kv_append.argtypes = [vp, vp, vp]              # (structures by address, or packed as bytes)
    lib.ee_attend_workspace.argtypes = [vp, vp, P(sz)]
    lib.ee_attend.argtypes = [vp, vp, vp, sz, vp]
    lib.ee_accept_workspace.argtypes = [vp, P(sz)]
    lib.ee_accept_drafts.argtypes = [vp, vp, sz, vp]
    for name in ("score", "distill", "norm_grad", "linear", "linear_grad"):
        getattr(lib, f"ee_{name}_workspace").argtypes = [vp, P(sz)]
        getattr(lib, "ee_score_tokens" if name == "score" else f"ee_{name}").argtypes = [vp, vp, sz, vp]
    lib.ee_norm.argtypes = [vp, vp]
    for name in EXPORTS:
        if name != "ee_last_error":
            getattr(lib, name).restype = ci
    _lib = lib
    return lib


def _check(rc: int) -> int:
    if rc < 0:
        raise EEError(rc, load_library().ee_last_error().decode(errors="replace"))
    return rc


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32).reshape(-1))


def _p(a: np.ndarray):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)) if a.size else None


def ee_device_synchronize(device: int = 0) -> None:
    _check(load_library().ee_device_synchronize(device))


def ee_verify_sampled_batch(sessions: List[Session], drafts: List[Sequence[int]], draft_probs, u, v, temperatures,
                            exit_layers: Sequence[int] = ()) -> None:
    """ee_verify_batch with each session's draft distributions [gamma][vocab], uniform numbers
    u [gamma], v [gamma+1] and temperature (lists, one entry per session)."""
    lib = load_library()
    n = len(sessions)
    hs = (ctypes.c_void_p * n)(*[s._h for s in sessions])
    ds = [_i32(d) for d in drafts]
    gamma = ds[0].size
    assert all(d.size == gamma for d in ds)
    dp = (ctypes.POINTER(ctypes.c_int32) * n)(*[_p(d) for d in ds])
    fp = ctypes.POINTER(ctypes.c_float)
    keep = []
    sms = (SamplingC * n)()
    for i in range(n):
        pr = np.ascontiguousarray(draft_probs[i], dtype=np.float32)
        uu = np.ascontiguousarray(u[i], dtype=np.float32)
        vv = np.ascontiguousarray(v[i], dtype=np.float32)
        if pr.shape != (gamma, sessions[i].model.vocab) or uu.size != gamma or vv.size != gamma + 1:
            raise ValueError("draft_probs [gamma][vocab], u [gamma], v [gamma+1] expected for every session")
        keep += [pr, uu, vv]
        sms[i] = SamplingC(pr.ctypes.data_as(fp), uu.ctypes.data_as(fp), vv.ctypes.data_as(fp), float(temperatures[i]))
    ex = _i32(exit_layers)
    outs = (ctypes.POINTER(VerifyResultC) * n)()
    _check(lib.ee_verify_sampled_batch(hs, n, dp, gamma, _p(ex), ex.size, sms, outs))
    for i, s in enumerate(sessions):
        s._res, s._n_exits, s._gamma = outs[i], ex.size, gamma


def ee_debug_mfma_layout(device: int = 0) -> None:
    _check(load_library().ee_debug_mfma_layout(device))


def ee_tune_k_split(kind_mask: int, log2_splits: int) -> None:
    _check(load_library().ee_tune_k_split(kind_mask, log2_splits))


def ee_debug_div_small(divisors, device: int = 0) -> int:
    d = np.ascontiguousarray(divisors, dtype=np.int32)
    bad = ctypes.c_longlong(-1)
    _check(load_library().ee_debug_div_small(device, d.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), int(d.size), ctypes.byref(bad)))
    return int(bad.value)


def ee_debug_linear_plan(n_rows: int, n_in: int, n_out: int, product: int = 0) -> tuple:
    """(rows and columns of a tile, parts of the sum, length of a part) of a product of ee_linear (0), or of ee_linear_grad (1: dx, 2: d_weight)."""
    plan = (ctypes.c_int32 * 4)()
    _check(load_library().ee_debug_linear_plan(n_rows, n_in, n_out, product, plan))
    return tuple(plan)


@dataclass
class VerifyOutput:
    gamma: int
    accept_len: int
    next_token: int
    final_tokens: np.ndarray
    exit_accept_len: np.ndarray
    exit_tokens: np.ndarray
    final_conf: np.ndarray = None   # [gamma+1] float32
    exit_conf: np.ndarray = None    # [n_exits][gamma+1] float32


class Model:
    """ee_model_load / ee_model_free / ee_model_info."""

    def __init__(self, path: str, device: int = 0, max_rows: int = 16, form: int = FORM_AUTO):
        self._l = load_library()
        h = ctypes.c_void_p()
        _check(self._l.ee_model_load_form(path.encode(), device, max_rows, form, ctypes.byref(h)))
        self._h = h
        c = ModelConfigC()
        _check(self._l.ee_model_info(h, ctypes.byref(c)))
        self.config = c
        self.n_layers, self.d_model, self.n_heads, self.head_dim = c.n_layers, c.d_model, c.n_heads, c.head_dim
        self.d_ffn, self.vocab, self.max_rows, self.n_workgroups = c.d_ffn, c.vocab, c.max_rows, c.n_workgroups
        self.exit_layers = [c.exit_layers[i] for i in range(c.n_exits)]

    def free(self):
        if self._h:
            self._l.ee_model_free(self._h)
            self._h = None

    def packed_bytes(self) -> int:
        n = ctypes.c_size_t()
        _check(self._l.ee_model_packed_bytes(self._h, ctypes.byref(n)))
        return int(n.value)

    def session(self, max_ctx: int, max_gamma: int = 8, flags: int = 0) -> "Session":
        return Session(self, max_ctx, max_gamma, flags)


class Session:
    """ee_session_create and the per-session calls, same names as the C ABI."""

    def __init__(self, model: Model, max_ctx: int, max_gamma: int = 8, flags: int = 0):
        self.model = model
        self._l = model._l
        h = ctypes.c_void_p()
        _check(self._l.ee_session_create(model._h, max_ctx, max_gamma, flags, ctypes.byref(h)))
        self._h = h
        self._res = None
        self._n_exits = 0
        self._gamma = 0

    def free(self):
        if self._h:
            self._l.ee_session_free(self._h)
            self._h = None

    def ee_session_fork(self, n: int, to: "Session") -> None:
        """`to` gets this session's first n cached positions."""
        _check(self._l.ee_session_fork(self._h, n, to._h))

    def ee_prefill(self, tokens: Sequence[int], flags: int = 0, emb: Optional[np.ndarray] = None) -> Optional[int]:
        t = _i32(tokens)
        first = ctypes.c_int32(-1)
        if emb is None:
            _check(self._l.ee_prefill(self._h, _p(t), t.size, flags, ctypes.byref(first)))
        else:
            e = np.ascontiguousarray(emb, dtype=np.uint16)
            _check(self._l.ee_prefill_embeds(self._h, e.ctypes.data, e.shape[0], _p(t), t.size, flags,
                                             ctypes.byref(first)))
        return None if flags & HOLD_LAST else int(first.value)

    def ee_verify(self, draft_tokens: Sequence[int], exit_layers: Sequence[int] = ()) -> None:
        """Asynchronous; results via ee_wait_exit / ee_wait_final + exit_result / final_result."""
        d, ex = _i32(draft_tokens), _i32(exit_layers)
        res = ctypes.POINTER(VerifyResultC)()
        _check(self._l.ee_verify(self._h, _p(d), d.size, _p(ex), ex.size, ctypes.byref(res)))
        self._res, self._n_exits, self._gamma = res, ex.size, d.size

    def ee_verify_static(self, draft_tokens: Sequence[int], exit_layers: Sequence[int] = ()) -> None:
        """ee_verify on the library's static scratch array (allocates nothing)."""
        d, ex = _i32(draft_tokens), _i32(exit_layers)
        res = ctypes.POINTER(VerifyResultC)()
        _check(self._l.ee_verify_static(self._h, _p(d), d.size, _p(ex), ex.size, ctypes.byref(res)))
        self._res, self._n_exits, self._gamma = res, ex.size, d.size

    def ee_verify_sampled(self, draft_tokens: Sequence[int], draft_probs, u, v, temperature: float = 1.0,
                          exit_layers: Sequence[int] = ()) -> None:
        """ee_verify with the draft model's distributions [gamma][vocab] and the caller's uniform numbers."""
        d, ex = _i32(draft_tokens), _i32(exit_layers)
        pr = np.ascontiguousarray(draft_probs, dtype=np.float32)
        uu = np.ascontiguousarray(u, dtype=np.float32)
        vv = np.ascontiguousarray(v, dtype=np.float32)
        if pr.ndim != 2 or pr.shape[0] != d.size or pr.shape[1] != self.model.vocab or uu.size != d.size or vv.size != d.size + 1:
            raise ValueError("draft_probs [gamma][vocab], u [gamma], v [gamma+1] expected")
        fp = ctypes.POINTER(ctypes.c_float)
        sm = SamplingC(pr.ctypes.data_as(fp), uu.ctypes.data_as(fp), vv.ctypes.data_as(fp), float(temperature))
        res = ctypes.POINTER(VerifyResultC)()
        _check(self._l.ee_verify_sampled(self._h, _p(d), d.size, _p(ex), ex.size, ctypes.byref(sm), ctypes.byref(res)))
        self._res, self._n_exits, self._gamma = res, ex.size, d.size

    def ee_wait_exit(self, exit_idx: int) -> None:
        _check(self._l.ee_wait_exit(self._h, exit_idx))

    def ee_query_exit(self, exit_idx: int) -> bool:
        return _check(self._l.ee_query_exit(self._h, exit_idx)) == EE_OK

    def ee_wait_final(self) -> None:
        _check(self._l.ee_wait_final(self._h))

    def ee_query_final(self) -> bool:
        return _check(self._l.ee_query_final(self._h)) == EE_OK

    def ee_pass_time_ms(self, exit_idx: int) -> float:
        ms = ctypes.c_float()
        _check(self._l.ee_pass_time_ms(self._h, exit_idx, ctypes.byref(ms)))
        return float(ms.value)

    def ee_kv_truncate(self, new_len: int) -> None:
        _check(self._l.ee_kv_truncate(self._h, new_len))

    def ee_set_pending(self, token: int) -> None:
        _check(self._l.ee_set_pending(self._h, token))

    def ee_kv_len(self) -> int:
        v = ctypes.c_int()
        _check(self._l.ee_kv_len(self._h, ctypes.byref(v)))
        return int(v.value)

    def ee_pending(self) -> int:
        v = ctypes.c_int32()
        _check(self._l.ee_pending(self._h, ctypes.byref(v)))
        return int(v.value)

    def ee_debug_logits(self, head_idx: int) -> np.ndarray:
        out = np.empty((self._gamma + 1, self.model.vocab), dtype=np.float32)
        _check(self._l.ee_debug_logits(self._h, head_idx, out.ctypes.data))
        return out

    def ee_exit_pop(self, wait: bool = True):
        """(status, exit index, score): status EE_OK, EE_NOT_READY or EE_DONE."""
        idx, sc = ctypes.c_int(-1), ctypes.c_float(0.0)
        rc = _check(self._l.ee_exit_pop(self._h, 1 if wait else 0, ctypes.byref(idx), ctypes.byref(sc)))
        return rc, int(idx.value), float(sc.value)

    def ee_exit_order(self):
        """([exit index], [score]) in the order the sender's queue releases them."""
        n = self._n_exits
        order, sc = (ctypes.c_int * max(n, 1))(), (ctypes.c_float * max(n, 1))()
        _check(self._l.ee_exit_order(self._h, order, sc))
        return [int(order[i]) for i in range(n)], [float(sc[i]) for i in range(n)]

    def ee_session_option(self, option: int, value: int) -> None:
        _check(self._l.ee_session_option(self._h, option, value))

    def ee_launch_times(self):
        """[(launch code, milliseconds)] of every launch of the last verify pass."""
        cap = 4096
        codes, ms, n = (ctypes.c_int32 * cap)(), (ctypes.c_float * cap)(), ctypes.c_int()
        _check(self._l.ee_launch_times(self._h, codes, ms, cap, ctypes.byref(n)))
        return [(int(codes[i]), float(ms[i])) for i in range(n.value)]

    # plain reads of the pinned result block (no computation)
    def exit_result(self, exit_idx: int):
        r, M = self._res.contents, self._gamma + 1
        return np.array(r.exit_tokens[exit_idx][:M], dtype=np.int32), int(r.exit_accept_len[exit_idx])

    def exit_conf(self, exit_idx: int) -> np.ndarray:
        r, M = self._res.contents, self._gamma + 1
        return np.array(r.exit_conf[exit_idx][:M], dtype=np.float32)

    def final_result(self) -> VerifyOutput:
        r, M, E = self._res.contents, self._gamma + 1, self._n_exits
        return VerifyOutput(
            gamma=self._gamma, accept_len=int(r.accept_len), next_token=int(r.next_token),
            final_tokens=np.array(r.final_tokens[:M], dtype=np.int32),
            exit_accept_len=np.array(r.exit_accept_len[:E], dtype=np.int32),
            exit_tokens=np.array([list(r.exit_tokens[e][:M]) for e in range(E)], dtype=np.int32).reshape(E, M),
            final_conf=np.array(r.final_conf[:M], dtype=np.float32),
            exit_conf=np.array([list(r.exit_conf[e][:M]) for e in range(E)], dtype=np.float32).reshape(E, M))

    def verify_sync(self, draft_tokens: Sequence[int], exit_layers: Sequence[int] = ()) -> VerifyOutput:
        self.ee_verify(draft_tokens, exit_layers)
        self.ee_wait_final()
        return self.final_result()


def ee_latency_model(T_p: float, T_q: float, T_c: float, tau: float, gamma: int = 4, n: int = 200, r: float = 1.0,
                     T_r: float = 0.0) -> dict:
    """The paper's AR / SD / FSD latency formulas and Eq. 9 (times in ms); plain marshalling."""
    p = LatencyParamsC(T_p, T_q, T_c, T_r, tau, r, gamma, n)
    out = LatencyC()
    _check(load_library().ee_latency_model(ctypes.byref(p), ctypes.byref(out)))
    return {k: getattr(out, k) for k, _ in LatencyC._fields_}


def ee_debug_copy(device: int, nbytes: int, reps: int) -> None:
    _check(load_library().ee_debug_copy(device, nbytes, reps))


def ee_verify_batch(sessions: List[Session], drafts: List[Sequence[int]], exit_layers: Sequence[int] = ()) -> None:
    """One pass for several sessions; wait on any of them, read each one's result."""
    lib = load_library()
    n = len(sessions)
    hs = (ctypes.c_void_p * n)(*[s._h for s in sessions])
    ds = [_i32(d) for d in drafts]
    gamma = ds[0].size
    assert all(d.size == gamma for d in ds)
    dp = (ctypes.POINTER(ctypes.c_int32) * n)(*[_p(d) for d in ds])
    ex = _i32(exit_layers)
    outs = (ctypes.POINTER(VerifyResultC) * n)()
    _check(lib.ee_verify_batch(hs, n, dp, gamma, _p(ex), ex.size, outs))
    for i, s in enumerate(sessions):
        s._res, s._n_exits, s._gamma = outs[i], ex.size, gamma


# ---------------------------------------------------------------- operators on device memory
#
# Arrays are objects in device memory with `data_ptr()`, `shape`, `stride()` (in elements), `dtype` and `device`, as a torch tensor has
# them (this module does not import torch; a program that uses both imports torch first, so that one HIP runtime is loaded).  `stream` is a
# hipStream_t as an integer (torch.cuda.current_stream().cuda_stream), 0 the device's default stream.
#
# A call of a few microseconds is bound by what happens here, so the checks read each attribute once and the arguments are packed
# in one go (a ctypes structure of 25 fields takes 4 us to fill, struct.pack 1).

_APPEND_PACK = struct.Struct("@6ifi6P8q3P").pack
_ATTEND_PACK = struct.Struct("@7if6P4q").pack
_ACCEPT_PACK = struct.Struct("@6i2Pq2Pq5P").pack

_TYPE_OF = {}
_FLOATS = {"bfloat16": BF16, "float16": FP16, "float32": FP32}


def _type(t) -> str:
    """Name of an array's element type: "float32", "bfloat16", "int32", ..."""
    name = _TYPE_OF.get(t.dtype)
    if name is None:
        name = _TYPE_OF[t.dtype] = str(t.dtype).rpartition(".")[2]
    return name


def _on(t, what: str) -> int:
    """Index of the GPU that holds the array."""
    d = t.device
    if d.type != "cuda":
        raise ValueError(f"{what} is not in device memory")
    return d.index or 0


def _vector(t, what: str, kind: str, device, n: int) -> int:
    """Address of a contiguous one-dimensional array of at least n elements (None: 0)."""
    if t is None:
        return 0
    shape = t.shape
    if len(shape) != 1 or shape[0] < n or _type(t) != kind or t.device != device or (shape[0] > 1 and t.stride()[0] != 1):
        raise ValueError(f"{what}: contiguous {kind} array of at least {n} elements on {device} expected")
    return t.data_ptr()


def _contiguous(t) -> bool:
    """Whether an array's elements follow each other (the stride of a dimension of one says nothing)."""
    at = 1
    for size, stride in zip(reversed(t.shape), reversed(t.stride())):
        if size > 1 and stride != at:
            return False
        at *= size
    return True


def _heads(t, what: str, rows, heads, dim: int, device):
    """(address, type, row stride, head stride, rows, heads) of [rows][heads][dim] with contiguous heads."""
    shape, s = t.shape, t.stride()
    kind = _FLOATS.get(_type(t))
    if len(shape) != 3 or shape[2] != dim or (rows is not None and shape[0] != rows) or (heads is not None and shape[1] != heads) or s[2] != 1:
        raise ValueError(f"{what}: [{rows if rows is not None else 'rows'}][{heads if heads is not None else 'heads'}][{dim}] with contiguous heads expected")
    if kind is None or t.device != device:
        raise ValueError(f"{what}: bf16, fp16 or fp32 on {device} expected")
    return t.data_ptr(), kind, s[0], s[1], shape[0], shape[1]


class PagedCache:
    """ee_paged_cache over a caller's arrays, which it keeps: k_pool bf16 [n_pages][n_kv_heads][16][terms][head_dim], v_pool bf16
    [n_pages][n_kv_heads][terms][head_dim][16], page_table int32 [n_seqs][pages of a sequence]."""

    def __init__(self, k_pool, v_pool, page_table):
        if len(k_pool.shape) != 5 or k_pool.shape[2] != 16 or len(v_pool.shape) != 5:
            raise ValueError("k_pool [n_pages][n_kv_heads][16][terms][head_dim] and v_pool [n_pages][n_kv_heads][terms][head_dim][16] expected")
        n, heads, _, terms, dim = k_pool.shape
        if tuple(v_pool.shape) != (n, heads, terms, dim, 16):
            raise ValueError("v_pool: the same pages, heads and terms as k_pool expected")
        device = _on(k_pool, "k_pool")
        self.device = k_pool.device
        for t, what in ((k_pool, "k_pool"), (v_pool, "v_pool")):
            if _type(t) != "bfloat16" or not _contiguous(t) or t.device != self.device:
                raise ValueError(f"{what}: contiguous bf16 on {self.device} expected")
        if len(page_table.shape) != 2 or _type(page_table) != "int32" or page_table.device != self.device:
            raise ValueError("page_table: int32 [n_seqs][entries] expected")
        self.n_kv_heads, self.head_dim, self.n_seqs = heads, dim, page_table.shape[0]
        if not _contiguous(page_table):
            raise ValueError("page_table: contiguous expected")
        self.k_pool, self.v_pool, self.page_table = k_pool, v_pool, page_table
        self.c = PagedCacheC(device, heads, dim, terms, n, self.n_seqs, page_table.shape[1], 0, k_pool.data_ptr(), v_pool.data_ptr(), page_table.data_ptr())
        self._at = ctypes.addressof(self.c)


def ee_kv_append(cache: PagedCache, row_start, kv_len, q, k, v, q_out, q_gain=None, k_gain=None, eps: float = 1e-5, rope=None, rope_pairs: bool = False,
                 stream: int = 0) -> None:
    """q, q_out [rows][heads][head_dim] (q may be None: keys and values only), k, v [rows][n_kv_heads][head_dim], gains fp32 [head_dim],
    rope fp32 [positions][head_dim / 2][2]."""
    dev, dim, n, kv_heads = cache.device, cache.head_dim, cache.n_seqs, cache.n_kv_heads
    kp, kind, ks, kh, rows, _ = _heads(k, "k", None, kv_heads, dim, dev)
    vp, kind_v, vs, vh, _, _ = _heads(v, "v", rows, kv_heads, dim, dev)
    qp = qs = qh = op = os_ = oh = heads = 0
    kind_q = kind_o = kind
    if q is not None:
        qp, kind_q, qs, qh, _, heads = _heads(q, "q", rows, None, dim, dev)
        op, kind_o, os_, oh, _, _ = _heads(q_out, "q_out", rows, heads, dim, dev)
    if kind_v != kind or kind_q != kind:
        raise ValueError("q, k and v must be of one type")
    rp = positions = 0
    if rope is not None:
        shape = rope.shape
        if len(shape) != 3 or shape[1] != dim // 2 or shape[2] != 2 or _type(rope) != "float32" or rope.device != dev or not _contiguous(rope):
            raise ValueError(f"rope: contiguous fp32 [positions][{dim // 2}][2] on {dev} expected")
        rp, positions = rope.data_ptr(), shape[0]
    a = _APPEND_PACK(kind, kind_o, heads, rows, positions, 1 if rope_pairs else 0, eps, 0, _vector(row_start, "row_start", "int32", dev, n + 1),
                     _vector(kv_len, "kv_len", "int32", dev, n), qp, kp, vp, op, qs, qh, ks, kh, vs, vh, os_, oh, _vector(q_gain, "q_gain", "float32", dev, dim),
                     _vector(k_gain, "k_gain", "float32", dev, dim), rp)
    _check((_lib or load_library()).ee_kv_append(cache._at, a, stream))


def _attend_args(cache: PagedCache, row_start, kv_len, q, out, scale, max_kv, group_start, group_pages, max_shared) -> bytes:
    dev, dim, n = cache.device, cache.head_dim, cache.n_seqs
    qp, kind, qs, qh, rows, heads = _heads(q, "q", None, None, dim, dev)
    op, kind_o, os_, oh = (0, kind, qs, qh) if out is None else _heads(out, "out", rows, heads, dim, dev)[:4]
    groups = 0
    if group_start is not None:
        groups = group_start.shape[0] - 1
        if group_pages is None or groups < 0:
            raise ValueError("group_start [groups + 1] comes with group_pages [groups]")
    return _ATTEND_PACK(kind, kind_o, heads, rows, groups, max_kv, max_shared, scale, _vector(row_start, "row_start", "int32", dev, n + 1),
                        _vector(kv_len, "kv_len", "int32", dev, n), _vector(group_start, "group_start", "int32", dev, 0),
                        _vector(group_pages, "group_pages", "int32", dev, groups), qp, op, qs, qh, os_, oh)


def ee_attend_workspace(cache: PagedCache, row_start, q, max_kv: int = 0, group_start=None, group_pages=None, max_shared: int = 0) -> int:
    """Bytes of workspace for calls of ee_attend with these sizes."""
    a = _attend_args(cache, row_start, None, q, None, 1.0, max_kv, group_start, group_pages, max_shared)
    n = ctypes.c_size_t()
    _check(load_library().ee_attend_workspace(cache._at, a, ctypes.byref(n)))
    return int(n.value)


def ee_attend(cache: PagedCache, row_start, kv_len, q, out, scale: float, max_kv: int = 0, group_start=None, group_pages=None, max_shared: int = 0,
              workspace=None, stream: int = 0) -> None:
    """q, out [rows][heads][head_dim]; group_start int32 [groups + 1] and group_pages int32 [groups] where sequences have pages in common."""
    a = _attend_args(cache, row_start, kv_len, q, out, scale, max_kv, group_start, group_pages, max_shared)
    _check((_lib or load_library()).ee_attend(cache._at, a, _vector(workspace, "workspace", "uint8", cache.device, 0), 0 if workspace is None else workspace.shape[0], stream))


def _accept_args(logits, row_start, drafts=None, draft_probs=None, u=None, v=None, temperature=None, accept_len=None, next_token=None) -> bytes:
    dev, shape, s = logits.device, logits.shape, logits.stride()
    kind = _FLOATS.get(_type(logits))
    if len(shape) != 2 or kind is None or s[1] != 1:
        raise ValueError("logits: [rows][vocab] of bf16, fp16 or fp32 with contiguous rows expected")
    rows, V = shape
    n = row_start.shape[0] - 1
    pp = ps = 0
    if draft_probs is not None:
        t = draft_probs.stride()
        if tuple(draft_probs.shape) != (rows, V) or _type(draft_probs) != "float32" or draft_probs.device != dev or t[1] != 1:
            raise ValueError(f"draft_probs: fp32 [{rows}][{V}] with contiguous rows on {dev} expected")
        pp, ps = draft_probs.data_ptr(), t[0] if rows > 1 else V
    # (a single row's stride says nothing)
    return _ACCEPT_PACK(_on(logits, "logits"), kind, n, rows, V, 0, _vector(row_start, "row_start", "int32", dev, 1), logits.data_ptr(), s[0] if rows > 1 else V,
                        _vector(drafts, "drafts", "int32", dev, rows), pp, ps, _vector(u, "u", "float32", dev, rows), _vector(v, "v", "float32", dev, rows),
                        _vector(temperature, "temperature", "float32", dev, n), _vector(accept_len, "accept_len", "int32", dev, n),
                        _vector(next_token, "next_token", "int32", dev, n))


def ee_accept_workspace(logits, row_start) -> int:
    """Bytes of workspace for calls of ee_accept_drafts with these sizes."""
    n = ctypes.c_size_t()
    _check(load_library().ee_accept_workspace(_accept_args(logits, row_start), ctypes.byref(n)))
    return int(n.value)


def ee_accept_drafts(logits, row_start, drafts, draft_probs, u, v, temperature, accept_len, next_token, workspace, stream: int = 0) -> None:
    """logits [rows][vocab], drafts int32 [rows], draft_probs fp32 [rows][vocab] or None, u and v fp32 [rows], temperature fp32 [sequences];
    results accept_len, next_token int32 [sequences]."""
    a = _accept_args(logits, row_start, drafts, draft_probs, u, v, temperature, accept_len, next_token)
    _check((_lib or load_library()).ee_accept_drafts(a, _vector(workspace, "workspace", "uint8", logits.device, 0), 0 if workspace is None else workspace.shape[0], stream))


# ---------------------------------------------------------------- operators around the LM head

_SCORE_PACK = struct.Struct("@5ifPq5P").pack
_DISTILL_PACK = struct.Struct("@7ifPq5Pq").pack
_NORM_PACK = struct.Struct("@6ifi4P2q").pack
_NORM_GRAD_PACK = struct.Struct("@7if6P3q").pack
_LINEAR_PACK = struct.Struct("@8i6P5q").pack
_LINEAR_GRAD_PACK = struct.Struct("@8i7P6q").pack


def _rows(t, what: str, rows, width, device):
    """(address, type, row stride, rows, width) of [rows][width] with contiguous rows; None: nothing."""
    if t is None:
        return 0, FP32, 0, rows, width
    shape, s = t.shape, t.stride()
    kind = _FLOATS.get(_type(t))
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (width is not None and shape[1] != width) or (shape[1] > 1 and s[1] != 1):
        raise ValueError(f"{what}: [{rows if rows is not None else 'rows'}][{width if width is not None else 'width'}] with contiguous rows expected")
    if kind is None or t.device != device:
        raise ValueError(f"{what}: bf16, fp16 or fp32 on {device} expected")
    return t.data_ptr(), kind, s[0], shape[0], shape[1]


def _lists(t, what: str, kind: str, device, rows: int, top: int) -> int:
    """Address of a contiguous array [rows][top] (None: 0)."""
    if t is None:
        return 0
    shape = t.shape
    if len(shape) != 2 or shape[0] != rows or shape[1] != top or _type(t) != kind or t.device != device or (tuple(t.stride()) != (top, 1) and not _contiguous(t)):
        raise ValueError(f"{what}: contiguous {kind} [{rows}][{top}] on {device} expected")
    return t.data_ptr()


def _space(workspace, device):
    return (0, 0) if workspace is None else (_vector(workspace, "workspace", "uint8", device, 0), workspace.shape[0])


def _bytes_of(call, args) -> int:
    n = ctypes.c_size_t()
    _check(call(args, ctypes.byref(n)))
    return int(n.value)


def _score_args(logits, tokens, logprob, entropy, top_ids, top_logprobs, top, temperature) -> bytes:
    dev = logits.device
    zp, kind, zs, rows, V = _rows(logits, "logits", None, None, dev)
    return _SCORE_PACK(_on(logits, "logits"), kind, rows, V, top, temperature, zp, zs, _vector(tokens, "tokens", "int32", dev, rows), _vector(logprob, "logprob", "float32", dev, rows),
                       _vector(entropy, "entropy", "float32", dev, rows), _lists(top_ids, "top_ids", "int32", dev, rows, top),
                       _lists(top_logprobs, "top_logprobs", "float32", dev, rows, top))


def ee_score_workspace(logits, top: int = 0) -> int:
    """Bytes of workspace for calls of ee_score_tokens with these sizes."""
    return _bytes_of(load_library().ee_score_workspace, _score_args(logits, None, None, None, None, None, top, 1.0))


def ee_score_tokens(logits, tokens=None, logprob=None, entropy=None, top_ids=None, top_logprobs=None, temperature: float = 1.0, workspace=None, stream: int = 0) -> None:
    """logits [rows][vocab], tokens int32 [rows]; results logprob, entropy fp32 [rows], top_ids int32 and top_logprobs fp32 [rows][top], each None where it is
    not wanted."""
    top = 0 if top_ids is None else top_ids.shape[-1]
    a = _score_args(logits, tokens, logprob, entropy, top_ids, top_logprobs, top, temperature)
    _check((_lib or load_library()).ee_score_tokens(a, *_space(workspace, logits.device), stream))


def _distill_args(logits, ids, logprobs, loss, d_loss, d_logits, top, rest, temperature) -> bytes:
    dev = logits.device
    zp, kind, zs, rows, V = _rows(logits, "logits", None, None, dev)
    gp, kind_g, gs, _, _ = _rows(d_logits, "d_logits", rows, V, dev)
    return _DISTILL_PACK(_on(logits, "logits"), kind, kind_g, rows, V, top, 1 if rest else 0, temperature, zp, zs, _lists(ids, "ids", "int32", dev, rows, top),
                         _lists(logprobs, "logprobs", "float32", dev, rows, top), _vector(loss, "loss", "float32", dev, rows),
                         _vector(d_loss, "d_loss", "float32", dev, rows), gp, gs)


def ee_distill_workspace(logits, top: int) -> int:
    """Bytes of workspace for calls of ee_distill with these sizes."""
    return _bytes_of(load_library().ee_distill_workspace, _distill_args(logits, None, None, None, None, None, top, True, 1.0))


def ee_distill(logits, ids, logprobs, loss=None, d_loss=None, d_logits=None, rest: bool = True, temperature: float = 1.0, workspace=None, stream: int = 0) -> None:
    """logits [rows][vocab], ids int32 and logprobs fp32 [rows][top]; results loss fp32 [rows] and d_logits [rows][vocab] (times d_loss fp32 [rows]), each None
    where it is not wanted."""
    a = _distill_args(logits, ids, logprobs, loss, d_loss, d_logits, ids.shape[-1], rest, temperature)
    _check((_lib or load_library()).ee_distill(a, *_space(workspace, logits.device), stream))


def ee_norm(x, y, gain=None, bias=None, eps: float = 1e-5, center: bool = False, stream: int = 0) -> None:
    """x, y [rows][dim]; gain, bias fp32 [dim]; center: layer norm instead of RMS norm."""
    dev = x.device
    xp, kind, xs, rows, dim = _rows(x, "x", None, None, dev)
    yp, kind_y, ys, _, _ = _rows(y, "y", rows, dim, dev)
    a = _NORM_PACK(_on(x, "x"), kind, kind_y, rows, dim, 1 if center else 0, eps, 0, xp, _vector(gain, "gain", "float32", dev, dim), _vector(bias, "bias", "float32", dev, dim), yp, xs, ys)
    _check((_lib or load_library()).ee_norm(a, stream))


def _norm_grad_args(x, dy, dx, gain, d_gain, d_bias, eps, center) -> bytes:
    dev = x.device
    xp, kind, xs, rows, dim = _rows(x, "x", None, None, dev)
    up, kind_u, us, _, _ = _rows(dy, "dy", rows, dim, dev)
    gp, kind_g, gs, _, _ = _rows(dx, "dx", rows, dim, dev)
    return _NORM_GRAD_PACK(_on(x, "x"), kind, kind_u, kind_g, rows, dim, 1 if center else 0, eps, xp, up, _vector(gain, "gain", "float32", dev, dim), gp,
                           _vector(d_gain, "d_gain", "float32", dev, dim), _vector(d_bias, "d_bias", "float32", dev, dim), xs, us, gs)


def ee_norm_grad_workspace(x) -> int:
    """Bytes of workspace for calls of ee_norm_grad with these sizes."""
    return _bytes_of(load_library().ee_norm_grad_workspace, _norm_grad_args(x, None, None, None, None, None, 0.0, False))


def ee_norm_grad(x, dy, dx=None, gain=None, d_gain=None, d_bias=None, eps: float = 1e-5, center: bool = False, workspace=None, stream: int = 0) -> None:
    """x, dy [rows][dim] and ee_norm's gain, eps and center; results dx [rows][dim], d_gain and d_bias fp32 [dim], each None where it is not wanted."""
    a = _norm_grad_args(x, dy, dx, gain, d_gain, d_bias, eps, center)
    _check((_lib or load_library()).ee_norm_grad(a, *_space(workspace, x.device), stream))


def _linear_args(x, weight, y, bias, act, residual, pre) -> bytes:
    dev = x.device
    xp, kind, xs, rows, n_in = _rows(x, "x", None, None, dev)
    wp, kind_w, ws, n_out, _ = _rows(weight, "weight", None, n_in, dev)
    yp, kind_y, ys, _, _ = _rows(y, "y", rows, n_out, dev)
    rp, kind_r, rs, _, _ = _rows(residual, "residual", rows, n_out, dev)
    pp, kind_p, ps, _, _ = _rows(pre, "pre", rows, n_out, dev)
    if kind_w != kind or (pre is not None and kind_p != kind):
        raise ValueError("x, weight and pre must be of one type")
    return _LINEAR_PACK(_on(x, "x"), kind, kind_y, kind_r, act, rows, n_in, n_out, xp, wp, _vector(bias, "bias", "float32", dev, n_out), rp, yp, pp, xs, ws, rs, ys, ps)


def ee_linear_workspace(x, weight) -> int:
    """Bytes of workspace for calls of ee_linear with these sizes."""
    return _bytes_of(load_library().ee_linear_workspace, _linear_args(x, weight, None, None, ACT_NONE, None, None))


def ee_linear(x, weight, y, bias=None, act: int = ACT_NONE, residual=None, pre=None, workspace=None, stream: int = 0) -> None:
    """x [rows][n_in], weight [n_out][n_in], bias fp32 [n_out], residual, y and pre [rows][n_out]."""
    a = _linear_args(x, weight, y, bias, act, residual, pre)
    _check((_lib or load_library()).ee_linear(a, *_space(workspace, x.device), stream))


def _linear_grad_args(x, weight, dy, pre, act, dx, d_weight, d_bias) -> bytes:
    dev = x.device
    xp, kind, xs, rows, n_in = _rows(x, "x", None, None, dev)
    wp, kind_w, ws, n_out, _ = _rows(weight, "weight", None, n_in, dev)
    up, kind_u, us, _, _ = _rows(dy, "dy", rows, n_out, dev)
    pp, kind_p, ps, _, _ = _rows(pre, "pre", rows, n_out, dev)
    gp, kind_g, gs, _, _ = _rows(dx, "dx", rows, n_in, dev)
    hp, kind_h, hs, _, _ = _rows(d_weight, "d_weight", n_out, n_in, dev)
    if kind_w != kind or (dy is not None and kind_u != kind) or (pre is not None and kind_p != kind):
        raise ValueError("x, weight, dy and pre must be of one type")
    return _LINEAR_GRAD_PACK(_on(x, "x"), kind, kind_g, kind_h, act, rows, n_in, n_out, xp, wp, up, pp, gp, hp, _vector(d_bias, "d_bias", "float32", dev, n_out), xs, ws, us, ps, gs, hs)


def ee_linear_grad_workspace(x, weight, act: int = ACT_NONE) -> int:
    """Bytes of workspace for calls of ee_linear_grad with these sizes, whatever the results' types."""
    return _bytes_of(load_library().ee_linear_grad_workspace, _linear_grad_args(x, weight, None, None, act, None, None, None))


def ee_linear_grad(x, weight, dy, pre=None, act: int = ACT_NONE, dx=None, d_weight=None, d_bias=None, workspace=None, stream: int = 0) -> None:
    """dy and pre [rows][n_out]; results dx [rows][n_in], d_weight [n_out][n_in], d_bias fp32 [n_out], each None where it is not wanted."""
    a = _linear_grad_args(x, weight, dy, pre, act, dx, d_weight, d_bias)
    _check((_lib or load_library()).ee_linear_grad(a, *_space(workspace, x.device), stream))
