"""ctypes binding of libcocodc.so with the same names as the C ABI (include/cocodc.h).

Argument marshalling only.  Tensors are torch CUDA tensors used as plain device
memory: the binding passes their addresses and the current CUDA stream.
"""

from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np
import torch

from . import build as _build

OK, ERR_INVALID_ARG, ERR_ALIGNMENT, ERR_ALIAS, ERR_NONFINITE, ERR_TIMEOUT, ERR_CUDA, ERR_NOMEM = range(8)
COMP_NONE, COMP_TAYLOR = 0, 1
SIGN_FORWARD, SIGN_PRINTED, SIGN_DESCENT = 0, 1, 2
BUDGET_COUNT, BUDGET_PARAMS, BUDGET_PARAMS_EXACT = 0, 1, 2
STAGE_OUTER, STAGE_MERGE, STAGE_SCORE, STAGE_ALL, STAGE_SUMSQ, STAGE_DEFER = 1, 2, 4, 7, 8, 16

EXPORTS = (
    "cocodc_create", "cocodc_destroy", "cocodc_sync_budget", "cocodc_fragment_scores",
    "cocodc_select_fragments", "cocodc_outer_step", "cocodc_outer_step_host", "cocodc_merge", "cocodc_snapshot", "cocodc_snapshot_host",
    "cocodc_poll_status", "cocodc_launch_count", "cocodc_status_string",
    "cocodc_fragment_scores_noalloc", "cocodc_selftest_bounded_wait",
    "cocodc_pseudo_gradient_sum", "cocodc_outer_step_received",
    "cocodc_select_fragments_at", "cocodc_outer_step_at", "cocodc_outer_step_received_peers",
    "cocodc_scores_from_sumsq", "cocodc_bind_in_flight", "cocodc_flush_scores", "cocodc_initiate", "cocodc_initiate_at",
    "cocodc_lm_create", "cocodc_lm_destroy", "cocodc_lm_poll_status", "cocodc_lm_launch_count",
    "cocodc_lm_embed", "cocodc_lm_embed_grad", "cocodc_lm_embed_grad_workspace",
    "cocodc_lm_glu", "cocodc_lm_glu_grad", "cocodc_lm_glu_grad_workspace",
    "cocodc_lm_logprobs", "cocodc_lm_logprobs_grad", "cocodc_lm_submit",
    "cocodc_lm_norm", "cocodc_lm_norm_grad", "cocodc_lm_norm_grad_workspace",
    "cocodc_lm_head", "cocodc_lm_head_workspace", "cocodc_lm_head_grad", "cocodc_lm_head_grad_workspace",
    "cocodc_lm_adam_create", "cocodc_lm_adam_destroy", "cocodc_lm_adamw",
)
NOALLOC_MAX_K, NOALLOC_MAX_SEGMENTS = 64, 64


class CocodcError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = int(code)
        super().__init__(f"{where}: {status_string(code)} (status {int(code)})")


class _Partition(ctypes.Structure):
    _fields_ = [("N", ctypes.c_int64), ("K", ctypes.c_int32), ("n_segments", ctypes.c_int32),
                ("frag_seg_ptr", ctypes.POINTER(ctypes.c_int32)),
                ("seg_offset", ctypes.POINTER(ctypes.c_int64)),
                ("seg_len", ctypes.POINTER(ctypes.c_int64))]


class _Hyper(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int32), ("comp_mode", ctypes.c_int32), ("sign_mode", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("H", ctypes.c_int64), ("tau", ctypes.c_int64),
                ("outer_lr", ctypes.c_float), ("momentum", ctypes.c_float),
                ("lam", ctypes.c_float), ("alpha", ctypes.c_float)]


class _Tensor(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("p", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("n", ctypes.c_int64), ("grad_type", ctypes.c_int32), ("copy_type", ctypes.c_int32), ("decay", ctypes.c_float),
        ("reserved", ctypes.c_int32)]


@dataclass
class Hyper:
    """Hyper-parameters of one completion, in the paper's symbols."""
    M: int
    H: int = 100
    tau: int = 1
    outer_lr: float = 0.7
    momentum: float = 0.9
    lam: float = 0.5
    alpha: float = 1.0
    comp_mode: int = COMP_TAYLOR
    sign_mode: int = SIGN_FORWARD

    def _c(self) -> _Hyper:
        return _Hyper(self.M, self.comp_mode, self.sign_mode, 0, self.H, self.tau,
                      self.outer_lr, self.momentum, self.lam, self.alpha)


def _load() -> ctypes.CDLL:
    path = _build.LIBRARY
    if not os.path.exists(path):
        raise ImportError(
            f"{path} is missing: build the CUDA library first "
            "(python -m paper_2504_17672_b200.build, or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(path)
    vp, i32, i64, u32, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_double
    lib.cocodc_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(_Partition), i32, i32]
    lib.cocodc_destroy.argtypes = [vp]
    lib.cocodc_sync_budget.argtypes = [i32, i64, f64, f64, f64, ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.cocodc_fragment_scores.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.cocodc_scores_from_sumsq.argtypes = [vp, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp]
    lib.cocodc_bind_in_flight.argtypes = [vp, vp]
    lib.cocodc_flush_scores.argtypes = [vp, vp]
    lib.cocodc_initiate.argtypes = [vp, vp, vp, vp, i64, i64, i32, i64, vp, vp, vp, vp, vp, vp, i64, i64, i32, vp]
    lib.cocodc_initiate_at.argtypes = [vp, vp, vp, vp, vp, i64, i32, i64, vp, vp, vp, vp, vp, vp, i64, i64, i32, vp]
    lib.cocodc_select_fragments.argtypes = [vp, vp, vp, vp, i64, i64, i32, i64, vp, vp, vp, vp, vp]
    lib.cocodc_outer_step.argtypes = [vp, ctypes.POINTER(_Hyper), vp, vp, i64, i64, vp, vp, vp, vp, vp, vp,
                                      i64, i64, vp, vp, vp, vp, u32, vp]
    lib.cocodc_outer_step_host.argtypes = [vp, ctypes.POINTER(_Hyper), vp, vp, i64, i64, vp, vp, vp, vp, vp, i32,
                                           i64, i64, vp, vp, vp, i32, vp, ctypes.c_uint64, vp]
    lib.cocodc_snapshot_host.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, i32, vp]
    lib.cocodc_merge.argtypes = [vp, ctypes.POINTER(_Hyper), vp, vp, i64, i64, vp, vp, vp, vp, vp]
    lib.cocodc_snapshot.argtypes = [vp, vp, vp, i64, i64, vp, i32, vp, vp, vp]
    lib.cocodc_fragment_scores_noalloc.argtypes = [ctypes.POINTER(_Partition), vp, vp, vp, vp, i32, vp]
    lib.cocodc_selftest_bounded_wait.argtypes = [vp, i32, vp]
    lib.cocodc_select_fragments_at.argtypes = [vp, vp, vp, vp, vp, i64, i32, i64, vp, vp, vp, vp, vp]
    lib.cocodc_outer_step_at.argtypes = [vp, ctypes.POINTER(_Hyper), vp, vp, i64, i64, vp, vp, vp, vp, vp, vp,
                                         vp, vp, vp, vp, vp, vp, u32, vp]
    lib.cocodc_pseudo_gradient_sum.argtypes = [vp, vp, i64, vp, vp, i32, vp, vp, vp, vp]
    lib.cocodc_outer_step_received.argtypes = [vp, ctypes.POINTER(_Hyper), i32, vp, vp, i64, i64, vp, vp, vp, vp,
                                               vp, vp, vp, i64, i64, vp, vp, vp, vp]
    lib.cocodc_outer_step_received_peers.argtypes = [vp, ctypes.POINTER(_Hyper), i32, vp, vp, i64, i64, vp, vp, vp,
                                                     ctypes.POINTER(vp), i32, vp, vp, vp, i64, i64, vp, vp, vp, vp]
    lib.cocodc_poll_status.argtypes = [vp, vp]
    lib.cocodc_launch_count.argtypes = [vp]
    lib.cocodc_status_string.argtypes = [ctypes.c_int]
    f32, u64 = ctypes.c_float, ctypes.c_uint64
    lib.cocodc_lm_create.argtypes = [ctypes.POINTER(vp), i32]
    lib.cocodc_lm_destroy.argtypes = [vp]
    lib.cocodc_lm_poll_status.argtypes = [vp, vp]
    lib.cocodc_lm_launch_count.argtypes = [vp]
    lib.cocodc_lm_embed.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, i64, f32, vp, i32, i64, vp]
    lib.cocodc_lm_embed_grad.argtypes = [vp, vp, i32, i64, vp, i32, i64, i64, i64, f32, i32, vp, i32, i64, vp, u64, vp]
    lib.cocodc_lm_embed_grad_workspace.argtypes = [i64, i64, i64]
    lib.cocodc_lm_glu.argtypes = [vp, i32, i32, vp, i64, vp, vp, i64, i64, i64, i64, vp, i64, vp, vp, i64, vp]
    lib.cocodc_lm_glu_grad.argtypes = [vp, i32, i32, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, i64, i64, i64,
                                       vp, i64, vp, vp, i64, vp, u64, vp]
    lib.cocodc_lm_glu_grad_workspace.argtypes = [i64, i64, i64]
    lib.cocodc_lm_logprobs.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, f32, vp, vp, vp, i32, vp, vp, vp]
    lib.cocodc_lm_logprobs_grad.argtypes = [vp, vp, i32, i64, i64, i64, vp, i32, f32, vp, vp, vp, vp, vp, i64, vp]
    lib.cocodc_lm_submit.argtypes = [vp, ctypes.c_char_p]
    lib.cocodc_lm_norm.argtypes = [vp, vp, i32, i64, vp, i64, i32, vp, i32, i64, i64, f32, vp, i64, vp, i32, i64, vp, i64, vp, vp]
    lib.cocodc_lm_norm_grad.argtypes = [vp, vp, i32, i64, vp, i32, i64, vp, i32, vp, i64, i64, vp, i64, vp, i64, vp, i32, i32, vp, u64, vp]
    lib.cocodc_lm_norm_grad_workspace.argtypes = [i64, i64]
    lib.cocodc_lm_head.argtypes = [vp, i32, vp, i64, vp, i64, i64, i64, i64, vp, i32, f32, vp, vp, vp, u64, vp]
    lib.cocodc_lm_head_grad.argtypes = [vp, i32, vp, i64, vp, i64, i64, i64, i64, vp, i32, f32, vp, vp, vp, vp, i64, vp, i32, i64, i32,
                                        vp, u64, vp]
    lib.cocodc_lm_head_workspace.argtypes = lib.cocodc_lm_head_grad_workspace.argtypes = [i64, i64, i64]
    lib.cocodc_lm_adam_create.argtypes = [ctypes.POINTER(vp), vp, ctypes.POINTER(_Tensor), i64, i32]
    lib.cocodc_lm_adam_destroy.argtypes = [vp]
    lib.cocodc_lm_adamw.argtypes = [vp, vp, f64, f64, f64, f64, i64, vp, vp, vp, i64, vp]
    other = {"cocodc_launch_count": i64, "cocodc_status_string": ctypes.c_char_p, "cocodc_lm_launch_count": i64,
             "cocodc_lm_embed_grad_workspace": u64, "cocodc_lm_glu_grad_workspace": u64, "cocodc_lm_norm_grad_workspace": u64,
             "cocodc_lm_head_workspace": u64, "cocodc_lm_head_grad_workspace": u64}
    for name, restype in other.items():
        getattr(lib, name).restype = restype
    for name in EXPORTS:
        if name not in other:
            getattr(lib, name).restype = ctypes.c_int
    return lib


_lib = _load()


def library() -> ctypes.CDLL:
    return _lib


def status_string(code: int) -> str:
    return _lib.cocodc_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != OK:
        raise CocodcError(code, where)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def cocodc_sync_budget(K: int, H: int, gamma: float, Tc: float, Ts: float):
    """Eq. 8-9 on the host: returns (N, h)."""
    N, h = ctypes.c_int64(), ctypes.c_int64()
    _check(_lib.cocodc_sync_budget(K, H, gamma, Tc, Ts, ctypes.byref(N), ctypes.byref(h)), "cocodc_sync_budget")
    return N.value, h.value


def cocodc_fragment_scores_noalloc(N: int, frag_seg_ptr, seg_offset, seg_len, delta_g, interval, norms, scores,
                                   device: int = 0, stream=None) -> None:
    """Fragment norms and scores without a context and without any device allocation.

    For callers that may not allocate on the device (allocator hooks, pre-partitioned memory,
    allocation-free hot paths): the library's own fixed scratch array is used instead of context
    memory.  At most NOALLOC_MAX_K fragments / NOALLOC_MAX_SEGMENTS segments; calls that overlap on
    the GPU race on that array, so keep them on one stream.  The fragment table is host data."""
    ptr = np.ascontiguousarray(frag_seg_ptr, dtype=np.int32)
    off = np.ascontiguousarray(seg_offset, dtype=np.int64)
    ln = np.ascontiguousarray(seg_len, dtype=np.int64)
    part = _Partition(int(N), len(ptr) - 1, len(off),
                      ptr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                      off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                      ln.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)))
    _check(_lib.cocodc_fragment_scores_noalloc(ctypes.byref(part), _p(delta_g), _p(interval), _p(norms), _p(scores),
                                               int(device), _stream(stream)), "cocodc_fragment_scores_noalloc")


class Context:
    """Owns a cocodc_ctx for one fragment partition on one device."""

    def __init__(self, N: int, frag_seg_ptr: Sequence[int], seg_offset: Sequence[int],
                 seg_len: Sequence[int], max_M: int, device: int = 0):
        self._h = ctypes.c_void_p()
        ptr = np.ascontiguousarray(frag_seg_ptr, dtype=np.int32)
        off = np.ascontiguousarray(seg_offset, dtype=np.int64)
        ln = np.ascontiguousarray(seg_len, dtype=np.int64)
        part = _Partition(int(N), len(ptr) - 1, len(off),
                          ptr.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                          off.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)),
                          ln.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)))
        self.N, self.K, self.device = int(N), len(ptr) - 1, int(device)
        _check(_lib.cocodc_create(ctypes.byref(self._h), ctypes.byref(part), int(max_M), int(device)), "cocodc_create")

    def close(self) -> None:
        if self._h:
            _lib.cocodc_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launch_count(self) -> int:
        return int(_lib.cocodc_launch_count(self._h))

    def cocodc_fragment_scores(self, delta_g, interval, norms, scores, sumsq_out=None, stream=None) -> None:
        _check(_lib.cocodc_fragment_scores(self._h, _p(delta_g), _p(interval), _p(norms), _p(scores),
                                           _p(sumsq_out), _stream(stream)), "cocodc_fragment_scores")

    def cocodc_scores_from_sumsq(self, sumsq, ids, n_ids, interval, t_p: int, t_l: int, last_sync, norms, scores,
                                 stream=None) -> None:
        """Eq. 10 from fp64 sums of squares [K]: completion mode with an id list, stand-alone (all K) without."""
        _check(_lib.cocodc_scores_from_sumsq(self._h, _p(sumsq), _p(ids), _p(n_ids), _p(interval), int(t_p),
                                             int(t_l), _p(last_sync), _p(norms), _p(scores), _stream(stream)),
               "cocodc_scores_from_sumsq")

    def cocodc_bind_in_flight(self, in_flight) -> None:
        """Bind (or, with None, unbind) the caller's device uint8[K] mask of fragments in flight."""
        self._in_flight = in_flight          # keeps the tensor alive while the context points at it
        _check(_lib.cocodc_bind_in_flight(self._h, _p(in_flight)), "cocodc_bind_in_flight")

    def cocodc_flush_scores(self, stream=None) -> None:
        """Form the scores a completion launched with STAGE_DEFER left unformed (no-op when there is none)."""
        _check(_lib.cocodc_flush_scores(self._h, _stream(stream)), "cocodc_flush_scores")

    def cocodc_select_fragments(self, scores, last_sync, ineligible, t_now: int, H: int, budget_kind: int,
                                budget: int, mask, ids, n_sel, pool_offset=None, stream=None) -> None:
        _check(_lib.cocodc_select_fragments(self._h, _p(scores), _p(last_sync), _p(ineligible), int(t_now), int(H),
                                            int(budget_kind), int(budget), _p(mask), _p(ids), _p(n_sel),
                                            _p(pool_offset), _stream(stream)), "cocodc_select_fragments")

    def cocodc_initiate(self, scores, last_sync, ineligible, t_now: int, H: int, budget_kind: int, budget: int,
                        mask, ids, n_sel, pool_offset, w_now, w_snap, now_stride: int, snap_stride: int, M: int,
                        stream=None) -> None:
        """Algorithm 2 and the snapshot of what it picks, one launch (cocodc_select_fragments + cocodc_snapshot)."""
        _check(_lib.cocodc_initiate(self._h, _p(scores), _p(last_sync), _p(ineligible), int(t_now), int(H),
                                    int(budget_kind), int(budget), _p(mask), _p(ids), _p(n_sel), _p(pool_offset),
                                    _p(w_now), _p(w_snap), int(now_stride), int(snap_stride), int(M),
                                    _stream(stream)), "cocodc_initiate")

    def cocodc_initiate_at(self, scores, last_sync, ineligible, t_now, H: int, budget_kind: int, budget: int,
                           mask, ids, n_sel, pool_offset, w_now, w_snap, now_stride: int, snap_stride: int, M: int,
                           stream=None) -> None:
        """As cocodc_initiate with t_now a device int64[1] tensor."""
        _check(_lib.cocodc_initiate_at(self._h, _p(scores), _p(last_sync), _p(ineligible), _p(t_now), int(H),
                                       int(budget_kind), int(budget), _p(mask), _p(ids), _p(n_sel), _p(pool_offset),
                                       _p(w_now), _p(w_snap), int(now_stride), int(snap_stride), int(M),
                                       _stream(stream)), "cocodc_initiate_at")

    def cocodc_outer_step(self, hyper: Hyper, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset,
                          theta_g, momentum, delta_g_out, ids, n_ids, t_p: int, t_l: int, last_sync,
                          norms, scores, stages: int = STAGE_ALL, stream=None, sumsq_out=None) -> None:
        h = hyper._c()
        _check(_lib.cocodc_outer_step(self._h, ctypes.byref(h), _p(w_now), _p(w_snap), int(now_stride),
                                      int(snap_stride), _p(snap_offset), _p(theta_g), _p(momentum),
                                      _p(delta_g_out), _p(ids), _p(n_ids), int(t_p), int(t_l), _p(last_sync),
                                      _p(norms), _p(scores), _p(sumsq_out), int(stages), _stream(stream)),
               "cocodc_outer_step")

    def cocodc_outer_step_host(self, hyper: Hyper, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset,
                               theta_g, momentum, delta_g_out, ids, n_ids: int, t_p: int, t_l: int,
                               last_sync, norms, scores, workspace, snap_on_device: bool = False,
                               stream=None) -> None:
        """Host-buffer variant: every tensor is a CPU tensor, except `workspace` (CUDA) and, with
        snap_on_device, `w_snap` (CUDA)."""
        h = hyper._c()
        _check(_lib.cocodc_outer_step_host(self._h, ctypes.byref(h), _p(w_now), _p(w_snap), int(now_stride),
                                           int(snap_stride), _p(snap_offset), _p(theta_g), _p(momentum),
                                           _p(delta_g_out), _p(ids), int(n_ids), int(t_p), int(t_l),
                                           _p(last_sync), _p(norms), _p(scores), 1 if snap_on_device else 0, _p(workspace),
                                           workspace.numel() * workspace.element_size(), _stream(stream)),
               "cocodc_outer_step_host")

    def cocodc_select_fragments_at(self, scores, last_sync, ineligible, t_now, H: int, budget_kind: int,
                                   budget: int, mask, ids, n_sel, pool_offset=None, stream=None) -> None:
        """As cocodc_select_fragments with t_now a device int64[1] tensor."""
        _check(_lib.cocodc_select_fragments_at(self._h, _p(scores), _p(last_sync), _p(ineligible), _p(t_now), int(H),
                                               int(budget_kind), int(budget), _p(mask), _p(ids), _p(n_sel),
                                               _p(pool_offset), _stream(stream)), "cocodc_select_fragments_at")

    def cocodc_outer_step_at(self, hyper: Hyper, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset,
                             theta_g, momentum, delta_g_out, ids, n_ids, t_p, t_l, last_sync,
                             norms, scores, stages: int = STAGE_ALL, stream=None, sumsq_out=None) -> None:
        """As cocodc_outer_step with t_p and t_l device int64[1] tensors."""
        h = hyper._c()
        _check(_lib.cocodc_outer_step_at(self._h, ctypes.byref(h), _p(w_now), _p(w_snap), int(now_stride),
                                         int(snap_stride), _p(snap_offset), _p(theta_g), _p(momentum),
                                         _p(delta_g_out), _p(ids), _p(n_ids), _p(t_p), _p(t_l), _p(last_sync),
                                         _p(norms), _p(scores), _p(sumsq_out), int(stages), _stream(stream)),
               "cocodc_outer_step_at")

    def cocodc_pseudo_gradient_sum(self, w_snap, snap_stride: int, snap_offset, theta_g, M: int, sum_out,
                                   ids, n_ids, stream=None) -> None:
        _check(_lib.cocodc_pseudo_gradient_sum(self._h, _p(w_snap), int(snap_stride), _p(snap_offset), _p(theta_g),
                                               int(M), _p(sum_out), _p(ids), _p(n_ids), _stream(stream)),
               "cocodc_pseudo_gradient_sum")

    def cocodc_outer_step_received(self, hyper: Hyper, M_total: int, w_now, w_snap, now_stride: int,
                                   snap_stride: int, snap_offset, theta_g, momentum, delta_sum, delta_g_out,
                                   ids, n_ids, t_p: int, t_l: int, last_sync, norms, scores, stream=None) -> None:
        h = hyper._c()
        _check(_lib.cocodc_outer_step_received(self._h, ctypes.byref(h), int(M_total), _p(w_now), _p(w_snap),
                                               int(now_stride), int(snap_stride), _p(snap_offset), _p(theta_g),
                                               _p(momentum), _p(delta_sum), _p(delta_g_out), _p(ids), _p(n_ids),
                                               int(t_p), int(t_l), _p(last_sync), _p(norms), _p(scores),
                                               _stream(stream)), "cocodc_outer_step_received")

    def cocodc_outer_step_received_peers(self, hyper: Hyper, M_total: int, w_now, w_snap, now_stride: int,
                                         snap_stride: int, snap_offset, theta_g, momentum, delta_sums, delta_g_out,
                                         ids, n_ids, t_p: int, t_l: int, last_sync, norms, scores,
                                         stream=None) -> None:
        """delta_sums: sequence of device tensors (or integer device addresses, e.g. of peer-mapped buffers)."""
        h = hyper._c()
        addrs = [int(x) if isinstance(x, int) else x.data_ptr() for x in delta_sums]
        arr = (ctypes.c_void_p * len(addrs))(*addrs)
        _check(_lib.cocodc_outer_step_received_peers(self._h, ctypes.byref(h), int(M_total), _p(w_now), _p(w_snap),
                                                     int(now_stride), int(snap_stride), _p(snap_offset), _p(theta_g),
                                                     _p(momentum), arr, len(addrs), _p(delta_g_out), _p(ids),
                                                     _p(n_ids), int(t_p), int(t_l), _p(last_sync), _p(norms),
                                                     _p(scores), _stream(stream)), "cocodc_outer_step_received_peers")

    def cocodc_merge(self, hyper: Hyper, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset,
                     theta_g_new, ids, n_ids, stream=None) -> None:
        h = hyper._c()
        _check(_lib.cocodc_merge(self._h, ctypes.byref(h), _p(w_now), _p(w_snap), int(now_stride), int(snap_stride),
                                 _p(snap_offset), _p(theta_g_new), _p(ids), _p(n_ids), _stream(stream)),
               "cocodc_merge")

    def cocodc_snapshot(self, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset, M: int,
                        ids, n_ids, stream=None) -> None:
        _check(_lib.cocodc_snapshot(self._h, _p(w_now), _p(w_snap), int(now_stride), int(snap_stride),
                                    _p(snap_offset), int(M), _p(ids), _p(n_ids), _stream(stream)),
               "cocodc_snapshot")

    def cocodc_snapshot_host(self, w_now, w_snap, now_stride: int, snap_stride: int, snap_offset, M: int,
                             ids, n_ids: int, stream=None) -> None:
        """S0 from a host w_now into a device w_snap; ids and snap_offset are CPU tensors."""
        _check(_lib.cocodc_snapshot_host(self._h, _p(w_now), _p(w_snap), int(now_stride), int(snap_stride),
                                         _p(snap_offset), int(M), _p(ids), int(n_ids), _stream(stream)),
               "cocodc_snapshot_host")

    def cocodc_selftest_bounded_wait(self, polls: int, stream=None) -> None:
        """Runs a bounded wait that must run out; the status word then reads ERR_TIMEOUT."""
        _check(_lib.cocodc_selftest_bounded_wait(self._h, int(polls), _stream(stream)), "cocodc_selftest_bounded_wait")

    def cocodc_poll_status(self, stream=None) -> int:
        """Waits for the stream; returns and clears the device status word."""
        return int(_lib.cocodc_poll_status(self._h, _stream(stream)))


# ---- operators of the local step (include/cocodc_lm.h) ------------------------------------------------------------

ACT_SILU, ACT_GELU = 0, 1
LM_MAX_TOP = 32
LM_ADAM_BLOCK = 256
E4M3 = 3                                                 # COCODC_E4M3: torch.float8_e4m3fn
_ACTS = {"silu": ACT_SILU, "gelu": ACT_GELU, ACT_SILU: ACT_SILU, ACT_GELU: ACT_GELU}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INDEX_TYPES = {torch.int32: 0, torch.int64: 1}
# records of cocodc_lm_submit: the operator's number, then its arguments (q: pointer or integer, d: scale)
_EMBED, _EMBED_GRAD, _GLU, _GLU_GRAD, _LOGPROBS, _LOGPROBS_GRAD, _NORM, _NORM_GRAD, _HEAD, _HEAD_GRAD, _ADAMW = (
    struct.Struct("=" + f).pack for f in ("9qd4q", "9qd7q", "17q", "24q", "8qd7q", "8qd7q", "11qd9q", "22q", "11qd5q", "11qd12q",
                                          "2q4d6q"))
_submit = _lib.cocodc_lm_submit


def _raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):      # the same number without a Stream object (2 us a call)
    _raw_stream = torch._C._cuda_getCurrentRawStream


def _matrix(t: torch.Tensor, name: str):
    """(address, row stride, rows, columns) of a row-major matrix; a single row (or column) may have any stride."""
    try:
        (rows, cols), (s0, s1) = t.shape, t.stride()
    except ValueError:
        raise ValueError(f"{name} must have two dimensions, not {t.dim()}") from None
    if s1 != 1 and cols > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), (s0 if rows > 1 or s0 > cols else cols), rows, cols


def _vector(t: Optional[torch.Tensor], name: str, n: int, dtype) -> int:
    """Address of a packed vector (or matrix) of n elements; 0 for None."""
    if t is None:
        return 0
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a packed {dtype} tensor of {n} elements")
    return t.data_ptr()


def _ids(t: torch.Tensor, name: str, n: int):
    kind = _INDEX_TYPES.get(t.dtype)
    if kind is None or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a packed int32 or int64 tensor of {n} elements")
    return t.data_ptr(), kind


def _type(t: torch.Tensor) -> int:
    kind = _TYPES.get(t.dtype)
    if kind is None:
        raise ValueError(f"type {t.dtype} is not supported (float32, bfloat16, float16)")
    return kind


def _one_type(*tensors) -> int:
    first = tensors[0].dtype
    for t in tensors:
        if t is not None and t.dtype is not first:
            raise ValueError("the tensors must have one type")
    return _type(tensors[0])


def _sized(name: str, rows: int, cols: int, want_rows: int, want_cols: int) -> None:
    if rows != want_rows or cols != want_cols:
        raise ValueError(f"{name} must be {want_rows} x {want_cols}, not {rows} x {cols}")


class AdamTensors:
    """Owns a cocodc_lm_adam: the tensors of a model as cocodc_lm_adamw steps them.

    params: packed float32 tensors; grads of any type; m and v float32, or float8_e4m3fn with their scales (m_scales, v_scales: one
    float32 for every 256 elements, begun at zero like m and v); decay: a number or one for each tensor; copies: 16-bit tensors
    (or None each) that receive the stepped parameters.  The tensors are kept alive and have to stay where they are."""

    def __init__(self, ops: "LmOps", params, grads, m, v, decay=0.0, copies=None, m_scales=None, v_scales=None):
        self._h = ctypes.c_void_p()
        params, grads, m, v = (list(x) for x in (params, grads, m, v))
        count = len(params)
        fill = lambda x: [None] * count if x is None else list(x)  # noqa: E731
        copies, m_scales, v_scales = fill(copies), fill(m_scales), fill(v_scales)
        decay = list(decay) if isinstance(decay, Sequence) else [float(decay)] * count
        lists = (params, grads, m, v, copies, m_scales, v_scales, decay)
        if any(len(x) != count for x in lists):
            raise ValueError("one of every list is needed for each tensor")
        self.tensors, self.count = lists, count
        state = torch.float32 if count == 0 or m[0] is None else m[0].dtype
        if state not in (torch.float32, torch.float8_e4m3fn):
            raise ValueError(f"states of type {state} are not supported (float32, float8_e4m3fn)")
        self.state_bits = 8 if state is torch.float8_e4m3fn else 32
        table = (_Tensor * max(1, count))()
        for i, (p, g, a, b, c, ms, vs, d) in enumerate(zip(*lists)):
            ops._on_device(p, g, a, b, c, ms, vs)
            n = p.numel()
            if g.numel() != n or not g.is_contiguous():
                raise ValueError(f"grads[{i}] must be packed, of {n} elements")
            if c is not None and (c.numel() != n or not c.is_contiguous() or c.dtype not in (torch.bfloat16, torch.float16)):
                raise ValueError(f"copies[{i}] must be packed, bfloat16 or float16, of {n} elements")
            blocks = (n + LM_ADAM_BLOCK - 1) // LM_ADAM_BLOCK
            table[i] = _Tensor(_vector(p, f"params[{i}]", n, torch.float32), g.data_ptr(), _vector(a, f"m[{i}]", n, state),
                               _vector(b, f"v[{i}]", n, state), _vector(ms, f"m_scales[{i}]", blocks, torch.float32),
                               _vector(vs, f"v_scales[{i}]", blocks, torch.float32), 0 if c is None else c.data_ptr(), n, _type(g),
                               0 if c is None else _type(c), float(d), 0)
        _check(_lib.cocodc_lm_adam_create(ctypes.byref(self._h), ops._h, table, count, self.state_bits), "cocodc_lm_adam_create")

    def close(self) -> None:
        if self._h:
            _lib.cocodc_lm_adam_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class LmOps:
    """Owns a cocodc_lm: the operators of a worker's local step on one device.

    Sizes, strides and types are read from the tensors; outputs are written to the tensors that are passed.  Calls run
    on `stream` (default: torch's current stream of the handle's device).  A workspace that is not passed is taken from
    torch's caching allocator on that stream."""

    def __init__(self, device: int = 0):
        self._h = ctypes.c_void_p()
        device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        self.device = torch.device("cuda", device.index or 0)
        self._index = self.device.index
        _check(_lib.cocodc_lm_create(ctypes.byref(self._h), self.device.index), "cocodc_lm_create")

    def close(self) -> None:
        if self._h:
            _lib.cocodc_lm_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launch_count(self) -> int:
        return int(_lib.cocodc_lm_launch_count(self._h))

    def cocodc_lm_poll_status(self, stream=None) -> int:
        """Waits for the stream; returns and clears the device status word."""
        return int(_lib.cocodc_lm_poll_status(self._h, self._stream(stream)))

    def _stream(self, stream) -> int:
        return _raw_stream(self._index) if stream is None else stream.cuda_stream

    def _on_device(self, *tensors) -> None:
        index = self._index
        for t in tensors:
            if t is not None and t.get_device() != index:      # -1 for a CPU tensor
                raise ValueError(f"a tensor is on {t.device}, the handle on {self.device}")

    def _scratch(self, workspace, need: int, stream):
        if workspace is None:
            if stream is None:
                return torch.empty(max(16, need), dtype=torch.uint8, device=self.device)
            with torch.cuda.stream(stream):
                return torch.empty(max(16, need), dtype=torch.uint8, device=self.device)
        self._on_device(workspace)
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
        return workspace

    def cocodc_lm_embed(self, table, ids, y, scale: float = 1.0, stream=None) -> None:
        """y[t] = scale * table[ids[t]]; zeros where ids[t] < 0."""
        self._on_device(table, ids, y)
        tp, ts, V, D = _matrix(table, "table")
        yp, ys, T, cols = _matrix(y, "y")
        if cols != D:
            _sized("y", T, cols, T, D)
        ip, it = _ids(ids, "ids", T)
        code = _submit(self._h, _EMBED(0, tp, _type(table), ts, V, D, ip, it, T, scale, yp, _type(y), ys, self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_embed")

    def cocodc_lm_embed_grad(self, dy, ids, dtable, scale: float = 1.0, accumulate: bool = False, workspace=None,
                             stream=None) -> None:
        """dtable[v] (+)= scale * sum of dy[t] over the t with ids[t] == v."""
        self._on_device(dy, ids, dtable)
        dp, ds, T, cols = _matrix(dy, "dy")
        gp, gs, V, D = _matrix(dtable, "dtable")
        if cols != D:
            _sized("dy", T, cols, T, D)
        ip, it = _ids(ids, "ids", T)
        w = self._scratch(workspace, _lib.cocodc_lm_embed_grad_workspace(V, D, T), stream)
        code = _submit(self._h, _EMBED_GRAD(1, dp, _type(dy), ds, ip, it, T, V, D, scale, bool(accumulate), gp, _type(dtable), gs,
                                            w.data_ptr(), w.numel() * w.element_size(), self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_embed_grad")

    def cocodc_lm_glu(self, x, wg, wu, h, gate=None, up=None, act="silu", stream=None) -> None:
        """h = act(x wg^T) * (x wu^T); gate and up receive the two products (both or neither)."""
        self._on_device(x, wg, wu, h)
        xp, xs, T, D = _matrix(x, "x")
        gp, gs, F, cols = _matrix(wg, "wg")
        up_, us, rows, cols2 = _matrix(wu, "wu")
        hp, hs, T2, F2 = _matrix(h, "h")
        if not (cols == cols2 == D and rows == F2 == F and T2 == T):
            _sized("wg", F, cols, F, D)
            _sized("wu", rows, cols2, F, D)
            _sized("h", T2, F2, T, F)
        if gs != us and F > 1:
            raise ValueError("wg and wu must have the same row stride")
        kind = _one_type(x, wg, wu, h, gate, up)
        gtp = utp = 0
        gus = F
        if gate is not None or up is not None:
            self._on_device(gate, up)
            strides = []
            for name, t in (("gate", gate), ("up", up)):
                if t is not None:
                    p, st, r, c = _matrix(t, name)
                    _sized(name, r, c, T, F)
                    strides.append(st)
                    gtp, utp = (p, utp) if name == "gate" else (gtp, p)
            gus = strides[0]
            if strides[-1] != gus and T > 1:
                raise ValueError("gate and up must have the same row stride")
        code = _submit(self._h, _GLU(2, _ACTS[act], kind, xp, xs, gp, up_, gs, T, D, F, hp, hs, gtp, utp, gus, self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_glu")

    def cocodc_lm_glu_grad(self, dh, gate, up, x, wg, wu, dx=None, dwg=None, dwu=None, act="silu", workspace=None,
                           stream=None) -> None:
        """dx, dwg, dwu of cocodc_lm_glu from dh and the gate and up that it wrote; dx, or dwg and dwu, may be None."""
        self._on_device(dh, gate, up, x, wg, wu, dx, dwg, dwu)
        xp, xs, T, D = _matrix(x, "x")
        gp, ws, F, cols = _matrix(wg, "wg")
        _sized("wg", F, cols, F, D)
        kind = _one_type(x, wg, wu, dh, gate, up, dx, dwg, dwu)

        def take(t, name, rows, cols):
            if t is None:
                return 0, cols
            p, stride, r, c = _matrix(t, name)
            _sized(name, r, c, rows, cols)
            return p, stride

        wup, ws2 = take(wu, "wu", F, D)
        hp, hs = take(dh, "dh", T, F)
        (gtp, gs), (utp, us) = take(gate, "gate", T, F), take(up, "up", T, F)
        dxp, dxs = take(dx, "dx", T, D)
        (dgp, dws), (dup, dws2) = take(dwg, "dwg", F, D), take(dwu, "dwu", F, D)
        if (gs != us and T > 1) or (ws != ws2 and F > 1):
            raise ValueError("gate and up, and wg and wu, must have the same row stride")
        if dwg is not None and dwu is not None and dws != dws2 and F > 1:
            raise ValueError("dwg and dwu must have the same row stride")
        w = self._scratch(workspace, _lib.cocodc_lm_glu_grad_workspace(T, D, F), stream)
        code = _submit(self._h, _GLU_GRAD(3, _ACTS[act], kind, hp, hs, gtp, utp, gs, xp, xs, gp, wup, ws, T, D, F, dxp, dxs, dgp, dup,
                                          dws, w.data_ptr(), w.numel() * w.element_size(), self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_glu_grad")

    def cocodc_lm_logprobs(self, logits, targets, logp, entropy=None, lse=None, top_ids=None, top_logp=None,
                           scale: float = 1.0, stream=None) -> None:
        """Per row of scale * logits: log probability of targets[t] (0 where it is negative), entropy, log-sum-exp, and the
        largest logits' ids and log probabilities (top_ids, top_logp: T x k).  targets and logp may both be None."""
        self._on_device(logits, targets, logp, entropy, lse, top_ids, top_logp)
        lp, ls, T, V = _matrix(logits, "logits")
        tp, tt = _ids(targets, "targets", T) if targets is not None else (0, 0)
        f32 = torch.float32
        k = kp = kl = 0
        if top_ids is not None or top_logp is not None:      # one without the other is refused by the call
            shape = (top_logp if top_ids is None else top_ids).shape
            if len(shape) != 2 or shape[0] != T:
                raise ValueError("top_ids and top_logp must be T x k")
            k = shape[1]
            kp, kl = _vector(top_ids, "top_ids", T * k, torch.int32), _vector(top_logp, "top_logp", T * k, f32)
        code = _submit(self._h, _LOGPROBS(4, lp, _type(logits), ls, T, V, tp, tt, scale, _vector(logp, "logp", T, f32),
                                          _vector(entropy, "entropy", T, f32), _vector(lse, "lse", T, f32), k, kp, kl,
                                          self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_logprobs")

    def cocodc_lm_logprobs_grad(self, logits, targets, lse, entropy, dlogp, dentropy, dlogits, scale: float = 1.0,
                                stream=None) -> None:
        """dlogits of cocodc_lm_logprobs given d/dlogp and d/dentropy (None for zero); dlogits may be logits itself."""
        self._on_device(logits, targets, lse, entropy, dlogp, dentropy, dlogits)
        lp, ls, T, V = _matrix(logits, "logits")
        dp, ds, T2, V2 = _matrix(dlogits, "dlogits")
        _sized("dlogits", T2, V2, T, V)
        kind = _one_type(logits, dlogits)
        tp, tt = _ids(targets, "targets", T) if targets is not None else (0, 0)
        f32 = torch.float32
        code = _submit(self._h, _LOGPROBS_GRAD(5, lp, kind, ls, T, V, tp, tt, scale, _vector(lse, "lse", T, f32),
                                               _vector(entropy, "entropy", T, f32), _vector(dlogp, "dlogp", T, f32),
                                               _vector(dentropy, "dentropy", T, f32), dp, ds, self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_logprobs_grad")

    def cocodc_lm_norm(self, x, weight, y, residual=None, total=None, rstd=None, y_scale=None, eps: float = 1e-6, stream=None) -> None:
        """total = x + residual (both or neither; total may be residual); y = total / rms(total) * weight, or of x.  y of type
        float8_e4m3fn takes y_scale: [T] or [T, 1] for a scale per row, [T, ceil(D / 128)] for one per 128 columns."""
        self._on_device(x, weight, y, residual, total, rstd, y_scale)
        xp, xs, T, D = _matrix(x, "x")
        yp, ys, rows, cols = _matrix(y, "y")
        if rows != T or cols != D:
            _sized("y", rows, cols, T, D)
        rp = tp = kind = sp = group = 0
        rs = ts = D
        if residual is not None:                             # one without the other is refused by the call
            kind = _type(residual)
            rp, rs, rows, cols = _matrix(residual, "residual")
            if rows != T or cols != D:
                _sized("residual", rows, cols, T, D)
        if total is not None:
            if residual is not None and total.dtype is not residual.dtype:
                raise ValueError("residual and total must have one type")
            kind = _type(total)
            tp, ts, rows, cols = _matrix(total, "total")
            if rows != T or cols != D:
                _sized("total", rows, cols, T, D)
        y_type = E4M3 if y.dtype is torch.float8_e4m3fn else _type(y)
        if y_scale is not None:
            groups, shape = (D + 127) // 128, tuple(y_scale.shape)
            if shape == (T, groups) and groups > 1:
                group = 128
            elif shape not in ((T,), (T, 1)):
                raise ValueError(f"y_scale must be {T}, {T} x 1 or {T} x {groups}, not {shape}")
            sp = _vector(y_scale, "y_scale", y_scale.numel(), torch.float32)
        code = _submit(self._h, _NORM(6, xp, _type(x), xs, rp, rs, kind, _vector(weight, "weight", D, weight.dtype), _type(weight), T, D, eps,
                                      tp, ts, yp, y_type, ys, sp, group, _vector(rstd, "rstd", T, torch.float32), self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_norm")

    def cocodc_lm_norm_grad(self, dy, total, weight, rstd, dx=None, dweight=None, dtotal=None, accumulate: bool = False, workspace=None,
                            stream=None) -> None:
        """dx = the gradient of total through the norm, plus dtotal (the one that reaches it otherwise; dx may be dtotal);
        dweight (+)= the weight's.  total and rstd are what cocodc_lm_norm wrote (total: x where it had no residual)."""
        self._on_device(dy, total, weight, rstd, dx, dweight, dtotal)
        yp, ys, T, D = _matrix(dy, "dy")
        kind = _type(total)

        def take(t, name):
            if t is None:
                return 0, D
            p, stride, r, c = _matrix(t, name)
            if r != T or c != D:
                _sized(name, r, c, T, D)
            if _type(t) != kind:
                raise ValueError("total, dtotal and dx must have one type")
            return p, stride

        (tp, ts), (dtp, dts), (xp, xs) = take(total, "total"), take(dtotal, "dtotal"), take(dx, "dx")
        wp = size = 0
        if dweight is not None:
            w = self._scratch(workspace, _lib.cocodc_lm_norm_grad_workspace(T, D), stream)
            wp, size = w.data_ptr(), w.numel() * w.element_size()
        code = _submit(self._h, _NORM_GRAD(7, yp, _type(dy), ys, tp, kind, ts, _vector(weight, "weight", D, weight.dtype), _type(weight),
                                           _vector(rstd, "rstd", T, torch.float32), T, D, dtp, dts, xp, xs,
                                           0 if dweight is None else _vector(dweight, "dweight", D, dweight.dtype),
                                           0 if dweight is None else _type(dweight), bool(accumulate), wp, size, self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_norm_grad")

    def cocodc_lm_head(self, x, table, targets, logp, lse=None, scale: float = 1.0, workspace=None, stream=None) -> None:
        """Log probability of targets[t] (0 where it is negative) and log-sum-exp of the logits scale * x table^T, which are not kept.
        targets and logp may both be None."""
        self._on_device(x, table, targets, logp, lse)
        xp, xs, T, D = _matrix(x, "x")
        wp, ws, V, cols = _matrix(table, "table")
        if cols != D:
            _sized("table", V, cols, V, D)
        kind = _one_type(x, table)
        tp, tt = _ids(targets, "targets", T) if targets is not None else (0, 0)
        w = self._scratch(workspace, _lib.cocodc_lm_head_workspace(T, D, V), stream)
        f32 = torch.float32
        code = _submit(self._h, _HEAD(8, kind, xp, xs, wp, ws, T, D, V, tp, tt, scale, _vector(logp, "logp", T, f32), _vector(lse, "lse", T, f32),
                                      w.data_ptr(), w.numel() * w.element_size(), self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_head")

    def cocodc_lm_head_grad(self, x, table, targets, lse, dlogp, dlse, dx=None, dtable=None, scale: float = 1.0, accumulate: bool = False,
                            workspace=None, stream=None) -> None:
        """dx and dtable of cocodc_lm_head from d/dlogp and d/dlse (None for zero) and the lse that it wrote; either output may be None.
        dtable of x's type or float32, added to what it holds with accumulate."""
        self._on_device(x, table, targets, lse, dlogp, dlse, dx, dtable)
        xp, xs, T, D = _matrix(x, "x")
        wp, ws, V, cols = _matrix(table, "table")
        if cols != D:
            _sized("table", V, cols, V, D)
        kind = _one_type(x, table, dx)
        tp, tt = _ids(targets, "targets", T) if targets is not None else (0, 0)
        dxp = dtp = dtt = 0
        dxs = dts = D
        if dx is not None:
            dxp, dxs, r, c = _matrix(dx, "dx")
            _sized("dx", r, c, T, D)
        if dtable is not None:
            dtp, dts, r, c = _matrix(dtable, "dtable")
            _sized("dtable", r, c, V, D)
            dtt = _type(dtable)
        w = self._scratch(workspace, _lib.cocodc_lm_head_grad_workspace(T, D, V), stream)
        f32 = torch.float32
        code = _submit(self._h, _HEAD_GRAD(9, kind, xp, xs, wp, ws, T, D, V, tp, tt, scale, _vector(lse, "lse", T, f32),
                                           _vector(dlogp, "dlogp", T, f32), _vector(dlse, "dlse", T, f32), dxp, dxs, dtp, dtt, dts,
                                           bool(accumulate), w.data_ptr(), w.numel() * w.element_size(), self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_head_grad")

    def cocodc_lm_adamw(self, plan: AdamTensors, lr: float, step: int = 0, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8,
                        step_at=None, grad_scale=None, lr_scale=None, seed: int = 0, stream=None) -> None:
        """One AdamW step of the plan's tensors.  step counts from 1; step_at (int64), grad_scale and lr_scale (float32) are device
        scalars, for captured steps, clipping and schedules; seed is the one of the random rounding of 8-bit states."""
        self._on_device(step_at, grad_scale, lr_scale)
        f32 = torch.float32
        code = _submit(self._h, _ADAMW(10, plan._h.value or 0, lr, beta1, beta2, eps, step, _vector(step_at, "step_at", 1, torch.int64),
                                       _vector(grad_scale, "grad_scale", 1, f32), _vector(lr_scale, "lr_scale", 1, f32), seed,
                                       self._stream(stream)))
        if code:
            raise CocodcError(code, "cocodc_lm_adamw")
