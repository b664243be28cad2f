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
    other = {"cocodc_launch_count": i64, "cocodc_status_string": ctypes.c_char_p, "cocodc_lm_launch_count": i64,
             "cocodc_lm_embed_grad_workspace": u64, "cocodc_lm_glu_grad_workspace": u64}
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
_ACTS = {"silu": ACT_SILU, "gelu": ACT_GELU, ACT_SILU: ACT_SILU, ACT_GELU: ACT_GELU}
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INDEX_TYPES = {torch.int32: 0, torch.int64: 1}
# records of cocodc_lm_submit: the operator's number, then its arguments (q: pointer or integer, d: scale)
_EMBED, _EMBED_GRAD, _GLU, _GLU_GRAD, _LOGPROBS, _LOGPROBS_GRAD = (
    struct.Struct("=" + f).pack for f in ("9qd4q", "9qd7q", "17q", "24q", "8qd7q", "8qd7q"))
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
