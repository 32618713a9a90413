"""ctypes binding of ``libstar.so`` (declared in ``include/star.h``).

Argument marshalling only: every function here has the name of the C entry
point it forwards to, turns torch tensors into device pointers and Python lists
into host arrays, and raises :class:`StarError` on a non-zero status.  PyTorch
supplies device memory and the current stream; nothing is computed in Python
and there is no fallback: if the library is missing, importing this module
raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import List, Optional, Sequence, Tuple

import torch

from .workloads import ModeDecision

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libstar.so")

STAR_OK = 0
STAR_ERR_NULL_POINTER = 1
STAR_ERR_INVALID_ARG = 2
STAR_ERR_BAD_SCHEDULE = 3
STAR_ERR_UNSUPPORTED = 4
STAR_ERR_WORKSPACE_TOO_SMALL = 5
STAR_ERR_CUDA = 6
STAR_ERR_TIMEOUT = 7

STAR_DTYPE_F32 = 0
STAR_DTYPE_BF16 = 1
STAR_MAX_WORKERS = 64
STAR_SUM_LINEAR = 0
STAR_SUM_TREE = 1


class StarError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        name = _lib.star_status_string(status).decode()
        extra = ""
        if status == STAR_ERR_CUDA:
            extra = " (cudaError %d)" % _lib.star_last_cuda_error()
        super().__init__("%s failed: %s%s" % (where, name, extra))


class star_multi_plan_t(ctypes.Structure):
    _fields_ = [
        ("magic", ctypes.c_uint64),
        ("d_workspace", ctypes.c_void_p),
        ("total_elements", ctypes.c_int64),
        ("n_tiles", ctypes.c_int64),
        ("complete_workers", ctypes.c_uint64),
        ("n_tensors", ctypes.c_int32),
        ("W", ctypes.c_int32),
        ("grad_dtype", ctypes.c_int32),
        ("tile_elements", ctypes.c_int32),
        ("n_snapshot_sets", ctypes.c_int32),
        ("snapshot_dtype", ctypes.c_int32),
    ]


def _load() -> ctypes.CDLL:
    # (Re)build in-tree when the library is missing or older than its sources and
    # nvcc is at hand; otherwise fail loudly: there is no CPU fallback.
    try:
        from . import build as _build
        if _build.is_stale():
            _build.build()
    except Exception as exc:
        if not os.path.exists(LIB_PATH):
            raise ImportError(
                "%s is missing and could not be built (%s): run "
                "`python -m paper_2512_09685_b200.build`; there is no CPU fallback" % (LIB_PATH, exc))
    lib = ctypes.CDLL(LIB_PATH)
    c_int, c_i64, c_vp, c_f = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float
    lib.star_status_string.argtypes = [c_int]
    lib.star_status_string.restype = ctypes.c_char_p
    lib.star_last_cuda_error.argtypes = []
    lib.star_last_cuda_error.restype = c_int
    lib.star_launch_count.argtypes = []
    lib.star_launch_count.restype = c_i64
    lib.star_schedule_validate.argtypes = [c_vp, c_vp, c_int, c_int]
    lib.star_schedule_static_x.argtypes = [c_vp, c_int, c_int, c_int, c_int, c_vp, c_vp, c_vp]
    lib.star_schedule_from_labels.argtypes = [c_vp, c_int, c_vp, c_vp, c_vp]
    lib.star_schedule_dynamic_x.argtypes = [c_vp, c_vp, c_int, c_vp, c_vp, c_vp]
    lib.star_group_update.argtypes = [c_vp, c_vp, c_vp, c_int, c_int, c_i64, c_vp, c_vp, c_int,
                                      c_f, c_f, c_f, c_vp]
    lib.star_multi_workspace_bytes.argtypes = [c_int, c_vp, c_int, c_vp]
    lib.star_multi_prepare.argtypes = [c_int, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_vp,
                                       ctypes.c_size_t, c_vp, c_vp]
    lib.star_group_update_multi.argtypes = [c_vp, c_vp, c_vp, c_int, c_f, c_f, c_f, c_vp]
    lib.star_group_update_multi_lrs.argtypes = [c_vp, c_vp, c_vp, c_int, c_vp, c_f, c_f, c_vp]
    lib.star_group_update_multi_lrs.restype = c_int
    lib.star_group_update_ex.argtypes = [c_vp, c_vp, c_vp, c_int, c_int, c_i64, c_vp, c_vp, c_int,
                                         c_vp, c_f, c_f, c_vp, c_int, c_int, c_vp]
    lib.star_group_update_ex.restype = c_int
    lib.star_cluster_iteration_times.argtypes = [c_vp, c_int, c_int, ctypes.c_double, c_vp, c_vp]
    lib.star_cluster_iteration_times.restype = c_int
    lib.star_mode_times.argtypes = [c_vp, c_vp, c_int, ctypes.c_double, ctypes.c_double, c_vp, c_vp]
    lib.star_mode_times.restype = c_int
    lib.star_choose_mode.argtypes = [c_vp, c_vp, c_int, ctypes.c_double, ctypes.c_double, c_vp, c_vp,
                                     c_vp, c_vp, c_vp]
    lib.star_choose_mode.restype = c_int
    lib.star_choose_all_reduce_mode.argtypes = [c_vp, c_vp, c_int] + [ctypes.c_double] * 4 + [c_vp] * 7
    lib.star_choose_all_reduce_mode.restype = c_int
    lib.star_assign_parents.argtypes = [c_vp, c_int, c_int, c_vp]
    lib.star_assign_parents.restype = c_int
    lib.star_build_tree.argtypes = [c_vp, c_int, c_int, c_vp]
    lib.star_build_tree.restype = c_int
    lib.star_shard_range.argtypes = [c_i64, c_int, c_int, c_i64, c_vp, c_vp]
    lib.star_shard_range.restype = c_int
    lib.star_host_workspace_bytes.argtypes = [c_int, c_int, c_i64, c_vp]
    lib.star_host_workspace_bytes.restype = c_int
    lib.star_group_update_host.argtypes = [c_vp, c_vp, c_vp, c_int, c_int, c_i64, c_vp, c_vp, c_int,
                                           c_f, c_f, c_f, c_vp, ctypes.c_size_t, c_vp]
    lib.star_group_update_host.restype = c_int
    lib.star_host_workspace_bytes_ex.argtypes = [c_int, c_int, c_int, c_int, c_i64, c_vp]
    lib.star_host_workspace_bytes_ex.restype = c_int
    lib.star_group_update_host_ex.argtypes = [c_vp, c_vp, c_vp, c_int, c_int, c_i64, c_vp, c_vp, c_int,
                                              c_vp, c_f, c_f, c_vp, c_int, c_int, c_vp, ctypes.c_size_t, c_vp]
    lib.star_group_update_host_ex.restype = c_int
    lib.star_group_update_multi_noalloc.argtypes = [c_int, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_vp, c_vp,
                                                    c_int, c_f, c_f, c_f, c_vp]
    lib.star_group_update_multi_noalloc.restype = c_int
    lib.star_group_reduce.argtypes = [c_vp, c_int, c_vp, c_int, c_int, c_i64, c_vp, c_int, c_int, c_vp]
    lib.star_group_reduce.restype = c_int
    lib.star_group_update_from_sums.argtypes = [c_vp, c_vp, c_vp, c_int, c_i64, c_int, c_f, c_f, c_f, c_vp]
    lib.star_group_update_from_sums.restype = c_int
    lib.star_multi_workspace_bytes_ex.argtypes = [c_int, c_vp, c_int, c_int, c_vp]
    lib.star_multi_workspace_bytes_ex.restype = c_int
    lib.star_multi_prepare_ex.argtypes = [c_int, c_vp, c_vp, c_vp, c_vp, c_int, c_int, c_int, c_vp, c_int, c_vp,
                                          ctypes.c_size_t, c_vp, c_vp]
    lib.star_multi_prepare_ex.restype = c_int
    lib.star_group_update_multi_ex.argtypes = [c_vp, c_vp, c_vp, c_int, c_vp, c_f, c_f, c_vp, c_int, c_vp]
    lib.star_group_update_multi_ex.restype = c_int
    lib.star_check_waits.argtypes = [c_vp]
    lib.star_check_waits.restype = c_int
    lib.star_set_wait_attempts.argtypes = [c_int]
    lib.star_set_wait_attempts.restype = c_int
    lib.star_token_logprobs.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_f, c_vp, c_vp, c_vp]
    lib.star_token_logprobs.restype = c_int
    lib.star_loss_workspace_bytes.argtypes = [c_i64, c_i64, c_vp]
    lib.star_loss_workspace_bytes.restype = c_int
    lib.star_policy_loss.argtypes = ([c_vp, c_int, c_i64, c_i64, c_i64] + [c_vp] * 5 + [c_f] * 4 + [c_vp] * 4
                                     + [c_i64, c_vp, ctypes.c_size_t, c_vp])
    lib.star_policy_loss.restype = c_int
    lib.star_preference_loss.argtypes = ([c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_vp, c_i64, c_vp, c_f, c_f, c_f, c_int,
                                          c_f] + [c_vp] * 5 + [c_i64, c_vp, ctypes.c_size_t, c_vp])
    lib.star_preference_loss.restype = c_int
    lib.star_token_alternatives.argtypes = [c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_f, c_int, c_vp, c_vp, c_i64, c_vp, c_vp, c_vp,
                                            c_vp]
    lib.star_token_alternatives.restype = c_int
    lib.star_token_alternatives_backward.argtypes = ([c_vp, c_i64, c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_f] + [c_vp] * 4
                                                     + [c_int, c_vp, c_i64, c_vp, c_i64, c_vp])
    lib.star_token_alternatives_backward.restype = c_int
    lib.star_distillation_loss.argtypes = ([c_vp, c_int, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_i64, c_int, c_int, c_f, c_vp, c_vp,
                                            c_f, c_f, c_f, c_vp, c_vp, c_vp, c_i64, c_vp, ctypes.c_size_t, c_vp])
    lib.star_distillation_loss.restype = c_int
    lib.star_rms_norm.argtypes = ([c_vp, c_i64] * 4 + [c_int, c_i64, c_i64, c_vp, c_int, c_f] + [c_vp] * 4)
    lib.star_rms_norm.restype = c_int
    lib.star_rms_norm_workspace_bytes.argtypes = [c_i64, c_i64, c_vp]
    lib.star_rms_norm_workspace_bytes.restype = c_int
    lib.star_rms_norm_backward.argtypes = [c_vp, c_i64, c_vp, c_int, c_int, c_vp, c_i64, c_vp, c_i64, c_vp, c_vp, c_vp, c_i64, c_int,
                                           c_i64, c_i64, c_vp, c_int, c_vp, c_vp, ctypes.c_size_t, c_vp]
    lib.star_rms_norm_backward.restype = c_int
    lib.star_checkpoint_sizes.argtypes = [c_i64, c_i64, c_vp, c_vp, c_vp]
    lib.star_checkpoint_sizes.restype = c_int
    lib.star_checkpoint_pack.argtypes = [c_vp, c_vp, c_vp, c_int, c_i64, c_i64, c_i64, c_int, c_vp, c_i64, c_vp]
    lib.star_checkpoint_pack.restype = c_int
    lib.star_checkpoint_unpack.argtypes = [c_vp, c_int, c_i64, c_vp, c_vp, c_i64, c_i64, c_int, c_vp]
    lib.star_checkpoint_unpack.restype = c_int
    lib.star_checkpoint_act_backward.argtypes = [c_vp, c_i64, c_vp, c_i64, c_int, c_vp, c_vp, c_i64, c_i64, c_int, c_vp]
    lib.star_checkpoint_act_backward.restype = c_int
    lib.star_checkpoint_weight_grad.argtypes = [c_vp, c_int, c_i64, c_int, c_vp, c_int, c_i64, c_vp, c_vp, c_i64, c_i64,
                                                c_i64, c_int, c_vp]
    lib.star_checkpoint_weight_grad.restype = c_int
    for name in ("star_schedule_validate", "star_schedule_static_x", "star_schedule_from_labels",
                 "star_schedule_dynamic_x", "star_group_update", "star_multi_workspace_bytes",
                 "star_multi_prepare", "star_group_update_multi"):
        getattr(lib, name).restype = c_int
    return lib


_lib = _load()


def _check(status: int, where: str) -> None:
    if status != STAR_OK:
        raise StarError(status, where)


def _i32(values: Sequence[int]):
    return (ctypes.c_int32 * max(len(values), 1))(*values)


def star_status_string(status: int) -> str:
    return _lib.star_status_string(status).decode()


def star_last_cuda_error() -> int:
    return _lib.star_last_cuda_error()


def star_launch_count() -> int:
    return _lib.star_launch_count()


# ---------------------------------------------------------------------------
# schedule encoding (host only)
# ---------------------------------------------------------------------------
Schedule = Tuple[List[int], List[int]]


def _unpack(offsets, members, n_groups) -> Schedule:
    K = n_groups.value
    off = list(offsets[: K + 1])
    return off, list(members[: off[K]])


def star_schedule_validate(group_offsets: Sequence[int], group_members: Sequence[int],
                           n_groups: int, W: int) -> int:
    """Returns the status code (does not raise)."""
    return _lib.star_schedule_validate(_i32(group_offsets), _i32(group_members), n_groups, W)


def star_schedule_static_x(arrival_order: Optional[Sequence[int]], W: int, x: int,
                           sort_members: bool = False) -> Schedule:
    offsets, members, K = _i32([0] * (W + 1)), _i32([0] * W), ctypes.c_int(0)
    if arrival_order is None:
        order, n_arrived = None, W
    else:
        if len(arrival_order) > W:
            raise StarError(STAR_ERR_INVALID_ARG, "star_schedule_static_x")
        order, n_arrived = _i32(arrival_order), len(arrival_order)
    _check(_lib.star_schedule_static_x(order, n_arrived, W, x, int(sort_members), offsets, members,
                                       ctypes.byref(K)), "star_schedule_static_x")
    return _unpack(offsets, members, K)


def star_schedule_from_labels(group_of_worker: Sequence[int]) -> Schedule:
    W = len(group_of_worker)
    offsets, members, K = _i32([0] * (W + 1)), _i32([0] * W), ctypes.c_int(0)
    _check(_lib.star_schedule_from_labels(_i32(group_of_worker), W, offsets, members,
                                          ctypes.byref(K)), "star_schedule_from_labels")
    return _unpack(offsets, members, K)


def star_schedule_dynamic_x(iter_time: Sequence[float], cluster_of_worker: Sequence[int]) -> Schedule:
    W = len(cluster_of_worker)
    if len(iter_time) != W:
        raise StarError(STAR_ERR_INVALID_ARG, "star_schedule_dynamic_x")
    offsets, members, K = _i32([0] * (W + 1)), _i32([0] * W), ctypes.c_int(0)
    times = (ctypes.c_double * max(W, 1))(*iter_time)
    _check(_lib.star_schedule_dynamic_x(times, _i32(cluster_of_worker), W, offsets, members,
                                        ctypes.byref(K)), "star_schedule_dynamic_x")
    return _unpack(offsets, members, K)


def _f64(values: Sequence[float]):
    return (ctypes.c_double * max(len(values), 1))(*values)


def star_cluster_iteration_times(iter_time: Sequence[float], n_clusters: int = 0,
                                 max_distance: float = -1.0) -> List[int]:
    """Cluster label per worker (average-linkage agglomerative clustering)."""
    W = len(iter_time)
    labels, K = _i32([0] * W), ctypes.c_int(0)
    _check(_lib.star_cluster_iteration_times(_f64(iter_time), W, n_clusters, max_distance, labels,
                                             ctypes.byref(K)), "star_cluster_iteration_times")
    return list(labels[:W])


def star_mode_times(iter_time: Sequence[float], cluster_of_worker: Optional[Sequence[int]], phi: float,
                    M: float) -> Tuple[List[float], Optional[float]]:
    """(T_x for x = 1..W by Eq. 1, T_d by Eq. 2 or None without clusters)."""
    W = len(iter_time)
    T_static, T_dynamic = _f64([0.0] * W), ctypes.c_double(0.0)
    clusters = None if cluster_of_worker is None else _i32(cluster_of_worker)
    _check(_lib.star_mode_times(_f64(iter_time), clusters, W, phi, M, T_static, ctypes.byref(T_dynamic)),
           "star_mode_times")
    return list(T_static[:W]), (None if clusters is None else T_dynamic.value)


def star_choose_mode(iter_time: Sequence[float], cluster_of_worker: Optional[Sequence[int]], phi: float,
                     M: float) -> Tuple[int, float, Schedule]:
    """(x, T, schedule): x = 0 means the dynamic mode."""
    W = len(iter_time)
    x, T, K = ctypes.c_int(0), ctypes.c_double(0.0), ctypes.c_int(0)
    offsets, members = _i32([0] * (W + 1)), _i32([0] * W)
    clusters = None if cluster_of_worker is None else _i32(cluster_of_worker)
    _check(_lib.star_choose_mode(_f64(iter_time), clusters, W, phi, M, ctypes.byref(x), ctypes.byref(T),
                                 offsets, members, ctypes.byref(K)), "star_choose_mode")
    return x.value, T.value, _unpack(offsets, members, K)


def star_choose_all_reduce_mode(iter_time: Sequence[float], child_time: Sequence[float], phi: float,
                                M: float, t_w_max: float, straggler_threshold: float = 0.2):
    """(x, t_w, T_a, removed workers, schedule of the one contributing group)."""
    W = len(iter_time)
    if len(child_time) != W:
        raise StarError(STAR_ERR_INVALID_ARG, "star_choose_all_reduce_mode")
    x, t_w, T, K = ctypes.c_int(0), ctypes.c_double(0.0), ctypes.c_double(0.0), ctypes.c_int(0)
    removed, offsets, members = _i32([0] * W), _i32([0] * (W + 1)), _i32([0] * W)
    _check(_lib.star_choose_all_reduce_mode(_f64(iter_time), _f64(child_time), W, phi, M, t_w_max,
                                            straggler_threshold, ctypes.byref(x), ctypes.byref(t_w),
                                            ctypes.byref(T), removed, offsets, members, ctypes.byref(K)),
           "star_choose_all_reduce_mode")
    return x.value, t_w.value, T.value, list(removed[: x.value]), _unpack(offsets, members, K)


def star_assign_parents(removed: Sequence[int], W: int) -> List[int]:
    """Parent of every worker (-1 for ring members) when ``removed`` leave the ring."""
    out = _i32([0] * W)
    _check(_lib.star_assign_parents(_i32(removed), len(removed), W, out), "star_assign_parents")
    return list(out[:W])


def star_build_tree(latency: Sequence[float], fanout: int) -> List[int]:
    """Parent of every worker (-1 = child of the root) in the latency-ordered tree."""
    W = len(latency)
    out = _i32([0] * W)
    _check(_lib.star_build_tree(_f64(latency), W, fanout, out), "star_build_tree")
    return list(out[:W])


def star_shard_range(n: int, world: int, rank: int, align: int = 16) -> Tuple[int, int]:
    """(first, count) of the element range rank ``rank`` of ``world`` owns."""
    first, count = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(_lib.star_shard_range(n, world, rank, align, ctypes.byref(first), ctypes.byref(count)),
           "star_shard_range")
    return first.value, count.value


def encode(decision: ModeDecision) -> Schedule:
    """Dispatch a mode decision to the matching C encoder."""
    if decision.kind == "labels":
        return star_schedule_from_labels(decision.labels)
    if decision.kind == "static_x":
        return star_schedule_static_x(decision.arrival_order, decision.W, decision.x,
                                      decision.sort_members)
    if decision.kind == "dynamic_x":
        return star_schedule_dynamic_x(decision.iter_time, decision.labels)
    raise ValueError(decision.kind)


# ---------------------------------------------------------------------------
# fused grouped update
# ---------------------------------------------------------------------------
def _grad_dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return STAR_DTYPE_F32
    if t.dtype == torch.bfloat16:
        return STAR_DTYPE_BF16
    raise TypeError("gradients must be float32 or bfloat16, got %s" % t.dtype)


def _state(t: torch.Tensor, what: str) -> int:
    if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous():
        raise TypeError("%s must be a contiguous float32 CUDA tensor" % what)
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)        # absent in a torch without CUDA
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:                                  # the current stream's handle, without a Stream object around it
        return _raw_stream(_current_device())
    return stream.cuda_stream


def star_group_update(params: torch.Tensor, momentum: torch.Tensor,
                      grads: Sequence[Optional[torch.Tensor]], group_offsets: Sequence[int],
                      group_members: Sequence[int], lr: float, mu: float, wd: float,
                      stream=None) -> None:
    """In-place fused grouped update of one flat tensor on the current device."""
    n = params.numel()
    p, v = _state(params, "params"), _state(momentum, "momentum")
    if momentum.numel() != n:
        raise ValueError("params and momentum differ in size")
    W = len(grads)
    ptrs = (ctypes.c_void_p * max(W, 1))()
    dt = None
    for w, g in enumerate(grads):
        if g is None:
            continue
        if not g.is_cuda or not g.is_contiguous() or g.numel() != n:
            raise ValueError("gradient %d must be a contiguous CUDA tensor of %d elements" % (w, n))
        d = _grad_dtype(g)
        if dt is not None and d != dt:
            raise TypeError("gradients differ in dtype")
        dt = d
        ptrs[w] = g.data_ptr()
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    _check(_lib.star_group_update(p, v, ptrs, W, STAR_DTYPE_F32 if dt is None else dt, n,
                                  _i32(group_offsets), _i32(group_members), K, lr, mu, wd,
                                  _stream(stream)), "star_group_update")


class FlatRoundBuffers:
    """The buffers of a flat round marshalled once: for callers that run many
    rounds on the same tensors (only the schedule and the scalars change per
    round), which saves building the pointer array and re-checking the tensors
    on every call -- on launch-bound sizes that is most of the host time.  Holds
    references to the tensors; computes nothing."""

    def __init__(self, params: torch.Tensor, momentum: torch.Tensor, grads: Sequence[Optional[torch.Tensor]]):
        self.n = params.numel()
        self.p, self.v = _state(params, "params"), _state(momentum, "momentum")
        if momentum.numel() != self.n:
            raise ValueError("params and momentum differ in size")
        self.W = len(grads)
        self.ptrs, self.dtype = _grad_pointers(grads, self.n)
        self._keep = (params, momentum, list(grads))

    def star_group_update(self, group_offsets: Sequence[int], group_members: Sequence[int], lr: float, mu: float,
                          wd: float, stream=None) -> None:
        K = len(group_offsets) - 1 if len(group_offsets) else 0
        _check(_lib.star_group_update(self.p, self.v, self.ptrs, self.W, self.dtype, self.n, _i32(group_offsets),
                                      _i32(group_members), K, lr, mu, wd, _stream(stream)), "star_group_update")


def star_group_update_ex(params: torch.Tensor, momentum: torch.Tensor,
                         grads: Sequence[Optional[torch.Tensor]], group_offsets: Sequence[int],
                         group_members: Sequence[int], lrs: Sequence[float], mu: float, wd: float,
                         snapshots: Optional[Sequence[Optional[torch.Tensor]]] = None,
                         sum_order: int = STAR_SUM_LINEAR, stream=None) -> None:
    """The round with one learning rate per group; ``snapshots[k]`` (CUDA tensor,
    all float32 or all bfloat16, or None) receives the parameters right after
    group k's update; ``sum_order`` is STAR_SUM_LINEAR or STAR_SUM_TREE."""
    n = params.numel()
    p, v = _state(params, "params"), _state(momentum, "momentum")
    if momentum.numel() != n:
        raise ValueError("params and momentum differ in size")
    W = len(grads)
    ptrs = (ctypes.c_void_p * max(W, 1))()
    dt = None
    for w, g in enumerate(grads):
        if g is None:
            continue
        if not g.is_cuda or not g.is_contiguous() or g.numel() != n:
            raise ValueError("gradient %d must be a contiguous CUDA tensor of %d elements" % (w, n))
        d = _grad_dtype(g)
        if dt is not None and d != dt:
            raise TypeError("gradients differ in dtype")
        dt = d
        ptrs[w] = g.data_ptr()
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    if len(lrs) != K:
        raise ValueError("need one learning rate per group")
    lr_arr = (ctypes.c_float * max(K, 1))(*lrs)
    snap_arr, snap_dt = None, STAR_DTYPE_F32
    if snapshots is not None:
        if len(snapshots) != K:
            raise ValueError("snapshots needs one entry (tensor or None) per group")
        snap_arr = (ctypes.c_void_p * max(K, 1))()
        kinds = set()
        for k, s in enumerate(snapshots):
            if s is None:
                continue
            if s.numel() != n or not s.is_cuda or not s.is_contiguous():
                raise ValueError("snapshot %d must be a contiguous CUDA tensor of %d elements" % (k, n))
            kinds.add(_grad_dtype(s))
            snap_arr[k] = s.data_ptr()
        if len(kinds) > 1:
            raise TypeError("snapshots differ in dtype")
        snap_dt = kinds.pop() if kinds else STAR_DTYPE_F32
    _check(_lib.star_group_update_ex(p, v, ptrs, W, STAR_DTYPE_F32 if dt is None else dt, n,
                                     _i32(group_offsets), _i32(group_members), K, lr_arr, mu, wd,
                                     snap_arr, snap_dt, sum_order, _stream(stream)), "star_group_update_ex")


def _grad_pointers(grads: Sequence[Optional[torch.Tensor]], n: int):
    """(ctypes array of W device pointers, dtype code) of a list of flat gradient tensors."""
    W = len(grads)
    ptrs = (ctypes.c_void_p * max(W, 1))()
    dt = None
    for w, g in enumerate(grads):
        if g is None:
            continue
        if not g.is_cuda or not g.is_contiguous() or g.numel() != n:
            raise ValueError("gradient %d must be a contiguous CUDA tensor of %d elements" % (w, n))
        d = _grad_dtype(g)
        if dt is not None and d != dt:
            raise TypeError("gradients differ in dtype")
        dt = d
        ptrs[w] = g.data_ptr()
    return ptrs, STAR_DTYPE_F32 if dt is None else dt


def star_group_reduce(out: torch.Tensor, grads: Sequence[Optional[torch.Tensor]], members: Sequence[int],
                      sum_order: int = STAR_SUM_LINEAR, stream=None) -> None:
    """``out[i] = grads[members[0]][i] + grads[members[1]][i] + ...`` (what a parent
    of the all-reduce architecture forwards to the ring); ``out`` is a float32
    or bfloat16 CUDA tensor."""
    n = out.numel()
    if not out.is_cuda or not out.is_contiguous():
        raise TypeError("out must be a contiguous CUDA tensor")
    ptrs, dt = _grad_pointers(grads, n)
    _check(_lib.star_group_reduce(out.data_ptr(), _grad_dtype(out), ptrs, len(grads), dt, n, _i32(members),
                                  len(members), sum_order, _stream(stream)), "star_group_reduce")


def star_group_update_from_sums(params: torch.Tensor, momentum: torch.Tensor, sums: Sequence[torch.Tensor],
                                n_reports: int, lr: float, mu: float, wd: float, stream=None) -> None:
    """One update from the ring members' aggregates ``sums`` (float32 CUDA tensors,
    added in the listed order), the mean taken over ``n_reports`` gradient reports."""
    n = params.numel()
    p, v = _state(params, "params"), _state(momentum, "momentum")
    if momentum.numel() != n:
        raise ValueError("params and momentum differ in size")
    for r, t in enumerate(sums):
        if t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
            raise ValueError("sum %d must be a contiguous float32 CUDA tensor of %d elements" % (r, n))
    ptrs = (ctypes.c_void_p * max(len(sums), 1))(*[t.data_ptr() for t in sums])
    _check(_lib.star_group_update_from_sums(p, v, ptrs, len(sums), n, n_reports, lr, mu, wd, _stream(stream)),
           "star_group_update_from_sums")


def star_multi_workspace_bytes(sizes: Sequence[int], W: int) -> int:
    out = ctypes.c_size_t(0)
    arr = (ctypes.c_int64 * max(len(sizes), 1))(*sizes)
    _check(_lib.star_multi_workspace_bytes(len(sizes), arr, W, ctypes.byref(out)),
           "star_multi_workspace_bytes")
    return out.value


def star_multi_prepare(params: Sequence[torch.Tensor], momentum: Sequence[torch.Tensor],
                       grads: Sequence[Sequence[Optional[torch.Tensor]]], workspace: torch.Tensor,
                       stream=None) -> star_multi_plan_t:
    """``grads[w][t]`` = worker w's gradient for tensor t.  ``workspace`` is a
    uint8 CUDA tensor of at least :func:`star_multi_workspace_bytes` bytes; the
    returned plan refers to it (keep the tensor alive)."""
    T, W = len(params), len(grads)
    if len(momentum) != T or any(len(g) != T for g in grads):
        raise ValueError("params, momentum and every worker's gradient list need one entry per tensor")
    sizes = [p.numel() for p in params]
    P = (ctypes.c_void_p * max(T, 1))(*[_state(p, "params") if p.numel() else None for p in params])
    V = (ctypes.c_void_p * max(T, 1))(*[_state(v, "momentum") if v.numel() else None for v in momentum])
    G = (ctypes.c_void_p * max(T * W, 1))()
    dt = None
    for w in range(W):
        for t in range(T):
            g = grads[w][t]
            if g is None:
                continue
            if not g.is_cuda or not g.is_contiguous() or g.numel() != sizes[t]:
                raise ValueError("gradient [%d][%d] must be a contiguous CUDA tensor of %d elements"
                                 % (w, t, sizes[t]))
            d = _grad_dtype(g)
            if dt is not None and d != dt:
                raise TypeError("gradients differ in dtype")
            dt = d
            G[t * W + w] = g.data_ptr() if sizes[t] else None
    if momentum and any(v.numel() != s for v, s in zip(momentum, sizes)):
        raise ValueError("params and momentum differ in size")
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 CUDA tensor")
    plan = star_multi_plan_t()
    S = (ctypes.c_int64 * max(T, 1))(*sizes)
    _check(_lib.star_multi_prepare(T, P, V, G, S, W, STAR_DTYPE_F32 if dt is None else dt,
                                   workspace.data_ptr(), workspace.numel(), _stream(stream),
                                   ctypes.byref(plan)), "star_multi_prepare")
    return plan


def star_group_update_multi(plan: star_multi_plan_t, group_offsets: Sequence[int],
                            group_members: Sequence[int], lr: float, mu: float, wd: float,
                            stream=None) -> None:
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    _check(_lib.star_group_update_multi(ctypes.byref(plan), _i32(group_offsets), _i32(group_members),
                                        K, lr, mu, wd, _stream(stream)), "star_group_update_multi")


def star_group_update_multi_lrs(plan: star_multi_plan_t, group_offsets: Sequence[int],
                                group_members: Sequence[int], lrs: Sequence[float], mu: float, wd: float,
                                stream=None) -> None:
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    if len(lrs) != K:
        raise ValueError("need one learning rate per group")
    _check(_lib.star_group_update_multi_lrs(ctypes.byref(plan), _i32(group_offsets), _i32(group_members), K,
                                            (ctypes.c_float * max(K, 1))(*lrs), mu, wd, _stream(stream)),
           "star_group_update_multi_lrs")


def star_multi_workspace_bytes_ex(sizes: Sequence[int], W: int, n_snapshot_sets: int) -> int:
    out = ctypes.c_size_t(0)
    arr = (ctypes.c_int64 * max(len(sizes), 1))(*sizes)
    _check(_lib.star_multi_workspace_bytes_ex(len(sizes), arr, W, n_snapshot_sets, ctypes.byref(out)),
           "star_multi_workspace_bytes_ex")
    return out.value


def _list_pointers(params, momentum, grads):
    """Pointer arrays (P, V, G, sizes array, dtype code) of a tensor list;
    ``grads[w][t]`` = worker w's gradient for tensor t."""
    T, W = len(params), len(grads)
    if len(momentum) != T or any(len(g) != T for g in grads):
        raise ValueError("params, momentum and every worker's gradient list need one entry per tensor")
    sizes = [p.numel() for p in params]
    if any(v.numel() != s for v, s in zip(momentum, sizes)):
        raise ValueError("params and momentum differ in size")
    P = (ctypes.c_void_p * max(T, 1))(*[_state(p, "params") if p.numel() else None for p in params])
    V = (ctypes.c_void_p * max(T, 1))(*[_state(v, "momentum") if v.numel() else None for v in momentum])
    G = (ctypes.c_void_p * max(T * W, 1))()
    dt = None
    for w in range(W):
        for t in range(T):
            g = grads[w][t]
            if g is None or sizes[t] == 0:
                continue
            if not g.is_cuda or not g.is_contiguous() or g.numel() != sizes[t]:
                raise ValueError("gradient [%d][%d] must be a contiguous CUDA tensor of %d elements"
                                 % (w, t, sizes[t]))
            d = _grad_dtype(g)
            if dt is not None and d != dt:
                raise TypeError("gradients differ in dtype")
            dt = d
            G[t * W + w] = g.data_ptr()
    S = (ctypes.c_int64 * max(T, 1))(*sizes)
    return P, V, G, S, sizes, STAR_DTYPE_F32 if dt is None else dt


def star_multi_prepare_ex(params: Sequence[torch.Tensor], momentum: Sequence[torch.Tensor],
                          grads: Sequence[Sequence[Optional[torch.Tensor]]],
                          snapshot_sets: Sequence[Sequence[Optional[torch.Tensor]]], workspace: torch.Tensor,
                          stream=None) -> star_multi_plan_t:
    """As :func:`star_multi_prepare`, registering ``snapshot_sets[s][t]`` (tensor
    t's buffer of snapshot set s, all float32 or all bfloat16, or None)."""
    T, W, S_sets = len(params), len(grads), len(snapshot_sets)
    P, V, G, S, sizes, dt = _list_pointers(params, momentum, grads)
    if any(len(one) != T for one in snapshot_sets):
        raise ValueError("every snapshot set needs one entry (tensor or None) per tensor")
    snaps = (ctypes.c_void_p * max(T * S_sets, 1))()
    kinds = set()
    for s_index, one in enumerate(snapshot_sets):
        for t, buf in enumerate(one):
            if buf is None or sizes[t] == 0:
                continue
            if not buf.is_cuda or not buf.is_contiguous() or buf.numel() != sizes[t]:
                raise ValueError("snapshot [%d][%d] must be a contiguous CUDA tensor of %d elements"
                                 % (s_index, t, sizes[t]))
            kinds.add(_grad_dtype(buf))
            snaps[t * S_sets + s_index] = buf.data_ptr()
    if len(kinds) > 1:
        raise TypeError("snapshots differ in dtype")
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 CUDA tensor")
    plan = star_multi_plan_t()
    _check(_lib.star_multi_prepare_ex(T, P, V, G, S, W, dt, S_sets, snaps, kinds.pop() if kinds else STAR_DTYPE_F32,
                                      workspace.data_ptr(), workspace.numel(), _stream(stream),
                                      ctypes.byref(plan)), "star_multi_prepare_ex")
    return plan


def star_group_update_multi_ex(plan: star_multi_plan_t, group_offsets: Sequence[int],
                               group_members: Sequence[int], lrs: Sequence[float], mu: float, wd: float,
                               snapshot_set_of_group: Optional[Sequence[int]] = None,
                               sum_order: int = STAR_SUM_LINEAR, stream=None) -> None:
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    if len(lrs) != K or (snapshot_set_of_group is not None and len(snapshot_set_of_group) != K):
        raise ValueError("need one learning rate (and one snapshot set index) per group")
    sets = None if snapshot_set_of_group is None else _i32(snapshot_set_of_group)
    _check(_lib.star_group_update_multi_ex(ctypes.byref(plan), _i32(group_offsets), _i32(group_members), K,
                                           (ctypes.c_float * max(K, 1))(*lrs), mu, wd, sets, sum_order,
                                           _stream(stream)), "star_group_update_multi_ex")


def star_host_workspace_bytes(max_scheduled: int, grad_dtype: torch.dtype, chunk_elements: int) -> int:
    out = ctypes.c_size_t(0)
    dt = STAR_DTYPE_BF16 if grad_dtype == torch.bfloat16 else STAR_DTYPE_F32
    _check(_lib.star_host_workspace_bytes(max_scheduled, dt, chunk_elements, ctypes.byref(out)),
           "star_host_workspace_bytes")
    return out.value


def star_group_update_host(params: torch.Tensor, momentum: torch.Tensor,
                           grads: Sequence[Optional[torch.Tensor]], group_offsets: Sequence[int],
                           group_members: Sequence[int], lr: float, mu: float, wd: float,
                           workspace: torch.Tensor, stream=None) -> None:
    """Fused grouped update of HOST tensors (ideally pinned), streamed through the
    device workspace in chunks.  Results are in ``params`` / ``momentum`` once the
    stream has been synchronized."""
    n = params.numel()
    for t, what in ((params, "params"), (momentum, "momentum")):
        if t.dtype != torch.float32 or t.is_cuda or not t.is_contiguous():
            raise TypeError("%s must be a contiguous float32 host tensor" % what)
    if momentum.numel() != n:
        raise ValueError("params and momentum differ in size")
    W = len(grads)
    ptrs = (ctypes.c_void_p * max(W, 1))()
    dt = None
    for w, g in enumerate(grads):
        if g is None:
            continue
        if g.is_cuda or not g.is_contiguous() or g.numel() != n:
            raise ValueError("gradient %d must be a contiguous host tensor of %d elements" % (w, n))
        d = _grad_dtype(g)
        if dt is not None and d != dt:
            raise TypeError("gradients differ in dtype")
        dt = d
        ptrs[w] = g.data_ptr()
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 CUDA tensor")
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    _check(_lib.star_group_update_host(params.data_ptr(), momentum.data_ptr(), ptrs, W,
                                       STAR_DTYPE_F32 if dt is None else dt, n, _i32(group_offsets),
                                       _i32(group_members), K, lr, mu, wd, workspace.data_ptr(),
                                       workspace.numel(), _stream(stream)), "star_group_update_host")


def star_host_workspace_bytes_ex(max_scheduled: int, grad_dtype: torch.dtype, max_snapshots: int,
                                 snapshot_dtype: torch.dtype, chunk_elements: int) -> int:
    out = ctypes.c_size_t(0)
    code = lambda dt: STAR_DTYPE_BF16 if dt == torch.bfloat16 else STAR_DTYPE_F32       # noqa: E731
    _check(_lib.star_host_workspace_bytes_ex(max_scheduled, code(grad_dtype), max_snapshots, code(snapshot_dtype),
                                             chunk_elements, ctypes.byref(out)), "star_host_workspace_bytes_ex")
    return out.value


def star_group_update_host_ex(params: torch.Tensor, momentum: torch.Tensor,
                              grads: Sequence[Optional[torch.Tensor]], group_offsets: Sequence[int],
                              group_members: Sequence[int], lrs: Sequence[float], mu: float, wd: float,
                              workspace: torch.Tensor, snapshots: Optional[Sequence[Optional[torch.Tensor]]] = None,
                              sum_order: int = STAR_SUM_LINEAR, stream=None) -> None:
    """The host-buffer round with per-group rates, host snapshot tensors
    (``snapshots[k]``: float32 or bfloat16 host tensor or None) and the summation order."""
    n = params.numel()
    for t, what in ((params, "params"), (momentum, "momentum")):
        if t.dtype != torch.float32 or t.is_cuda or not t.is_contiguous():
            raise TypeError("%s must be a contiguous float32 host tensor" % what)
    if momentum.numel() != n:
        raise ValueError("params and momentum differ in size")
    W = len(grads)
    ptrs = (ctypes.c_void_p * max(W, 1))()
    dt = None
    for w, g in enumerate(grads):
        if g is None:
            continue
        if g.is_cuda or not g.is_contiguous() or g.numel() != n:
            raise ValueError("gradient %d must be a contiguous host tensor of %d elements" % (w, n))
        d = _grad_dtype(g)
        if dt is not None and d != dt:
            raise TypeError("gradients differ in dtype")
        dt = d
        ptrs[w] = g.data_ptr()
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    if len(lrs) != K:
        raise ValueError("need one learning rate per group")
    snap_arr, snap_dt = None, STAR_DTYPE_F32
    if snapshots is not None:
        if len(snapshots) != K:
            raise ValueError("snapshots needs one entry (tensor or None) per group")
        snap_arr = (ctypes.c_void_p * max(K, 1))()
        kinds = set()
        for k, s in enumerate(snapshots):
            if s is None:
                continue
            if s.is_cuda or not s.is_contiguous() or s.numel() != n:
                raise ValueError("snapshot %d must be a contiguous host tensor of %d elements" % (k, n))
            kinds.add(_grad_dtype(s))
            snap_arr[k] = s.data_ptr()
        if len(kinds) > 1:
            raise TypeError("snapshots differ in dtype")
        snap_dt = kinds.pop() if kinds else STAR_DTYPE_F32
    if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
        raise TypeError("workspace must be a contiguous uint8 CUDA tensor")
    _check(_lib.star_group_update_host_ex(params.data_ptr(), momentum.data_ptr(), ptrs, W,
                                          STAR_DTYPE_F32 if dt is None else dt, n, _i32(group_offsets),
                                          _i32(group_members), K, (ctypes.c_float * max(K, 1))(*lrs), mu, wd,
                                          snap_arr, snap_dt, sum_order, workspace.data_ptr(), workspace.numel(),
                                          _stream(stream)), "star_group_update_host_ex")


STAR_STATIC_SCRATCH_BYTES = 1 << 20


def star_group_update_multi_noalloc(params: Sequence[torch.Tensor], momentum: Sequence[torch.Tensor],
                                    grads: Sequence[Sequence[Optional[torch.Tensor]]],
                                    group_offsets: Sequence[int], group_members: Sequence[int],
                                    lr: float, mu: float, wd: float, stream=None) -> None:
    """One round over a tensor list for callers that have no way to obtain a
    device workspace (``grads[w][t]`` = worker w's gradient for tensor t).

    The pointer table goes into a fixed array inside the library
    (``STAR_STATIC_SCRATCH_BYTES``) that every call on the device shares; lists
    whose table is larger are rejected with ``STAR_ERR_WORKSPACE_TOO_SMALL``.
    Results equal :func:`star_multi_prepare` + :func:`star_group_update_multi`.
    The caller must serialize calls that could overlap on the GPU, and should
    make the first call on each device outside stream capture."""
    T, W = len(params), len(grads)
    if len(momentum) != T or any(len(g) != T for g in grads):
        raise ValueError("params, momentum and every worker's gradient list need one entry per tensor")
    sizes = [p.numel() for p in params]
    if any(v.numel() != s for v, s in zip(momentum, sizes)):
        raise ValueError("params and momentum differ in size")
    P = (ctypes.c_void_p * max(T, 1))(*[_state(p, "params") if p.numel() else None for p in params])
    V = (ctypes.c_void_p * max(T, 1))(*[_state(v, "momentum") if v.numel() else None for v in momentum])
    G = (ctypes.c_void_p * max(T * W, 1))()
    dt = None
    for w in range(W):
        for t in range(T):
            g = grads[w][t]
            if g is None or sizes[t] == 0:
                continue
            if not g.is_cuda or not g.is_contiguous() or g.numel() != sizes[t]:
                raise ValueError("gradient [%d][%d] must be a contiguous CUDA tensor of %d elements"
                                 % (w, t, sizes[t]))
            d = _grad_dtype(g)
            if dt is not None and d != dt:
                raise TypeError("gradients differ in dtype")
            dt = d
            G[t * W + w] = g.data_ptr()
    S = (ctypes.c_int64 * max(T, 1))(*sizes)
    K = len(group_offsets) - 1 if len(group_offsets) else 0
    _check(_lib.star_group_update_multi_noalloc(T, P, V, G, S, W, STAR_DTYPE_F32 if dt is None else dt,
                                                _i32(group_offsets), _i32(group_members), K, lr, mu, wd,
                                                _stream(stream)), "star_group_update_multi_noalloc")


# ---------------------------------------------------------------------------
# a worker's step: losses over the vocabulary, activations kept in 8 bits
# ---------------------------------------------------------------------------
STAR_ACT_NONE = 0
STAR_ACT_GELU_TANH = 1
STAR_ACT_GELU_ERF = 2
STAR_ACT_SILU = 3
_ACTS = {"none": STAR_ACT_NONE, "gelu_tanh": STAR_ACT_GELU_TANH, "gelu_erf": STAR_ACT_GELU_ERF, "silu": STAR_ACT_SILU}
_DTYPES = {torch.float32: STAR_DTYPE_F32, torch.bfloat16: STAR_DTYPE_BF16}


def _matrix(t: torch.Tensor, what: str, shape=None, dtype=None) -> Tuple[int, int, int]:
    """(address, dtype code, row stride) of a CUDA matrix whose rows are contiguous."""
    kind, own = t.dtype, t.shape
    code = _DTYPES.get(kind)
    if code is None or len(own) != 2 or not t.is_cuda or (dtype is not None and kind is not dtype):
        raise TypeError("%s must be a 2-D %s CUDA tensor" % (what, "float32 or bfloat16" if dtype is None else dtype))
    rows, cols = own
    if shape is not None and (rows, cols) != shape:
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(own), shape))
    ld, step = t.stride()
    if step == 1 and ld >= cols:
        return t.data_ptr(), code, ld
    if (step != 1 and cols > 1) or (ld < cols and rows > 1):
        raise TypeError("%s must have contiguous rows that do not overlap" % what)
    return t.data_ptr(), code, max(ld, cols)


def _vector(t: Optional[torch.Tensor], n: int, what: str, dtype=torch.float32) -> Optional[int]:
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s CUDA tensor" % (what, dtype))
    if t.numel() != n:
        raise ValueError("%s has %d elements, expected %d" % (what, t.numel(), n))
    return t.data_ptr()


def _act(act) -> int:
    if act not in _ACTS:
        raise ValueError("unknown activation %r (one of %s)" % (act, ", ".join(_ACTS)))
    return _ACTS[act]


def star_token_logprobs(logits: torch.Tensor, labels: torch.Tensor, logp: torch.Tensor,
                        lse: Optional[torch.Tensor] = None, temperature: float = 1.0, stream=None) -> None:
    """logp (and lse) of every row's label; labels outside [0, vocab) give 0."""
    rows, vocab = logits.shape
    x, dtype, ld = _matrix(logits, "logits")
    _check(_lib.star_token_logprobs(x, dtype, rows, vocab, ld, _vector(labels, rows, "labels", torch.int64),
                                    temperature, _vector(logp, rows, "logp"), _vector(lse, rows, "lse"),
                                    _stream(stream)), "star_token_logprobs")


def star_loss_workspace_bytes(rows: int, sequences: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.star_loss_workspace_bytes(rows, sequences, ctypes.byref(out)), "star_loss_workspace_bytes")
    return out.value


def _workspace(t: torch.Tensor) -> Tuple[int, int]:
    if not t.is_cuda or not t.is_contiguous():
        raise TypeError("workspace must be a contiguous CUDA tensor")
    return t.data_ptr(), t.numel() * t.element_size()


def star_policy_loss(logits: torch.Tensor, labels: torch.Tensor, advantages: torch.Tensor, logp: torch.Tensor,
                     token_loss: torch.Tensor, sums: torch.Tensor, workspace: torch.Tensor,
                     dlogits: Optional[torch.Tensor] = None, weights: Optional[torch.Tensor] = None,
                     old_logp: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                     clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0, temperature: float = 1.0,
                     stream=None) -> None:
    """Clipped policy loss with a KL term: logp, token_loss, the four sums and,
    unless None, the gradient of the logits (which may be the logits)."""
    rows, vocab = logits.shape
    x, dtype, ld = _matrix(logits, "logits")
    d, _, ld_d = (None, dtype, vocab) if dlogits is None else _matrix(dlogits, "dlogits", (rows, vocab), logits.dtype)
    ws, ws_bytes = _workspace(workspace)
    _check(_lib.star_policy_loss(x, dtype, rows, vocab, ld, _vector(labels, rows, "labels", torch.int64),
                                 _vector(weights, rows, "weights"), _vector(advantages, rows, "advantages"),
                                 _vector(old_logp, rows, "old_logp"), _vector(ref_logp, rows, "ref_logp"), temperature,
                                 clip_low, clip_high, kl_coef, _vector(logp, rows, "logp"),
                                 _vector(token_loss, rows, "token_loss"), _vector(sums, 4, "sums"), d, ld_d, ws,
                                 ws_bytes, _stream(stream)), "star_policy_loss")


def star_preference_loss(logits: torch.Tensor, labels: torch.Tensor, seq_offsets: torch.Tensor, seq_logp: torch.Tensor,
                         pair_loss: torch.Tensor, margin: torch.Tensor, loss: torch.Tensor, workspace: torch.Tensor,
                         dlogits: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                         beta: float = 0.1, label_smoothing: float = 0.0, average: bool = False,
                         loss_scale: float = 1.0, temperature: float = 1.0, stream=None) -> None:
    """Preference loss of pairs of sequences (chosen, rejected, chosen, ...):
    sequence log-probabilities, losses, margins, the total and, unless None, the
    gradient of the logits (which may be the logits)."""
    rows, vocab = logits.shape
    pairs = pair_loss.numel()
    x, dtype, ld = _matrix(logits, "logits")
    d, _, ld_d = (None, dtype, vocab) if dlogits is None else _matrix(dlogits, "dlogits", (rows, vocab), logits.dtype)
    ws, ws_bytes = _workspace(workspace)
    _check(_lib.star_preference_loss(x, dtype, rows, vocab, ld, _vector(labels, rows, "labels", torch.int64),
                                     _vector(seq_offsets, 2 * pairs + 1, "seq_offsets", torch.int32), pairs,
                                     _vector(ref_logp, 2 * pairs, "ref_logp"), temperature, beta, label_smoothing,
                                     int(average), loss_scale, _vector(seq_logp, 2 * pairs, "seq_logp"),
                                     _vector(pair_loss, pairs, "pair_loss"), _vector(margin, pairs, "margin"),
                                     _vector(loss, 1, "loss"), d, ld_d, ws, ws_bytes, _stream(stream)),
           "star_preference_loss")


STAR_MAX_ALTERNATIVES = 128


def _like(t: torch.Tensor, what: str, shape, dtype) -> Tuple[int, int]:
    """(address, row stride) of a matrix of a shape and dtype that another argument gave."""
    if t.shape == shape and t.dtype is dtype and t.is_cuda:
        ld, step = t.stride()
        if step == 1 and ld >= shape[1]:
            return t.data_ptr(), ld
    p, _, ld = _matrix(t, what, tuple(shape), dtype)
    return p, ld


def _listed(t: torch.Tensor, rows: int, k: int, what: str, dtype) -> Tuple[int, int]:
    """(address, row stride) of a rows x k matrix of a teacher's or of top entries."""
    if t.dtype is not dtype or t.dim() != 2 or not t.is_cuda:
        raise TypeError("%s must be a 2-D %s CUDA tensor" % (what, dtype))
    if t.shape != (rows, k):
        raise ValueError("%s has shape %s, expected %s" % (what, tuple(t.shape), (rows, k)))
    ld, step = t.stride()
    if (step != 1 and k > 1) or (ld < k and rows > 1):
        raise TypeError("%s must have contiguous rows that do not overlap" % what)
    return t.data_ptr(), ld if ld > k else k


def star_token_alternatives(logits: torch.Tensor, top_ids: Optional[torch.Tensor] = None,
                            top_logp: Optional[torch.Tensor] = None, labels: Optional[torch.Tensor] = None,
                            logp: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                            entropy: Optional[torch.Tensor] = None, temperature: float = 1.0, stream=None) -> None:
    """The largest logits' ids (int32, rows x k) and log-probabilities, with lse,
    entropy and the labels' logp where asked for; without labels every row takes part."""
    x, dtype, ld = _matrix(logits, "logits")
    rows, vocab = logits.shape
    k = ld_top = 0
    ids = top = None
    if top_ids is not None and top_logp is not None:
        k = top_ids.shape[-1]
        ids, ld_top = _listed(top_ids, rows, k, "top_ids", torch.int32)
        top, ld_logp = _listed(top_logp, rows, k, "top_logp", torch.float32)
        if ld_logp != ld_top and rows > 1:
            raise ValueError("top_ids and top_logp must have one row stride")
    elif top_ids is not top_logp:
        raise ValueError("top_ids and top_logp come together")
    _check(_lib.star_token_alternatives(x, dtype, rows, vocab, ld, _vector(labels, rows, "labels", torch.int64), temperature, k,
                                        ids, top, ld_top, _vector(logp, rows, "logp"), _vector(lse, rows, "lse"),
                                        _vector(entropy, rows, "entropy"), _stream(stream)), "star_token_alternatives")


def star_token_alternatives_backward(dlogits: torch.Tensor, logits: torch.Tensor, lse: torch.Tensor,
                                     labels: Optional[torch.Tensor] = None, d_logp: Optional[torch.Tensor] = None,
                                     entropy: Optional[torch.Tensor] = None, d_entropy: Optional[torch.Tensor] = None,
                                     top_ids: Optional[torch.Tensor] = None, d_top_logp: Optional[torch.Tensor] = None,
                                     temperature: float = 1.0, stream=None) -> None:
    """The gradient of the logits (which it may replace) from those of
    star_token_alternatives' results, with that call's lse and entropy."""
    x, dtype, ld = _matrix(logits, "logits")
    shape = logits.shape
    rows, vocab = shape
    d, ld_d = _like(dlogits, "dlogits", shape, logits.dtype)
    k = ld_ids = ld_top = 0
    ids = top = None
    if top_ids is not None and d_top_logp is not None:
        k = top_ids.shape[-1]
        ids, ld_ids = _listed(top_ids, rows, k, "top_ids", torch.int32)
        top, ld_top = _listed(d_top_logp, rows, k, "d_top_logp", torch.float32)
    elif top_ids is not d_top_logp:
        raise ValueError("top_ids and d_top_logp come together")
    _check(_lib.star_token_alternatives_backward(d, ld_d, x, dtype, rows, vocab, ld, _vector(labels, rows, "labels", torch.int64),
                                                 temperature, _vector(lse, rows, "lse"), _vector(entropy, rows, "entropy"),
                                                 _vector(d_logp, rows, "d_logp"), _vector(d_entropy, rows, "d_entropy"), k, ids,
                                                 ld_ids, top, ld_top, _stream(stream)), "star_token_alternatives_backward")


def star_distillation_loss(logits: torch.Tensor, teacher_ids: torch.Tensor, teacher_values: torch.Tensor,
                           token_loss: torch.Tensor, sums: torch.Tensor, workspace: torch.Tensor,
                           dlogits: Optional[torch.Tensor] = None, labels: Optional[torch.Tensor] = None,
                           weights: Optional[torch.Tensor] = None, temperature: float = 1.0, teacher_temperature: float = 1.0,
                           rest: bool = False, soft_coef: float = 1.0, label_coef: float = 0.0, stream=None) -> None:
    """Distillation from a teacher's k ids and values a row (logits, or with
    ``rest`` log-probabilities whose remainder counts too): token_loss, the four
    sums and, unless None, the gradient of the logits (which may be the logits)."""
    x, dtype, ld = _matrix(logits, "logits")
    shape = logits.shape
    rows, vocab = shape
    d, ld_d = (None, vocab) if dlogits is None else _like(dlogits, "dlogits", shape, logits.dtype)
    k = teacher_ids.shape[-1]
    ids, ld_ids = _listed(teacher_ids, rows, k, "teacher_ids", torch.int32)
    values, ld_values = _listed(teacher_values, rows, k, "teacher_values", torch.float32)
    ws, ws_bytes = _workspace(workspace)
    _check(_lib.star_distillation_loss(x, dtype, rows, vocab, ld, ids, ld_ids, values, ld_values, k, rest, teacher_temperature,
                                       _vector(labels, rows, "labels", torch.int64), _vector(weights, rows, "weights"), temperature,
                                       soft_coef, label_coef, _vector(token_loss, rows, "token_loss"), _vector(sums, 4, "sums"), d,
                                       ld_d, ws, ws_bytes, _stream(stream)), "star_distillation_loss")


def star_checkpoint_sizes(rows: int, cols: int) -> Tuple[int, int, int]:
    """(pitch, bytes of codes, bytes of scales) of a checkpoint of rows x cols values."""
    pitch, code_bytes, scale_bytes = ctypes.c_int64(0), ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(_lib.star_checkpoint_sizes(rows, cols, ctypes.byref(pitch), ctypes.byref(code_bytes), ctypes.byref(scale_bytes)),
           "star_checkpoint_sizes")
    return pitch.value, code_bytes.value, scale_bytes.value


def star_checkpoint_empty(rows: int, cols: int, device="cuda") -> Tuple[torch.Tensor, torch.Tensor]:
    """Uninitialized codes (int8, rows x pitch) and scales (uint8, tiles x tall x 4) for rows x cols values."""
    pitch, _, scale_bytes = star_checkpoint_sizes(rows, cols)
    tiles = (cols + 127) // 128
    return (torch.empty((rows, pitch), dtype=torch.int8, device=device),
            torch.empty((tiles, scale_bytes // (4 * max(tiles, 1)), 4), dtype=torch.uint8, device=device))


def _kept(codes: torch.Tensor, scales: torch.Tensor, rows: int, cols: int) -> Tuple[int, int]:
    pitch, tiles, tall = (cols + 15) // 16 * 16, (cols + 127) // 128, (rows + 63) // 64 * 64
    if codes.dtype != torch.int8 or scales.dtype != torch.uint8 or not codes.is_cuda or not scales.is_cuda \
            or not codes.is_contiguous() or not scales.is_contiguous():
        raise TypeError("codes / scales must be contiguous int8 / uint8 CUDA tensors")
    if codes.numel() != rows * pitch or scales.numel() != tiles * tall * 4:
        raise ValueError("codes / scales do not have the sizes of a checkpoint of %d x %d values" % (rows, cols))
    return codes.data_ptr(), scales.data_ptr()


def star_checkpoint_pack(codes: torch.Tensor, scales: torch.Tensor, x: torch.Tensor, act: str = "none",
                         act_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Keep x in 8 bits; with act_out also write act(x) (which may be x)."""
    rows, cols = x.shape
    p, dtype, ld = _matrix(x, "x")
    q, s = _kept(codes, scales, rows, cols)
    h, _, ld_h = (None, dtype, cols) if act_out is None else _matrix(act_out, "act_out", (rows, cols), x.dtype)
    _check(_lib.star_checkpoint_pack(q, s, p, dtype, rows, cols, ld, _act(act), h, ld_h, _stream(stream)),
           "star_checkpoint_pack")


def star_checkpoint_unpack(out: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, act: str = "none",
                           stream=None) -> None:
    """out = act(kept value)."""
    rows, cols = out.shape
    p, dtype, ld = _matrix(out, "out")
    q, s = _kept(codes, scales, rows, cols)
    _check(_lib.star_checkpoint_unpack(p, dtype, ld, q, s, rows, cols, _act(act), _stream(stream)),
           "star_checkpoint_unpack")


def star_checkpoint_act_backward(dx: torch.Tensor, dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                                 act: str, stream=None) -> None:
    """dx = dy * act'(kept value); dx may be dy."""
    rows, cols = dy.shape
    p, dtype, ld = _matrix(dy, "dy")
    d, _, ld_d = _matrix(dx, "dx", (rows, cols), dy.dtype)
    q, s = _kept(codes, scales, rows, cols)
    _check(_lib.star_checkpoint_act_backward(d, ld_d, p, ld, dtype, q, s, rows, cols, _act(act), _stream(stream)),
           "star_checkpoint_act_backward")


def star_checkpoint_weight_grad(dw: torch.Tensor, dy: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor,
                                transposed: bool = False, accumulate: bool = False, stream=None) -> None:
    """dw (outs x cols, or cols x outs if transposed) = or += dy^T times the kept values."""
    rows, outs = dy.shape
    w, w_dtype, ld_w = _matrix(dw, "dw")
    cols = dw.shape[0 if transposed else 1]
    if dw.shape[1 if transposed else 0] != outs:
        raise ValueError("dw has shape %s, dy has %d columns" % (tuple(dw.shape), outs))
    p, dtype, ld = _matrix(dy, "dy")
    q, s = _kept(codes, scales, rows, cols)
    _check(_lib.star_checkpoint_weight_grad(w, w_dtype, ld_w, int(transposed), p, dtype, ld, q, s, rows, cols, outs,
                                            int(accumulate), _stream(stream)), "star_checkpoint_weight_grad")


def _gain(t: Optional[torch.Tensor], cols: int, what: str) -> Tuple[Optional[int], int]:
    """(address, dtype code) of a vector of float32 or bfloat16."""
    if t is None:
        return None, STAR_DTYPE_F32
    kind = t.dtype
    code = _DTYPES.get(kind)
    if code is None:
        raise TypeError("%s must be a contiguous float32 or bfloat16 CUDA tensor" % what)
    return _vector(t, cols, what, kind), code


def _optional_kept(codes, scales, rows: int, cols: int) -> Tuple[Optional[int], Optional[int]]:
    if (codes is None) != (scales is None):
        raise ValueError("codes and scales come together")
    return (None, None) if codes is None else _kept(codes, scales, rows, cols)


def star_rms_norm(y: torch.Tensor, x: torch.Tensor, gain: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                  total: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None,
                  codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  stream=None) -> None:
    """y = the root-mean-square norm of x + residual; the sum goes to total (which may
    be x or the residual), and y is kept in 8 bits in codes and scales, where given (for
    what reads y; star_rms_norm_backward takes the stream's)."""
    p, dtype, ld = _matrix(x, "x")
    shape, kind = x.shape, x.dtype
    rows, cols = shape
    o, ld_o = _like(y, "y", shape, kind)
    r, ld_r = (None, cols) if residual is None else _like(residual, "residual", shape, kind)
    s, ld_s = (None, cols) if total is None else _like(total, "total", shape, kind)
    g, g_dtype = _gain(gain, cols, "gain")
    q, b = (None, None) if codes is None and scales is None else _optional_kept(codes, scales, rows, cols)
    _check(_lib.star_rms_norm(o, ld_o, p, ld, r, ld_r, s, ld_s, dtype, rows, cols, g, g_dtype, eps, _vector(rstd, rows, "rstd"),
                              q, b, _stream(stream)), "star_rms_norm")


def star_rms_norm_workspace_bytes(rows: int, cols: int) -> int:
    out = ctypes.c_size_t(0)
    _check(_lib.star_rms_norm_workspace_bytes(rows, cols, ctypes.byref(out)), "star_rms_norm_workspace_bytes")
    return out.value


def star_rms_norm_backward(dx: torch.Tensor, dgain: Optional[torch.Tensor], dy: torch.Tensor, gain: Optional[torch.Tensor],
                           rstd: torch.Tensor, workspace: Optional[torch.Tensor] = None, total: Optional[torch.Tensor] = None,
                           codes: Optional[torch.Tensor] = None, scales: Optional[torch.Tensor] = None,
                           d_total: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None) -> None:
    """dx (which may be dy or d_total) and, unless None, dgain = or += its sums, from
    the normalized stream: total, or a checkpoint of it in codes and scales, which
    star_checkpoint_pack makes of total.  (star_rms_norm's codes are y's: not these.)"""
    p, dtype, ld = _matrix(dy, "dy")
    shape, kind = dy.shape, dy.dtype
    rows, cols = shape
    d, ld_d = _like(dx, "dx", shape, kind)
    s, ld_s = (None, cols) if total is None else _like(total, "total", shape, kind)
    e, ld_e = (None, cols) if d_total is None else _like(d_total, "d_total", shape, kind)
    g, g_dtype = _gain(gain, cols, "gain")
    dg, dg_dtype = _gain(dgain, cols, "dgain")
    q, b = (None, None) if codes is None and scales is None else _optional_kept(codes, scales, rows, cols)
    ws, ws_bytes = (None, 0) if workspace is None else _workspace(workspace)
    _check(_lib.star_rms_norm_backward(d, ld_d, dg, dg_dtype, accumulate, p, ld, s, ld_s, q, b, e, ld_e, dtype, rows, cols, g,
                                       g_dtype, _vector(rstd, rows, "rstd"), ws, ws_bytes, _stream(stream)),
           "star_rms_norm_backward")


def star_check_waits(stream=None) -> None:
    """Waits for the stream; raises if a wait inside a kernel ran out since the last check."""
    _check(_lib.star_check_waits(_stream(stream)), "star_check_waits")


STAR_WAIT_ATTEMPTS = 1 << 24


def star_set_wait_attempts(attempts: int = STAR_WAIT_ATTEMPTS) -> None:
    """Attempts of a wait inside a kernel, for launches from now on; 0: every wait has run out at once."""
    _check(_lib.star_set_wait_attempts(attempts), "star_set_wait_attempts")
