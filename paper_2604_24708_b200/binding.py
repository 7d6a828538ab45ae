"""ctypes binding of libhdet (include/hdet.h): same names, argument marshalling only.

Every step of the path runs inside the library's CUDA kernels; nothing here computes.
There is no fallback: if the shared library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import List, Optional, Sequence

HDET_MAX_REPLICAS = 32
HDET_MAX_GROUPS = 8

HDET_OK = 0
HDET_ERR_INVALID_ARG = 1
HDET_ERR_STATE = 2
HDET_ERR_ALIGN = 3
HDET_ERR_UNSUPPORTED = 4
HDET_ERR_CUDA = 5
HDET_ERR_NONFINITE = 6
HDET_ERR_TIMEOUT = 7

HDET_OPT_SGD, HDET_OPT_ADAMW = 0, 1
HDET_DTYPE_F32, HDET_DTYPE_BF16, HDET_DTYPE_F64, HDET_DTYPE_I32, HDET_DTYPE_I64 = 0, 1, 2, 3, 4
HDET_GRAD_AS_GIVEN, HDET_GRAD_REPLICA_MEAN = 0, 1
HDET_SCHED_CONSTANT, HDET_SCHED_ONECYCLE_COS, HDET_SCHED_ONECYCLE_LINEAR = 0, 1, 2

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lib", "libhdet.so")


class HdetError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"hdet status {status}: {message}")
        self.status = status
        self.message = message


class hdet_tensor(C.Structure):
    _fields_ = [
        ("param", C.c_void_p), ("grad", C.c_void_p), ("exp_avg", C.c_void_p), ("exp_avg_sq", C.c_void_p),
        ("numel", C.c_int64), ("param_stride", C.c_int64), ("grad_stride", C.c_int64), ("state_stride", C.c_int64),
        ("group", C.c_int32), ("reserved", C.c_int32), ("param_bf16", C.c_void_p),
    ]


class hdet_config(C.Structure):
    _fields_ = [
        ("n_replicas", C.c_int32), ("n_groups", C.c_int32), ("optimizer", C.c_int32), ("grad_dtype", C.c_int32),
        ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("momentum", C.c_double),
        ("alpha_lr", C.c_double), ("alpha_wd", C.c_double), ("sync_interval", C.c_int64),
        ("reshuffle", C.c_int32), ("fuse_converge", C.c_int32), ("seed", C.c_uint64),
        ("device", C.c_int32), ("grad_mode", C.c_int32),
        ("n_replicas_global", C.c_int32), ("replica_offset", C.c_int32),
    ]


class hdet_schedule(C.Structure):
    _fields_ = [
        ("kind", C.c_int32), ("autolr", C.c_int32), ("total_steps", C.c_int64),
        ("max_lr", C.POINTER(C.c_double)), ("weight_decay", C.POINTER(C.c_double)),
        ("pct_start", C.c_double), ("div_factor", C.c_double), ("final_div_factor", C.c_double),
        ("warmup_steps", C.c_int64), ("beta", C.c_double), ("sigma", C.c_double), ("lambda_", C.c_double),
        ("f_div", C.c_double), ("f_final", C.c_double), ("auto_wd", C.c_int32), ("reserved", C.c_int32),
    ]


class hdet_embedding(C.Structure):
    _fields_ = [
        ("tokens", C.c_void_p), ("rows", C.c_void_p), ("table", C.c_void_p),
        ("n_tokens", C.c_int64), ("vocab", C.c_int64), ("width", C.c_int64), ("token_stride", C.c_int64),
        ("rows_stride", C.c_int64), ("rows_row", C.c_int64), ("table_stride", C.c_int64), ("table_row", C.c_int64),
        ("scale", C.c_double), ("n_replicas", C.c_int32), ("token_dtype", C.c_int32), ("rows_dtype", C.c_int32),
        ("table_dtype", C.c_int32), ("device", C.c_int32), ("reserved", C.c_int32),
    ]


class hdet_token_loss_args(C.Structure):
    _fields_ = [
        ("hidden", C.c_void_p), ("weight", C.c_void_p), ("targets", C.c_void_p), ("loss", C.c_void_p),
        ("token_loss", C.c_void_p), ("d_hidden", C.c_void_p), ("d_weight", C.c_void_p),
        ("n_tokens", C.c_int64), ("vocab", C.c_int64), ("width", C.c_int64),
        ("hidden_stride", C.c_int64), ("hidden_row", C.c_int64), ("weight_stride", C.c_int64), ("weight_row", C.c_int64),
        ("target_stride", C.c_int64), ("token_loss_stride", C.c_int64), ("d_hidden_stride", C.c_int64),
        ("d_hidden_row", C.c_int64), ("d_weight_stride", C.c_int64), ("d_weight_row", C.c_int64),
        ("grad_scale", C.c_double), ("piece_bytes", C.c_int64), ("n_replicas", C.c_int32), ("hidden_dtype", C.c_int32),
        ("weight_dtype", C.c_int32), ("target_dtype", C.c_int32), ("loss_dtype", C.c_int32), ("d_hidden_dtype", C.c_int32),
        ("d_weight_dtype", C.c_int32), ("accumulate", C.c_int32), ("device", C.c_int32), ("reserved", C.c_int32),
    ]


class hdet_token_scores_args(C.Structure):
    _fields_ = [
        ("hidden", C.c_void_p), ("weight", C.c_void_p), ("targets", C.c_void_p), ("logprob", C.c_void_p), ("entropy", C.c_void_p),
        ("lse", C.c_void_p), ("top_ids", C.c_void_p), ("top_logprob", C.c_void_p), ("d_logprob", C.c_void_p), ("d_entropy", C.c_void_p),
        ("d_hidden", C.c_void_p), ("d_weight", C.c_void_p),
        ("n_tokens", C.c_int64), ("vocab", C.c_int64), ("width", C.c_int64), ("hidden_stride", C.c_int64), ("hidden_row", C.c_int64),
        ("weight_stride", C.c_int64), ("weight_row", C.c_int64), ("target_stride", C.c_int64), ("logprob_stride", C.c_int64),
        ("entropy_stride", C.c_int64), ("lse_stride", C.c_int64), ("top_ids_stride", C.c_int64), ("top_logprob_stride", C.c_int64),
        ("d_logprob_stride", C.c_int64), ("d_entropy_stride", C.c_int64), ("d_hidden_stride", C.c_int64), ("d_hidden_row", C.c_int64),
        ("d_weight_stride", C.c_int64), ("d_weight_row", C.c_int64), ("piece_bytes", C.c_int64),
        ("n_replicas", C.c_int32), ("n_top", C.c_int32), ("hidden_dtype", C.c_int32), ("weight_dtype", C.c_int32), ("target_dtype", C.c_int32),
        ("d_hidden_dtype", C.c_int32), ("d_weight_dtype", C.c_int32), ("accumulate", C.c_int32), ("device", C.c_int32), ("reserved", C.c_int32),
    ]


_GD = C.c_double * HDET_MAX_GROUPS
_ND = C.c_double * HDET_MAX_REPLICAS
_GND = (C.c_double * HDET_MAX_REPLICAS) * HDET_MAX_GROUPS
_GNI = (C.c_int32 * HDET_MAX_REPLICAS) * HDET_MAX_GROUPS


class hdet_state(C.Structure):
    _fields_ = [
        ("step", C.c_int64), ("n_acc", C.c_int64), ("fired", C.c_int32), ("round_ended", C.c_int32),
        ("device_status", C.c_uint32), ("reserved", C.c_int32),
        ("base", _GD), ("ctrl_base", _GD), ("velocity", _GD), ("delta", _GD),
        ("lr", _GND), ("wd", _GND), ("perm_lr", _GNI), ("perm_wd", _GNI),
        ("weights", _ND), ("loss_acc", _ND), ("loss_round", _ND), ("gamma", C.c_double),
        ("wd_base", _GD), ("wd_velocity", _GD), ("wd_delta", _GD),
    ]


def _load() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2604_24708_b200.build` "
            "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    H = C.c_void_p
    lib.hdet_create.argtypes = [C.POINTER(hdet_config), C.POINTER(hdet_tensor), C.c_int64, C.POINTER(H)]
    lib.hdet_set_schedule.argtypes = [H, C.POINTER(hdet_schedule)]
    lib.hdet_step.argtypes = [H, C.POINTER(C.c_double), C.c_void_p, C.POINTER(C.c_int32)]
    lib.hdet_step_device.argtypes = [H, C.c_void_p, C.c_int32, C.c_void_p, C.POINTER(C.c_int32)]
    lib.hdet_step_device.restype = C.c_int
    lib.hdet_step_host_grads.argtypes = [H, C.POINTER(C.c_void_p), C.POINTER(C.c_double), C.c_void_p,
                                         C.POINTER(C.c_int32)]
    lib.hdet_step_host_grads.restype = C.c_int
    lib.hdet_step_sharded.argtypes = [H, C.POINTER(C.c_double), C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
    lib.hdet_step_sharded.restype = C.c_int
    lib.hdet_apply_mean.argtypes = [H, C.c_void_p, C.c_void_p]
    lib.hdet_apply_mean.restype = C.c_int
    lib.hdet_apply_mean_peers.argtypes = [H, C.POINTER(C.c_void_p), C.c_int32, C.c_void_p]
    lib.hdet_apply_mean_peers.restype = C.c_int
    lib.hdet_partial_layout.argtypes = [H, C.POINTER(C.c_int64), C.c_int64, C.POINTER(C.c_int64)]
    lib.hdet_partial_layout.restype = C.c_int
    lib.hdet_grad_norm.argtypes = [H, C.c_void_p, C.c_int32, C.c_void_p]
    lib.hdet_grad_norm.restype = C.c_int
    lib.hdet_set_clip.argtypes = [H, C.c_double, C.c_void_p, C.c_int32]
    lib.hdet_set_clip.restype = C.c_int
    lib.hdet_warm_init.argtypes = [H, C.c_double, C.c_uint64, C.c_void_p]
    lib.hdet_warm_init.restype = C.c_int
    lib.hdet_converge.argtypes = [H, C.c_void_p]
    lib.hdet_autolr_update.argtypes = [H, C.POINTER(C.c_double), C.c_void_p]
    lib.hdet_get_state.argtypes = [H, C.POINTER(hdet_state)]
    lib.hdet_set_state.argtypes = [H, C.POINTER(hdet_state)]
    lib.hdet_destroy.argtypes = [H]
    lib.hdet_last_error.argtypes = [H]
    lib.hdet_last_error.restype = C.c_char_p
    lib.hdet_kernel_launches.argtypes = [H]
    lib.hdet_kernel_launches.restype = C.c_int64
    lib.hdet_converge_static.argtypes = [C.POINTER(hdet_tensor), C.c_int64, C.c_int32, C.c_int32, C.c_void_p]
    lib.hdet_converge_static.restype = C.c_int
    lib.hdet_plan_tiles.argtypes = [C.POINTER(hdet_config), C.POINTER(hdet_tensor), C.c_int64, C.POINTER(C.c_int32),
                                    C.POINTER(C.c_int32), C.c_int64, C.POINTER(C.c_int64), C.POINTER(C.c_int32),
                                    C.POINTER(C.c_int64)]
    lib.hdet_plan_tiles.restype = C.c_int
    lib.hdet_selftest_bounded_wait.argtypes = [H, C.c_void_p]
    lib.hdet_selftest_bounded_wait.restype = C.c_int
    # descriptors of these calls are given as byref(struct) or as its packed bytes
    lib.hdet_embed.argtypes = [C.c_void_p, C.c_void_p]
    lib.hdet_embed.restype = C.c_int
    lib.hdet_embed_grad_workspace.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
    lib.hdet_embed_grad_workspace.restype = C.c_int
    lib.hdet_embed_grad.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
    lib.hdet_embed_grad.restype = C.c_int
    lib.hdet_token_loss_workspace.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
    lib.hdet_token_loss_workspace.restype = C.c_int
    for f in (lib.hdet_token_scores_workspace, lib.hdet_token_scores_grad_workspace):
        f.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        f.restype = C.c_int
    for f in (lib.hdet_token_loss, lib.hdet_selftest_token_loss_wait, lib.hdet_token_scores, lib.hdet_token_scores_grad,
              lib.hdet_selftest_token_scores_wait, lib.hdet_selftest_token_scores_grad_wait):
        f.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        f.restype = C.c_int
    for f in ("hdet_create", "hdet_set_schedule", "hdet_step", "hdet_converge", "hdet_autolr_update",
              "hdet_get_state", "hdet_set_state", "hdet_destroy"):
        getattr(lib, f).restype = C.c_int
    return lib


_lib = _load()


def _check(status: int, handle) -> None:
    if status != HDET_OK:
        msg = _lib.hdet_last_error(handle)
        raise HdetError(status, msg.decode() if msg else "")


def _doubles(values: Optional[Sequence[float]]):
    if values is None:
        return None
    return (C.c_double * len(values))(*[float(v) for v in values])


def tensor_from_torch(param, grad, exp_avg=None, exp_avg_sq=None, group: int = 0) -> hdet_tensor:
    """Descriptor for tensors whose first axis is the replica axis ([N, ...], inner axes contiguous).

    ``grad`` may lack the replica axis (same shape as one replica): it is then shared (stride 0).
    """
    n = param.shape[0]
    numel = param[0].numel()
    if not param[0].is_contiguous():
        raise ValueError("each replica of param must be contiguous")
    shared = grad.dim() == param.dim() - 1 or (grad.shape[0] == 1 and n > 1)
    g0 = grad if grad.dim() == param.dim() - 1 else grad[0]
    if g0.numel() != numel or not g0.is_contiguous():
        raise ValueError("grad must match one replica of param and be contiguous")
    t = hdet_tensor()
    t.param = param.data_ptr()
    t.grad = grad.data_ptr()
    t.numel = numel
    t.param_stride = param.stride(0) if n > 1 else numel
    t.grad_stride = 0 if shared else (grad.stride(0) if n > 1 else numel)
    if exp_avg is not None:
        if not (exp_avg[0].is_contiguous() and exp_avg_sq[0].is_contiguous()) or exp_avg.stride(0) != exp_avg_sq.stride(0):
            raise ValueError("moments must be contiguous per replica and share one replica stride")
        t.exp_avg = exp_avg.data_ptr()
        t.exp_avg_sq = exp_avg_sq.data_ptr()
        t.state_stride = exp_avg.stride(0) if n > 1 else numel
    t.group = group
    return t


def make_schedule(kind: int, total_steps: int, max_lr: Sequence[float], weight_decay: Optional[Sequence[float]] = None,
                  pct_start: float = 0.3, div_factor: float = 25.0, final_div_factor: float = 1e4, autolr: int = 0,
                  warmup_steps: int = 0, beta: float = 0.9, sigma: float = 0.1, lambda_: float = 0.5,
                  f_div: float = 25.0, f_final: float = 1.0, auto_wd: int = 0) -> hdet_schedule:
    s = hdet_schedule()
    s.kind, s.autolr, s.total_steps = kind, int(autolr), total_steps
    s._max_lr = _doubles(max_lr)            # keep the host arrays alive with the struct
    s._weight_decay = _doubles(weight_decay)
    s.max_lr = C.cast(s._max_lr, C.POINTER(C.c_double))
    s.weight_decay = C.cast(s._weight_decay, C.POINTER(C.c_double)) if weight_decay is not None else None
    s.pct_start, s.div_factor, s.final_div_factor = pct_start, div_factor, final_div_factor
    s.warmup_steps, s.beta, s.sigma, s.lambda_ = warmup_steps, beta, sigma, lambda_
    s.f_div, s.f_final = f_div, f_final
    s.auto_wd = int(auto_wd)
    return s


def hdet_create(cfg: hdet_config, tensors: Sequence[hdet_tensor]) -> C.c_void_p:
    arr = (hdet_tensor * len(tensors))(*tensors) if tensors else None
    h = C.c_void_p()
    status = _lib.hdet_create(C.byref(cfg), arr, len(tensors), C.byref(h))
    _check(status, None)
    h.n_replicas, h.device = int(cfg.n_replicas), int(cfg.device)
    return h


def hdet_set_schedule(h, sched: hdet_schedule) -> None:
    _check(_lib.hdet_set_schedule(h, C.byref(sched)), h)


def hdet_step(h, step_losses: Optional[Sequence[float]] = None, stream: int = 0) -> bool:
    """Runs one update; returns True when it ended a round (the replicas were averaged)."""
    flag = C.c_int32(0)
    _check(_lib.hdet_step(h, _doubles(step_losses), C.c_void_p(stream), C.byref(flag)), h)
    return bool(flag.value)


def hdet_step_device(h, d_step_losses=None, stream: int = 0) -> bool:
    """One device-resident update; ``d_step_losses`` is a CUDA tensor of N float32 or float64 losses (or None)."""
    flag = C.c_int32(0)
    ptr, dtype = None, HDET_DTYPE_F32
    if d_step_losses is not None:
        import torch
        if not d_step_losses.is_cuda or not d_step_losses.is_contiguous():
            raise ValueError("d_step_losses must be a contiguous CUDA tensor")
        dtype = {torch.float32: HDET_DTYPE_F32, torch.float64: HDET_DTYPE_F64}[d_step_losses.dtype]
        ptr = C.c_void_p(d_step_losses.data_ptr())
    _check(_lib.hdet_step_device(h, ptr, dtype, C.c_void_p(stream), C.byref(flag)), h)
    return bool(flag.value)


def hdet_step_host_grads(h, host_grad_ptrs: Sequence[int], step_losses: Optional[Sequence[float]] = None,
                         stream: int = 0) -> bool:
    """hdet_step with the gradients taken from host memory (one pointer per tensor, laid out like the device gradient)."""
    flag = C.c_int32(0)
    arr = (C.c_void_p * max(1, len(host_grad_ptrs)))(*host_grad_ptrs) if host_grad_ptrs else None
    _check(_lib.hdet_step_host_grads(h, arr, _doubles(step_losses), C.c_void_p(stream), C.byref(flag)), h)
    return bool(flag.value)


def hdet_step_sharded(h, step_losses, d_partial, stream: int = 0) -> bool:
    """One update of a handle that holds a shard of the replica axis; ``d_partial`` is a CUDA float32 tensor."""
    flag = C.c_int32(0)
    ptr = C.c_void_p(d_partial.data_ptr()) if d_partial is not None else None
    _check(_lib.hdet_step_sharded(h, _doubles(step_losses), ptr, C.c_void_p(stream), C.byref(flag)), h)
    return bool(flag.value)


def hdet_apply_mean(h, d_sum, stream: int = 0) -> None:
    _check(_lib.hdet_apply_mean(h, C.c_void_p(d_sum.data_ptr()), C.c_void_p(stream)), h)


def hdet_apply_mean_peers(h, d_partials, stream: int = 0) -> None:
    """Every local replica <- (sum over the ranks' staging buffers, in the given rank order) / N, read by the kernel itself."""
    ptrs = [p.data_ptr() if hasattr(p, "data_ptr") else int(p) for p in d_partials]
    arr = (C.c_void_p * len(ptrs))(*ptrs)
    _check(_lib.hdet_apply_mean_peers(h, arr, len(ptrs), C.c_void_p(stream)), h)


def hdet_partial_layout(h, n_tensors: int):
    """(offsets per tensor, total elements) of the partial-sum staging buffer."""
    offs = (C.c_int64 * max(1, n_tensors))()
    total = C.c_int64(0)
    _check(_lib.hdet_partial_layout(h, offs if n_tensors else None, n_tensors, C.byref(total)), h)
    return list(offs)[:n_tensors], int(total.value)


def hdet_plan_tiles(cfg: hdet_config, tensors: Sequence[hdet_tensor]):
    """The work plan hdet_create would build, computed on the host: (tile_tensor, tile_index, access per tensor,
    partial-sum offset per tensor)."""
    arr = (hdet_tensor * len(tensors))(*tensors) if tensors else None
    count = C.c_int64(0)
    _check(_lib.hdet_plan_tiles(C.byref(cfg), arr, len(tensors), None, None, 0, C.byref(count), None, None), None)
    n = int(count.value)
    tt, ti = (C.c_int32 * max(1, n))(), (C.c_int32 * max(1, n))()
    acc, offs = (C.c_int32 * max(1, len(tensors)))(), (C.c_int64 * max(1, len(tensors)))()
    _check(_lib.hdet_plan_tiles(C.byref(cfg), arr, len(tensors), tt, ti, n, C.byref(count), acc, offs), None)
    return list(tt)[:n], list(ti)[:n], list(acc)[:len(tensors)], list(offs)[:len(tensors)]


def hdet_selftest_bounded_wait(h, stream: int = 0) -> None:
    """Launches a kernel whose bounded wait runs out (about a second): sets the timeout bit of the status word."""
    _check(_lib.hdet_selftest_bounded_wait(h, C.c_void_p(stream)), h)


def _norms(h, norms):
    """(pointer, dtype code) of a contiguous tensor of N float32 or float64 norms on the handle's device."""
    if not norms.is_cuda or norms.get_device() != h.device or norms.shape != (h.n_replicas,) or not norms.is_contiguous():
        raise ValueError("norms must be a contiguous tensor on the handle's CUDA device with one value per replica")
    return norms.data_ptr(), _dtype_code[norms.dtype]


def hdet_grad_norm(h, norms, stream: int = 0) -> None:
    """norms [N] (CUDA, float32 or float64) = every replica's global gradient norm over the handle's tensors."""
    ptr, code = _norms(h, norms)
    _check(_lib.hdet_grad_norm(h, ptr, code, stream), h)


def hdet_set_clip(h, max_norm: float, norms=None) -> None:
    """Every step from now on clips each replica's gradient to ``max_norm`` (0: none) and leaves the norms in ``norms`` [N]
    (CUDA, float32 or float64, kept by the caller while clipping is on), if given."""
    ptr, code = (None, HDET_DTYPE_F32) if norms is None else _norms(h, norms)
    _check(_lib.hdet_set_clip(h, max_norm, ptr, code), h)


def hdet_warm_init(h, nu: float = 0.01, seed: int = 0, stream: int = 0) -> None:
    """Eq. 10: every replica <- replica 0 (the checkpoint) + Gaussian noise of relative scale nu."""
    _check(_lib.hdet_warm_init(h, nu, seed, C.c_void_p(stream)), h)


def hdet_converge(h, stream: int = 0) -> None:
    _check(_lib.hdet_converge(h, C.c_void_p(stream)), h)


HDET_STATIC_MAX_TENSORS = 1024
HDET_STATIC_MAX_TILES = 65536


def hdet_converge_static(tensors: Sequence[hdet_tensor], n_replicas: int, device: int = 0, stream: int = 0) -> None:
    """Replica mean of every listed tensor without a handle and without any device allocation.

    For callers that cannot allocate at that point (all device memory owned by a framework pool, or a
    loop that must not risk the synchronisation an allocation can cause).  The work tables go into a
    static device array shared by all calls, so calls that overlap on the GPU must be serialised.
    """
    arr = (hdet_tensor * len(tensors))(*tensors) if tensors else None
    _check(_lib.hdet_converge_static(arr, len(tensors), n_replicas, device, C.c_void_p(stream)), None)


HDET_MAX_TOKENS = 1 << 24
HDET_MAX_VOCAB = 1 << 24
HDET_MAX_WIDTH = 1 << 16
HDET_MAX_ROW_STRIDE = 1 << 36
HDET_MAX_REPLICA_STRIDE = 1 << 48
HDET_MAX_TOP = 20


class _DtypeCodes(dict):
    """torch dtype -> HDET_DTYPE_*; filled on first use, so that importing this module does not import torch."""

    def __missing__(self, dtype):
        import torch
        self.update({torch.float32: HDET_DTYPE_F32, torch.bfloat16: HDET_DTYPE_BF16, torch.float64: HDET_DTYPE_F64,
                     torch.int32: HDET_DTYPE_I32, torch.int64: HDET_DTYPE_I64})
        if dtype not in self:
            raise ValueError(f"dtype {dtype} is not supported")
        return self[dtype]


_dtype_code = _DtypeCodes()


# The calls below are used once per token by a model that is sampled, so their checks read every attribute once and their
# descriptors are packed without building a ctypes struct (same layouts: hdet_embedding, hdet_token_loss_args, hdet_token_scores_args).
_EMBEDDING = struct.Struct("@3Q8qd6i")
_TOKEN_LOSS = struct.Struct("@7Q13qdq10i")
_TOKEN_SCORES = struct.Struct("@12Q20q10i")
assert _EMBEDDING.size == C.sizeof(hdet_embedding) and _TOKEN_LOSS.size == C.sizeof(hdet_token_loss_args)
assert _TOKEN_SCORES.size == C.sizeof(hdet_token_scores_args)


def _rows_layout(tensor, n: int, what: str):
    """(replica stride, row stride) of [n, rows, width], or of [rows, width] (replica stride 0: one copy for all)."""
    shape, stride = tensor.shape, tensor.stride()
    axes = len(shape)
    if axes == 3 and shape[0] == n:
        replica = stride[0]
    elif axes == 2:
        replica = 0
    else:
        raise ValueError(f"{what}: expected 2 axes, or 3 with {n} replicas first")
    width = shape[-1]
    if stride[-1] != 1 and width > 1:
        raise ValueError(f"{what}: the last axis must be contiguous")
    return replica, (stride[-2] if shape[-2] > 1 else width)


def _ids_stride(tensor, n: int, what: str) -> int:
    """Replica stride of [n, T] (or [T]: 0)."""
    shape, stride = tensor.shape, tensor.stride()
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the last axis must be contiguous")
    if len(shape) == 1:
        return 0
    if len(shape) != 2 or shape[0] != n:
        raise ValueError(f"{what}: expected 1 axis, or 2 with {n} replicas first")
    return stride[0]


def _embedding(tokens, rows, table, n: int, scale: float) -> bytes:
    shape = rows.shape
    T, D = shape[-2], shape[-1]
    V, width = table.shape[-2:]
    if tokens.shape[-1] != T or width != D:
        raise ValueError("tokens, rows and table disagree on the number of tokens or the width")
    device = tokens.get_device()
    if device < 0 or rows.get_device() != device or table.get_device() != device:
        raise ValueError("all tensors must be on one CUDA device")
    rows_stride, rows_row = _rows_layout(rows, n, "rows")
    table_stride, table_row = _rows_layout(table, n, "table")
    return _EMBEDDING.pack(tokens.data_ptr(), rows.data_ptr(), table.data_ptr(), T, V, D, _ids_stride(tokens, n, "tokens"),
                           rows_stride, rows_row, table_stride, table_row, scale, n, _dtype_code[tokens.dtype],
                           _dtype_code[rows.dtype], _dtype_code[table.dtype], device, 0)


def hdet_embed(tokens, table, out, scale: float = 1.0, stream: int = 0) -> None:
    """out[r, t] = scale * table[r, tokens[r, t]] for CUDA tensors tokens [N, T] or [T] (int32 or int64), table [N, V, D] or
    [V, D] (one for all replicas) and out [N, T, D], float32 or bfloat16 each.  Tokens outside 0 .. V-1 give zeros."""
    if out.dim() != 3:
        raise ValueError("out must be [N, T, D]")
    status = _lib.hdet_embed(_embedding(tokens, out, table, out.shape[0], scale), stream)
    if status:
        _check(status, None)


def hdet_embed_grad_workspace(tokens, d_out, d_table) -> int:
    """Bytes of workspace that hdet_embed_grad needs for these tensors."""
    d = _embedding(tokens, d_out, d_table, d_table.shape[0], 1.0)
    need = C.c_int64(0)
    _check(_lib.hdet_embed_grad_workspace(d, C.byref(need)), None)
    return int(need.value)


def hdet_embed_grad(tokens, d_out, d_table, workspace, scale: float = 1.0, accumulate: bool = False, stream: int = 0) -> None:
    """Gradient of hdet_embed: d_table [N, V, D] (+)= scale * the sums of d_out's rows ([N, T, D], or [T, D] for all replicas)
    by token.  ``workspace`` is a contiguous CUDA tensor of at least hdet_embed_grad_workspace bytes."""
    if d_table.dim() != 3:
        raise ValueError("d_table must be [N, V, D]")
    d = _embedding(tokens, d_out, d_table, d_table.shape[0], scale)
    ptr, size = _workspace(workspace, tokens.get_device())
    status = _lib.hdet_embed_grad(d, 1 if accumulate else 0, ptr, size, stream)
    if status:
        _check(status, None)


def _token_loss_args(hidden, weight, targets, loss, token_loss, d_hidden, d_weight, n, grad_scale, accumulate, piece_bytes) -> bytes:
    T, D = hidden.shape[-2:]
    V, width = weight.shape[-2:]
    if targets.shape[-1] != T or width != D:
        raise ValueError("hidden, weight and targets disagree on the number of tokens or the width")
    device = hidden.get_device()
    if device < 0 or weight.get_device() != device or targets.get_device() != device:
        raise ValueError("all tensors must be on one CUDA device")
    hidden_stride, hidden_row = _rows_layout(hidden, n, "hidden")
    weight_stride, weight_row = _rows_layout(weight, n, "weight")
    loss_at = loss_code = token_at = token_stride = dh_at = dh_stride = dh_code = dw_at = dw_stride = dw_code = 0
    dh_row = dw_row = D
    if loss is not None:
        if loss.shape != (n,) or loss.get_device() != device or (n > 1 and loss.stride(0) != 1):
            raise ValueError("loss must be a contiguous [N] on the inputs' device")
        loss_at, loss_code = loss.data_ptr(), _dtype_code[loss.dtype]
    if token_loss is not None:
        if token_loss.shape != (n, T) or token_loss.get_device() != device or _dtype_code[token_loss.dtype] != HDET_DTYPE_F32:
            raise ValueError("token_loss must be float32 [N, T] on the inputs' device")
        token_at, token_stride = token_loss.data_ptr(), _ids_stride(token_loss, n, "token_loss")
    if d_hidden is not None:
        if d_hidden.shape != (n, T, D) or d_hidden.get_device() != device:
            raise ValueError("d_hidden must be [N, T, D] on the inputs' device")
        dh_at, dh_code = d_hidden.data_ptr(), _dtype_code[d_hidden.dtype]
        dh_stride, dh_row = _rows_layout(d_hidden, n, "d_hidden")
    if d_weight is not None:
        if d_weight.shape != (n, V, D) or d_weight.get_device() != device:
            raise ValueError("d_weight must be [N, V, D] on the inputs' device")
        dw_at, dw_code = d_weight.data_ptr(), _dtype_code[d_weight.dtype]
        dw_stride, dw_row = _rows_layout(d_weight, n, "d_weight")
    return _TOKEN_LOSS.pack(
        hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), loss_at, token_at, dh_at, dw_at, T, V, D, hidden_stride, hidden_row,
        weight_stride, weight_row, _ids_stride(targets, n, "targets"), token_stride, dh_stride, dh_row, dw_stride, dw_row, grad_scale,
        piece_bytes, n, _dtype_code[hidden.dtype], _dtype_code[weight.dtype], _dtype_code[targets.dtype], loss_code, dh_code, dw_code,
        1 if accumulate else 0, device, 0)


def _replicas(*tensors) -> int:
    """N, from the first of (tensor, axes of one replica) that has a replica axis; 1 when none has."""
    for t, dims in tensors:
        if t is not None and t.dim() == dims + 1:
            return t.shape[0]
    return 1


def hdet_token_loss_workspace(hidden, weight, targets, d_hidden=None, d_weight=None, piece_bytes: int = 0) -> int:
    """Bytes of workspace that hdet_token_loss needs for these tensors and gradients."""
    n = _replicas((hidden, 2), (weight, 2), (targets, 1), (d_hidden, 2), (d_weight, 2))
    a = _token_loss_args(hidden, weight, targets, None, None, d_hidden, d_weight, n, 1.0, False, piece_bytes)
    need = C.c_int64(0)
    _check(_lib.hdet_token_loss_workspace(a, C.byref(need)), None)
    return int(need.value)


def hdet_token_loss(hidden, weight, targets, loss, workspace, token_loss=None, d_hidden=None, d_weight=None,
                    grad_scale: float = 1.0, accumulate: bool = False, piece_bytes: int = 0, stream: int = 0) -> None:
    """Softmax cross entropy of hidden [N, T, D] against the table weight [N, V, D] (or [V, D] for all replicas), both bf16,
    with targets [N, T] (or [T]; int32 or int64; outside 0 .. V-1: padding).  Writes the replicas' means to ``loss`` [N]
    (float32 or float64, as hdet_step_device reads them) and, where given, ``token_loss`` [N, T] and the gradients
    ``d_hidden`` [N, T, D] and ``d_weight`` [N, V, D] (float32 or bfloat16; ``accumulate`` adds d_weight to what is there)."""
    a = _token_loss_args(hidden, weight, targets, loss, token_loss, d_hidden, d_weight, loss.shape[0], grad_scale, accumulate,
                         piece_bytes)
    ptr, size = _workspace(workspace, hidden.get_device())
    status = _lib.hdet_token_loss(a, ptr, size, stream)
    if status:
        _check(status, None)


def hdet_selftest_token_loss_wait(hidden, weight, targets, loss, workspace, d_hidden=None, d_weight=None, piece_bytes: int = 0, stream: int = 0) -> None:
    """hdet_token_loss whose kernels' waits run out after some milliseconds: every loss becomes NaN, gradients are not defined."""
    a = _token_loss_args(hidden, weight, targets, loss, None, d_hidden, d_weight, loss.shape[0], 1.0, False, piece_bytes)
    ptr, size = _workspace(workspace, hidden.get_device())
    _check(_lib.hdet_selftest_token_loss_wait(a, ptr, size, stream), None)


def _per_token(tensor, n: int, T: int, device: int, what: str, dtype_code: int = HDET_DTYPE_F32, read: bool = False):
    """(address, replica stride) of one value a token: [n, T], or with ``read`` [T] for all replicas; (0, 0) for None."""
    if tensor is None:
        return 0, 0
    shape = tensor.shape
    if (shape != (n, T) and not (read and shape == (T,))) or tensor.get_device() != device or _dtype_code[tensor.dtype] != dtype_code:
        raise ValueError(f"{what} must be {'int32' if dtype_code == HDET_DTYPE_I32 else 'float32'} [N, T] on the inputs' device")
    return tensor.data_ptr(), _ids_stride(tensor, n, what)


def _per_alternative(tensor, n: int, T: int, device: int, what: str, dtype_code: int):
    """(address, replica stride) of n_top values a token, [n, T, n_top] with the last two axes contiguous; (0, 0) for None."""
    if tensor is None:
        return 0, 0
    shape, stride = tensor.shape, tensor.stride()
    if len(shape) != 3 or shape[:2] != (n, T) or tensor.get_device() != device or _dtype_code[tensor.dtype] != dtype_code:
        raise ValueError(f"{what} must be {'int32' if dtype_code == HDET_DTYPE_I32 else 'float32'} [N, T, n_top] on the inputs' device")
    if (shape[2] > 1 and stride[2] != 1) or (T > 1 and stride[1] != shape[2]):
        raise ValueError(f"{what}: the last two axes must be contiguous")
    return tensor.data_ptr(), stride[0]


def _token_scores_args(hidden, weight, targets, n, logprob=None, entropy=None, lse=None, top_ids=None, top_logprob=None, n_top=0,
                       d_logprob=None, d_entropy=None, d_hidden=None, d_weight=None, accumulate=False, piece_bytes=0, read=False) -> bytes:
    T, D = hidden.shape[-2:]
    V, width = weight.shape[-2:]
    if width != D or (targets is not None and targets.shape[-1] != T):
        raise ValueError("hidden, weight and targets disagree on the number of tokens or the width")
    device = hidden.get_device()
    if device < 0 or weight.get_device() != device or (targets is not None and targets.get_device() != device):
        raise ValueError("all tensors must be on one CUDA device")
    hidden_stride, hidden_row = _rows_layout(hidden, n, "hidden")
    weight_stride, weight_row = _rows_layout(weight, n, "weight")
    y_at = y_stride = dh_at = dh_stride = dh_code = dw_at = dw_stride = dw_code = 0
    y_code, dh_row, dw_row = HDET_DTYPE_I32, D, D
    if targets is not None:
        y_at, y_stride, y_code = targets.data_ptr(), _ids_stride(targets, n, "targets"), _dtype_code[targets.dtype]
    lp_at, lp_stride = _per_token(logprob, n, T, device, "logprob", read=read)
    en_at, en_stride = _per_token(entropy, n, T, device, "entropy", read=read)
    ls_at, ls_stride = _per_token(lse, n, T, device, "lse", read=read)
    id_at, id_stride = _per_alternative(top_ids, n, T, device, "top_ids", HDET_DTYPE_I32)
    tl_at, tl_stride = _per_alternative(top_logprob, n, T, device, "top_logprob", HDET_DTYPE_F32)
    if top_ids is not None:
        n_top = top_ids.shape[2]
        if top_logprob is not None and top_logprob.shape[2] != n_top:
            raise ValueError("top_ids and top_logprob disagree on the number of alternatives")
    dl_at, dl_stride = _per_token(d_logprob, n, T, device, "d_logprob", read=True)
    de_at, de_stride = _per_token(d_entropy, n, T, device, "d_entropy", read=True)
    if d_hidden is not None:
        if d_hidden.shape != (n, T, D) or d_hidden.get_device() != device:
            raise ValueError("d_hidden must be [N, T, D] on the inputs' device")
        dh_at, dh_code = d_hidden.data_ptr(), _dtype_code[d_hidden.dtype]
        dh_stride, dh_row = _rows_layout(d_hidden, n, "d_hidden")
    if d_weight is not None:
        if d_weight.shape != (n, V, D) or d_weight.get_device() != device:
            raise ValueError("d_weight must be [N, V, D] on the inputs' device")
        dw_at, dw_code = d_weight.data_ptr(), _dtype_code[d_weight.dtype]
        dw_stride, dw_row = _rows_layout(d_weight, n, "d_weight")
    return _TOKEN_SCORES.pack(
        hidden.data_ptr(), weight.data_ptr(), y_at, lp_at, en_at, ls_at, id_at, tl_at, dl_at, de_at, dh_at, dw_at, T, V, D,
        hidden_stride, hidden_row, weight_stride, weight_row, y_stride, lp_stride, en_stride, ls_stride, id_stride, tl_stride, dl_stride,
        de_stride, dh_stride, dh_row, dw_stride, dw_row, piece_bytes, n, n_top, _dtype_code[hidden.dtype], _dtype_code[weight.dtype], y_code,
        dh_code, dw_code, 1 if accumulate else 0, device, 0)


def _scores_replicas(hidden, weight, targets, *outputs) -> int:
    for t in outputs:
        if t is not None:
            return t.shape[0]
    return _replicas((hidden, 2), (weight, 2), (targets, 1))


def hdet_token_scores_workspace(hidden, weight, targets=None, n_top: int = 0) -> int:
    """Bytes of workspace that hdet_token_scores needs for these tensors and ``n_top`` alternatives a token."""
    a = _token_scores_args(hidden, weight, targets, _scores_replicas(hidden, weight, targets), n_top=n_top)
    need = C.c_int64(0)
    _check(_lib.hdet_token_scores_workspace(a, C.byref(need)), None)
    return int(need.value)


def hdet_token_scores(hidden, weight, targets, workspace, logprob=None, entropy=None, lse=None, top_ids=None, top_logprob=None,
                      stream: int = 0) -> None:
    """Of hidden [N, T, D] (or [T, D] for all replicas) against the table weight [N, V, D] (or [V, D]), both bf16, whichever is given:
    ``logprob`` of the tokens in targets [N, T] (or [T]; int32 or int64; outside 0 .. V-1: padding), ``entropy`` and ``lse`` (log sum
    exp), each float32 [N, T], and the best alternatives, ``top_ids`` (int32) and ``top_logprob`` (float32) [N, T, n_top].
    Without targets (None) every token counts."""
    n = _scores_replicas(hidden, weight, targets, logprob, entropy, lse, top_ids)
    a = _token_scores_args(hidden, weight, targets, n, logprob, entropy, lse, top_ids, top_logprob)
    ptr, size = _workspace(workspace, hidden.get_device())
    status = _lib.hdet_token_scores(a, ptr, size, stream)
    if status:
        _check(status, None)


def hdet_selftest_token_scores_wait(hidden, weight, targets, workspace, logprob=None, entropy=None, lse=None, top_ids=None, top_logprob=None,
                                    stream: int = 0) -> None:
    """hdet_token_scores whose kernels' waits run out after some milliseconds: every counted token has NaN, and -1 for its ids."""
    n = _scores_replicas(hidden, weight, targets, logprob, entropy, lse, top_ids)
    a = _token_scores_args(hidden, weight, targets, n, logprob, entropy, lse, top_ids, top_logprob)
    ptr, size = _workspace(workspace, hidden.get_device())
    _check(_lib.hdet_selftest_token_scores_wait(a, ptr, size, stream), None)


def hdet_token_scores_grad_workspace(hidden, weight, targets=None, d_hidden=None, d_weight=None, piece_bytes: int = 0) -> int:
    """Bytes of workspace that hdet_token_scores_grad needs for these tensors and gradients."""
    n = _scores_replicas(hidden, weight, targets, d_hidden, d_weight)
    a = _token_scores_args(hidden, weight, targets, n, d_hidden=d_hidden, d_weight=d_weight, piece_bytes=piece_bytes)
    need = C.c_int64(0)
    _check(_lib.hdet_token_scores_grad_workspace(a, C.byref(need)), None)
    return int(need.value)


def hdet_token_scores_grad(hidden, weight, targets, workspace, lse, logprob=None, entropy=None, d_logprob=None, d_entropy=None,
                           d_hidden=None, d_weight=None, accumulate: bool = False, piece_bytes: int = 0, stream: int = 0) -> None:
    """Gradients of a loss of log probabilities and entropies: given d_logprob and / or d_entropy (float32 [N, T] or [T]) and what
    hdet_token_scores left (``lse``; ``logprob`` with targets; ``entropy`` with d_entropy), writes ``d_hidden`` [N, T, D] and / or
    ``d_weight`` [N, V, D] (float32 or bfloat16; ``accumulate`` adds d_weight to what is there)."""
    n = _scores_replicas(hidden, weight, targets, d_hidden, d_weight)
    a = _token_scores_args(hidden, weight, targets, n, logprob, entropy, lse, d_logprob=d_logprob, d_entropy=d_entropy, d_hidden=d_hidden,
                           d_weight=d_weight, accumulate=accumulate, piece_bytes=piece_bytes, read=True)
    ptr, size = _workspace(workspace, hidden.get_device())
    status = _lib.hdet_token_scores_grad(a, ptr, size, stream)
    if status:
        _check(status, None)


def hdet_selftest_token_scores_grad_wait(hidden, weight, targets, workspace, lse, logprob=None, entropy=None, d_logprob=None, d_entropy=None,
                                         d_hidden=None, d_weight=None, accumulate: bool = False, piece_bytes: int = 0, stream: int = 0) -> None:
    """hdet_token_scores_grad whose kernels' waits run out after some milliseconds: the first element of every replica's gradients is NaN."""
    n = _scores_replicas(hidden, weight, targets, d_hidden, d_weight)
    a = _token_scores_args(hidden, weight, targets, n, logprob, entropy, lse, d_logprob=d_logprob, d_entropy=d_entropy, d_hidden=d_hidden,
                           d_weight=d_weight, accumulate=accumulate, piece_bytes=piece_bytes, read=True)
    ptr, size = _workspace(workspace, hidden.get_device())
    _check(_lib.hdet_selftest_token_scores_grad_wait(a, ptr, size, stream), None)


def _workspace(workspace, device: int):
    if workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on the inputs' CUDA device")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def hdet_autolr_update(h, round_losses: Optional[Sequence[float]] = None, stream: int = 0) -> None:
    _check(_lib.hdet_autolr_update(h, _doubles(round_losses), C.c_void_p(stream)), h)


def hdet_get_state(h, raise_on_nonfinite: bool = True) -> hdet_state:
    st = hdet_state()
    status = _lib.hdet_get_state(h, C.byref(st))
    if status in (HDET_ERR_NONFINITE, HDET_ERR_TIMEOUT) and not raise_on_nonfinite:   # sticky device flags: *out is filled
        return st
    _check(status, h)
    return st


def hdet_set_state(h, st: hdet_state) -> None:
    _check(_lib.hdet_set_state(h, C.byref(st)), h)


def hdet_destroy(h) -> None:
    _check(_lib.hdet_destroy(h), None)


def hdet_last_error(h=None) -> str:
    msg = _lib.hdet_last_error(h)
    return msg.decode() if msg else ""


def hdet_kernel_launches(h) -> int:
    return int(_lib.hdet_kernel_launches(h))


def raw_library() -> C.CDLL:
    """The loaded CDLL (for tests that call the C ABI with hand-built arguments)."""
    return _lib
