"""Thin ctypes binding of ``libpsops.so`` -- argument marshalling only.

Every function has the name and meaning of the C entry point declared in
``include/psops.h``; every step of the synchronisation runs in the CUDA
library.  PyTorch is used for device memory and streams, nothing else.  If the
shared library is missing the import of a symbol fails with an error: there is
no CPU path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

from .build import LIBRARY

PSOPS_OK = 0
PSOPS_EINVAL, PSOPS_EALIGN, PSOPS_ESTATE, PSOPS_ENAN = -1, -2, -3, -4
PSOPS_EWORKSPACE, PSOPS_ECUDA, PSOPS_ENOMEM, PSOPS_ELIMIT = -5, -6, -7, -8
PSOPS_STATIC_SCRATCH_DOUBLES = 1 << 20
PSOPS_MAX_K = 1024
PSOPS_KEEP_GBEST, PSOPS_QUADRATIC, PSOPS_GBEST_HISTORY, PSOPS_SEPARATE_SELECT = 1, 2, 4, 8
PSOPS_X, PSOPS_V, PSOPS_PBEST, PSOPS_GBEST = 0, 1, 2, 3
PSOPS_NONE, PSOPS_F32, PSOPS_F16, PSOPS_BF16 = 0, 1, 2, 3
PSOPS_MEAN, PSOPS_SUM, PSOPS_PER_TOKEN = 0, 1, 2
PSOPS_XENT_GRADS, PSOPS_XENT_STAGED = 1, 2
PSOPS_ATTENTION_GRADS = 1
PSOPS_RELU, PSOPS_SILU, PSOPS_GELU = 0, 1, 2

EXPORTS = [
    "psops_workspace_bytes", "psops_create", "psops_set_losses", "psops_sync",
    "psops_sync_host", "psops_average", "psops_get_weights", "psops_set_weights",
    "psops_sync_info", "psops_get_losses", "psops_set_quadratic",
    "psops_eval_quadratic", "psops_get_state", "psops_set_state", "psops_inertia",
    "psops_launch_count", "psops_strerror", "psops_last_error", "psops_destroy",
    "psops_quadratic_fitness_static", "psops_shard_select", "psops_shard_update",
    "psops_shard_update_range", "psops_get_history", "psops_set_history", "psops_ssgd",
    "psops_host_register", "psops_host_unregister",
    "psops_adamw_workspace_bytes", "psops_adamw_create", "psops_adamw_set_grads", "psops_adamw_step",
    "psops_adamw_steps", "psops_adamw_set_stream", "psops_adamw_launch_count", "psops_adamw_last_error",
    "psops_adamw_destroy",
    "psops_gradnorm_workspace_bytes", "psops_gradnorm_create", "psops_gradnorm_set_grads", "psops_gradnorm_run",
    "psops_gradnorm_set_stream", "psops_gradnorm_launch_count", "psops_gradnorm_last_error",
    "psops_gradnorm_destroy",
    "psops_xent_workspace_bytes", "psops_xent_create", "psops_xent_forward", "psops_xent_backward",
    "psops_xent_set_stream", "psops_xent_launch_count", "psops_xent_last_error", "psops_xent_destroy",
    "psops_attention_workspace_bytes", "psops_attention_create", "psops_attention_forward", "psops_attention_backward",
    "psops_attention_set_stream", "psops_attention_launch_count", "psops_attention_last_error",
    "psops_attention_destroy",
    "psops_keep_create", "psops_keep_pack", "psops_keep_unpack", "psops_keep_activate",
    "psops_keep_activate_backward", "psops_keep_set_stream", "psops_keep_launch_count", "psops_keep_last_error",
    "psops_keep_destroy",
]


class psops_config(ctypes.Structure):
    _fields_ = [("K", ctypes.c_int32), ("k_first", ctypes.c_int32), ("N", ctypes.c_int64),
                ("ld", ctypes.c_int64), ("m_max", ctypes.c_float), ("m_min", ctypes.c_float),
                ("t_max", ctypes.c_int64), ("c1", ctypes.c_float), ("c2", ctypes.c_float),
                ("seed", ctypes.c_uint64), ("flags", ctypes.c_uint32), ("K_total", ctypes.c_int32)]


class psops_adamw_config(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("steps_done", ctypes.c_int64), ("state_bits", ctypes.c_int32), ("grad_type", ctypes.c_int32),
                ("copy_type", ctypes.c_int32), ("n_tensors", ctypes.c_int32)]


class psops_adamw_tensor(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("g", ctypes.c_void_p), ("copy", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("weight_decay", ctypes.c_double)]


class psops_xent_config(ctypes.Structure):
    _fields_ = [("max_tokens", ctypes.c_int64), ("dim", ctypes.c_int64), ("vocab", ctypes.c_int64),
                ("type", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class psops_attention_config(ctypes.Structure):
    _fields_ = [("max_tokens", ctypes.c_int64), ("max_sequences", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("dim", ctypes.c_int32), ("type", ctypes.c_int32),
                ("buckets", ctypes.c_int32), ("first", ctypes.POINTER(ctypes.c_int32)), ("scale", ctypes.c_float),
                ("flags", ctypes.c_uint32)]


class psops_heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class PsopsError(RuntimeError):
    def __init__(self, code: int, where: str, detail: str = ""):
        self.code = code
        msg = f"{where}: {_strerror(code)} ({code})"
        if detail:
            msg += f": {detail}"
        super().__init__(msg)


_lib = None
_vp, _f32p, _u32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
_i32, _i64 = ctypes.c_int32, ctypes.c_int64


def load() -> ctypes.CDLL:
    """Load the CUDA library; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBRARY):
        raise ImportError(
            f"{LIBRARY} is missing: build it with "
            "`python -m paper_2009_03816_b200.build` (needs nvcc). "
            "There is no CPU fallback.")
    lib = ctypes.CDLL(LIBRARY)
    cfgp = ctypes.POINTER(psops_config)
    xcfgp = ctypes.POINTER(psops_xent_config)
    tcfgp, hp = ctypes.POINTER(psops_attention_config), ctypes.POINTER(psops_heads)
    acfgp, atensp = ctypes.POINTER(psops_adamw_config), ctypes.POINTER(psops_adamw_tensor)
    sig = {
        "psops_workspace_bytes": (ctypes.c_size_t, [cfgp]),
        "psops_create": (ctypes.c_int, [ctypes.POINTER(_vp), cfgp, _f32p, _f32p, _f32p, _vp,
                                        ctypes.c_size_t, _vp]),
        "psops_set_losses": (ctypes.c_int, [_vp, _f32p, ctypes.c_int]),
        "psops_sync": (ctypes.c_int, [_vp, ctypes.c_int64, ctypes.c_float]),
        "psops_sync_host": (ctypes.c_int, [_vp, _f32p, ctypes.c_int64, _f32p, ctypes.c_int64,
                                           ctypes.c_float, _f32p, ctypes.c_int64]),
        "psops_average": (ctypes.c_int, [_vp]),
        "psops_get_weights": (ctypes.c_int, [_vp, ctypes.c_int, ctypes.c_int, _f32p, ctypes.c_int]),
        "psops_set_weights": (ctypes.c_int, [_vp, ctypes.c_int, ctypes.c_int, _f32p, ctypes.c_int]),
        "psops_sync_info": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_int), _u32p, _f32p]),
        "psops_get_losses": (ctypes.c_int, [_vp, _f32p, ctypes.c_int]),
        "psops_set_quadratic": (ctypes.c_int, [_vp, _f32p, _f32p]),
        "psops_eval_quadratic": (ctypes.c_int, [_vp]),
        "psops_get_state": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_uint32), _f32p]),
        "psops_set_state": (ctypes.c_int, [_vp, ctypes.c_uint32, _f32p]),
        "psops_inertia": (ctypes.c_float, [cfgp, ctypes.c_int64]),
        "psops_launch_count": (ctypes.c_int64, [_vp]),
        "psops_strerror": (ctypes.c_char_p, [ctypes.c_int]),
        "psops_last_error": (ctypes.c_char_p, [_vp]),
        "psops_destroy": (ctypes.c_int, [_vp]),
        "psops_shard_select": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_int)]),
        "psops_shard_update": (ctypes.c_int, [_vp, ctypes.c_int64, ctypes.c_float, _f32p]),
        "psops_shard_update_range": (ctypes.c_int, [_vp, ctypes.c_int64, ctypes.c_float, _f32p,
                                                    ctypes.c_int64, ctypes.c_int64]),
        "psops_get_history": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int)]),
        "psops_set_history": (ctypes.c_int, [_vp, ctypes.c_float, _f32p, ctypes.c_int]),
        "psops_ssgd": (ctypes.c_int, [_vp, _f32p, ctypes.c_int64, ctypes.c_float]),
        "psops_host_register": (ctypes.c_int, [_vp, ctypes.c_size_t]),
        "psops_host_unregister": (ctypes.c_int, [_vp]),
        "psops_quadratic_fitness_static": (ctypes.c_int, [_f32p, ctypes.c_int64, ctypes.c_int32,
                                                          ctypes.c_int64, _f32p, _f32p, _f32p, _vp]),
        "psops_adamw_workspace_bytes": (ctypes.c_size_t, [acfgp, atensp]),
        "psops_adamw_create": (ctypes.c_int, [ctypes.POINTER(_vp), acfgp, atensp, _vp, ctypes.c_size_t, _vp]),
        "psops_adamw_set_grads": (ctypes.c_int, [_vp, ctypes.POINTER(_vp)]),
        "psops_adamw_step": (ctypes.c_int, [_vp, ctypes.c_double, _f32p]),
        "psops_adamw_steps": (ctypes.c_int, [_vp, ctypes.POINTER(ctypes.c_int64)]),
        "psops_adamw_set_stream": (ctypes.c_int, [_vp, _vp]),
        "psops_adamw_launch_count": (ctypes.c_int64, [_vp]),
        "psops_adamw_last_error": (ctypes.c_char_p, [_vp]),
        "psops_adamw_destroy": (ctypes.c_int, [_vp]),
        "psops_gradnorm_workspace_bytes": (ctypes.c_size_t, [ctypes.c_int32, ctypes.POINTER(ctypes.c_int64)]),
        "psops_gradnorm_create": (ctypes.c_int, [ctypes.POINTER(_vp), ctypes.c_int32, ctypes.POINTER(_vp),
                                                 ctypes.POINTER(ctypes.c_int64), ctypes.c_int32, _vp,
                                                 ctypes.c_size_t, _vp]),
        "psops_gradnorm_set_grads": (ctypes.c_int, [_vp, ctypes.POINTER(_vp)]),
        "psops_gradnorm_run": (ctypes.c_int, [_vp, ctypes.c_float, _f32p]),
        "psops_gradnorm_set_stream": (ctypes.c_int, [_vp, _vp]),
        "psops_gradnorm_launch_count": (ctypes.c_int64, [_vp]),
        "psops_gradnorm_last_error": (ctypes.c_char_p, [_vp]),
        "psops_gradnorm_destroy": (ctypes.c_int, [_vp]),
        "psops_xent_workspace_bytes": (ctypes.c_size_t, [xcfgp]),
        "psops_xent_create": (ctypes.c_int, [ctypes.POINTER(_vp), xcfgp, _vp, ctypes.c_size_t, _vp]),
        "psops_xent_forward": (ctypes.c_int, [_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                              ctypes.c_int32, _f32p, _f32p, _f32p]),
        "psops_xent_backward": (ctypes.c_int, [_vp, _vp, ctypes.c_int64, _vp, ctypes.c_int64, _vp, ctypes.c_int64,
                                               _f32p, _f32p, _f32p, ctypes.c_int32, _vp, ctypes.c_int64, _vp,
                                               ctypes.c_int64]),
        "psops_xent_set_stream": (ctypes.c_int, [_vp, _vp]),
        "psops_xent_launch_count": (ctypes.c_int64, [_vp]),
        "psops_xent_last_error": (ctypes.c_char_p, [_vp]),
        "psops_xent_destroy": (ctypes.c_int, [_vp]),
        "psops_attention_workspace_bytes": (ctypes.c_size_t, [tcfgp]),
        "psops_attention_create": (ctypes.c_int, [ctypes.POINTER(_vp), tcfgp, _vp, ctypes.c_size_t, _vp]),
        "psops_attention_forward": (ctypes.c_int, [_vp, hp, hp, hp, _vp, ctypes.c_int32, ctypes.c_int64, _vp,
                                                   ctypes.c_int32, hp, _f32p, ctypes.c_int32]),
        "psops_attention_backward": (ctypes.c_int, [_vp, hp, hp, hp, _vp, ctypes.c_int32, ctypes.c_int64, _vp,
                                                    ctypes.c_int32, hp, _f32p, hp, hp, hp, hp, _vp, ctypes.c_int32]),
        "psops_attention_set_stream": (ctypes.c_int, [_vp, _vp]),
        "psops_attention_launch_count": (ctypes.c_int64, [_vp]),
        "psops_attention_last_error": (ctypes.c_char_p, [_vp]),
        "psops_attention_destroy": (ctypes.c_int, [_vp]),
        "psops_keep_create": (ctypes.c_int, [ctypes.POINTER(_vp), _vp]),
        "psops_keep_pack": (ctypes.c_int, [_vp, _i32, _i64, _i64, _vp, _i64, _vp, _f32p]),
        "psops_keep_unpack": (ctypes.c_int, [_vp, _i32, _i64, _i64, _vp, _f32p, _vp, _i64]),
        "psops_keep_activate": (ctypes.c_int, [_vp, _i32, _i32, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _f32p,
                                                _vp, _f32p]),
        "psops_keep_activate_backward": (ctypes.c_int, [_vp, _i32, _i32, _i64, _i64, _vp, _f32p, _vp, _f32p, _vp, _i64,
                                                         _vp, _i64, _vp, _i64, _vp, _i64]),
        "psops_keep_set_stream": (ctypes.c_int, [_vp, _vp]),
        "psops_keep_launch_count": (ctypes.c_int64, [_vp]),
        "psops_keep_last_error": (ctypes.c_char_p, [_vp]),
        "psops_keep_destroy": (ctypes.c_int, [_vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)            # AttributeError if a symbol is missing
        fn.restype, fn.argtypes = res, args
    _lib = lib
    return lib


def _strerror(code: int) -> str:
    try:
        return load().psops_strerror(int(code)).decode()
    except Exception:  # pragma: no cover
        return "error"


def _check(rc: int, where: str, ctx=None, last_error="psops_last_error") -> None:
    if rc != PSOPS_OK:
        detail = ""
        if ctx is not None and rc == PSOPS_ECUDA:
            detail = getattr(load(), last_error)(ctx).decode()
        raise PsopsError(rc, where, detail)


def _ptr(buf) -> int:
    """Address of a torch tensor or numpy array (0 for None)."""
    if isinstance(buf, torch.Tensor):
        return buf.data_ptr()
    if buf is None:
        return 0
    if isinstance(buf, np.ndarray):
        return buf.ctypes.data
    if isinstance(buf, int):
        return buf
    raise TypeError(f"cannot take the address of {type(buf)!r}")


def _on_device(buf) -> int:
    return int(isinstance(buf, torch.Tensor) and buf.is_cuda)


def make_config(K, N, ld=None, *, m_max, m_min, t_max=1, c1, c2, seed, flags=0,
                k_first=0, K_total=0) -> psops_config:
    ld = (int(N) + 3) // 4 * 4 if ld is None else int(ld)
    return psops_config(int(K), int(k_first), int(N), ld, float(m_max), float(m_min), int(t_max),
                        float(c1), float(c2), int(seed), int(flags), int(K_total))


# ---- one function per C entry point --------------------------------------

def psops_workspace_bytes(cfg: psops_config) -> int:
    return int(load().psops_workspace_bytes(ctypes.byref(cfg)))


def psops_inertia(cfg: psops_config, t_iter: int) -> float:
    return float(load().psops_inertia(ctypes.byref(cfg), int(t_iter)))


def psops_create(cfg, d_x, d_v, d_pbest, d_workspace, workspace_bytes=None, stream=None):
    handle = _vp()
    if workspace_bytes is None:
        workspace_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    rc = load().psops_create(ctypes.byref(handle), ctypes.byref(cfg), _ptr(d_x), _ptr(d_v),
                             _ptr(d_pbest), _ptr(d_workspace), int(workspace_bytes),
                             int(stream) if stream else None)
    _check(rc, "psops_create")
    return handle


def psops_set_losses(ctx, losses) -> None:
    _check(load().psops_set_losses(ctx, _ptr(losses), _on_device(losses)), "psops_set_losses", ctx)


def psops_sync(ctx, t_iter: int = 0, lam: float = 1.0) -> None:
    _check(load().psops_sync(ctx, int(t_iter), float(lam)), "psops_sync", ctx)


def psops_sync_host(ctx, h_x_in, h_in_ld, h_losses, t_iter, lam, h_x_out, h_out_ld) -> None:
    _check(load().psops_sync_host(ctx, _ptr(h_x_in), int(h_in_ld), _ptr(h_losses), int(t_iter),
                                  float(lam), _ptr(h_x_out), int(h_out_ld)), "psops_sync_host", ctx)


def psops_shard_select(ctx) -> int:
    g = ctypes.c_int(-1)
    _check(load().psops_shard_select(ctx, ctypes.byref(g)), "psops_shard_select", ctx)
    return int(g.value)


def psops_shard_update(ctx, t_iter, lam, d_gbest_row) -> None:
    _check(load().psops_shard_update(ctx, int(t_iter), float(lam), _ptr(d_gbest_row)),
           "psops_shard_update", ctx)


def psops_shard_update_range(ctx, t_iter, lam, d_gbest_row, first_elem, last_elem) -> None:
    _check(load().psops_shard_update_range(ctx, int(t_iter), float(lam), _ptr(d_gbest_row),
                                           int(first_elem), int(last_elem)),
           "psops_shard_update_range", ctx)


def psops_get_history(ctx):
    loss, valid = ctypes.c_float(0.0), ctypes.c_int(0)
    _check(load().psops_get_history(ctx, ctypes.byref(loss), ctypes.byref(valid)), "psops_get_history", ctx)
    return float(loss.value), bool(valid.value)


def psops_set_history(ctx, gbest_loss, gbest_row) -> None:
    _check(load().psops_set_history(ctx, float(gbest_loss), _ptr(gbest_row), _on_device(gbest_row)),
           "psops_set_history", ctx)


def psops_ssgd(ctx, d_grad, grad_ld, alpha) -> None:
    _check(load().psops_ssgd(ctx, _ptr(d_grad), int(grad_ld), float(alpha)), "psops_ssgd", ctx)


def psops_host_register(buf) -> None:
    """Pin a host buffer (numpy array or CPU tensor) in place for psops_sync_host."""
    nbytes = buf.nbytes if isinstance(buf, np.ndarray) else buf.numel() * buf.element_size()
    _check(load().psops_host_register(_ptr(buf), int(nbytes)), "psops_host_register")


def psops_host_unregister(buf) -> None:
    _check(load().psops_host_unregister(_ptr(buf)), "psops_host_unregister")


def psops_average(ctx) -> None:
    _check(load().psops_average(ctx), "psops_average", ctx)


def psops_get_weights(ctx, which: int, k: int, dst) -> None:
    _check(load().psops_get_weights(ctx, int(which), int(k), _ptr(dst), _on_device(dst)),
           "psops_get_weights", ctx)


def psops_set_weights(ctx, which: int, k: int, src) -> None:
    _check(load().psops_set_weights(ctx, int(which), int(k), _ptr(src), _on_device(src)),
           "psops_set_weights", ctx)


def psops_sync_info(ctx, K: int):
    g = ctypes.c_int(-1)
    words = np.zeros((K + 31) // 32, dtype=np.uint32)
    pl = np.zeros(K, dtype=np.float32)
    _check(load().psops_sync_info(ctx, ctypes.byref(g), _ptr(words), _ptr(pl)), "psops_sync_info", ctx)
    improved = np.array([(int(words[i >> 5]) >> (i & 31)) & 1 for i in range(K)], dtype=bool)
    return int(g.value), improved, pl


def psops_get_losses(ctx, dst) -> None:
    _check(load().psops_get_losses(ctx, _ptr(dst), _on_device(dst)), "psops_get_losses", ctx)


def psops_set_quadratic(ctx, d_dvec, d_tvec) -> None:
    _check(load().psops_set_quadratic(ctx, _ptr(d_dvec), _ptr(d_tvec)), "psops_set_quadratic", ctx)


def psops_eval_quadratic(ctx) -> None:
    _check(load().psops_eval_quadratic(ctx), "psops_eval_quadratic", ctx)


def psops_get_state(ctx, K: int):
    step = ctypes.c_uint32(0)
    pl = np.zeros(K, dtype=np.float32)
    _check(load().psops_get_state(ctx, ctypes.byref(step), _ptr(pl)), "psops_get_state", ctx)
    return int(step.value), pl


def psops_set_state(ctx, sync_step: int, pbest_loss) -> None:
    pl = np.ascontiguousarray(pbest_loss, dtype=np.float32)
    _check(load().psops_set_state(ctx, int(sync_step), _ptr(pl)), "psops_set_state", ctx)


def psops_launch_count(ctx) -> int:
    return int(load().psops_launch_count(ctx))


def psops_destroy(ctx) -> None:
    _check(load().psops_destroy(ctx), "psops_destroy")


def psops_quadratic_fitness_static(d_x, ld, K, N, d_dvec, d_tvec, d_loss, stream=None) -> None:
    """Fitness of K device rows into d_loss[K] using the library's built-in
    scratch array: no workspace, no context, no allocation (for callers that
    cannot allocate device memory).  Work is enqueued on `stream`."""
    _check(load().psops_quadratic_fitness_static(_ptr(d_x), int(ld), int(K), int(N), _ptr(d_dvec),
                                                 _ptr(d_tvec), _ptr(d_loss),
                                                 int(stream) if stream else None),
           "psops_quadratic_fitness_static")


# ---- operators of the training steps ---------------------------------------

def _addresses(buffers):
    return (_vp * len(buffers))(*[_ptr(b) or None for b in buffers])


def psops_adamw_workspace_bytes(cfg: psops_adamw_config, tensors) -> int:
    return int(load().psops_adamw_workspace_bytes(ctypes.byref(cfg), tensors))


def psops_adamw_create(cfg, tensors, d_workspace, workspace_bytes=None, stream=None):
    """`tensors`: a ctypes array of psops_adamw_tensor, cfg.n_tensors of them."""
    handle = _vp()
    if workspace_bytes is None:
        workspace_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    rc = load().psops_adamw_create(ctypes.byref(handle), ctypes.byref(cfg), tensors, _ptr(d_workspace),
                                   int(workspace_bytes), int(stream) if stream else None)
    _check(rc, "psops_adamw_create")
    return handle


def psops_adamw_set_grads(opt, grads) -> None:
    _check(load().psops_adamw_set_grads(opt, _addresses(grads)), "psops_adamw_set_grads", opt,
           "psops_adamw_last_error")


def psops_adamw_step(opt, lr: float, d_scale=None) -> None:
    _check(load().psops_adamw_step(opt, float(lr), _ptr(d_scale)), "psops_adamw_step", opt, "psops_adamw_last_error")


def psops_adamw_steps(opt) -> int:
    steps = ctypes.c_int64(0)
    _check(load().psops_adamw_steps(opt, ctypes.byref(steps)), "psops_adamw_steps", opt, "psops_adamw_last_error")
    return int(steps.value)


def psops_adamw_set_stream(ctx, stream) -> None:
    _check(load().psops_adamw_set_stream(ctx, int(stream) if stream else None), "psops_adamw_set_stream", ctx,
           "psops_adamw_last_error")


def psops_adamw_launch_count(opt) -> int:
    return int(load().psops_adamw_launch_count(opt))


def psops_adamw_destroy(opt) -> None:
    _check(load().psops_adamw_destroy(opt), "psops_adamw_destroy")


def psops_gradnorm_workspace_bytes(sizes) -> int:
    return int(load().psops_gradnorm_workspace_bytes(len(sizes), (ctypes.c_int64 * len(sizes))(*sizes)))


def psops_gradnorm_create(grads, sizes, grad_type, d_workspace, workspace_bytes=None, stream=None):
    handle = _vp()
    if workspace_bytes is None:
        workspace_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    rc = load().psops_gradnorm_create(ctypes.byref(handle), len(sizes), _addresses(grads),
                                      (ctypes.c_int64 * len(sizes))(*sizes), int(grad_type), _ptr(d_workspace),
                                      int(workspace_bytes), int(stream) if stream else None)
    _check(rc, "psops_gradnorm_create")
    return handle


def psops_gradnorm_set_grads(gn, grads) -> None:
    _check(load().psops_gradnorm_set_grads(gn, _addresses(grads)), "psops_gradnorm_set_grads", gn,
           "psops_gradnorm_last_error")


def psops_gradnorm_run(gn, max_norm: float, d_out) -> None:
    _check(load().psops_gradnorm_run(gn, float(max_norm), _ptr(d_out)), "psops_gradnorm_run", gn,
           "psops_gradnorm_last_error")


def psops_gradnorm_set_stream(ctx, stream) -> None:
    _check(load().psops_gradnorm_set_stream(ctx, int(stream) if stream else None), "psops_gradnorm_set_stream", ctx,
           "psops_gradnorm_last_error")


def psops_gradnorm_launch_count(gn) -> int:
    return int(load().psops_gradnorm_launch_count(gn))


def psops_gradnorm_destroy(gn) -> None:
    _check(load().psops_gradnorm_destroy(gn), "psops_gradnorm_destroy")


def psops_xent_workspace_bytes(cfg: psops_xent_config) -> int:
    return int(load().psops_xent_workspace_bytes(ctypes.byref(cfg)))


def psops_xent_create(cfg, d_workspace, workspace_bytes=None, stream=None):
    handle = _vp()
    if workspace_bytes is None:
        workspace_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    rc = load().psops_xent_create(ctypes.byref(handle), ctypes.byref(cfg), _ptr(d_workspace), int(workspace_bytes),
                                  int(stream) if stream else None)
    _check(rc, "psops_xent_create")
    return handle


def psops_xent_forward(x, d_h, h_ld, d_w, w_ld, d_targets, tokens, reduction, d_loss, d_rows, d_lse) -> None:
    _check(load().psops_xent_forward(x, _ptr(d_h), int(h_ld), _ptr(d_w), int(w_ld), _ptr(d_targets), int(tokens),
                                     int(reduction), _ptr(d_loss), _ptr(d_rows), _ptr(d_lse)),
           "psops_xent_forward", x, "psops_xent_last_error")


def psops_xent_backward(x, d_h, h_ld, d_w, w_ld, d_targets, tokens, d_lse, d_rows, d_grad, reduction, d_dh, dh_ld,
                        d_dw, dw_ld) -> None:
    _check(load().psops_xent_backward(x, _ptr(d_h), int(h_ld), _ptr(d_w), int(w_ld), _ptr(d_targets), int(tokens),
                                      _ptr(d_lse), _ptr(d_rows), _ptr(d_grad), int(reduction), _ptr(d_dh), int(dh_ld),
                                      _ptr(d_dw), int(dw_ld)),
           "psops_xent_backward", x, "psops_xent_last_error")


def psops_xent_set_stream(ctx, stream) -> None:
    _check(load().psops_xent_set_stream(ctx, int(stream) if stream else None), "psops_xent_set_stream", ctx,
           "psops_xent_last_error")


def psops_xent_launch_count(x) -> int:
    return int(load().psops_xent_launch_count(x))


def psops_xent_destroy(x) -> None:
    _check(load().psops_xent_destroy(x), "psops_xent_destroy")


def psops_attention_workspace_bytes(cfg: psops_attention_config) -> int:
    return int(load().psops_attention_workspace_bytes(ctypes.byref(cfg)))


def psops_attention_create(cfg, d_workspace, workspace_bytes=None, stream=None):
    handle = _vp()
    if workspace_bytes is None:
        workspace_bytes = d_workspace.numel() * d_workspace.element_size() if d_workspace is not None else 0
    rc = load().psops_attention_create(ctypes.byref(handle), ctypes.byref(cfg), _ptr(d_workspace), int(workspace_bytes),
                                       int(stream) if stream else None)
    _check(rc, "psops_attention_create")
    return handle


def psops_attention_forward(a, q, k, v, d_offsets, sequences, tokens, d_bias, bias_type, out, d_lse, zero_rest) -> None:
    """q, k, v, out: psops_heads."""
    _check(load().psops_attention_forward(a, q, k, v, _ptr(d_offsets), int(sequences), int(tokens), _ptr(d_bias),
                                          int(bias_type), out, _ptr(d_lse), int(zero_rest)),
           "psops_attention_forward", a, "psops_attention_last_error")


def psops_attention_backward(a, q, k, v, d_offsets, sequences, tokens, d_bias, bias_type, out, d_lse, grad, dq, dk, dv,
                             d_dbias, zero_rest) -> None:
    """q, k, v, out, grad and, where not None, dq, dk, dv: psops_heads."""
    _check(load().psops_attention_backward(a, q, k, v, _ptr(d_offsets), int(sequences), int(tokens), _ptr(d_bias),
                                           int(bias_type), out, _ptr(d_lse), grad, dq, dk, dv, _ptr(d_dbias),
                                           int(zero_rest)),
           "psops_attention_backward", a, "psops_attention_last_error")


def psops_attention_set_stream(ctx, stream) -> None:
    _check(load().psops_attention_set_stream(ctx, int(stream) if stream else None), "psops_attention_set_stream", ctx,
           "psops_attention_last_error")


def psops_attention_launch_count(a) -> int:
    return int(load().psops_attention_launch_count(a))


def psops_attention_destroy(a) -> None:
    _check(load().psops_attention_destroy(a), "psops_attention_destroy")


def psops_keep_create(stream=None):
    handle = _vp()
    _check(load().psops_keep_create(ctypes.byref(handle), int(stream) if stream else None), "psops_keep_create")
    return handle


def psops_keep_pack(k, type_, rows, cols, d_x, x_ld, d_codes, d_scales) -> None:
    _check(load().psops_keep_pack(k, type_, rows, cols, _ptr(d_x), x_ld, _ptr(d_codes), _ptr(d_scales)),
           "psops_keep_pack", k, "psops_keep_last_error")


def psops_keep_unpack(k, type_, rows, cols, d_codes, d_scales, d_x, x_ld) -> None:
    _check(load().psops_keep_unpack(k, type_, rows, cols, _ptr(d_codes), _ptr(d_scales), _ptr(d_x), x_ld),
           "psops_keep_unpack", k, "psops_keep_last_error")


def psops_keep_activate(k, kind, type_, rows, cols, d_a, a_ld, d_b, b_ld, d_y, y_ld, d_a_codes, d_a_scales, d_b_codes,
                         d_b_scales) -> None:
    _check(load().psops_keep_activate(k, kind, type_, rows, cols, _ptr(d_a), a_ld, _ptr(d_b), b_ld, _ptr(d_y), y_ld,
                                       _ptr(d_a_codes), _ptr(d_a_scales), _ptr(d_b_codes), _ptr(d_b_scales)),
           "psops_keep_activate", k, "psops_keep_last_error")


def psops_keep_activate_backward(k, kind, type_, rows, cols, d_a_codes, d_a_scales, d_b_codes, d_b_scales, d_dy, dy_ld,
                                  d_da, da_ld, d_db, db_ld, d_y, y_ld) -> None:
    _check(load().psops_keep_activate_backward(k, kind, type_, rows, cols, _ptr(d_a_codes), _ptr(d_a_scales),
                                                _ptr(d_b_codes), _ptr(d_b_scales), _ptr(d_dy), dy_ld, _ptr(d_da), da_ld,
                                                _ptr(d_db), db_ld, _ptr(d_y), y_ld),
           "psops_keep_activate_backward", k, "psops_keep_last_error")


def psops_keep_set_stream(ctx, stream) -> None:
    _check(load().psops_keep_set_stream(ctx, int(stream) if stream else None), "psops_keep_set_stream", ctx,
           "psops_keep_last_error")


def psops_keep_launch_count(k) -> int:
    return int(load().psops_keep_launch_count(k))


def psops_keep_destroy(k) -> None:
    _check(load().psops_keep_destroy(k), "psops_keep_destroy")


# ---- convenience holder of the tensors a context borrows ------------------

class Swarm:
    """Owns the device tensors (torch) that one psops context borrows and
    forwards to the C entry points.  No arithmetic happens here."""

    def __init__(self, x, v, pbest, *, N=None, m_max, m_min, t_max=1, c1, c2, seed, flags=0,
                 stream=None, k_first=0, K_total=0):
        for t in (x, v, pbest):
            assert t.is_cuda and t.dtype == torch.float32 and t.dim() == 2 and t.stride(1) == 1
        self.x, self.v, self.pbest = x, v, pbest
        self.K = x.shape[0]
        self.ld = x.stride(0)
        assert v.stride(0) == self.ld and pbest.stride(0) == self.ld
        self.N = int(N) if N is not None else x.shape[1]
        self.cfg = make_config(self.K, self.N, self.ld, m_max=m_max, m_min=m_min, t_max=t_max,
                               c1=c1, c2=c2, seed=seed, flags=flags, k_first=k_first, K_total=K_total)
        self.Kt = K_total if K_total else self.K
        nbytes = psops_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise PsopsError(PSOPS_EINVAL, "psops_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(x.device).cuda_stream
        self._refs = []
        self.ctx = psops_create(self.cfg, x, v, pbest, self.workspace, nbytes, self.stream)

    def set_losses(self, losses):
        if isinstance(losses, (list, tuple)):
            losses = np.asarray(losses, dtype=np.float32)
        if isinstance(losses, np.ndarray):
            losses = np.ascontiguousarray(losses, dtype=np.float32)
        count = losses.size if isinstance(losses, np.ndarray) else losses.numel()
        assert count == self.Kt
        self._loss_ref = losses        # a device buffer is read by the next sync: keep it alive
        psops_set_losses(self.ctx, losses)

    def sync(self, t_iter=0, lam=1.0):
        psops_sync(self.ctx, t_iter, lam)

    def sync_host(self, h_x_in, h_losses, t_iter=0, lam=1.0, h_x_out=None):
        h_x_out = h_x_in if h_x_out is None else h_x_out
        h_losses = np.ascontiguousarray(h_losses, dtype=np.float32) \
            if not isinstance(h_losses, torch.Tensor) else h_losses
        psops_sync_host(self.ctx, h_x_in, _ld_of(h_x_in), h_losses, t_iter, lam, h_x_out, _ld_of(h_x_out))

    def average(self):
        psops_average(self.ctx)

    def info(self):
        return psops_sync_info(self.ctx, self.Kt)

    def shard_select(self) -> int:
        return psops_shard_select(self.ctx)

    def shard_update(self, d_gbest_row, t_iter=0, lam=1.0):
        psops_shard_update(self.ctx, t_iter, lam, d_gbest_row)

    def shard_update_range(self, d_gbest_row, first_elem, last_elem, t_iter=0, lam=1.0):
        psops_shard_update_range(self.ctx, t_iter, lam, d_gbest_row, first_elem, last_elem)

    def ssgd(self, d_grad, alpha):
        psops_ssgd(self.ctx, d_grad, d_grad.stride(0), alpha)

    def history(self):
        return psops_get_history(self.ctx)

    def losses(self) -> np.ndarray:
        out = np.zeros(self.Kt, dtype=np.float32)
        psops_get_losses(self.ctx, out)
        return out

    def row(self, which, k=0) -> np.ndarray:
        out = np.empty(self.N, dtype=np.float32)
        psops_get_weights(self.ctx, which, k, out)
        return out

    def set_quadratic(self, dvec, tvec):
        self._refs = [dvec, tvec]
        psops_set_quadratic(self.ctx, dvec, tvec)

    def eval_quadratic(self):
        psops_eval_quadratic(self.ctx)

    def state(self):
        return psops_get_state(self.ctx, self.Kt)

    def set_state(self, step, pbest_loss):
        psops_set_state(self.ctx, step, pbest_loss)

    @property
    def launches(self) -> int:
        return psops_launch_count(self.ctx)

    def close(self):
        ctx, self.ctx = self.ctx, None             # it is freed even where the entry reports an error
        if ctx is not None:
            psops_destroy(ctx)

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass


def _ld_of(buf) -> int:
    if isinstance(buf, torch.Tensor):
        return buf.stride(0)
    return buf.strides[0] // buf.itemsize
