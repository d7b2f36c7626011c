"""Python binding of libchoco (the CHOCO-Gossip / CHOCO-SGD step on one B200).

Argument marshalling only: every function forwards to the C entry point of the same
name in ``libchoco.so`` (declared in ``include/choco.h``); all arithmetic runs in the
library's CUDA kernels.  PyTorch tensors are used for device memory and streams.
There is no CPU path: if the library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libchoco.so")

Q_IDENTITY, Q_TOPK, Q_RANDK, Q_QSGD, Q_SIGN = 0, 1, 2, 3, 4
Q_KINDS = {"identity": Q_IDENTITY, "topk": Q_TOPK, "randk": Q_RANDK, "qsgd": Q_QSGD, "sign": Q_SIGN}

EXPORTS = [
    "choco_init", "choco_destroy", "choco_gossip_step", "choco_sgd_step",
    "choco_sgd_momentum_step", "choco_sgd_step_host", "choco_invalidate", "choco_set_carry",
    "choco_get_step", "choco_set_graphs", "choco_set_rescue", "choco_set_select_blocks", "choco_set_nesterov",
    "choco_set_step", "choco_message_bytes", "choco_get_message", "choco_read_message",
    "choco_consensus_error", "choco_consensus_error_noalloc",
    "choco_get_stats", "choco_profile_enable", "choco_profile_set_stride", "choco_profile_read", "choco_strerror",
    "choco_last_cuda_error", "choco_debug_set_wait_polls", "choco_debug_set_candidate_slot",
    "choco_layers_init", "choco_layers_destroy", "choco_layers_gossip_step", "choco_layers_sgd_step",
    "choco_layers_sgd_momentum_step", "choco_layers_message_bytes", "choco_layers_get_layer",
    "choco_layers_invalidate", "choco_layers_set_step", "choco_layers_set_nesterov", "choco_layers_set_graphs", "choco_layers_combined_steps",
    "choco_embedding_init", "choco_embedding_destroy", "choco_embedding_forward", "choco_embedding_backward",
    "choco_adamw_init", "choco_adamw_destroy", "choco_adamw_state_size", "choco_adamw_set_grads", "choco_adamw_grad_norm",
    "choco_adamw_set_rounding", "choco_adamw_step", "choco_adamw_read_state", "choco_adamw_get_steps", "choco_adamw_set_steps",
    "choco_muon_init", "choco_muon_destroy", "choco_muon_state_size", "choco_muon_set_grads", "choco_muon_step", "choco_muon_orthogonalize",
    "choco_muon_status", "choco_debug_muon_set_wait_polls",
    "choco_group_norm_init", "choco_group_norm_destroy", "choco_group_norm_forward", "choco_group_norm_backward",
]

DTYPES = {"float32": 0, "bfloat16": 1, "float16": 2}   # choco_dtype


ERR_TIMEOUT = -8


class ChocoError(RuntimeError):
    """A libchoco call returned a negative status; `code` holds it."""

    def __init__(self, message: str, code: int = 0):
        super().__init__(message)
        self.code = code


class choco_params(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("s", ctypes.c_int32), ("bucket", ctypes.c_int32),
                ("qsgd_biased", ctypes.c_int32), ("k", ctypes.c_int64)]


class choco_stats(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_uint64), ("prepared_rows", ctypes.c_uint64),
                ("recompressed_rows", ctypes.c_uint64), ("exact_rows", ctypes.c_uint64),
                ("kernel_launches", ctypes.c_uint64), ("device_timeouts", ctypes.c_uint64),
                ("graph_replays", ctypes.c_uint64), ("rescued_rows", ctypes.c_uint64)]


class choco_embedding_params(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("scale", ctypes.c_float), ("vocab", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("table_row", ctypes.c_int64), ("table_ld", ctypes.c_int64), ("max_tokens", ctypes.c_int64),
                ("padding", ctypes.c_int64)]


class choco_adamw_params(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("state_bits", ctypes.c_int32), ("groups", ctypes.c_int32)]


class choco_muon_params(ctypes.Structure):
    _fields_ = [("beta", ctypes.c_double), ("a", ctypes.c_double), ("b", ctypes.c_double), ("c", ctypes.c_double), ("nesterov", ctypes.c_int32),
                ("steps", ctypes.c_int32), ("products", ctypes.c_int32), ("groups", ctypes.c_int32)]


# choco_adamw_tensor as a numpy record: a list of tensors is an array of these
ADAMW_TENSOR = [("x", "<u8"), ("g", "<u8"), ("copy", "<u8"), ("numel", "<i8"), ("x_dtype", "<i4"), ("g_dtype", "<i4"),
                ("copy_dtype", "<i4"), ("group", "<i4"), ("weight_decay", "<f8"), ("lr_scale", "<f8")]
ADAMW_BLOCK = 256   # elements that share a scale; tensors start on multiples of it in the moments

# choco_muon_matrix likewise
MUON_MATRIX = [("x", "<u8"), ("g", "<u8"), ("copy", "<u8"), ("rows", "<i8"), ("cols", "<i8"), ("x_ld", "<i8"), ("g_ld", "<i8"), ("copy_ld", "<i8"),
               ("x_dtype", "<i4"), ("g_dtype", "<i4"), ("copy_dtype", "<i4"), ("group", "<i4"), ("weight_decay", "<f8"), ("lr_scale", "<f8")]
MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)

ACTIVATIONS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}   # choco_activation


class choco_group_norm_params(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int32), ("groups", ctypes.c_int32), ("channels", ctypes.c_int64), ("max_images", ctypes.c_int64),
                ("eps", ctypes.c_double), ("activation", ctypes.c_int32), ("unused", ctypes.c_int32)]


class choco_pixels(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("worker", ctypes.c_int64), ("image", ctypes.c_int64), ("pixel", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("unused", ctypes.c_int32)]


_lib = None


def load() -> ctypes.CDLL:
    """dlopen libchoco.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ChocoError(f"{LIB_PATH} is missing: run `python -m paper_1907_09356_b200.build` "
                             "(there is no fallback implementation)")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, u64, f32 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64,
                                  ctypes.c_float)
        lib.choco_init.argtypes = [ctypes.POINTER(vp), i32, i64, i64, vp, vp, vp,
                                   ctypes.POINTER(choco_params), u64]
        lib.choco_destroy.argtypes = [vp]
        lib.choco_gossip_step.argtypes = [vp, vp, vp, vp, f32, vp]
        lib.choco_sgd_step.argtypes = [vp, vp, vp, vp, vp, f32, f32, vp]
        lib.choco_sgd_momentum_step.argtypes = [vp, vp, vp, vp, vp, vp, f32, f32, f32, f32, vp]
        lib.choco_sgd_step_host.argtypes = [vp, vp, vp, vp, vp, f32, f32, vp]
        lib.choco_invalidate.argtypes = [vp]
        lib.choco_set_carry.argtypes = [vp, i32]
        lib.choco_set_graphs.argtypes = [vp, i32]
        lib.choco_set_rescue.argtypes = [vp, i32]
        lib.choco_set_select_blocks.argtypes = [vp, i32]
        lib.choco_set_nesterov.argtypes = [vp, i32]
        lib.choco_debug_set_candidate_slot.argtypes = [vp, i32]
        lib.choco_get_step.argtypes = [vp, ctypes.POINTER(u64)]
        lib.choco_set_step.argtypes = [vp, u64]
        lib.choco_message_bytes.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        lib.choco_get_message.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(i64)]
        lib.choco_read_message.argtypes = [vp, i32, i32, vp, i64, ctypes.POINTER(i64), vp]
        lib.choco_consensus_error.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_double), vp]
        lib.choco_consensus_error_noalloc.argtypes = [vp, i32, i64, i64, vp, vp]
        lib.choco_get_stats.argtypes = [vp, ctypes.POINTER(choco_stats), vp]
        lib.choco_profile_enable.argtypes = [vp, i32]
        lib.choco_profile_set_stride.argtypes = [vp, i32]
        lib.choco_profile_read.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_double), vp]
        lib.choco_strerror.argtypes = [ctypes.c_int]
        lib.choco_strerror.restype = ctypes.c_char_p
        lib.choco_last_cuda_error.argtypes = [vp]
        lib.choco_debug_set_wait_polls.argtypes = [vp, ctypes.c_uint32]
        lib.choco_layers_init.argtypes = [ctypes.POINTER(vp), i32, i32, vp, i64, vp, vp, vp,
                                          ctypes.POINTER(choco_params), i64, i64, u64]
        lib.choco_layers_destroy.argtypes = [vp]
        lib.choco_layers_gossip_step.argtypes = [vp, vp, vp, vp, f32, vp]
        lib.choco_layers_sgd_step.argtypes = [vp, vp, vp, vp, vp, f32, f32, vp]
        lib.choco_layers_sgd_momentum_step.argtypes = [vp, vp, vp, vp, vp, vp, f32, f32, f32, f32, vp]
        lib.choco_layers_message_bytes.argtypes = [vp, ctypes.POINTER(i64), ctypes.POINTER(i64)]
        lib.choco_layers_get_layer.argtypes = [vp, i32, ctypes.POINTER(vp), ctypes.POINTER(i64),
                                               ctypes.POINTER(i64)]
        lib.choco_layers_invalidate.argtypes = [vp]
        lib.choco_layers_set_step.argtypes = [vp, u64]
        lib.choco_layers_set_nesterov.argtypes = [vp, i32]
        lib.choco_layers_set_graphs.argtypes = [vp, i32, ctypes.POINTER(u64)]
        lib.choco_layers_combined_steps.argtypes = [vp, ctypes.POINTER(u64)]
        lib.choco_embedding_init.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(choco_embedding_params)]
        lib.choco_embedding_destroy.argtypes = [vp]
        lib.choco_embedding_forward.argtypes = [vp, vp, i32, vp, i32, i64, i64, vp, i32, i64, i64, vp]
        lib.choco_embedding_backward.argtypes = [vp, vp, i32, i64, i64, vp, i32, i64, i64, vp, i32, i32, vp]
        f64 = ctypes.c_double
        lib.choco_adamw_init.argtypes = [ctypes.POINTER(vp), i32, vp, ctypes.POINTER(choco_adamw_params)]
        lib.choco_adamw_destroy.argtypes = [vp]
        lib.choco_adamw_state_size.argtypes = [vp, ctypes.POINTER(i64), vp]
        lib.choco_adamw_set_grads.argtypes = [vp, vp, vp]
        lib.choco_adamw_set_rounding.argtypes = [vp, i32, u64]
        lib.choco_adamw_grad_norm.argtypes = [vp, f32, f32, vp, vp, vp]
        lib.choco_adamw_step.argtypes = [vp, vp, vp, vp, vp, f64, vp, vp]
        lib.choco_adamw_read_state.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp]
        lib.choco_adamw_get_steps.argtypes = [vp, vp, vp]
        lib.choco_adamw_set_steps.argtypes = [vp, vp, vp]
        lib.choco_muon_init.argtypes = [ctypes.POINTER(vp), i32, vp, ctypes.POINTER(choco_muon_params)]
        lib.choco_muon_destroy.argtypes = [vp]
        lib.choco_muon_state_size.argtypes = [vp, ctypes.POINTER(i64), vp]
        lib.choco_muon_set_grads.argtypes = [vp, vp, vp]
        lib.choco_muon_step.argtypes = [vp, vp, f64, vp, vp]
        lib.choco_muon_orthogonalize.argtypes = [vp, vp]
        lib.choco_muon_status.argtypes = [vp, vp]
        lib.choco_debug_muon_set_wait_polls.argtypes = [vp, ctypes.c_uint32]
        px = ctypes.POINTER(choco_pixels)
        lib.choco_group_norm_init.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(choco_group_norm_params)]
        lib.choco_group_norm_destroy.argtypes = [vp]
        lib.choco_group_norm_forward.argtypes = [vp, i64, i64, px, px, vp, vp, i64, i32, vp, vp, vp]
        lib.choco_group_norm_backward.argtypes = [vp, i64, i64, px, px, px, vp, vp, i64, i32, vp, vp, vp, vp, i64, i32, i32, vp]
        for name in EXPORTS:
            if name not in ("choco_strerror",):
                getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


def _check(rc: int, ctx=None) -> None:
    if rc != 0:
        lib = load()
        msg = lib.choco_strerror(rc).decode()
        if ctx is not None and rc == -4:
            msg += f" (cudaError {lib.choco_last_cuda_error(ctx)})"
        raise ChocoError(f"libchoco: {msg} [{rc}]", rc)


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


_raw_stream = None


def _find_raw_stream():
    """Current stream's handle by device index."""
    global _raw_stream
    import torch
    # the handle itself where torch gives it (0.1 us); its Stream object takes 3 us to make
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        _raw_stream = lambda device: torch.cuda.current_stream(device).cuda_stream  # noqa: E731
    return _raw_stream


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = (_raw_stream or _find_raw_stream())(torch.cuda.current_device())
        return stream or None
    return stream.cuda_stream or None


def _stream_of(stream, device: int) -> Optional[int]:
    """The same for a call whose tensors are known to be on `device`."""
    if stream is None:
        return (_raw_stream or _find_raw_stream())(device) or None
    return stream.cuda_stream or None


def _on_one_device(what: str, *tensors, of: int) -> int:
    """`of`, the index of the handle's GPU, which all of them are on."""
    for t in tensors:
        if t.get_device() != of:
            raise ChocoError(f"libchoco: {what} must be on one GPU, that of the handle ({of})", -1)
    return of


# --------------------------------------------------------------------------- C names


def choco_init(n: int, d: int, ld: int, w_row_ptr, w_col, w_val, kind, k: int = 0, s: int = 16,
               bucket: int = 0, qsgd_biased: bool = True, seed: int = 0):
    """W as host numpy arrays (int32, int32, float32).  Returns the context handle."""
    import numpy as np
    rp = np.ascontiguousarray(w_row_ptr, dtype=np.int32)
    col = np.ascontiguousarray(w_col, dtype=np.int32)
    val = np.ascontiguousarray(w_val, dtype=np.float32)
    p = choco_params(Q_KINDS[kind] if isinstance(kind, str) else int(kind), int(s), int(bucket),
                     1 if qsgd_biased else 0, int(k))
    ctx = ctypes.c_void_p()
    _check(load().choco_init(ctypes.byref(ctx), n, d, ld, rp.ctypes.data, col.ctypes.data,
                             val.ctypes.data, ctypes.byref(p), seed))
    return ctx


def choco_destroy(ctx) -> None:
    _check(load().choco_destroy(ctx))


def choco_gossip_step(ctx, X, Xhat, S, gamma: float, stream=None) -> None:
    _check(load().choco_gossip_step(ctx, _ptr(X), _ptr(Xhat), _ptr(S), gamma, _stream(stream)), ctx)


def choco_sgd_step(ctx, X, Xhat, S, G, eta: float, gamma: float, stream=None) -> None:
    _check(load().choco_sgd_step(ctx, _ptr(X), _ptr(Xhat), _ptr(S), _ptr(G), eta, gamma,
                                 _stream(stream)), ctx)


def choco_sgd_momentum_step(ctx, X, Xhat, S, G, M, eta: float, gamma: float, lam: float,
                            beta: float, stream=None) -> None:
    _check(load().choco_sgd_momentum_step(ctx, _ptr(X), _ptr(Xhat), _ptr(S), _ptr(G), _ptr(M), eta,
                                          gamma, lam, beta, _stream(stream)), ctx)


def choco_sgd_step_host(ctx, X, Xhat, S, G, eta: float, gamma: float, stream=None) -> None:
    """X, Xhat, S, G: host tensors (CPU torch tensors or numpy arrays), updated in place."""
    def hp(a):
        if a is None:
            return None
        return a.data_ptr() if hasattr(a, "data_ptr") else a.ctypes.data
    _check(load().choco_sgd_step_host(ctx, hp(X), hp(Xhat), hp(S), hp(G), eta, gamma,
                                      _stream(stream)), ctx)


def choco_invalidate(ctx) -> None:
    _check(load().choco_invalidate(ctx))


def choco_set_carry(ctx, enable: bool) -> None:
    _check(load().choco_set_carry(ctx, 1 if enable else 0))


def choco_set_graphs(ctx, enable: bool) -> None:
    _check(load().choco_set_graphs(ctx, 1 if enable else 0), ctx)


def choco_set_rescue(ctx, enable: bool) -> None:
    _check(load().choco_set_rescue(ctx, 1 if enable else 0), ctx)


def choco_set_select_blocks(ctx, blocks: int) -> None:
    _check(load().choco_set_select_blocks(ctx, blocks), ctx)


def choco_debug_set_candidate_slot(ctx, slot: int) -> None:
    _check(load().choco_debug_set_candidate_slot(ctx, slot), ctx)


def choco_set_nesterov(ctx, enable: bool) -> None:
    _check(load().choco_set_nesterov(ctx, 1 if enable else 0), ctx)


def choco_get_step(ctx) -> int:
    t = ctypes.c_uint64()
    _check(load().choco_get_step(ctx, ctypes.byref(t)))
    return t.value


def choco_set_step(ctx, t: int) -> None:
    _check(load().choco_set_step(ctx, t))


def choco_message_bytes(ctx) -> tuple[int, int]:
    a, b = ctypes.c_int64(), ctypes.c_int64()
    _check(load().choco_message_bytes(ctx, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def choco_get_message(ctx, worker: int, plane: int) -> tuple[int, int]:
    """(device pointer, size in bytes) of one plane of a worker's last message."""
    p, nb = ctypes.c_void_p(), ctypes.c_int64()
    _check(load().choco_get_message(ctx, worker, plane, ctypes.byref(p), ctypes.byref(nb)))
    return (p.value or 0), nb.value


def choco_read_message(ctx, worker: int, plane: int, stream=None):
    """One plane of a worker's last message, copied to the host as a numpy uint8 array."""
    import numpy as np
    _, size = choco_get_message(ctx, worker, plane)
    out = np.empty(size, dtype=np.uint8)
    nb = ctypes.c_int64()
    if size:
        _check(load().choco_read_message(ctx, worker, plane, out.ctypes.data, size,
                                         ctypes.byref(nb), _stream(stream)), ctx)
    return out


def choco_consensus_error(ctx, X, stream=None) -> float:
    out = ctypes.c_double()
    _check(load().choco_consensus_error(ctx, _ptr(X), ctypes.byref(out), _stream(stream)), ctx)
    return out.value


def choco_consensus_error_noalloc(X, n: int, d: int, ld: int, out_dev, stream=None) -> None:
    """Consensus distance into `out_dev` (a device tensor holding one float64) without any
    allocation by the library: for callers that must not allocate device memory, e.g. while
    a pool or a capture session owns allocation.  d is limited to 4 194 304; asynchronous."""
    _check(load().choco_consensus_error_noalloc(_ptr(X), n, d, ld, _ptr(out_dev), _stream(stream)))


def choco_get_stats(ctx, stream=None) -> dict:
    st = choco_stats()
    _check(load().choco_get_stats(ctx, ctypes.byref(st), _stream(stream)), ctx)
    return {f: getattr(st, f) for f, _ in choco_stats._fields_}


def choco_debug_set_wait_polls(ctx, polls: int) -> None:
    """Test hook: polls a kernel spends on its first wait for staged copies (0 = give up at once)."""
    _check(load().choco_debug_set_wait_polls(ctx, polls), ctx)


def choco_profile_enable(ctx, max_steps: int) -> None:
    _check(load().choco_profile_enable(ctx, max_steps), ctx)


def choco_profile_set_stride(ctx, stride: int) -> None:
    _check(load().choco_profile_set_stride(ctx, stride), ctx)


def choco_profile_read(ctx, stream=None) -> tuple[int, float]:
    """(steps recorded, total milliseconds spent in the update kernel over them)."""
    n, ms = ctypes.c_int32(), ctypes.c_double()
    _check(load().choco_profile_read(ctx, ctypes.byref(n), ctypes.byref(ms), _stream(stream)), ctx)
    return n.value, ms.value


def choco_layers_init(n: int, layer_off, ld: int, w_row_ptr, w_col, w_val, kind, a_num: int = 1,
                      a_den: int = 1, s: int = 16, bucket: int = 0, qsgd_biased: bool = True,
                      seed: int = 0):
    """Per-layer compression: layer_off is a host array of n_layers + 1 offsets; top-k and
    random-k keep max(1, floor(a_num / a_den * d_l)) entries of layer l."""
    import numpy as np
    off = np.ascontiguousarray(layer_off, dtype=np.int64)
    rp = np.ascontiguousarray(w_row_ptr, dtype=np.int32)
    col = np.ascontiguousarray(w_col, dtype=np.int32)
    val = np.ascontiguousarray(w_val, dtype=np.float32)
    p = choco_params(Q_KINDS[kind] if isinstance(kind, str) else int(kind), int(s), int(bucket),
                     1 if qsgd_biased else 0, 0)
    h = ctypes.c_void_p()
    _check(load().choco_layers_init(ctypes.byref(h), n, len(off) - 1, off.ctypes.data, ld, rp.ctypes.data,
                                    col.ctypes.data, val.ctypes.data, ctypes.byref(p), a_num, a_den, seed))
    return h


def choco_layers_destroy(layers) -> None:
    _check(load().choco_layers_destroy(layers))


def choco_layers_gossip_step(layers, X, Xhat, S, gamma: float, stream=None) -> None:
    _check(load().choco_layers_gossip_step(layers, _ptr(X), _ptr(Xhat), _ptr(S), gamma, _stream(stream)))


def choco_layers_sgd_step(layers, X, Xhat, S, G, eta: float, gamma: float, stream=None) -> None:
    _check(load().choco_layers_sgd_step(layers, _ptr(X), _ptr(Xhat), _ptr(S), _ptr(G), eta, gamma,
                                        _stream(stream)))


def choco_layers_sgd_momentum_step(layers, X, Xhat, S, G, M, eta: float, gamma: float, lam: float,
                                   beta: float, stream=None) -> None:
    _check(load().choco_layers_sgd_momentum_step(layers, _ptr(X), _ptr(Xhat), _ptr(S), _ptr(G), _ptr(M),
                                                 eta, gamma, lam, beta, _stream(stream)))


def choco_layers_message_bytes(layers) -> tuple[int, int]:
    a, b = ctypes.c_int64(), ctypes.c_int64()
    _check(load().choco_layers_message_bytes(layers, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def choco_layers_get_layer(layers, layer: int):
    """(context handle of the layer, its first coordinate, its length)."""
    c, o, n = ctypes.c_void_p(), ctypes.c_int64(), ctypes.c_int64()
    _check(load().choco_layers_get_layer(layers, layer, ctypes.byref(c), ctypes.byref(o), ctypes.byref(n)))
    return c, o.value, n.value


def choco_layers_set_graphs(layers, enable: int = -1) -> int:
    """Turn the CUDA-graph replay of steady-state steps off (0) / on (1), or leave it (-1);
    returns the number of steps replayed so far."""
    n = ctypes.c_uint64()
    _check(load().choco_layers_set_graphs(layers, enable, ctypes.byref(n)))
    return n.value


def choco_layers_combined_steps(layers) -> int:
    """Step calls so far that were enqueued as launches over all layers at once."""
    n = ctypes.c_uint64()
    _check(load().choco_layers_combined_steps(layers, ctypes.byref(n)))
    return n.value


def choco_layers_invalidate(layers) -> None:
    _check(load().choco_layers_invalidate(layers))


def choco_layers_set_step(layers, t: int) -> None:
    _check(load().choco_layers_set_step(layers, t))


def choco_layers_set_nesterov(layers, enable: bool) -> None:
    _check(load().choco_layers_set_nesterov(layers, 1 if enable else 0))


_dtype_codes: dict = {}    # by torch dtype, filled as they are met
_index_codes: dict = {}


def _dtype(t) -> int:
    """choco_dtype of a tensor (or of a torch dtype)."""
    dtype = getattr(t, "dtype", t)
    code = _dtype_codes.get(dtype)
    if code is None:
        name = str(dtype).rpartition(".")[2]
        if name not in DTYPES:
            raise ChocoError(f"libchoco: {name} arrays are not supported (float32, bfloat16 or float16)", -1)
        code = _dtype_codes[dtype] = DTYPES[name]
    return code


def _index_bits(t) -> int:
    code = _index_codes.get(t.dtype)
    if code is None:
        name = str(t.dtype).rpartition(".")[2]
        if name not in ("int32", "int64"):
            raise ChocoError(f"libchoco: tokens are int32 or int64, not {name}", -1)
        code = _index_codes[t.dtype] = 32 if name == "int32" else 64
    return code


def _token_rows(tokens, rows, n, dim) -> tuple:
    """(tokens per worker, stride of the tokens' rows, strides of `rows` from token to token and from
    worker to worker) for tokens [n, T] and rows [n, T, dim] with unit stride inside their rows."""
    a, b = tokens.shape, rows.shape
    if len(a) == 2 and len(b) == 3 and a[0] == b[0] == n and a[1] == b[1] and b[2] == dim:
        count = a[1]
        ld, one = tokens.stride()
        worker, row, inside = rows.stride()
        if count == 0:
            return 0, ld, b[2], 0
        if (one == 1 or count == 1) and (inside == 1 or b[2] == 1):
            return count, ld, (row if count > 1 else max(b[2], row)), worker
    raise ChocoError(f"libchoco: tokens must be [{n}, T] and the rows [{n}, T, {dim}], both contiguous inside "
                     f"their rows, not {list(a)} and {list(b)}", -1)


class EmbeddingHandle(ctypes.c_void_p):
    """What choco_embedding_init returns: the library's handle, with the device it belongs to and the layout of
    the tables it serves."""

    def describe(self, device: int, n: int, vocab: int, dim: int, table_row: int, table_ld: int) -> None:
        self.device, self.n, self.vocab, self.dim = device, n, vocab, dim
        self.table_row = table_row or dim
        self.table_ld = table_ld or vocab * self.table_row
        self.table_span = (vocab - 1) * self.table_row + dim      # elements from a table's first to its last
        self.row_strides = (self.table_ld, 1)


def _check_table(emb, what: str, t) -> None:
    """The arrays whose address alone goes to the library hold all n tables, where the handle says: rows of X or G
    [n, >= span], tables [n, vocab, dim], one table [vocab, dim], or the elements in a row."""
    shape, strides, n = t.shape, t.stride(), emb.n
    if strides == emb.row_strides and shape[0] >= n and shape[1] >= emb.table_span:
        return                                                    # rows of X or G, as nearly all are
    k = len(shape)
    if k == 2:
        if shape[0] >= n and shape[1] >= emb.table_span and (strides[1] == 1 or shape[1] == 1) and (strides[0] == emb.table_ld or n == 1):
            return
        if n == 1 and shape[0] >= emb.vocab and shape[1] >= emb.dim and strides == (emb.table_row, 1):
            return
    elif k == 3:
        if shape[0] >= n and shape[1] >= emb.vocab and shape[2] >= emb.dim and (strides[0] == emb.table_ld or n == 1) and (
                strides[1] == emb.table_row or emb.vocab == 1) and (strides[2] == 1 or emb.dim == 1):
            return
    elif k == 1 and shape[0] >= (n - 1) * emb.table_ld + emb.table_span and strides[0] == 1:
        return
    raise ChocoError(f"libchoco: {what} of {list(shape)}, strides {list(strides)}, does not hold {n} tables of {emb.vocab} x {emb.dim} with rows "
                     f"{emb.table_row} and tables {emb.table_ld} elements apart", -1)


def choco_embedding_init(n: int, vocab: int, dim: int, max_tokens: int, table_row: int = 0, table_ld: int = 0,
                         scale: float = 1.0, padding: int = -1):
    """Handle for the token tables of n workers (see choco.h) on the current device; max_tokens = 0 serves lookups only."""
    import torch
    p = choco_embedding_params(n, scale, vocab, dim, table_row, table_ld, max_tokens, padding)
    h = EmbeddingHandle()
    _check(load().choco_embedding_init(ctypes.byref(h), ctypes.byref(p)))
    h.describe(torch.cuda.current_device(), n, vocab, dim, table_row, table_ld)
    return h


def choco_embedding_destroy(emb) -> None:
    _check(load().choco_embedding_destroy(emb))


def choco_embedding_forward(emb, table, tokens, out, stream=None, n=None, dim=None) -> None:
    """out[i, t] = scale * table_i[tokens[i, t]].  `table` is a tensor that starts at worker 0's first
    row; tokens [n, T] int32 or int64; out [n, T, dim].  n and dim, if given, are the handle's."""
    if (n or dim) and ((n or emb.n) != emb.n or (dim or emb.dim) != emb.dim):
        raise ChocoError(f"libchoco: the handle is for n = {emb.n}, dim = {emb.dim}", -1)
    count, tokens_ld, row, ld = _token_rows(tokens, out, emb.n, emb.dim)
    device = _on_one_device("table, tokens and out", out, tokens, table, of=emb.device)
    _check_table(emb, "a table", table)
    _check(load().choco_embedding_forward(emb, table.data_ptr(), _dtype(table), tokens.data_ptr(), _index_bits(tokens), count,
                                          tokens_ld, out.data_ptr(), _dtype(out), row, ld, _stream_of(stream, device)))


def choco_embedding_backward(emb, tokens, dout, grad, accumulate: bool = False, stream=None, n=None, dim=None) -> None:
    """grad_i[r] (+)= scale * sum of dout[i, t] over the t with tokens[i, t] = r, in the table's layout."""
    if (n or dim) and ((n or emb.n) != emb.n or (dim or emb.dim) != emb.dim):
        raise ChocoError(f"libchoco: the handle is for n = {emb.n}, dim = {emb.dim}", -1)
    count, tokens_ld, row, ld = _token_rows(tokens, dout, emb.n, emb.dim)
    device = _on_one_device("tokens, dout and grad", grad, tokens, dout, of=emb.device)
    _check_table(emb, "a grad", grad)
    _check(load().choco_embedding_backward(emb, tokens.data_ptr(), _index_bits(tokens), count, tokens_ld, dout.data_ptr(),
                                           _dtype(dout), row, ld, grad.data_ptr(), _dtype(grad), 1 if accumulate else 0,
                                           _stream_of(stream, device)))


class AdamWHandle(ctypes.c_void_p):
    """What choco_adamw_init returns: the library's handle, with the device it belongs to and the sizes of what its
    calls take."""

    def describe(self, device: int, n_tensors: int, groups: int, state_bits: int, elements: int) -> None:
        self.device, self.n_tensors, self.groups, self.state_bits, self.elements = device, n_tensors, groups, state_bits, elements

    def state_arrays(self) -> list:
        """(type, length) of m, v and, with 8-bit moments, their scales."""
        if self.state_bits == 32:
            return [("float32", self.elements)] * 2
        scales = ("float32", self.elements // ADAMW_BLOCK)
        return [("int8", self.elements), ("uint8", self.elements), scales, scales]


def _check_groups(opt, what: str, *tensors) -> None:
    """Arrays of one float32 per group."""
    for t in tensors:
        if t.get_device() != opt.device or _dtype(t) != 0 or t.numel() < opt.groups or not t.is_contiguous():
            raise ChocoError(f"libchoco: {what} must be contiguous float32 with one element for each of {opt.groups} groups, on GPU {opt.device}, "
                             f"not {t.dtype} {list(t.shape)} on {t.device}", -1)


def _check_states(opt, states, need: bool = True) -> None:
    """Moments as the handle's calls take them: (m, v) or (m, v, m_scale, v_scale), all of them if `need`."""
    want = opt.state_arrays()
    got = [None if a is None else (str(a.dtype).rpartition(".")[2], a.numel()) for a in states]
    good = len(got) >= len(want) and not any(got[len(want):])
    for a, g, w in zip(states, got, want):
        good = good and (g is None and (not need or opt.elements == 0) or g == w and a.is_contiguous() and a.get_device() == opt.device)
    if not good:
        raise ChocoError(f"libchoco: the moments must be contiguous arrays of {want} on GPU {opt.device}, not {got} on "
                         f"{[str(a.device) for a in states if a is not None]}", -1)


def choco_adamw_init(tensors, groups: int = 1, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                     state_bits: int = 32):
    """tensors: numpy array of ADAMW_TENSOR records (see adamw_layer_tensors), on the current device."""
    import numpy as np
    import torch
    t = np.ascontiguousarray(tensors, dtype=ADAMW_TENSOR)
    p = choco_adamw_params(beta1, beta2, eps, state_bits, groups)
    h, e = AdamWHandle(), ctypes.c_int64()
    _check(load().choco_adamw_init(ctypes.byref(h), len(t), t.ctypes.data if len(t) else None, ctypes.byref(p)))
    _check(load().choco_adamw_state_size(h, ctypes.byref(e), None))
    h.describe(torch.cuda.current_device(), len(t), groups, state_bits, e.value)
    return h


def choco_adamw_destroy(opt) -> None:
    _check(load().choco_adamw_destroy(opt))


def choco_adamw_state_size(opt, n_tensors: int = 0):
    """(elements of the moments, first element of every tensor: an int64 array of n_tensors, all of the list)."""
    import numpy as np
    if n_tensors not in (0, opt.n_tensors):
        raise ChocoError(f"libchoco: the list has {opt.n_tensors} tensors, not {n_tensors}", -1)
    e = ctypes.c_int64()
    off = np.zeros(n_tensors, dtype=np.int64)
    _check(load().choco_adamw_state_size(opt, ctypes.byref(e), off.ctypes.data if n_tensors else None))
    return e.value, off


def choco_adamw_set_grads(opt, pointers, stream=None) -> None:
    """New gradient addresses, one per tensor of the list."""
    import numpy as np
    g = np.ascontiguousarray(pointers, dtype=np.uint64)
    if g.shape != (opt.n_tensors,):
        raise ChocoError(f"libchoco: one address for each of {opt.n_tensors} tensors", -1)
    _check(load().choco_adamw_set_grads(opt, g.ctypes.data, _stream_of(stream, opt.device)))


def choco_adamw_set_rounding(opt, random: bool, seed: int = 0) -> None:
    """8-bit codes to the nearest, or at random with the right expected value (see choco.h)."""
    _check(load().choco_adamw_set_rounding(opt, 1 if random else 0, seed))


def choco_adamw_grad_norm(opt, max_norm: float, norm, factor, unscale: float = 1.0, stream=None) -> None:
    _check_groups(opt, "norm and factor", norm, factor)
    _check(load().choco_adamw_grad_norm(opt, max_norm, unscale, norm.data_ptr(), factor.data_ptr(), _stream_of(stream, opt.device)))


def choco_adamw_step(opt, m, v, m_scale, v_scale, lr: float, factor=None, stream=None) -> None:
    _check_states(opt, (m, v, m_scale, v_scale))
    _adamw_step(opt, m, v, m_scale, v_scale, lr, factor, stream)


def _adamw_step(opt, m, v, m_scale, v_scale, lr, factor, stream) -> None:
    """The step with moments that have been checked."""
    if factor is not None:
        _check_groups(opt, "factor", factor)
    _check(load().choco_adamw_step(opt, _ptr(m), _ptr(v), _ptr(m_scale), _ptr(v_scale), lr, _ptr(factor), _stream_of(stream, opt.device)))


def choco_adamw_read_state(opt, m, v, m_scale, v_scale, m_out, v_out, stream=None) -> None:
    """The values of the moments; m_out and v_out (either may be None) have one type."""
    _check_states(opt, (m, v, m_scale, v_scale), need=False)
    _adamw_read_state(opt, m, v, m_scale, v_scale, m_out, v_out, stream)


def _adamw_read_state(opt, m, v, m_scale, v_scale, m_out, v_out, stream) -> None:
    """The same with moments that have been checked."""
    out = m_out if m_out is not None else v_out
    if m_out is not None and v_out is not None and m_out.dtype != v_out.dtype:
        raise ChocoError("libchoco: m_out and v_out have one type", -1)
    for t in (m_out, v_out):
        if t is not None and (t.get_device() != opt.device or t.numel() != opt.elements or not t.is_contiguous()):
            raise ChocoError(f"libchoco: outputs must be contiguous with {opt.elements} elements on GPU {opt.device}", -1)
    _check(load().choco_adamw_read_state(opt, _ptr(m), _ptr(v), _ptr(m_scale), _ptr(v_scale), _ptr(m_out), _ptr(v_out),
                                         0 if out is None else _dtype(out), _stream_of(stream, opt.device)))


def choco_adamw_get_steps(opt, groups: int, stream=None):
    """Steps that every group has taken (int64 array)."""
    import numpy as np
    if groups != opt.groups:
        raise ChocoError(f"libchoco: the list has {opt.groups} groups, not {groups}", -1)
    steps = np.zeros(groups, dtype=np.int64)
    _check(load().choco_adamw_get_steps(opt, steps.ctypes.data, _stream_of(stream, opt.device)))
    return steps


def choco_adamw_set_steps(opt, steps, stream=None) -> None:
    import numpy as np
    s = np.ascontiguousarray(steps, dtype=np.int64)
    if s.shape != (opt.groups,):
        raise ChocoError(f"libchoco: one step count for each of {opt.groups} groups", -1)
    _check(load().choco_adamw_set_steps(opt, s.ctypes.data, _stream_of(stream, opt.device)))


class MuonHandle(ctypes.c_void_p):
    """What choco_muon_init returns: the library's handle, with the device it belongs to and the sizes of what its
    calls take."""

    def describe(self, device: int, n_matrices: int, groups: int, elements: int) -> None:
        self.device, self.n_matrices, self.groups, self.elements = device, n_matrices, groups, elements


def _check_momentum(opt, m) -> None:
    if m is None and opt.elements == 0:
        return
    if m is None or m.get_device() != opt.device or _dtype(m) != 0 or m.numel() != opt.elements or not m.is_contiguous():
        raise ChocoError(f"libchoco: the momentum must be a contiguous float32 array of {opt.elements} elements on GPU {opt.device}, not "
                         f"{None if m is None else (m.dtype, list(m.shape), str(m.device))}", -1)


def choco_muon_init(matrices, groups: int = 1, beta: float = 0.95, nesterov: bool = True, steps: int = 5, coefficients=MUON_COEFFICIENTS,
                    products: int = 0):
    """matrices: numpy array of MUON_MATRIX records (see muon_layer_matrices), on the current device."""
    import numpy as np
    import torch
    t = np.ascontiguousarray(matrices, dtype=MUON_MATRIX)
    a, b, c = coefficients
    p = choco_muon_params(beta, a, b, c, 1 if nesterov else 0, steps, products, groups)
    h, e = MuonHandle(), ctypes.c_int64()
    _check(load().choco_muon_init(ctypes.byref(h), len(t), t.ctypes.data if len(t) else None, ctypes.byref(p)))
    _check(load().choco_muon_state_size(h, ctypes.byref(e), None))
    h.describe(torch.cuda.current_device(), len(t), groups, e.value)
    return h


def choco_muon_destroy(opt) -> None:
    _check(load().choco_muon_destroy(opt))


def choco_muon_state_size(opt):
    """(elements of the momentum, first element of every matrix: an int64 array)."""
    import numpy as np
    e, off = ctypes.c_int64(), np.zeros(opt.n_matrices, dtype=np.int64)
    _check(load().choco_muon_state_size(opt, ctypes.byref(e), off.ctypes.data))
    return e.value, off


def choco_muon_set_grads(opt, pointers, stream=None) -> None:
    """New gradient addresses, one per matrix of the list."""
    import numpy as np
    g = np.ascontiguousarray(pointers, dtype=np.uint64)
    if g.shape != (opt.n_matrices,):
        raise ChocoError(f"libchoco: one address for each of {opt.n_matrices} matrices", -1)
    _check(load().choco_muon_set_grads(opt, g.ctypes.data, _stream_of(stream, opt.device)))


def choco_muon_step(opt, m, lr: float, factor=None, stream=None) -> None:
    _check_momentum(opt, m)
    _muon_step(opt, m, lr, factor, stream)


def _muon_step(opt, m, lr, factor, stream) -> None:
    """The step with a momentum that has been checked."""
    if factor is not None:
        _check_groups(opt, "factor", factor)
    _check(load().choco_muon_step(opt, _ptr(m), lr, _ptr(factor), _stream_of(stream, opt.device)))


def choco_muon_orthogonalize(opt, stream=None) -> None:
    _check(load().choco_muon_orthogonalize(opt, _stream_of(stream, opt.device)))


def choco_muon_status(opt, stream=None) -> None:
    """Waits for `stream`; raises if a bounded wait in a kernel ever ran out."""
    _check(load().choco_muon_status(opt, _stream_of(stream, opt.device)))


def choco_debug_muon_set_wait_polls(opt, polls: int) -> None:
    """Test hook: see choco.h."""
    _check(load().choco_debug_muon_set_wait_polls(opt, polls))


class GroupNormHandle(ctypes.c_void_p):
    """What choco_group_norm_init returns: the library's handle, with the device it belongs to, its sizes, and the layouts of arrays that
    its calls have found to be in order."""

    def describe(self, device: int, n: int, channels: int, groups: int) -> None:
        self.device, self.n, self.channels, self.groups = device, n, channels, groups
        self.layouts: dict = {}


def _pixels_of(gn, what: str, t):
    """(choco_pixels, images, pixels) of an array [n, images, ..., channels]: what lies between images and channels are pixels, which
    have one stride."""
    key = (what, t.shape, t.stride(), t.dtype)
    found = gn.layouts.get(key)
    if found is None:
        if len(gn.layouts) > 1000:       # batches of ever new shapes
            gn.layouts.clear()
        found = gn.layouts[key] = _pixel_layout(gn, what, t)
    if t.get_device() != gn.device:
        raise ChocoError(f"libchoco: {what} must be on the handle's GPU ({gn.device}), not {t.device}", -1)
    found[0].data = t.data_ptr()
    return found


def _pixel_layout(gn, what: str, t):
    shape, strides = t.shape, t.stride()
    if len(shape) < 3 or shape[0] != gn.n or shape[-1] != gn.channels or (strides[-1] != 1 and shape[-1] > 1):
        raise ChocoError(f"libchoco: {what} must be [{gn.n}, images, pixels, {gn.channels}] with neighbouring channels, not {list(shape)}, "
                         f"strides {list(strides)}", -1)
    pixels, step = 1, 0
    for k in range(len(shape) - 2, 1, -1):
        if shape[k] == 1:
            continue
        if pixels == 1:
            step = strides[k]
        elif strides[k] != pixels * step and pixels > 0 and shape[k] > 0:
            raise ChocoError(f"libchoco: the pixels of {what} must have one stride, not {list(strides)} for {list(shape)}", -1)
        pixels *= shape[k]
    return choco_pixels(None, strides[0], strides[1], step, _dtype(t), 0), shape[1], pixels


def _channels_of(gn, what: str, first, second):
    """(stride from worker to worker, type) of arrays [n, channels] with neighbouring channels; None is left out."""
    found = None
    for t in (first, second):
        if t is None:
            continue
        key = (what, t.shape, t.stride(), t.dtype)
        this = gn.layouts.get(key)
        if this is None:
            if t.dim() != 2 or t.shape[0] != gn.n or t.shape[1] != gn.channels or (t.stride(1) != 1 and gn.channels > 1):
                raise ChocoError(f"libchoco: {what} must be [{gn.n}, {gn.channels}] with neighbouring channels, not {list(t.shape)}, "
                                 f"strides {list(t.stride())}", -1)
            this = gn.layouts[key] = (t.stride(0), _dtype(t))
        if t.get_device() != gn.device:
            raise ChocoError(f"libchoco: {what} must be on GPU {gn.device}, not on {t.device}", -1)
        if found is not None and this != found and (gn.n > 1 or this[1] != found[1]):
            raise ChocoError(f"libchoco: {what} have one type and one stride from worker to worker", -1)
        found = found or this
    return found or (gn.channels, 0)


def _check_stats(gn, images: int, *tensors) -> None:
    for t in tensors:
        if t is not None and (t.get_device() != gn.device or _dtype(t) != 0 or t.shape != (gn.n, images, gn.groups) or not t.is_contiguous()):
            raise ChocoError(f"libchoco: mean and rstd must be contiguous float32 [{gn.n}, {images}, {gn.groups}] on GPU {gn.device}, not {t.dtype} "
                             f"{list(t.shape)} on {t.device}", -1)


def choco_group_norm_init(n: int, channels: int, groups: int, max_images: int = 0, eps: float = 1e-5, activation: str = "none"):
    """Handle for the norms of n workers (see choco.h) on the current device; max_images = 0: no gradients of parameters."""
    import torch
    if activation not in ACTIVATIONS:
        raise ChocoError(f"libchoco: activations are {', '.join(ACTIVATIONS)}, not {activation}", -1)
    p = choco_group_norm_params(n, groups, channels, max_images, eps, ACTIVATIONS[activation], 0)
    h = GroupNormHandle()
    _check(load().choco_group_norm_init(ctypes.byref(h), ctypes.byref(p)))
    h.describe(torch.cuda.current_device(), n, channels, groups)
    return h


def choco_group_norm_destroy(gn) -> None:
    _check(load().choco_group_norm_destroy(gn))


def choco_group_norm_forward(gn, x, weight, bias, y, mean=None, rstd=None, stream=None) -> None:
    """y = act(weight xhat + bias).  x and y [n, images, pixels, channels] (or with more axes of pixels); weight and bias [n, channels],
    or None; mean and rstd [n, images, groups] receive the statistics."""
    ax, images, pixels = _pixels_of(gn, "x", x)
    ay, *same = _pixels_of(gn, "y", y)
    if same != [images, pixels]:
        raise ChocoError(f"libchoco: y must have the shape of x, {list(x.shape)}, not {list(y.shape)}", -1)
    ld, kind = _channels_of(gn, "weight and bias", weight, bias)
    _check_stats(gn, images, mean, rstd)
    _check(load().choco_group_norm_forward(gn, images, pixels, ax, ay, _ptr(weight), _ptr(bias), ld, kind, _ptr(mean), _ptr(rstd),
                                           _stream_of(stream, gn.device)))


def choco_group_norm_backward(gn, x, dy, weight, bias, mean, rstd, dx, dweight, dbias, accumulate: bool = False, stream=None) -> None:
    """The gradients of that; dx, dweight and dbias may be None."""
    ax, images, pixels = _pixels_of(gn, "x", x)
    ay, *same = _pixels_of(gn, "dy", dy)
    ad = None
    if dx is not None:
        ad, *other = _pixels_of(gn, "dx", dx)
        same += other
    if any(s != (images, pixels)[k % 2] for k, s in enumerate(same)):
        raise ChocoError(f"libchoco: dy and dx must have the shape of x, {list(x.shape)}", -1)
    ld, kind = _channels_of(gn, "weight and bias", weight, bias)
    gld, gkind = _channels_of(gn, "dweight and dbias", dweight, dbias)
    if mean is None or rstd is None:
        raise ChocoError("libchoco: mean and rstd of the forward call are needed", -1)
    _check_stats(gn, images, mean, rstd)
    _check(load().choco_group_norm_backward(gn, images, pixels, ax, ay, ad, _ptr(weight), _ptr(bias), ld, kind, _ptr(mean), _ptr(rstd),
                                            _ptr(dweight), _ptr(dbias), gld, gkind, 1 if accumulate else 0, _stream_of(stream, gn.device)))


# --------------------------------------------------------------------------- convenience


def adamw_layer_tensors(X, G, layer_off, weight_decay=0.0, lr_scale=1.0, copy=None, layers=None):
    """The list of tensors (worker by worker, layer by layer, group = worker) for rows of X and G
    [n, >= layer_off[-1]] cut at layer_off; weight_decay and lr_scale are numbers or one per layer.
    X may be None (a list for norms only).  layers: which of them are in the list (others are another optimizer's), all without it."""
    import numpy as np
    off = np.asarray(layer_off, dtype=np.int64)
    which, n, layers = layers, G.shape[0], len(off) - 1
    if layers < 1 or off[0] != 0 or np.any(np.diff(off) < 0):
        raise ChocoError("libchoco: layer_off must start at 0 and not decrease", -1)
    if which is not None and (len(which) == 0 or len(set(which)) < len(which) or min(which) < 0 or max(which) >= layers):
        raise ChocoError(f"libchoco: layers must be different ones of 0 .. {layers - 1}, one at least", -1)
    t = np.zeros((n, layers), dtype=ADAMW_TENSOR)
    rows = np.arange(n, dtype=np.int64)[:, None]
    for name, a in (("x", X), ("g", G), ("copy", copy)):
        if a is None:
            continue
        if a.get_device() != G.get_device():
            raise ChocoError(f"libchoco: {name} is on {a.device} and G on {G.device}", -1)
        if not a.is_cuda or a.dim() != 2 or a.shape[0] != n or a.shape[1] < off[-1] or (a.shape[1] > 1 and a.stride(1) != 1):
            raise ChocoError(f"libchoco: {name} must be [{n}, >= {int(off[-1])}] on the GPU with contiguous rows", -1)
        t[name] = (a.data_ptr() + (rows * a.stride(0) + off[None, :-1]) * a.element_size()).astype(np.uint64)
        t[name + "_dtype"] = _dtype(a)
    t["numel"] = np.diff(off)[None]
    t["group"] = rows
    t["weight_decay"] = np.broadcast_to(np.asarray(weight_decay, dtype=np.float64), (layers,))[None]
    t["lr_scale"] = np.broadcast_to(np.asarray(lr_scale, dtype=np.float64), (layers,))[None]
    return (t if which is None else t[:, list(which)]).reshape(-1)


def muon_layer_matrices(X, G, layer_off, shapes, weight_decay=0.0, lr_scale=None, copy=None):
    """The list of matrices (worker by worker, layer by layer, group = worker) for rows of X and G [n, >= layer_off[-1]] cut at
    layer_off.  shapes: (rows, cols) of a layer, with as many elements as the layer has, or None for one that is no
    matrix (a bias, a table) and left out.  weight_decay and lr_scale are numbers or one per layer; without
    lr_scale a matrix has sqrt(max(1, rows / cols))."""
    import numpy as np
    off = np.asarray(layer_off, dtype=np.int64)
    n, layers = G.shape[0], len(off) - 1
    if layers < 1 or off[0] != 0 or np.any(np.diff(off) < 0) or len(shapes) != layers:
        raise ChocoError("libchoco: layer_off must start at 0 and not decrease, with a shape (or None) for each layer", -1)
    which = [k for k in range(layers) if shapes[k] is not None]
    dims = np.array([shapes[k] for k in which], dtype=np.int64).reshape(-1, 2)
    if not which or np.any(dims < 0) or np.any(dims[:, 0] * dims[:, 1] != np.diff(off)[which]):
        raise ChocoError("libchoco: the shapes must be those of the layers' elements, one matrix at least", -1)
    t = np.zeros((n, len(which)), dtype=MUON_MATRIX)
    rows = np.arange(n, dtype=np.int64)[:, None]
    for name, a in (("x", X), ("g", G), ("copy", copy)):
        if a is None:
            continue
        if a.get_device() != G.get_device():
            raise ChocoError(f"libchoco: {name} is on {a.device} and G on {G.device}", -1)
        if not a.is_cuda or a.dim() != 2 or a.shape[0] != n or a.shape[1] < off[-1] or (a.shape[1] > 1 and a.stride(1) != 1):
            raise ChocoError(f"libchoco: {name} must be [{n}, >= {int(off[-1])}] on the GPU with contiguous rows", -1)
        t[name] = (a.data_ptr() + (rows * a.stride(0) + off[which][None]) * a.element_size()).astype(np.uint64)
        t[name + "_dtype"] = _dtype(a)
    t["rows"], t["cols"] = dims[None, :, 0], dims[None, :, 1]
    t["group"] = rows
    if lr_scale is None:
        t["lr_scale"] = np.sqrt(np.maximum(1.0, dims[:, 0] / np.maximum(dims[:, 1], 1)))[None]
    else:
        t["lr_scale"] = np.broadcast_to(np.asarray(lr_scale, dtype=np.float64), (layers,))[which][None]
    t["weight_decay"] = np.broadcast_to(np.asarray(weight_decay, dtype=np.float64), (layers,))[which][None]
    return t.reshape(-1)


def _matrix_records(name, tensors):
    """Addresses, types, sizes and row pitches of 2-D tensors, or of the matrices of 3-D ones."""
    import numpy as np
    parts = []
    for a in tensors:
        if not a.is_cuda or a.dim() not in (2, 3) or (a.shape[-1] > 1 and a.stride(-1) != 1) or a.device != tensors[0].device:
            raise ChocoError(f"libchoco: {name} are matrices, or stacks of them, with contiguous rows on one GPU", -1)
        count, step = (1, 0) if a.dim() == 2 else (a.shape[0], a.stride(0))
        t = np.zeros(count, dtype=[("at", "<u8"), ("kind", "<i4"), ("rows", "<i8"), ("cols", "<i8"), ("ld", "<i8")])
        t["at"] = (a.data_ptr() + np.arange(count, dtype=np.int64) * step * a.element_size()).astype(np.uint64)
        t["kind"], t["rows"], t["cols"] = _dtype(a), a.shape[-2], a.shape[-1]
        t["ld"] = a.stride(-2) if a.shape[-2] > 1 else a.shape[-1]
        parts.append(t)
    return np.concatenate(parts)


@dataclasses.dataclass
class Choco:
    """Owns a context; `w` is any object with n, row_ptr, col, val (host arrays)."""

    w: object
    d: int
    kind: str
    k: int = 0
    s: int = 16
    bucket: int = 0
    qsgd_biased: bool = True
    seed: int = 0
    ld: int = 0

    def __post_init__(self):
        self.ld = self.ld or self.d
        self.ctx = choco_init(self.w.n, self.d, self.ld, self.w.row_ptr, self.w.col, self.w.val,
                              self.kind, self.k, self.s, self.bucket, self.qsgd_biased, self.seed)

    def gossip_step(self, X, Xhat, S, gamma, stream=None):
        choco_gossip_step(self.ctx, X, Xhat, S, gamma, stream)

    def sgd_step(self, X, Xhat, S, G, eta, gamma, stream=None):
        choco_sgd_step(self.ctx, X, Xhat, S, G, eta, gamma, stream)

    def sgd_momentum_step(self, X, Xhat, S, G, M, eta, gamma, lam, beta, stream=None):
        choco_sgd_momentum_step(self.ctx, X, Xhat, S, G, M, eta, gamma, lam, beta, stream)

    def close(self):
        if getattr(self, "ctx", None) is not None:
            choco_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Embedding:
    """Owns a choco_embedding handle; see choco_embedding_init."""

    def __init__(self, n: int, vocab: int, dim: int, max_tokens: int, table_row: int = 0, table_ld: int = 0,
                 scale: float = 1.0, padding: int = -1):
        self.n, self.vocab, self.dim = n, vocab, dim
        self.handle = choco_embedding_init(n, vocab, dim, max_tokens, table_row, table_ld, scale, padding)

    def forward(self, table, tokens, out, stream=None):
        choco_embedding_forward(self.handle, table, tokens, out, stream)

    def backward(self, tokens, dout, grad, accumulate: bool = False, stream=None):
        choco_embedding_backward(self.handle, tokens, dout, grad, accumulate, stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            choco_embedding_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW:
    """AdamW over the layers of all workers' rows: X and G are [n, ld] tensors, every worker a group.
    Owns the handle and (unless `states` hands them over) the moments: (m, v), or with 8-bit
    moments (m, v, m_scale, v_scale), flat arrays in the layout choco.h gives.  With X = None only
    grad_norm can be called.  rounding: of 8-bit moments, "nearest" or "random" (drawn from `seed`); long
    runs want "random", see choco_adamw_set_rounding.  layers: those that it has, where another optimizer (Muon) has the rest;
    grad_norm then is that of these layers."""

    def __init__(self, X, G, layer_off, weight_decay=0.0, lr_scale=1.0, copy=None, beta1: float = 0.9,
                 beta2: float = 0.999, eps: float = 1e-8, state_bits: int = 32, states=None, step: int = 0,
                 rounding: str = "nearest", seed: int = 0, layers=None):
        import torch
        if rounding not in ("nearest", "random"):
            raise ChocoError(f"libchoco: rounding is nearest or random, not {rounding}", -1)
        tensors = adamw_layer_tensors(X, G, layer_off, weight_decay, lr_scale, copy, layers)
        if G.get_device() != torch.cuda.current_device():
            raise ChocoError(f"libchoco: a handle belongs to the current device ({torch.cuda.current_device()}), and G is on {G.device}", -1)
        self.groups = G.shape[0]
        self._keep = (X, G, copy)      # the list holds their addresses
        self.handle = choco_adamw_init(tensors, self.groups, beta1, beta2, eps, state_bits)
        if rounding == "random":
            choco_adamw_set_rounding(self.handle, True, seed)
        self.m = self.v = self.m_scale = self.v_scale = None
        self.elements, self.offsets = choco_adamw_state_size(self.handle, len(tensors))
        if X is not None:
            if states is None:
                states = [torch.zeros(count, dtype=getattr(torch, kind), device=X.device) for kind, count in self.handle.state_arrays()]
            _check_states(self.handle, states)
            self.m, self.v, self.m_scale, self.v_scale = (tuple(states) + (None, None))[:4]
        if step:
            self.set_steps([step] * self.groups)

    def grad_norm(self, max_norm: float, norm, factor, unscale: float = 1.0, stream=None):
        choco_adamw_grad_norm(self.handle, max_norm, norm, factor, unscale, stream)

    def step(self, lr: float, factor=None, stream=None):
        _adamw_step(self.handle, self.m, self.v, self.m_scale, self.v_scale, lr, factor, stream)

    def read_state(self, m_out, v_out, stream=None):
        _adamw_read_state(self.handle, self.m, self.v, self.m_scale, self.v_scale, m_out, v_out, stream)

    def get_steps(self, stream=None):
        return choco_adamw_get_steps(self.handle, self.groups, stream)

    def set_steps(self, steps, stream=None):
        choco_adamw_set_steps(self.handle, steps, stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            choco_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Orthogonalizer:
    """outputs[k] = the orthogonalised inputs[k] (see choco.h): lists of matrices, or of stacks [count, rows, cols] of them.
    The arrays have to stay where they are; outputs may not overlap.  products = 1: factors of 11 bits, results 0.002 off, in half the time."""

    def __init__(self, inputs, outputs, steps: int = 5, coefficients=MUON_COEFFICIENTS, products: int = 0):
        import numpy as np
        import torch
        inputs, outputs = list(inputs), list(outputs)
        if not inputs or [tuple(a.shape) for a in inputs] != [tuple(a.shape) for a in outputs]:
            raise ChocoError("libchoco: inputs and outputs have the same shapes, one matrix at least", -1)
        a, b = _matrix_records("inputs", inputs), _matrix_records("outputs", outputs)
        if inputs[0].device != outputs[0].device or inputs[0].get_device() != torch.cuda.current_device():
            raise ChocoError(f"libchoco: a handle belongs to the current device ({torch.cuda.current_device()}), and the matrices are on "
                             f"{inputs[0].device} and {outputs[0].device}", -1)
        if len(a) == 0:
            raise ChocoError("libchoco: one matrix at least", -1)
        t = np.zeros(len(a), dtype=MUON_MATRIX)
        t["g"], t["g_dtype"], t["g_ld"] = a["at"], a["kind"], a["ld"]
        t["x"], t["x_dtype"], t["x_ld"] = b["at"], b["kind"], b["ld"]
        t["rows"], t["cols"] = a["rows"], a["cols"]
        self._keep = (inputs, outputs)
        self.handle = choco_muon_init(t, steps=steps, coefficients=coefficients, products=products)

    def apply(self, stream=None):
        choco_muon_orthogonalize(self.handle, stream)

    def status(self, stream=None):
        choco_muon_status(self.handle, stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            choco_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Muon:
    """Muon over the matrices among the layers of all workers' rows: X and G are [n, ld] tensors, every worker a
    group; shapes names the matrices (see muon_layer_matrices), other layers are left alone.  Owns the handle and (unless
    `states` hands it over) the momentum, a flat array in the layout choco.h gives.  products: see Orthogonalizer."""

    def __init__(self, X, G, layer_off, shapes, weight_decay=0.0, lr_scale=None, copy=None, beta: float = 0.95, nesterov: bool = True,
                 steps: int = 5, coefficients=MUON_COEFFICIENTS, products: int = 0, states=None):
        import torch
        matrices = muon_layer_matrices(X, G, layer_off, shapes, weight_decay, lr_scale, copy)
        if G.get_device() != torch.cuda.current_device():
            raise ChocoError(f"libchoco: a handle belongs to the current device ({torch.cuda.current_device()}), and G is on {G.device}", -1)
        self.groups = G.shape[0]
        self._keep = (X, G, copy)      # the list holds their addresses
        self.handle = choco_muon_init(matrices, self.groups, beta, nesterov, steps, coefficients, products)
        self.elements, self.offsets = choco_muon_state_size(self.handle)
        self.m = torch.zeros(self.elements, dtype=torch.float32, device=X.device) if states is None else states
        _check_momentum(self.handle, self.m)

    def step(self, lr: float, factor=None, stream=None):
        _muon_step(self.handle, self.m, lr, factor, stream)

    def status(self, stream=None):
        choco_muon_status(self.handle, stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            choco_muon_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class GroupNorm:
    """Owns a choco_group_norm handle; see choco_group_norm_init.  Used by one host thread at a time; calls for gradients of parameters
    (and replays of captured ones) follow one another."""

    def __init__(self, n: int, channels: int, groups: int, max_images: int = 0, eps: float = 1e-5, activation: str = "none"):
        self.n, self.channels, self.groups = n, channels, groups
        self.handle = choco_group_norm_init(n, channels, groups, max_images, eps, activation)

    def forward(self, x, weight, bias, y, mean=None, rstd=None, stream=None):
        choco_group_norm_forward(self.handle, x, weight, bias, y, mean, rstd, stream)

    def backward(self, x, dy, weight, bias, mean, rstd, dx, dweight, dbias, accumulate: bool = False, stream=None):
        choco_group_norm_backward(self.handle, x, dy, weight, bias, mean, rstd, dx, dweight, dbias, accumulate, stream)

    def close(self):
        if getattr(self, "handle", None) is not None:
            choco_group_norm_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
