"""ctypes binding of libls.so (include/ls.h).

Argument marshalling only: every arithmetic step runs inside the CUDA library.
torch is used for device memory and streams.  If the library cannot be built
or loaded this module raises; there is no other implementation to fall back to.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
from typing import Optional, Sequence

import numpy as np

from . import build as _build

LS_MAX_LAYERS = 8
LS_MAX_REPLICAS = 64

LS_OK = 0
LS_ERR_INVALID_ARG = -1
LS_ERR_BAD_HANDLE = -2
LS_ERR_STATE_SIZE = -3
LS_ERR_NO_DATASET = -4
LS_ERR_ROW_RANGE = -5
LS_ERR_CUDA = -6
LS_ERR_UNSUPPORTED = -7
LS_ERR_OVERFLOW = -8
LS_ERR_DEVICE_TIMEOUT = -9
LS_ERR_TOO_LARGE = -10
LS_ERR_EXCHANGE = -11

LOSS = {"softmax_ce": 0, "mse_half": 1}
GEMM = {"fp32": 0, "bf16": 1}
MOMENTUM_MODE = {"average": 0, "keep": 1, "reset": 2, "block": 3}
KERNEL_CLASSES = ("fwd", "loss", "dx", "dw", "bias", "avg")


class AdacommOpts(C.Structure):
    _fields_ = [("gamma", C.c_double), ("slack", C.c_int32), ("n_decay", C.c_int32), ("decay_at", C.c_void_p),
                ("decay_factor", C.c_double)]


class ModelSpec(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int32),
        ("dims", C.c_int32 * (LS_MAX_LAYERS + 1)),
        ("loss", C.c_int32),
        ("has_bias", C.c_int32),
        ("gemm_dtype", C.c_int32),
        ("momentum_mode", C.c_int32),
        ("weight_decay", C.c_float),
        ("block_momentum", C.c_float),
    ]


# int exchange(void* ctx, const float* partial_dev, float* gathered_dev, size_t bytes, int n_gpus)
EXCHANGE_FN = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_int)


class LsError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_lib().ls_strerror(code).decode()} ({code})")


_LIB = None


def _lib():
    global _LIB
    if _LIB is not None:
        return _LIB
    path = _build.build()          # compiles with nvcc when missing or stale; raises on failure
    lib = C.CDLL(path)
    vp, i64, f32 = C.c_void_p, C.c_int64, C.c_float
    P = C.POINTER
    sig = {
        "ls_strerror": (C.c_char_p, [C.c_int]),
        "ls_param_count": (C.c_int, [P(ModelSpec), P(i64)]),
        "ls_state_bytes": (C.c_int, [C.c_int, P(ModelSpec), C.c_int, P(C.c_size_t)]),
        "ls_create": (C.c_int, [P(vp), C.c_int, P(ModelSpec), f32, f32, C.c_int, vp, C.c_size_t, vp]),
        "ls_destroy": (C.c_int, [vp]),
        "ls_sync": (C.c_int, [vp]),
        "ls_selftest_wait_timeout": (C.c_int, [vp, i64]),
        "ls_last_cuda_error": (C.c_int, [vp]),
        "ls_set_lr": (C.c_int, [vp, f32]),
        "ls_set_params": (C.c_int, [vp, vp]),
        "ls_set_state": (C.c_int, [vp, C.c_int, vp, vp]),
        "ls_get_state": (C.c_int, [vp, C.c_int, vp, vp]),
        "ls_state_view": (C.c_int, [vp, P(vp), P(vp), P(i64)]),
        "ls_bind_dataset": (C.c_int, [vp, vp, vp, i64]),
        "ls_local_steps": (C.c_int, [vp, C.c_int, vp, vp]),
        "ls_local_steps_avg": (C.c_int, [vp, C.c_int, vp, vp]),
        "ls_local_steps_host": (C.c_int, [vp, C.c_int, vp, vp, vp]),
        "ls_average": (C.c_int, [vp]),
        "ls_average_flat": (C.c_int, [vp, C.c_int, i64, i64, vp]),
        "ls_block_average_flat": (C.c_int, [vp, vp, vp, C.c_int, i64, i64, C.c_float, C.c_float, vp]),
        "ls_set_block_state": (C.c_int, [vp, vp, vp]),
        "ls_run_timed": (C.c_int, [vp, i64, C.c_int, C.c_double, i64, vp, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp]),
        "ls_delay": (C.c_int, [C.c_double, C.c_int, C.c_int, vp]),
        "ls_speedup": (C.c_int, [C.c_double, C.c_int, vp]),
        "ls_error_bound": (C.c_int, [C.c_double] * 6 + [C.c_int, C.c_int, C.c_double, C.c_double, vp]),
        "ls_tau_star": (C.c_int, [C.c_double] * 7 + [vp]),
        "ls_simulate_runtime": (C.c_int, [C.c_int, C.c_int, i64, C.c_double, C.c_double, C.c_uint64, C.c_int, vp, vp]),
        "ls_philox4x32_10": (C.c_int, [vp, vp, vp]),
        "ls_get_block_state": (C.c_int, [vp, vp, vp]),
        "ls_eval_loss": (C.c_int, [vp, C.c_int, i64, i64, P(f32)]),
        "adacomm_next_tau": (C.c_int, [C.c_double, C.c_double, C.c_int]),
        "ls_run": (C.c_int, [vp, i64, C.c_int, C.c_int, i64, vp, vp, vp, i64, P(i64), vp, vp, vp, i64, P(i64),
                             P(f32)]),
        "ls_launch_count": (C.c_int, [vp, P(i64)]),
        "adacomm_next_tau_refined": (C.c_int, [C.c_double, C.c_double, C.c_int, C.c_int, C.c_double, C.c_int,
                                               C.c_double, C.c_double, C.c_int]),
        "ls_run_refined": (C.c_int, [vp, i64, C.c_int, C.c_int, i64, vp, vp, P(AdacommOpts), vp, i64, P(i64), vp, vp,
                                     vp, i64, P(i64), P(f32)]),
        "ls_get_lr": (C.c_int, [vp, P(f32)]),
        "ls_linear_loss_static": (C.c_int, [vp, vp, vp, vp, i64, C.c_int, C.c_int, C.c_int, C.c_int, vp, vp]),
        "ls_device_status": (C.c_int, [vp]),
        "ls_selftest_device_timeout": (C.c_int, [i64, vp]),
        "ls_layer_norm": (C.c_int, [vp, vp, vp, C.c_int, i64, C.c_int, i64, i64, C.c_int, f32, vp, i64, vp, vp, vp]),
        "ls_layer_norm_grad_ws_bytes": (C.c_int, [C.c_int, i64, C.c_int, P(C.c_size_t)]),
        "ls_layer_norm_grad": (C.c_int, [vp, vp, vp, vp, vp, C.c_int, i64, C.c_int, i64, i64, i64, C.c_int, vp, i64, vp, vp,
                                         i64, vp, C.c_size_t, vp]),
        "ls_vocab_loss_ws_bytes": (C.c_int, [C.c_int, i64, i64, C.c_int, C.c_int, C.c_int, P(C.c_size_t)]),
        "ls_vocab_loss": (C.c_int, [vp, vp, vp, C.c_int, i64, i64, C.c_int, i64, i64, C.c_int, vp, vp, vp, vp, C.c_size_t,
                                    vp]),
        "ls_vocab_loss_grad": (C.c_int, [vp, vp, vp, C.c_int, i64, i64, C.c_int, i64, i64, C.c_int, f32, vp, vp, vp, vp, i64,
                                         vp, i64, vp, C.c_size_t, vp]),
        "ls_orthogonalize_ws_bytes": (C.c_int, [C.c_int, C.c_int, C.c_int, P(C.c_size_t)]),
        "ls_orthogonalize": (C.c_int, [vp, C.c_int, C.c_int, C.c_int, i64, C.c_int, C.c_int, vp, i64, vp, C.c_size_t, vp]),
        "ls_muon_step": (C.c_int, [vp, vp, vp, C.c_int, C.c_int, C.c_int, i64, i64, i64, C.c_int, f32, f32, C.c_int, C.c_int,
                                   vp, C.c_size_t, vp]),
        "ls_muon_step_layer": (C.c_int, [vp, C.c_int, vp, i64, C.c_int, f32, f32, C.c_int, C.c_int, vp, C.c_size_t]),
        "ls_shard_buffer_floats": (C.c_int, [vp, P(i64)]),
        "ls_set_shard": (C.c_int, [vp, C.c_int, C.c_int, vp, vp, EXCHANGE_FN, vp]),
        "ls_shard_partial_sum": (C.c_int, [vp, vp]),
        "ls_shard_average": (C.c_int, [vp, vp, C.c_int, C.c_int]),
        "ls_partial_sum_flat": (C.c_int, [vp, C.c_int, i64, i64, vp, vp]),
        "ls_combine_partials_flat": (C.c_int, [vp, C.c_int, i64, C.c_int, i64, vp, C.c_int, i64, vp]),
        "ls_profile_begin": (C.c_int, [vp, C.c_uint32, C.c_int]),
        "ls_profile_end": (C.c_int, [vp, P(C.c_double), P(i64)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _LIB = lib
    return lib


def library_path() -> str:
    _lib()
    return _build.LIB_PATH


def _check(code: int, where: str):
    if code != LS_OK:
        raise LsError(code, where)


def make_spec(dims: Sequence[int], loss: str = "softmax_ce", has_bias: bool = True, gemm_dtype: str = "fp32",
              momentum_mode: str = "average", weight_decay: float = 0.0, block_momentum: float = 0.0) -> ModelSpec:
    s = ModelSpec()
    if not (2 <= len(dims) <= LS_MAX_LAYERS + 1):
        raise ValueError("1..8 layers")
    s.n_layers = len(dims) - 1
    for i, d in enumerate(dims):
        s.dims[i] = int(d)
    s.loss = LOSS[loss]
    s.has_bias = int(bool(has_bias))
    s.gemm_dtype = GEMM[gemm_dtype]
    s.momentum_mode = MOMENTUM_MODE[momentum_mode]
    s.weight_decay = float(weight_decay)
    s.block_momentum = float(block_momentum)
    return s


def param_count(spec: ModelSpec) -> int:
    n = C.c_int64()
    _check(_lib().ls_param_count(C.byref(spec), C.byref(n)), "ls_param_count")
    return n.value


def state_bytes(m: int, spec: ModelSpec, batch: int) -> int:
    n = C.c_size_t()
    _check(_lib().ls_state_bytes(m, C.byref(spec), batch, C.byref(n)), "ls_state_bytes")
    return n.value


def adacomm_next_tau(F_t: float, F_0: float, tau_0: int) -> int:
    r = _lib().adacomm_next_tau(float(F_t), float(F_0), int(tau_0))
    if r < 0:
        raise LsError(r, "adacomm_next_tau")
    return r


def adacomm_next_tau_refined(F_t: float, F_0: float, tau_0: int, tau_prev: int, gamma: float = 0.5, slack: int = 0,
                             lr_0: float = 1.0, lr_l: float = 1.0, lr_changed: bool = False) -> int:
    r = _lib().adacomm_next_tau_refined(float(F_t), float(F_0), int(tau_0), int(tau_prev), float(gamma), int(slack),
                                        float(lr_0), float(lr_l), int(bool(lr_changed)))
    if r < 0:
        raise LsError(r, "adacomm_next_tau_refined")
    return r


def _stream_ptr(stream) -> int:
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


def average_flat(buf, m: int, P: int, stride: Optional[int] = None, stream=None) -> None:
    """Average m float32 vectors of P elements held in the CUDA tensor `buf`
    (vector j starts at element j*stride) in place."""
    import torch
    if not (buf.is_cuda and buf.dtype == torch.float32 and buf.is_contiguous()):
        raise ValueError("buf must be a contiguous float32 CUDA tensor")
    stride = int(P if stride is None else stride)
    if buf.numel() < (m - 1) * stride + P:
        raise ValueError("buf too small")
    _check(_lib().ls_average_flat(buf.data_ptr(), int(m), int(P), stride, _stream_ptr(stream)), "ls_average_flat")


def partial_sum_flat(buf, m: int, P: int, out, stride: Optional[int] = None, stream=None) -> None:
    """out[0..P) = sum of the m vectors of buf (vector j at j*stride) in index order, fp32 (ls_partial_sum_flat)."""
    stride = int(P if stride is None else stride)
    _check(_lib().ls_partial_sum_flat(buf.data_ptr(), int(m), int(P), stride, out.data_ptr(), _stream_ptr(stream)),
           "ls_partial_sum_flat")


def combine_partials_flat(partials, G: int, part_stride: int, m_total: int, P: int, dst, m_local: int,
                          dst_stride: Optional[int] = None, stream=None) -> None:
    """Every one of the m_local vectors of dst = (partials[0] + ... + partials[G-1], in that order) / m_total
    (ls_combine_partials_flat)."""
    dst_stride = int(P if dst_stride is None else dst_stride)
    _check(_lib().ls_combine_partials_flat(partials.data_ptr(), int(G), int(part_stride), int(m_total), int(P),
                                           dst.data_ptr(), int(m_local), dst_stride, _stream_ptr(stream)),
           "ls_combine_partials_flat")


def block_average_flat(buf, anchor, u, m: int, P: int, lr: float, beta: float, stride: Optional[int] = None,
                       stream=None) -> None:
    """Block-momentum averaging step (Section 5.3) on raw CUDA tensors: buf as for average_flat, anchor and u
    float32 vectors of P elements (the period-start model and the global buffer), all updated in place."""
    import torch
    for t in (buf, anchor, u):
        if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            raise ValueError("contiguous float32 CUDA tensors expected")
    stride = int(P if stride is None else stride)
    if buf.numel() < (m - 1) * stride + P or anchor.numel() < P or u.numel() < P:
        raise ValueError("buffer too small")
    _check(_lib().ls_block_average_flat(buf.data_ptr(), anchor.data_ptr(), u.data_ptr(), int(m), int(P), stride,
                                        float(lr), float(beta), _stream_ptr(stream)), "ls_block_average_flat")


# ---- runtime model (host only; Sections 2-4) ----------------------------------------------------------
DELAY_SCALING = {"constant": 0, "log2": 1, "tree": 2, "linear": 3}


def delay(D0: float, m: int, scaling: str = "tree") -> float:
    out = C.c_double()
    _check(_lib().ls_delay(float(D0), int(m), DELAY_SCALING[scaling], C.byref(out)), "ls_delay")
    return out.value


def speedup(alpha: float, tau: int) -> float:
    out = C.c_double()
    _check(_lib().ls_speedup(float(alpha), int(tau), C.byref(out)), "ls_speedup")
    return out.value


def error_bound(T, F1, Finf, lr, L, sigma2, m, tau, Y, D) -> float:
    out = C.c_double()
    _check(_lib().ls_error_bound(float(T), float(F1), float(Finf), float(lr), float(L), float(sigma2), int(m), int(tau),
                                 float(Y), float(D), C.byref(out)), "ls_error_bound")
    return out.value


def tau_star(F1, Finf, D, lr, L, sigma2, T) -> float:
    out = C.c_double()
    _check(_lib().ls_tau_star(float(F1), float(Finf), float(D), float(lr), float(L), float(sigma2), float(T),
                              C.byref(out)), "ls_tau_star")
    return out.value


def simulate_runtime(m: int, tau: int, n_periods: int, y_mean: float, D: float, seed: int, exponential: bool = True):
    """(mean T_sync, mean T_P-Avg) per iteration over n_periods periods (Section 3.1)."""
    a, b = C.c_double(), C.c_double()
    _check(_lib().ls_simulate_runtime(int(m), int(tau), int(n_periods), float(y_mean), float(D), int(seed),
                                      int(bool(exponential)), C.byref(a), C.byref(b)), "ls_simulate_runtime")
    return a.value, b.value


def philox4x32_10(counter, key):
    c = (C.c_uint32 * 4)(*counter)
    k = (C.c_uint32 * 2)(*key)
    o = (C.c_uint32 * 4)()
    _check(_lib().ls_philox4x32_10(c, k, o), "ls_philox4x32_10")
    return tuple(int(v) for v in o)


def linear_loss_static(W, bias, x, y, chunk_rows: int, chunk_loss, loss: str = "softmax_ce", stream=None) -> None:
    """Per-chunk mean loss of z = W x + b on the rows of x, computed by the library without allocating
    any memory (its scratch is a fixed array inside the library).  W [d_out][d_in], bias [d_out] or None,
    x [n_rows][d_in] float32, y int32 labels / float32 targets, chunk_loss float32 [n_rows // chunk_rows]:
    all CUDA tensors owned by the caller.  Calls that overlap on the GPU must be serialised."""
    _check(_lib().ls_linear_loss_static(W.data_ptr(), None if bias is None else bias.data_ptr(), x.data_ptr(),
                                        y.data_ptr(), int(x.shape[0]), int(x.shape[1]), int(W.shape[0]), LOSS[loss],
                                        int(chunk_rows), chunk_loss.data_ptr(), _stream_ptr(stream)),
           "ls_linear_loss_static")


# ---- operators of a language model's last layers and its weight update ---------------------------------------
# Every tensor takes the replicas first ([m][rows][d], ...); one replica may leave that axis out.  A replica is dense,
# the distance between replicas is free (views into packed replica vectors are fine).  Outputs that are not given are
# allocated.  `workspace`: a uint8 tensor of the size the matching *_workspace function names, for callers that keep
# one; calls that may overlap on the GPU need their own.  `stream`: a torch stream, the current one by default.

_TORCH = None
_OP_DTYPE = {}


def _op_torch():
    """torch, imported once (importing this module stays cheap)."""
    global _TORCH
    if _TORCH is None:
        import torch
        _OP_DTYPE.update({torch.float32: 0, torch.bfloat16: 1})
        _TORCH = torch
    return _TORCH


def _op_dtype(t, name: str) -> int:
    dt = _OP_DTYPE.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return dt


class _Op:
    """Checks the tensors of one call, lends out its workspace and keeps track of what the stream uses.  The common
    case (contiguous tensors, the current stream and device) takes a few attribute reads per tensor: a call of a
    small operator costs what its Python does."""

    __slots__ = ("torch", "device", "stream", "raw")

    def __init__(self, first, stream):
        self.torch = torch = _op_torch()
        if not (isinstance(first, torch.Tensor) and first.is_cuda):
            raise ValueError("CUDA tensors expected")
        self.device = first.device
        if stream is None:
            self.stream = None
            self.raw = torch._C._cuda_getCurrentRawStream(self.device.index)
        else:
            if stream.device != self.device:
                raise ValueError("the stream belongs to another device than the tensors")
            self.raw = int(stream.cuda_stream)
            # None where it is the current one
            self.stream = stream if stream != torch.cuda.current_stream(self.device) else None

    def stack(self, t, name: str, tail, m: Optional[int], dtype=None):
        """t as [m][*tail] (m None: from t); returns (pointer, m, stride between replicas)."""
        torch = self.torch
        if not isinstance(t, torch.Tensor) or t.device != self.device:
            raise ValueError(f"{name} must be a tensor on {self.device}")
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
        shape = tuple(t.shape)
        lead = len(shape) - len(tail)
        if lead not in (0, 1) or shape[lead:] != tail or (m is not None and (shape[0] if lead else 1) != m):
            raise ValueError(f"{name} has shape {shape}, expected [{'m' if m is None else m}] + {list(tail)}")
        n = 1
        for size in tail:
            n *= size
        k = shape[0] if lead else 1
        step = n
        if not t.is_contiguous():
            want = 1
            for size, st in zip(reversed(tail), reversed(t.stride()[lead:])):
                if size > 1 and st != want:
                    raise ValueError(f"{name}: a replica must be dense and row-major")
                want *= size
            if k > 1:
                step = t.stride(0)
                if step < n:
                    raise ValueError(f"{name}: the replicas overlap")
        if self.stream is not None:
            t.record_stream(self.stream)
        return t.data_ptr(), k, step

    def dense(self, t, name: str, shape, dtype):
        """t as a dense tensor of this shape (one replica may leave the first axis out)."""
        if not (isinstance(t, self.torch.Tensor) and t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous")
        return self.stack(t, name, shape[1:], shape[0], dtype)[0]

    def new(self, like, shape, dtype):
        if self.stream is None:
            return like.new_empty(shape, dtype=dtype)
        return self.elsewhere(lambda: like.new_empty(shape, dtype=dtype))

    def elsewhere(self, make):
        """A new tensor for a call on a stream that is not the current one: out of that stream's memory (a block that the
        current stream has given back may still be read by what is queued there), and kept from reuse until the current
        stream, where the caller will read it, is through with it."""
        with self.torch.cuda.stream(self.stream):
            t = make()
        t.record_stream(self.torch.cuda.current_stream(self.device))
        return t

    def out(self, given, like, name: str, shape, dtype):
        """An output [m][*tail]: the caller's tensor, or a new dense one.  Returns (tensor, pointer, stride)."""
        if given is None:
            if self.stream is None and like.shape == shape and like.dtype == dtype and like.is_contiguous():
                t = self.torch.empty_like(like)
            else:
                t = self.new(like, shape, dtype)
            return t, t.data_ptr(), math.prod(shape[1:])
        ptr, _, step = self.stack(given, name, shape[1:], shape[0], dtype)
        return given, ptr, step

    def out_dense(self, given, like, name: str, shape, dtype):
        if given is None:
            t = self.new(like, shape, dtype)
            return t, t.data_ptr()
        return given, self.dense(given, name, shape, dtype)

    def workspace(self, like, given, nbytes: int):
        t = given
        if t is None:
            t = self.new(like, (nbytes + 256,), self.torch.uint8)
        elif not (t.is_cuda and t.device == self.device and t.dtype == self.torch.uint8 and t.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 tensor on the device of the call")
        elif self.stream is not None:
            t.record_stream(self.stream)
        start = t.data_ptr()
        base = (start + 255) & -256
        # (a view that ends before the first 256-byte boundary holds nothing)
        return base, max(0, start + t.numel() - base), t

    def call(self, name: str, *args):
        fn = getattr(_LIB or _lib(), name)
        if self.torch._C._cuda_getDevice() == self.device.index:
            code = fn(*args, self.raw)
        else:
            with self.torch.cuda.device(self.device):
                code = fn(*args, self.raw)
        if code != LS_OK:
            raise LsError(code, name)


def _like(t, lead, out):
    """An output without the replica axis when the call's first tensor had none."""
    return out if t.dim() == lead else out.squeeze(0)


def _int32(v: int, code: int, name: str) -> int:
    """v as the C int that the library takes; ctypes would keep its low 32 bits."""
    if not -2 ** 31 <= v < 2 ** 31:
        raise LsError(code, name)
    return v


@functools.lru_cache(maxsize=256)
def _ws_bytes(name: str, *args) -> int:
    for v in args:                       # (no operator takes a size beyond 2^31 - 1, whatever the type of its argument)
        _int32(v, LS_ERR_TOO_LARGE, name)
    n = C.c_size_t()
    _check(getattr(_lib(), name)(*args, C.byref(n)), name)
    return n.value


def device_status(stream=None) -> None:
    """Wait for the stream; raises LsError(LS_ERR_DEVICE_TIMEOUT) if a bounded wait of an operator ran out on its
    device since the last call (ls_device_status)."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    with torch.cuda.device(s.device):
        _check(_lib().ls_device_status(int(s.cuda_stream)), "ls_device_status")


def selftest_device_timeout(limit_cycles: int = 2_000_000, stream=None) -> None:
    """Enqueue the kernel whose bounded wait runs out (ls_selftest_device_timeout); the next device_status() of that device
    raises LsError(LS_ERR_DEVICE_TIMEOUT)."""
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    with torch.cuda.device(s.device):
        _check(_lib().ls_selftest_device_timeout(int(limit_cycles), int(s.cuda_stream)), "ls_selftest_device_timeout")


def layer_norm(x, weight, bias=None, eps: float = 1e-5, out=None, mean=None, rstd=None, stream=None):
    """Layer norm of the rows of x [m][rows][d] (float32 or bfloat16) with float32 weight and bias [m][d]
    (ls_layer_norm).  Returns (y, mean, rstd), the last two float32 [m][rows]."""
    op = _Op(x, stream)
    dt = _op_dtype(x, "x")
    if x.dim() not in (2, 3):
        raise ValueError("x must be [m][rows][d] or [rows][d]")
    rows, d = x.shape[-2:]
    xp, m, xs = op.stack(x, "x", (rows, d), None)
    if d >= 2 ** 31 or m >= 2 ** 31:
        raise LsError(LS_ERR_TOO_LARGE, "ls_layer_norm")
    f32 = op.torch.float32
    wp, _, ws = op.stack(weight, "weight", (d,), m, f32)
    bp = None
    if bias is not None:
        bp, _, bs = op.stack(bias, "bias", (d,), m, f32)
        if m > 1 and bs != ws:
            raise ValueError("weight and bias must have the same distance between replicas")
    y, yp, ys = op.out(out, x, "out", (m, rows, d), x.dtype)
    mean_t, mp = op.out_dense(mean, x, "mean", (m, rows), f32)
    rstd_t, rp = op.out_dense(rstd, x, "rstd", (m, rows), f32)
    op.call("ls_layer_norm", xp, wp, bp, m, rows, d, xs, ws, dt, eps, yp, ys, mp, rp)
    if x.dim() == 3:
        return y, mean_t, rstd_t
    return (y if out is not None else y.squeeze(0), mean_t if mean is not None else mean_t.squeeze(0),
            rstd_t if rstd is not None else rstd_t.squeeze(0))


def layer_norm_grad_workspace(m: int, rows: int, d: int) -> int:
    return _ws_bytes("ls_layer_norm_grad_ws_bytes", int(m), int(rows), int(d)) + 256


def layer_norm_grad(dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, workspace=None, stream=None):
    """Gradient of layer_norm from dy, x and the forward call's mean and rstd (ls_layer_norm_grad).  Returns
    (dx like x, dweight, dbias float32 [m][d])."""
    op = _Op(x, stream)
    dt = _op_dtype(x, "x")
    if x.dim() not in (2, 3):
        raise ValueError("x must be [m][rows][d] or [rows][d]")
    rows, d = x.shape[-2:]
    f32 = op.torch.float32
    xp, m, xs = op.stack(x, "x", (rows, d), None)
    dyp, _, dys = op.stack(dy, "dy", (rows, d), m, x.dtype)
    wp, _, ws = op.stack(weight, "weight", (d,), m, f32)
    mp, rp = op.dense(mean, "mean", (m, rows), f32), op.dense(rstd, "rstd", (m, rows), f32)
    dx_t, dxp, dxs = op.out(dx, x, "dx", (m, rows, d), x.dtype)
    dw_t, dwp, dps = op.out(dweight, x, "dweight", (m, d), f32)
    if dbias is None and (m == 1 or dps == d):
        db_t = op.new(x, (m, d), f32)
    elif dbias is None:
        # beside dweight, with its distance between replicas
        def beside():
            return op.torch.empty_strided((m, d), (dps, 1), dtype=f32, device=op.device)
        db_t = beside() if op.stream is None else op.elsewhere(beside)
    else:
        db_t = dbias
    dbp, _, dbs = op.stack(db_t, "dbias", (d,), m, f32)
    if m > 1 and dbs != dps:
        raise ValueError("dweight and dbias must have the same distance between replicas")
    base, nbytes, keep = op.workspace(x, workspace, _ws_bytes("ls_layer_norm_grad_ws_bytes", m, rows, d))
    op.call("ls_layer_norm_grad", dyp, xp, wp, mp, rp, m, rows, d, dys, xs, ws, dt, dxp, dxs, dwp, dbp, dps, base, nbytes)
    return (dx_t if dx is not None else _like(x, 3, dx_t), dw_t if dweight is not None else _like(x, 3, dw_t),
            db_t if dbias is not None else _like(x, 3, db_t))


def vocab_loss_workspace(m: int, rows: int, vocab: int, d: int, dtype: str = "bf16", grad: bool = False) -> int:
    return _ws_bytes("ls_vocab_loss_ws_bytes", int(m), int(rows), int(vocab), int(d), GEMM[dtype], int(bool(grad))) + 256


def _vocab_args(op, h, W, labels):
    torch = op.torch
    dt = _op_dtype(h, "h")
    if h.dim() not in (2, 3):
        raise ValueError("h must be [m][rows][d] or [rows][d]")
    rows, d = h.shape[-2:]
    hp, m, hs = op.stack(h, "h", (rows, d), None)
    if W.dim() not in (2, 3) or W.shape[-1] != d:
        raise ValueError(f"W must be [m][vocab][{d}]")
    vocab = W.shape[-2]
    wp, _, ws = op.stack(W, "W", (vocab, d), m, h.dtype)
    lp = op.dense(labels, "labels", (m, rows), torch.int32)
    return dt, m, rows, d, vocab, hp, hs, wp, ws, lp


def vocab_loss(h, W, labels, loss=None, row_loss=None, lse=None, workspace=None, stream=None):
    """Mean softmax cross entropy of the logits h W^T, h [m][rows][d], W [m][vocab][d] (both float32 or both
    bfloat16), labels int32 [m][rows] (outside [0, vocab): no label), without storing the logits (ls_vocab_loss).
    Returns (loss [m], row_loss [m][rows], log-sum-exp [m][rows]), float32."""
    op = _Op(h, stream)
    dt, m, rows, d, vocab, hp, hs, wp, ws, lp = _vocab_args(op, h, W, labels)
    f32 = op.torch.float32
    loss_t, loss_p = op.out_dense(loss, h, "loss", (m,), f32)
    rl_t, rl_p = op.out_dense(row_loss, h, "row_loss", (m, rows), f32)
    lse_t, lse_p = op.out_dense(lse, h, "lse", (m, rows), f32)
    outs = (loss_p, rl_p, lse_p)
    base, nbytes, keep = op.workspace(h, workspace, _ws_bytes("ls_vocab_loss_ws_bytes", m, rows, vocab, d, dt, 0))
    op.call("ls_vocab_loss", hp, wp, lp, m, rows, vocab, d, hs, ws, dt, *outs, base, nbytes)
    return (loss_t, rl_t if row_loss is not None else _like(h, 3, rl_t), lse_t if lse is not None else _like(h, 3, lse_t))


def vocab_loss_grad(h, W, labels, scale: float = 1.0, dh=None, dW=None, loss=None, row_loss=None, lse=None,
                    workspace=None, stream=None):
    """vocab_loss and the gradients of scale * loss (ls_vocab_loss_grad).  Returns (loss, row_loss, lse, dh like h,
    dW like W)."""
    op = _Op(h, stream)
    dt, m, rows, d, vocab, hp, hs, wp, ws, lp = _vocab_args(op, h, W, labels)
    f32 = op.torch.float32
    loss_t, loss_p = op.out_dense(loss, h, "loss", (m,), f32)
    rl_t, rl_p = op.out_dense(row_loss, h, "row_loss", (m, rows), f32)
    lse_t, lse_p = op.out_dense(lse, h, "lse", (m, rows), f32)
    outs = (loss_p, rl_p, lse_p)
    dh_t, dhp, dhs = op.out(dh, h, "dh", (m, rows, d), h.dtype)
    dW_t, dwp, dws = op.out(dW, h, "dW", (m, vocab, d), h.dtype)
    base, nbytes, keep = op.workspace(h, workspace, _ws_bytes("ls_vocab_loss_ws_bytes", m, rows, vocab, d, dt, 1))
    op.call("ls_vocab_loss_grad", hp, wp, lp, m, rows, vocab, d, hs, ws, dt, float(scale), *outs, dhp, dhs, dwp, dws, base,
            nbytes)
    return (loss_t, rl_t if row_loss is not None else _like(h, 3, rl_t), lse_t if lse is not None else _like(h, 3, lse_t),
            dh_t if dh is not None else _like(h, 3, dh_t), dW_t if dW is not None else _like(h, 3, dW_t))


def orthogonalize_workspace(m: int, rows: int, cols: int) -> int:
    """Workspace of orthogonalize and muon_step."""
    return _ws_bytes("ls_orthogonalize_ws_bytes", int(m), int(rows), int(cols)) + 256


def orthogonalize(u, steps: int = 5, out=None, workspace=None, stream=None):
    """Newton-Schulz orthogonalisation of the matrices u [m][rows][cols], float32 or bfloat16 (ls_orthogonalize)."""
    op = _Op(u, stream)
    dt = _op_dtype(u, "u")
    if u.dim() not in (2, 3):
        raise ValueError("u must be [m][rows][cols] or [rows][cols]")
    rows, cols = u.shape[-2:]
    up, m, us = op.stack(u, "u", (rows, cols), None)
    o, outp, outs = op.out(out, u, "out", (m, rows, cols), u.dtype)
    base, nbytes, keep = op.workspace(u, workspace, _ws_bytes("ls_orthogonalize_ws_bytes", m, rows, cols))
    op.call("ls_orthogonalize", up, m, rows, cols, us, dt, _int32(int(steps), LS_ERR_INVALID_ARG, "steps"), outp, outs, base, nbytes)
    return o if out is not None else _like(u, 3, o)


def muon_step(w, v, g, lr: float, momentum: float = 0.95, nesterov: bool = True, steps: int = 5, workspace=None,
              stream=None) -> None:
    """One orthogonalised momentum step of the float32 matrices w [m][rows][cols] with momentum buffers v, in place,
    from gradients g (float32 or bfloat16) (ls_muon_step).  w and v may be views into packed replica vectors of the
    caller's; the weights of a LocalSGD take LocalSGD.muon_step."""
    op = _Op(w, stream)
    dt = _op_dtype(g, "g")
    if w.dim() not in (2, 3):
        raise ValueError("w must be [m][rows][cols] or [rows][cols]")
    rows, cols = w.shape[-2:]
    f32 = op.torch.float32
    wp, m, ws = op.stack(w, "w", (rows, cols), None, f32)
    vp, _, vs = op.stack(v, "v", (rows, cols), m, f32)
    gp, _, gs = op.stack(g, "g", (rows, cols), m)
    base, nbytes, keep = op.workspace(w, workspace, _ws_bytes("ls_orthogonalize_ws_bytes", m, rows, cols))
    op.call("ls_muon_step", wp, vp, gp, m, rows, cols, ws, vs, gs, dt, float(lr), float(momentum), int(bool(nesterov)),
            _int32(int(steps), LS_ERR_INVALID_ARG, "steps"), base, nbytes)


class LocalSGD:
    """m replicas of a fully connected model on one GPU, trained by local SGD
    steps and periodic averaging.  Thin wrapper over the ls_* calls."""

    def __init__(self, m: int, dims: Sequence[int], loss: str = "softmax_ce", has_bias: bool = True,
                 gemm_dtype: str = "fp32", lr: float = 0.05, momentum: float = 0.0, batch: int = 32,
                 momentum_mode: str = "average", device: str = "cuda:0", stream=None, block_momentum: float = 0.0):
        import torch
        self._torch = torch
        self.lib = _lib()
        self.m, self.batch, self.dims = int(m), int(batch), tuple(int(d) for d in dims)
        self.gemm_dtype = gemm_dtype
        self.loss_kind = loss
        self.spec = make_spec(dims, loss, has_bias, gemm_dtype, momentum_mode, block_momentum=block_momentum)
        self.P = param_count(self.spec)
        nbytes = state_bytes(self.m, self.spec, self.batch)
        self.device = torch.device(device)
        with torch.cuda.device(self.device):
            self.state = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.state.data_ptr()
            self._state_ptr = (base + 255) // 256 * 256
            self.stream = stream if stream is not None else torch.cuda.current_stream()
            h = C.c_void_p()
            _check(self.lib.ls_create(C.byref(h), self.m, C.byref(self.spec), float(lr), float(momentum), self.batch,
                                      self._state_ptr, nbytes, int(self.stream.cuda_stream)), "ls_create")
        self.h = h
        self._x = self._y = None

    # -- life cycle -------------------------------------------------------
    def close(self):
        if getattr(self, "h", None) is not None and self.h.value:
            self.lib.ls_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sync(self):
        _check(self.lib.ls_sync(self.h), "ls_sync")

    def selftest_wait_timeout(self, limit_cycles: int = 2_000_000):
        """Enqueue the kernel whose bounded wait runs out (ls_selftest_wait_timeout); the next call that waits
        for the stream raises LsError(LS_ERR_DEVICE_TIMEOUT)."""
        _check(self.lib.ls_selftest_wait_timeout(self.h, int(limit_cycles)), "ls_selftest_wait_timeout")

    def set_lr(self, lr: float):
        _check(self.lib.ls_set_lr(self.h, float(lr)), "ls_set_lr")

    # -- state ------------------------------------------------------------
    def set_params(self, x1: np.ndarray):
        a = np.ascontiguousarray(x1, dtype=np.float32)
        if a.size != self.P:
            raise ValueError("x1 has the wrong size")
        _check(self.lib.ls_set_params(self.h, a.ctypes.data), "ls_set_params")

    def set_state(self, replica: int, params: Optional[np.ndarray] = None, momentum: Optional[np.ndarray] = None):
        p = None if params is None else np.ascontiguousarray(params, dtype=np.float32)
        v = None if momentum is None else np.ascontiguousarray(momentum, dtype=np.float32)
        for a in (p, v):
            if a is not None and a.size != self.P:
                raise ValueError("wrong size")
        _check(self.lib.ls_set_state(self.h, int(replica), None if p is None else p.ctypes.data,
                                     None if v is None else v.ctypes.data), "ls_set_state")

    def set_block_state(self, anchor: Optional[np.ndarray] = None, u: Optional[np.ndarray] = None):
        a = None if anchor is None else np.ascontiguousarray(anchor, dtype=np.float32)
        b = None if u is None else np.ascontiguousarray(u, dtype=np.float32)
        for t in (a, b):
            if t is not None and t.size != self.P:
                raise ValueError("wrong size")
        _check(self.lib.ls_set_block_state(self.h, None if a is None else a.ctypes.data,
                                           None if b is None else b.ctypes.data), "ls_set_block_state")

    def get_block_state(self):
        a = np.empty(self.P, dtype=np.float32)
        b = np.empty(self.P, dtype=np.float32)
        _check(self.lib.ls_get_block_state(self.h, a.ctypes.data, b.ctypes.data), "ls_get_block_state")
        return a, b

    def get_state(self, replica: int):
        p = np.empty(self.P, dtype=np.float32)
        v = np.empty(self.P, dtype=np.float32)
        _check(self.lib.ls_get_state(self.h, int(replica), p.ctypes.data, v.ctypes.data), "ls_get_state")
        return p, v

    def get_all(self):
        ps, vs = zip(*(self.get_state(i) for i in range(self.m)))
        return np.stack(ps), np.stack(vs)

    def state_view(self):
        """(params, momentum) as float32 CUDA tensors [m][stride] aliasing the state block, to be read: the handle does
        not see what is written through them (ls_state_view)."""
        torch = self._torch
        pp, vp, st = C.c_void_p(), C.c_void_p(), C.c_int64()
        _check(self.lib.ls_state_view(self.h, C.byref(pp), C.byref(vp), C.byref(st)), "ls_state_view")
        base = self.state.data_ptr()
        out = []
        for ptr in (pp.value, vp.value):
            off = ptr - base
            out.append(self.state[off:off + self.m * st.value * 4].view(torch.float32).view(self.m, st.value))
        return out[0], out[1]

    def muon_step(self, layer: int, g, lr: float, momentum: float = 0.95, nesterov: bool = True, steps: int = 5,
                  workspace=None) -> None:
        """One orthogonalised momentum step of layer `layer`'s matrix (0-based) of all replicas, from gradients g
        [m][dims[layer + 1]][dims[layer]] (float32 or bfloat16), on the handle's stream (ls_muon_step_layer)."""
        if not 0 <= layer < len(self.dims) - 1:
            raise ValueError("no such layer")
        op = _Op(g, self.stream)
        dt = _op_dtype(g, "g")
        rows, cols = self.dims[layer + 1], self.dims[layer]
        gp, _, gs = op.stack(g, "g", (rows, cols), self.m)
        base, nbytes, keep = op.workspace(g, workspace, _ws_bytes("ls_orthogonalize_ws_bytes", self.m, rows, cols))
        with self._torch.cuda.device(self.device):
            _check(self.lib.ls_muon_step_layer(self.h, int(layer), gp, gs, dt, float(lr), float(momentum),
                                               int(bool(nesterov)), _int32(int(steps), LS_ERR_INVALID_ARG, "steps"), base,
                                               nbytes), "ls_muon_step_layer")

    # -- data ---------------------------------------------------------------
    def bind_dataset(self, x, y):
        torch = self._torch
        want = torch.bfloat16 if self.gemm_dtype == "bf16" else torch.float32
        ywant = torch.int32 if self.loss_kind == "softmax_ce" else torch.float32
        if not (x.is_cuda and x.dtype == want and x.is_contiguous() and x.dim() == 2 and x.shape[1] == self.dims[0]):
            raise ValueError(f"x must be a contiguous CUDA {want} tensor [n_rows][{self.dims[0]}]")
        if not (y.is_cuda and y.dtype == ywant and y.is_contiguous() and y.numel() == x.shape[0]):
            raise ValueError(f"y must be a contiguous CUDA {ywant} tensor [n_rows]")
        self._x, self._y = x, y
        _check(self.lib.ls_bind_dataset(self.h, x.data_ptr(), y.data_ptr(), int(x.shape[0])), "ls_bind_dataset")

    # -- hot path -----------------------------------------------------------
    def local_steps(self, tau: int, row_offsets: np.ndarray, loss_out=None, average: bool = False):
        """tau local steps; average=True: followed by the averaging step (one whole period, ls_local_steps_avg)."""
        offs = np.ascontiguousarray(row_offsets, dtype=np.int64)
        if offs.size != tau * self.m:
            raise ValueError("row_offsets must be [tau][m]")
        lp = None
        if loss_out is not None:
            torch = self._torch
            if not (loss_out.is_cuda and loss_out.dtype == torch.float32 and loss_out.is_contiguous()
                    and loss_out.numel() >= tau * self.m):
                raise ValueError("loss_out must be a contiguous float32 CUDA tensor [tau][m]")
            lp = loss_out.data_ptr()
        if average:
            _check(self.lib.ls_local_steps_avg(self.h, int(tau), offs.ctypes.data, lp), "ls_local_steps_avg")
        else:
            _check(self.lib.ls_local_steps(self.h, int(tau), offs.ctypes.data, lp), "ls_local_steps")

    def local_steps_host(self, tau: int, x_host, y_host, loss_host):
        """x_host [tau][m][batch][d_in], y_host [tau][m][batch], loss_host float32 [tau][m]: CPU torch
        tensors (pinned for overlap)."""
        _check(self.lib.ls_local_steps_host(self.h, int(tau), x_host.data_ptr(), y_host.data_ptr(),
                                            loss_host.data_ptr()), "ls_local_steps_host")

    def average(self):
        _check(self.lib.ls_average(self.h), "ls_average")

    def eval_loss(self, replica: int, row_offset: int, n_rows: int) -> float:
        f = C.c_float()
        _check(self.lib.ls_eval_loss(self.h, int(replica), int(row_offset), int(n_rows), C.byref(f)), "ls_eval_loss")
        return float(f.value)

    def run(self, K: int, tau_0: int, row_offsets: np.ndarray, interval: int = 0, probe_rows: int = 0, loss_out=None):
        """K iterations of local steps + averaging in native code; AdaComm when interval > 0."""
        offs = np.ascontiguousarray(row_offsets, dtype=np.int64)
        if offs.size != K * self.m:
            raise ValueError("row_offsets must be [K][m]")
        max_p = int(K) + 1
        period_tau = np.zeros(max_p, dtype=np.int32)
        dk = np.zeros(max_p, dtype=np.int64)
        dF = np.zeros(max_p, dtype=np.float32)
        dt = np.zeros(max_p, dtype=np.int32)
        n_p, n_d, F0 = C.c_int64(), C.c_int64(), C.c_float()
        lp = None if loss_out is None else loss_out.data_ptr()
        _check(self.lib.ls_run(self.h, int(K), int(tau_0), int(interval), int(probe_rows), offs.ctypes.data, lp,
                               period_tau.ctypes.data, max_p, C.byref(n_p), dk.ctypes.data, dF.ctypes.data,
                               dt.ctypes.data, max_p, C.byref(n_d), C.byref(F0)), "ls_run")
        n_p, n_d = n_p.value, n_d.value
        return {"taus": period_tau[:n_p].tolist(), "decision_k": dk[:n_d].tolist(), "decision_F": dF[:n_d].copy(),
                "decision_tau": dt[:n_d].tolist(), "F_0": float(F0.value) if interval > 0 else None}

    def run_timed(self, K: int, tau_0: int, T0_ms: float, row_offsets: np.ndarray, probe_rows: int, loss_out=None):
        """K iterations with AdaComm decisions at wall-clock intervals of T0_ms (Section 4)."""
        offs = np.ascontiguousarray(row_offsets, dtype=np.int64)
        if offs.size != K * self.m:
            raise ValueError("row_offsets must be [K][m]")
        max_p = int(K) + 1
        period_tau = np.zeros(max_p, dtype=np.int32)
        dk = np.zeros(max_p, dtype=np.int64)
        dF = np.zeros(max_p, dtype=np.float32)
        dt = np.zeros(max_p, dtype=np.int32)
        dms = np.zeros(max_p, dtype=np.float64)
        n_p, n_d, F0 = C.c_int64(), C.c_int64(), C.c_float()
        lp = None if loss_out is None else loss_out.data_ptr()
        _check(self.lib.ls_run_timed(self.h, int(K), int(tau_0), float(T0_ms), int(probe_rows), offs.ctypes.data, lp,
                                     period_tau.ctypes.data, max_p, C.byref(n_p), dk.ctypes.data, dF.ctypes.data,
                                     dt.ctypes.data, dms.ctypes.data, max_p, C.byref(n_d), C.byref(F0)),
               "ls_run_timed")
        n_p, n_d = n_p.value, n_d.value
        return {"taus": period_tau[:n_p].tolist(), "decision_k": dk[:n_d].tolist(), "decision_F": dF[:n_d].copy(),
                "decision_tau": dt[:n_d].tolist(), "decision_ms": dms[:n_d].copy(), "F_0": float(F0.value)}

    def profile_begin(self, classes: Sequence[str] = KERNEL_CLASSES, layer: int = -1):
        mask = 0
        for c in classes:
            mask |= 1 << KERNEL_CLASSES.index(c)
        _check(self.lib.ls_profile_begin(self.h, mask, int(layer)), "ls_profile_begin")

    def profile_end(self):
        """{(class, layer): (total ms, launches)} for what ran since profile_begin()."""
        n = len(KERNEL_CLASSES) * LS_MAX_LAYERS
        ms = (C.c_double * n)()
        cnt = (C.c_int64 * n)()
        _check(self.lib.ls_profile_end(self.h, ms, cnt), "ls_profile_end")
        out = {}
        for ci, cname in enumerate(KERNEL_CLASSES):
            for l in range(LS_MAX_LAYERS):
                if cnt[ci * LS_MAX_LAYERS + l]:
                    out[(cname, l)] = (ms[ci * LS_MAX_LAYERS + l], cnt[ci * LS_MAX_LAYERS + l])
        return out

    def run_refined(self, K: int, tau_0: int, row_offsets: np.ndarray, interval: int, probe_rows: int,
                    gamma: float = 0.5, slack: int = 0, decay_at: Sequence[int] = (), decay_factor: float = 0.1,
                    loss_out=None):
        """ls_run_refined: AdaComm with the saturation decay and the learning-rate coupling (Section 4.3)."""
        offs = np.ascontiguousarray(row_offsets, dtype=np.int64)
        if offs.size != K * self.m:
            raise ValueError("row_offsets must be [K][m]")
        dec = np.ascontiguousarray(decay_at, dtype=np.int64)
        opts = AdacommOpts(float(gamma), int(slack), int(dec.size), dec.ctypes.data if dec.size else None,
                           float(decay_factor))
        max_p = int(K) + 1
        period_tau = np.zeros(max_p, dtype=np.int32)
        dk = np.zeros(max_p, dtype=np.int64)
        dF = np.zeros(max_p, dtype=np.float32)
        dt = np.zeros(max_p, dtype=np.int32)
        n_p, n_d, F0 = C.c_int64(), C.c_int64(), C.c_float()
        lp = None if loss_out is None else loss_out.data_ptr()
        _check(self.lib.ls_run_refined(self.h, int(K), int(tau_0), int(interval), int(probe_rows), offs.ctypes.data, lp,
                                       C.byref(opts), period_tau.ctypes.data, max_p, C.byref(n_p), dk.ctypes.data,
                                       dF.ctypes.data, dt.ctypes.data, max_p, C.byref(n_d), C.byref(F0)),
               "ls_run_refined")
        lr = C.c_float()
        _check(self.lib.ls_get_lr(self.h, C.byref(lr)), "ls_get_lr")
        n_p, n_d = n_p.value, n_d.value
        return {"taus": period_tau[:n_p].tolist(), "decision_k": dk[:n_d].tolist(), "decision_F": dF[:n_d].copy(),
                "decision_tau": dt[:n_d].tolist(), "F_0": float(F0.value), "lr": float(lr.value)}

    # -- one job on several GPUs ----------------------------------------------
    def shard_buffer_floats(self) -> int:
        n = C.c_int64()
        _check(self.lib.ls_shard_buffer_floats(self.h, C.byref(n)), "ls_shard_buffer_floats")
        return n.value

    def set_shard(self, n_gpus: int, m_total: int, partial=None, gathered=None, exchange=None):
        """ls_set_shard: this handle's replicas are one rank's share of a job of m_total replicas.  `exchange` is
        a Python callable (partial_ptr, gathered_ptr, nbytes, n_gpus) -> 0 on success; the buffers and the
        callback object are kept alive by this wrapper."""
        if n_gpus == 0:
            _check(self.lib.ls_set_shard(self.h, 0, 0, None, None, EXCHANGE_FN(0), None), "ls_set_shard")
            self._shard = None
            return
        cb = EXCHANGE_FN(0) if exchange is None else EXCHANGE_FN(lambda ctx, p, g, nbytes, n: int(exchange(p, g, nbytes, n)))
        _check(self.lib.ls_set_shard(self.h, int(n_gpus), int(m_total), partial.data_ptr(),
                                     None if gathered is None else gathered.data_ptr(), cb, None), "ls_set_shard")
        self._shard = (partial, gathered, cb)

    def shard_partial_sum(self, partial):
        _check(self.lib.ls_shard_partial_sum(self.h, partial.data_ptr()), "ls_shard_partial_sum")

    def shard_average(self, gathered, n_gpus: int, m_total: int):
        _check(self.lib.ls_shard_average(self.h, gathered.data_ptr(), int(n_gpus), int(m_total)), "ls_shard_average")

    def launch_count(self) -> int:
        n = C.c_int64()
        _check(self.lib.ls_launch_count(self.h, C.byref(n)), "ls_launch_count")
        return n.value
