"""Oscars local-SGD hot path on MI355X (gfx950): Python binding.

A thin ctypes layer over the C ABI declared in ``include/oscars.h``.  It only
marshals arguments (torch tensors become device pointers, the current torch
stream becomes the HIP stream); every step of the hot path runs in the HIP
library ``_lib/liboscars.so``.  If that library is missing the import of this
package fails: there is no CPU fallback.

Build with ``python paper_2102_08550_amd/build.py`` (or
``__graft_entry__.build()``).
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
import os
from typing import List, Optional, Sequence, Tuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "liboscars.so")

OK, E_INVALID, E_NOMEM, E_HIP, E_INFEASIBLE, E_STATE = 0, -1, -2, -3, -4, -5
FP32, BF16 = 0, 1
MAX_K = 64
EVAL_NOALLOC_MAX_ROWS = 262144
MAX_MATRICES = 32
# Newton-Schulz steps (a, b, c) of ``orthogonalize``: the quintic whose slope at
# zero is steep, five times (singular values end between about 0.7 and 1.2).
NEWTON_SCHULZ = ((3.4445, -4.7750, 2.0315),) * 5
(KERNEL_CAST, KERNEL_FWD, KERNEL_SOFTMAX, KERNEL_DGRAD, KERNEL_WGRAD, KERNEL_AGGREGATE,
 KERNEL_BWD_FUSED) = range(7)
KERNEL_NAMES = ("cast_bf16", "gemm_fwd", "softmax_ce", "gemm_dgrad", "gemm_wgrad_update",
                "aggregate", "gemm_bwd_fused")

_i32, _i64, _u32, _u64, _f32, _vp = (ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32,
                                     ctypes.c_uint64, ctypes.c_float, ctypes.c_void_p)
_P = ctypes.POINTER


class OscarsError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {_lib().oscars_status_str(status).decode()} (status {status}"
                         + (f", hip error {_lib().oscars_last_hip_error()}" if status == E_HIP
                            else "") + ")")


class _Model(ctypes.Structure):
    _fields_ = [("n_layers", _i32), ("dims", _P(_i32)), ("dtype", _i32)]


class _CnnModel(ctypes.Structure):
    _fields_ = [("height", _i32), ("width", _i32), ("channels", _i32), ("n_conv", _i32),
                ("conv_channels", _P(_i32)), ("conv_strides", _P(_i32)), ("classes", _i32),
                ("conv_skip", _P(_i32))]


class _Matrix(ctypes.Structure):
    _fields_ = [("rows", _i32), ("cols", _i32), ("x", _vp), ("x_ld", _i64), ("out", _vp),
                ("out_ld", _i64)]


class _ServerOptions(ctypes.Structure):
    _fields_ = [("lr", _f32), ("beta", _f32), ("weight_decay", _f32), ("plain_lr", _f32),
                ("nesterov", _i32), ("plain_layers", _u32), ("coeffs", _P(_f32)),
                ("steps", _i32)]


class _Dropout(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", _u64), ("offset", _u64), ("offset_device", _vp)]


class _Gradients(ctypes.Structure):
    _fields_ = [("rows", _i64), ("inputs", _i64), ("outs", _i64), ("dy", _vp), ("y", _vp),
                ("x", _vp), ("dy_ld", _i64), ("y_ld", _i64), ("x_ld", _i64), ("y_dtype", _i32),
                ("x_dtype", _i32), ("wtq", _vp), ("wtscale", _vp), ("wt_ld", _i64),
                ("wts_ld", _i64), ("dx", _vp), ("dw", _vp), ("db", _vp), ("dx_ld", _i64),
                ("dw_ld", _i64), ("dropout", _vp)]


class _Shards(ctypes.Structure):
    _fields_ = [("x", _vp), ("y", _vp), ("n_rows", _i64), ("offsets", _P(_i64)), ("seed", _u64)]


_LIB = None
_SAME_DEVICE = contextlib.nullcontext()

# name -> (restype, argtypes)
_SIGS = {
    "oscars_create": (_i32, [_P(_vp), _P(_Model), _i32, _i32, _vp]),
    "oscars_create_cnn": (_i32, [_P(_vp), _P(_CnnModel), _i32, _i32, _vp]),
    "oscars_destroy": (None, [_vp]),
    "oscars_set_stream": (_i32, [_vp, _vp]),
    "oscars_num_params": (_i64, [_vp]),
    "oscars_layer_offsets": (_i32, [_vp, _i32, _P(_i64), _P(_i64)]),
    "oscars_load_balance": (_i32, [_P(_i64), _i32, _i64, _P(_i64), _P(_i32)]),
    "oscars_paper_weights": (_i32, [_P(_i32), _i32, _P(_f32)]),
    "oscars_shard_offsets": (_i32, [_i64, _i32, _P(_i64)]),
    "oscars_sample_indices": (_i32, [_P(_Shards), _i32, _i32, _i64, _i32, _i32, _P(_i64)]),
    "oscars_local_steps": (_i32, [_vp, _vp, _P(_Shards), _P(_i32), _f32, _i32]),
    "oscars_round": (_i32, [_vp, _vp, _vp, _P(_Shards), _P(_i32), _f32, _i32, _P(_f32)]),
    "oscars_round_losses": (_i32, [_vp, _P(_f32)]),
    "oscars_aggregate": (_i32, [_vp, _vp, _P(_f32), _i32, _i64, _i64, _i32, _vp]),
    "oscars_get_cursors": (_i32, [_vp, _P(_i64)]),
    "oscars_set_cursors": (_i32, [_vp, _P(_i64)]),
    "oscars_profile_begin": (_i32, [_vp, _u32]),
    "oscars_profile_end": (_i32, [_vp, _P(ctypes.c_double), _P(_i64)]),
    "oscars_set_gemm_tiling": (_i32, [_vp, _i32]),
    "oscars_tuning_pending": (_i32, [_vp, _P(_i32)]),
    "oscars_set_backward": (_i32, [_vp, _i32]),
    "oscars_backward_path": (_i32, [_vp, _i32, _i32, _i32, _P(_i32)]),
    "oscars_broadcast": (_i32, [_vp, _vp, _i32, _i64, _i64, _vp]),
    "oscars_plan_tau": (_i32, [_P(ctypes.c_double), _i32, _i32, _i64, _P(_i64), _P(_i64), _P(_i32)]),
    "oscars_evaluate": (_i32, [_vp, _vp, _vp, _vp, _i64, _P(ctypes.c_double), _P(_i64)]),
    "oscars_evaluate_noalloc": (_i32, [_vp, _vp, _vp, _vp, _i64, _P(ctypes.c_double),
                                       _P(_i64)]),
    "oscars_orthogonalize_workspace": (_i64, [_P(_Matrix), _i32]),
    "oscars_orthogonalize": (_i32, [_P(_Matrix), _i32, _i32, _P(_f32), _i32, _vp, _i64, _vp]),
    "oscars_server_workspace": (_i64, [_vp]),
    "oscars_server_step": (_i32, [_vp, _vp, _vp, _P(_f32), _vp, _vp, _vp, _P(_ServerOptions), _vp,
                                  _i64]),
    "oscars_quantize_rows": (_i32, [_vp, _i64, _vp, _vp, _i64, _i32, _i64, _i32, _vp]),
    "oscars_matmul_quantized": (_i32, [_vp, _i64, _i32, _vp, _i64, _vp, _vp, _i64, _vp, _vp, _i32,
                                       _i64, _i32, _i32, _vp]),
    "oscars_linear_quantized_workspace": (_i64, [_i64, _i32]),
    "oscars_linear_quantized": (_i32, [_vp, _i64, _i32, _vp, _i64, _i32, _vp, _i64, _vp, _vp, _i32,
                                       _i64, _i32, _i32, _vp, _i64, _vp]),
    "oscars_quantize_micro": (_i32, [_vp, _i64, _vp, _i64, _vp, _i64, _i32, _i64, _i64, _i32, _vp]),
    "oscars_dequantize_micro": (_i32, [_vp, _i64, _i32, _vp, _i64, _vp, _i64, _i64, _i64, _vp]),
    "oscars_matmul_micro": (_i32, [_vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp,
                                   _i32, _P(_Dropout), _i64, _i64, _i64, _vp]),
    "oscars_linear_micro_workspace": (_i64, [_i64, _i64]),
    "oscars_linear_micro": (_i32, [_vp, _i64, _i32, _vp, _i64, _i32, _vp, _i64, _vp, _i64, _vp,
                                   _i32, _P(_Dropout), _i64, _i64, _i64, _vp, _i64, _vp]),
    "oscars_linear_micro_backward_workspace": (_i64, [_i64, _i64, _i64, _i32]),
    "oscars_linear_micro_backward": (_i32, [_P(_Gradients), _vp, _i64, _vp]),
    "oscars_dropout": (_i32, [_vp, _i64, _vp, _i64, _i32, _P(_Dropout), _i64, _i64, _vp]),
    "oscars_micro_model_bytes": (_i64, [_vp]),
    "oscars_quantize_model_micro": (_i32, [_vp, _vp, _vp]),
    "oscars_evaluate_micro": (_i32, [_vp, _vp, _vp, _vp, _i64, _P(ctypes.c_double), _P(_i64)]),
    "oscars_quantized_model_bytes": (_i64, [_vp]),
    "oscars_quantize_model": (_i32, [_vp, _vp, _vp]),
    "oscars_evaluate_quantized": (_i32, [_vp, _vp, _vp, _vp, _i64, _P(ctypes.c_double), _P(_i64)]),
    "oscars_status_str": (ctypes.c_char_p, [_i32]),
    "oscars_last_hip_error": (_i32, []),
}


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"HIP library not built: {LIB_PATH} is missing "
                              "(run python paper_2102_08550_amd/build.py)")
        # torch first: the library then binds to the HIP runtime torch has
        # loaded, so that both share one runtime (and one view of the GPU).
        import torch  # noqa: F401
        lib = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


_lib()  # fail at import time when the library is absent
import torch  # noqa: E402  (loaded by _lib, in front of the library)


def _check(status: int, what: str):
    if status != OK:
        raise OscarsError(status, what)


_CTYPES = {np.int32: _i32, np.int64: _i64, np.float32: _f32}


def _arr(a, dtype):
    """``a`` as a contiguous array of ``dtype`` and a C pointer to it.  (Through
    the buffer protocol: 1.3 us for five values, 5.8 us by way of
    ndarray.ctypes and a pointer type looked up per call; a round passes
    three such arrays, an average one.)"""
    a = np.ascontiguousarray(a, dtype=dtype)
    c = _CTYPES[dtype]
    if a.size and a.flags.writeable:
        return a, ctypes.pointer(c.from_buffer(a))
    return a, a.ctypes.data_as(_P(c))


# the handle alone where torch gives it (0.5 us, by way of a Stream object 4)
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream=None, device=None) -> Optional[int]:
    """``stream``'s handle, or the current one's of ``device`` (None: of the current device)."""
    if stream is not None:
        return stream.cuda_stream
    if _RAW_STREAM is not None:
        return _RAW_STREAM(torch.cuda.current_device() if device is None else device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _dev_ptr(t, dtype=None, what="tensor") -> int:
    import torch
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{what} must be a CUDA (HIP) tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {t.dtype}")
    return t.data_ptr()


# ---------------------------------------------------------------- host-only calls

def load_balance(t_iter: Sequence[int], M: int) -> Tuple[int, List[int]]:
    """Algorithm 1: (T*, tau) for integer iteration times t_iter and bound M."""
    t, tp = _arr(t_iter, np.int64)
    tau = np.zeros(len(t), np.int32)
    T = _i64(0)
    _check(_lib().oscars_load_balance(tp, len(t), int(M), ctypes.byref(T),
                                      tau.ctypes.data_as(_P(_i32))), "oscars_load_balance")
    return int(T.value), tau.tolist()


def plan_tau(t_measured: Sequence[float], resolution: int, M: int):
    """The controller's plan from measured iteration times: (ticks, T*, tau).
    The tick is min(t) / resolution; Algorithm 1 then runs on the ticks."""
    t = np.ascontiguousarray(t_measured, dtype=np.float64)
    ticks = np.zeros(len(t), np.int64)
    tau = np.zeros(len(t), np.int32)
    T = _i64(0)
    _check(_lib().oscars_plan_tau(t.ctypes.data_as(_P(ctypes.c_double)), len(t), int(resolution),
                                  int(M), ticks.ctypes.data_as(_P(_i64)), ctypes.byref(T),
                                  tau.ctypes.data_as(_P(_i32))), "oscars_plan_tau")
    return ticks.tolist(), int(T.value), tau.tolist()


def paper_weights(K: int, staleness: Optional[Sequence[int]] = None) -> np.ndarray:
    w = np.zeros(K, np.float32)
    st = None
    if staleness is not None:
        st, stp = _arr(staleness, np.int32)
    else:
        stp = None
    _check(_lib().oscars_paper_weights(stp, int(K), w.ctypes.data_as(_P(_f32))),
           "oscars_paper_weights")
    return w


def shard_offsets(n_rows: int, K: int) -> List[int]:
    off = np.zeros(K + 1, np.int64)
    _check(_lib().oscars_shard_offsets(int(n_rows), int(K), off.ctypes.data_as(_P(_i64))),
           "oscars_shard_offsets")
    return off.tolist()


def _shards(x_ptr, y_ptr, n_rows, offsets, seed):
    off, offp = _arr(offsets, np.int64)
    sh = _Shards(x_ptr, y_ptr, int(n_rows), offp, ctypes.c_uint64(seed & (2**64 - 1)).value)
    return sh, off  # keep `off` alive with the struct


def sample_indices(n_rows: int, offsets: Sequence[int], seed: int, k: int, first_step: int,
                   steps: int, batch: int) -> np.ndarray:
    sh, keep = _shards(None, None, n_rows, offsets, seed)
    out = np.zeros((steps, batch), np.int64)
    _check(_lib().oscars_sample_indices(ctypes.byref(sh), len(offsets) - 1, int(k),
                                        int(first_step), int(steps), int(batch),
                                        out.ctypes.data_as(_P(_i64))), "oscars_sample_indices")
    return out


# ---------------------------------------------------------------- GPU calls

# Forward / backward-data GEMM tilings (oscars_set_gemm_tiling); results are
# bit-identical for every tiling.
TILING_AUTO, TILING_L, TILING_M, TILING_S, TILING_W, TILING_WS, TILING_VS, TILING_LS = range(8)
TILINGS = {"auto": TILING_AUTO, "L": TILING_L, "M": TILING_M, "S": TILING_S, "W": TILING_W,
           "WS": TILING_WS, "VS": TILING_VS, "LS": TILING_LS}



# Backward pass of hidden bf16 layers (oscars_set_backward); results are
# bit-identical in every mode.
BACKWARD_AUTO, BACKWARD_SEPARATE, BACKWARD_FUSED, BACKWARD_FUSED_SPLIT = range(4)
BACKWARDS = {"auto": BACKWARD_AUTO, "separate": BACKWARD_SEPARATE, "fused": BACKWARD_FUSED,
             "fused_split": BACKWARD_FUSED_SPLIT}



def aggregate(global_, replicas, weights: Sequence[float], K: int, n: int, ld: int,
              broadcast: bool = False, stream=None):
    """global_[i] = pairwise-tree sum_k w_k replicas[k*ld + i]; optional broadcast."""
    import torch
    gp = _dev_ptr(global_, torch.float32, "global")
    rp = _dev_ptr(replicas, torch.float32, "replicas")
    if global_.numel() < n or replicas.numel() < (K - 1) * ld + n:
        raise ValueError("buffers smaller than K, n, ld imply")
    w, wp = _arr(weights, np.float32)
    if len(w) != K:
        raise ValueError("one weight per replica")
    _check(_lib().oscars_aggregate(gp, rp, wp, int(K), int(n), int(ld), int(bool(broadcast)),
                                   _stream_handle(stream)), "oscars_aggregate")


def broadcast(global_, replicas, K: int, n: int, ld: int, stream=None):
    """replicas[k*ld + i] = global_[i] for k < K, i < n (the step after Eq. 4's average)."""
    import torch
    gp = _dev_ptr(global_, torch.float32, "global")
    rp = _dev_ptr(replicas, torch.float32, "replicas")
    if global_.numel() < n or replicas.numel() < (K - 1) * ld + n:
        raise ValueError("buffers smaller than K, n, ld imply")
    _check(_lib().oscars_broadcast(gp, rp, int(K), int(n), int(ld), _stream_handle(stream)),
           "oscars_broadcast")


def _on_device(device):
    """The context in which a call's kernels go to ``device``."""
    if torch.cuda.current_device() == device.index:
        return _SAME_DEVICE
    return torch.cuda.device(device)


def _workspace(nbytes: int, device, stream=None):
    """Device memory for one call on ``stream`` (None: the current one): torch's
    allocator gives it to later work of that stream only."""
    if stream is None or stream == torch.cuda.current_stream(device):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _used_on(stream, *tensors):
    """What a call on ``stream`` reads or writes (None: the current one, whose work
    torch orders by itself): dropped by the caller, it is not given to other
    streams' work before the call has run."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


@functools.lru_cache(maxsize=16)
def _coeffs(coeffs):
    """((a, b, c), ...) as a C array, kept with its number of steps."""
    flat = [float(v) for step in coeffs for v in step]
    if not coeffs or any(len(step) != 3 for step in coeffs):
        raise ValueError("coeffs must be a sequence of (a, b, c)")
    return (_f32 * len(flat))(*flat), len(coeffs)


def _matrix_view(t, what):
    """(rows, cols, row stride, turned) of a 2-D tensor stored by rows, or by
    columns (then of its transpose).  A single row or column is a column of
    rows of one element each, whatever its stride."""
    if t.dim() != 2 or t.numel() == 0:
        raise ValueError(f"{what} must be a matrix that is not empty")
    (r, c), (sr, sc) = t.shape, t.stride()
    if r == 1 or c == 1:
        n, step = (r, sr) if c == 1 else (c, sc)
        if step >= 1 or n == 1:
            return n, 1, step if n > 1 else 1, False
    elif sc == 1 and sr >= c:
        return r, c, sr, False
    elif sr == 1 and sc >= r:
        return c, r, sc, True
    raise ValueError(f"{what} must have one unit stride and rows that do not overlap")


def orthogonalize(x, out=None, coeffs=NEWTON_SCHULZ, stream=None):
    """Newton-Schulz orthogonalisation (oscars_orthogonalize) of the matrix ``x``
    or of every matrix of a sequence, in one call: fp32 or bf16 device tensors
    of one type, stored by rows or by columns, with any stride between them.
    ``out``: where the results go (``x`` itself is allowed), stored the same
    way; new tensors by default.  ``coeffs``: each step's (a, b, c); steps that
    leave fp16's range are refused.  Returns ``out``."""
    import torch
    single = isinstance(x, torch.Tensor)
    xs = [x] if single else list(x)
    if not 1 <= len(xs) <= MAX_MATRICES:
        raise ValueError(f"1 to {MAX_MATRICES} matrices per call")
    dt, dev = xs[0].dtype, xs[0].device
    if dt not in (torch.float32, torch.bfloat16):
        raise TypeError("matrices must be fp32 or bf16")
    views = [_matrix_view(t, "x") for t in xs]
    if out is None:
        # dense results stored as x is, for work on the call's stream
        with torch.cuda.stream(stream):
            outs = [torch.empty_like(t.mT).mT if v[3] else torch.empty_like(t)
                    for t, v in zip(xs, views)]
    else:
        outs = [out] if single else list(out)
    if len(outs) != len(xs):
        raise ValueError("one output per matrix")
    mats = (_Matrix * len(xs))()
    for m, t, o, v in zip(mats, xs, outs, views):
        if not (t.is_cuda and o.is_cuda) or t.device != dev or o.device != dev:
            raise TypeError("matrices must be on one CUDA (HIP) device")
        if t.dtype != dt or o.dtype != dt:
            raise TypeError("matrices must have one type")
        if t.shape != o.shape:
            raise ValueError("an output must have its matrix's shape")
        ov = _matrix_view(o, "out")
        if v[3] != ov[3]:
            raise ValueError("out must be stored as x is")
        m.rows, m.cols, m.x, m.x_ld, m.out, m.out_ld = (v[0], v[1], t.data_ptr(), v[2],
                                                        o.data_ptr(), ov[2])
    ca, steps = _coeffs(tuple(map(tuple, coeffs)))
    with _on_device(dev):
        need = _lib().oscars_orthogonalize_workspace(mats, len(xs))
        ws = _workspace(need, dev, stream)
        _check(_lib().oscars_orthogonalize(mats, len(xs), FP32 if dt == torch.float32 else BF16,
                                           ca, steps, ws.data_ptr(), need,
                                           _stream_handle(stream)), "oscars_orthogonalize")
    _used_on(stream, *xs, *outs)
    return outs[0] if single else outs


def _float_type(dtype, what) -> int:
    if dtype == torch.float32:
        return FP32
    if dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"{what} must be fp32 or bf16, got {dtype}")


def _rows(t, dtype, device, what):
    """(pointer, rows, row stride, columns) of a 2-D device tensor stored by rows."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != device:
        raise TypeError(f"{what} must be a tensor on the input's CUDA (HIP) device")
    if t.dtype != dtype:
        raise TypeError(f"{what} must have dtype {dtype}, got {t.dtype}")
    shape, strides = t.shape, t.stride()
    if len(shape) != 2 or (shape[1] > 1 and strides[1] != 1) or (
            shape[0] > 1 and strides[0] < shape[1]):
        raise ValueError(f"{what} must be a matrix stored by rows that do not overlap")
    n, c = shape
    return t.data_ptr(), n, max(strides[0], c), c


def _vector(t, n, device, what):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.device != device:
        raise TypeError(f"{what} must be a tensor on the input's CUDA (HIP) device")
    if t.dtype != torch.float32 or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} must be {n} contiguous fp32 values")
    return t.data_ptr()


def _new(shape, dtype, device, stream):
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def quantize_rows(x, out=None, stream=None):
    """The rows of ``x`` (fp32 or bf16 matrix, any row stride) in 8 bits with a
    scale each (oscars_quantize_rows): ``(q, scale)``, q int8 [rows][columns
    rounded up to 128, zero behind the columns], scale fp32 [rows].  ``out``:
    such a pair to write into: the row stride of q a multiple of 16, and q as
    wide as the padding goes, to the next multiple of 128 columns or, where rows
    are shorter than that, to their end (a window of wider rows holds all of it)."""
    import torch
    dev = x.device
    xp, n, ld, cols = _rows(x, x.dtype, dev, "x")
    dt = _float_type(x.dtype, "x")
    if out is None:
        out = (_new((n, (cols + 127) // 128 * 128), torch.int8, dev, stream),
               _new((n,), torch.float32, dev, stream))
    q, scale = out
    qp, qn, qld, qc = _rows(q, torch.int8, dev, "q")
    if qn != n or qc < max(cols, min(qld, (cols + 127) // 128 * 128)):
        raise ValueError("q must have a row per row of x, of its columns and the zeros behind them")
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_quantize_rows(qp, qld, _vector(scale, n, dev, "scale"), xp, ld, dt, n,
                                           cols, _stream_handle(stream)), "oscars_quantize_rows")
    _used_on(stream, x, q, scale)
    return out


def matmul_i8(xq, xscale, wq, wscale, in_features: int, bias=None, relu: bool = False,
              out_dtype=None, out=None, stream=None):
    """xscale wscale (xq wq') + bias (oscars_matmul_quantized) for quantised rows ``xq``
    [rows][..] and weights ``wq`` [outputs][..] as quantize_rows gives them, of
    ``in_features`` columns; fp32 by default.  Returns ``out``."""
    import torch
    dev = xq.device
    xp, n, xld, xc = _rows(xq, torch.int8, dev, "xq")
    wp, outs, wld, wc = _rows(wq, torch.int8, dev, "wq")
    if xc < (in_features + 127) // 128 * 128 or wc < in_features:
        raise ValueError("xq must hold in_features columns rounded up to 128, wq in_features")
    if out is None:
        out = _new((n, outs), out_dtype or torch.float32, dev, stream)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError("out has another dtype than out_dtype")
    op, on, old, oc = _rows(out, out.dtype, dev, "out")
    if (on, oc) != (n, outs):
        raise ValueError("out must be [rows][outputs]")
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_matmul_quantized(
            op, old, _float_type(out.dtype, "out"), xp, xld, _vector(xscale, n, dev, "xscale"), wp,
            wld, _vector(wscale, outs, dev, "wscale"), _vector(bias, outs, dev, "bias"),
            int(bool(relu)), n, int(in_features), outs, _stream_handle(stream)),
            "oscars_matmul_quantized")
    _used_on(stream, xq, xscale, wq, wscale, bias, out)
    return out


def linear_i8(x, wq, wscale, bias=None, relu: bool = False, out_dtype=None, out=None, stream=None):
    """A linear layer in 8 bits (oscars_linear_quantized): the rows of ``x`` (fp32 or
    bf16) are quantised with a scale each, ``wq`` [outputs][inputs or more, the
    row stride a multiple of 16] and ``wscale`` are a weight matrix's
    quantize_rows.  The result has ``x``'s type by default.  Returns ``out``."""
    import torch
    dev = x.device
    xp, n, xld, cols = _rows(x, x.dtype, dev, "x")
    dt = _float_type(x.dtype, "x")
    wp, outs, wld, wc = _rows(wq, torch.int8, dev, "wq")
    if wc < cols:
        raise ValueError("wq must have as many columns as x, or more")
    if out is None:
        out = _new((n, outs), out_dtype or x.dtype, dev, stream)
    elif out_dtype is not None and out.dtype != out_dtype:
        raise TypeError("out has another dtype than out_dtype")
    op, on, old, oc = _rows(out, out.dtype, dev, "out")
    if (on, oc) != (n, outs):
        raise ValueError("out must be [rows][outputs]")
    if n == 0:
        return out
    lib = _lib()
    need = lib.oscars_linear_quantized_workspace(n, cols)
    ws = _workspace(need, dev, stream) if need else None
    with _on_device(dev):
        _check(lib.oscars_linear_quantized(
            op, old, _float_type(out.dtype, "out"), xp, xld, dt, wp, wld,
            _vector(wscale, outs, dev, "wscale"), _vector(bias, outs, dev, "bias"),
            int(bool(relu)), n, cols, outs, ws.data_ptr() if need else None, need,
            _stream_handle(stream)), "oscars_linear_quantized")
    _used_on(stream, x, wq, wscale, bias, out)
    return out


def _micro_shapes(rows: int, cols: int):
    """The shapes of ``rows`` rows of ``cols`` entries in 4 bits and of their scales."""
    return (rows, (cols + 255) // 256 * 128), (rows, (cols + 511) // 512 * 16)


def _count(q, what) -> int:
    if not isinstance(q, torch.Tensor) or q.dim() != 2:
        raise TypeError(f"{what} must be a matrix of quantised rows")
    return q.shape[0]


def _micro_rows(q, scale, rows, cols, device, what):
    """(pointer, row stride, scales' pointer, row stride) of quantised rows."""
    if (not isinstance(q, torch.Tensor) or not isinstance(scale, torch.Tensor)
            or q.device != device or scale.device != device or not q.is_cuda):
        raise TypeError(f"{what} and its scales must be tensors on the input's CUDA (HIP) device")
    if q.dtype != torch.uint8 or scale.dtype != torch.uint8:
        raise TypeError(f"{what} and its scales must have dtype uint8")
    width, blocks = (cols + 255) // 256 * 128, (cols + 511) // 512 * 16
    qs, ss = q.shape, scale.shape
    if (len(qs) != 2 or len(ss) != 2 or qs[0] != rows or ss[0] != rows or qs[1] < width
            or ss[1] < blocks):
        raise ValueError(f"{what} must hold {rows} rows of {width} bytes and {blocks} scales")
    if rows <= 1:  # the stride of a single row says nothing
        if (qs[1] > 1 and q.stride(1) != 1) or (ss[1] > 1 and scale.stride(1) != 1):
            raise ValueError(f"{what} must be stored by rows")
        return q.data_ptr(), width, scale.data_ptr(), blocks
    (qld, qstep), (sld, sstep) = q.stride(), scale.stride()
    if ((qs[1] > 1 and qstep != 1) or (ss[1] > 1 and sstep != 1) or qld < qs[1] or sld < ss[1]):
        raise ValueError(f"{what} must be stored by rows that do not overlap")
    return q.data_ptr(), qld, scale.data_ptr(), sld


def _dropout_options(dropout, device):
    """(options, the offset's tensor) of ``(p, seed[, offset])``; Nones for None."""
    if dropout is None:
        return None, None
    p, seed, offset = dropout if len(dropout) == 3 else (*dropout, 0)
    p, seed = float(p), int(seed)
    if not 0.0 <= p <= 1.0:
        raise ValueError("dropout's p must be from 0 to 1")
    if not 0 <= seed < 1 << 64:
        raise ValueError("dropout's seed must be of 64 bits, not negative")
    if isinstance(offset, torch.Tensor):
        if not offset.is_cuda or offset.device != device or offset.dtype != torch.int64:
            raise TypeError("dropout's offset must be an int, or int64 on the input's device")
        if offset.numel() != 1:
            raise ValueError("dropout's offset must be one number")
        return _Dropout(p, seed, 0, offset.data_ptr()), offset
    offset = int(offset)
    if not 0 <= offset < 1 << 64:
        raise ValueError("dropout's offset must be of 64 bits, not negative")
    return _Dropout(p, seed, offset, None), None


def _result(out, rows, cols, dtype, asked, device, stream):
    """(out, pointer, row stride, type): a new tensor of ``asked`` or ``dtype``, or
    the caller's, checked."""
    if out is None:
        out = _new((rows, cols), asked or dtype, device, stream)
        return out, out.data_ptr(), cols, _float_type(out.dtype, "out")
    if asked is not None and out.dtype != asked:
        raise TypeError("out has another dtype than the one asked for")
    op, on, old, oc = _rows(out, out.dtype, device, "out")
    if (on, oc) != (rows, cols):
        raise ValueError(f"out must be [{rows}][{cols}]")
    return out, op, old, _float_type(out.dtype, "out")


def quantize_mx4(x, transposed: bool = False, out=None, stream=None):
    """The rows of ``x`` (fp32 or bf16 matrix, any row stride) in microscaled 4-bit
    floating point (oscars_quantize_micro), or with ``transposed`` the rows of its
    transpose: ``(q, scale)``, uint8, two entries a byte and a scale for every 32.
    ``out``: such a pair to write into, row strides multiples of 16."""
    dev = x.device
    xp, n, ld, cols = _rows(x, x.dtype, dev, "x")
    dt = _float_type(x.dtype, "x")
    count, along = (cols, n) if transposed else (n, cols)
    if out is None:
        qs, ss = _micro_shapes(count, along)
        out = _new(qs, torch.uint8, dev, stream), _new(ss, torch.uint8, dev, stream)
    q, scale = out
    qp, qld, sp, sld = _micro_rows(q, scale, count, along, dev, "q")
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_quantize_micro(qp, qld, sp, sld, xp, ld, dt, n, cols,
                                            int(bool(transposed)), _stream_handle(stream, dev)),
               "oscars_quantize_micro")
    _used_on(stream, x, q, scale)
    return out


def dequantize_mx4(q, scale, columns: int, dtype=None, out=None, stream=None):
    """The values of quantised rows of ``columns`` entries (oscars_dequantize_micro), in
    fp32 by default."""
    n, dev = _count(q, "q"), q.device
    qp, qld, sp, sld = _micro_rows(q, scale, n, int(columns), dev, "q")
    out, op, old, odt = _result(out, n, int(columns), torch.float32, dtype, dev, stream)
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_dequantize_micro(op, old, odt, qp, qld, sp,
                                              sld, n, int(columns), _stream_handle(stream, dev)),
               "oscars_dequantize_micro")
    _used_on(stream, q, scale, out)
    return out


def matmul_mx4(xq, xscale, wq, wscale, in_features: int, bias=None, relu: bool = False,
               dropout=None, out_dtype=None, out=None, stream=None):
    """drop(relu(x w' + bias)) (oscars_matmul_micro) of quantised rows ``xq`` [rows][..]
    and weights ``wq`` [outputs][..] as quantize_mx4 gives them, of ``in_features``
    entries each; ``dropout``: ``(p, seed)`` or ``(p, seed, offset)`` as in ``dropout``;
    fp32 by default.  Returns ``out``, which autograd does not follow."""
    n, outs, cols, dev = _count(xq, "xq"), _count(wq, "wq"), int(in_features), xq.device
    xp, xld, xsp, xsld = _micro_rows(xq, xscale, n, cols, dev, "xq")
    wp, wld, wsp, wsld = _micro_rows(wq, wscale, outs, cols, dev, "wq")
    out, op, old, odt = _result(out, n, outs, torch.float32, out_dtype, dev, stream)
    drop, offset = _dropout_options(dropout, dev)
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_matmul_micro(
            op, old, odt, xp, xld, xsp, xsld, wp, wld, wsp, wsld,
            _vector(bias, outs, dev, "bias"), int(bool(relu)), drop, n, cols, outs,
            _stream_handle(stream, dev)), "oscars_matmul_micro")
    _used_on(stream, xq, xscale, wq, wscale, bias, offset, out)
    return out


def linear_mx4(x, wq, wscale, bias=None, relu: bool = False, dropout=None, out_dtype=None,
               out=None, stream=None):
    """A linear layer in microscaled 4-bit floating point (oscars_linear_micro): the rows of
    ``x`` (fp32 or bf16) are quantised on the way, ``wq`` and ``wscale`` are a weight
    matrix's quantize_mx4.  ``dropout`` (training): ``(p, seed)`` or ``(p, seed,
    offset)`` as in ``dropout``.  The result has ``x``'s type by default.  Returns
    ``out``.  Autograd does not follow the call, whatever requires a gradient: a
    program's training step calls linear_mx4_backward."""
    dev = x.device
    xp, n, xld, cols = _rows(x, x.dtype, dev, "x")
    dt = _float_type(x.dtype, "x")
    outs = _count(wq, "wq")
    wp, wld, wsp, wsld = _micro_rows(wq, wscale, outs, cols, dev, "wq")
    out, op, old, odt = _result(out, n, outs, x.dtype, out_dtype, dev, stream)
    drop, offset = _dropout_options(dropout, dev)
    if n == 0:
        return out
    lib = _lib()
    need = lib.oscars_linear_micro_workspace(n, cols)
    ws = _workspace(need, dev, stream) if need else None
    with _on_device(dev):
        _check(lib.oscars_linear_micro(
            op, old, odt, xp, xld, dt, wp, wld, wsp, wsld,
            _vector(bias, outs, dev, "bias"), int(bool(relu)), drop, n, cols, outs,
            ws.data_ptr() if need else None, need, _stream_handle(stream, dev)),
            "oscars_linear_micro")
    _used_on(stream, x, wq, wscale, bias, offset, out)
    return out


def linear_mx4_backward(dy, x, wtq=None, wtscale=None, y=None, dropout=None, want_dx: bool = True,
                        out=None, stream=None):
    """The gradients of linear_mx4's layer (oscars_linear_micro_backward), straight through the
    rounding to 4 bits: ``(dx, dw, db)`` from the output's gradient ``dy``, the
    layer's input ``x`` and ``quantize_mx4(w, transposed=True)``.  ``y``: the layer's
    output, for a layer with a ReLU.  ``dropout``: as in the forward call.  dx has
    ``x``'s type (None without ``want_dx``, which needs no weights), dw and db are
    fp32.  ``out``: such a triple to write into."""
    dev = dy.device
    dyp, n, dyld, outs = _rows(dy, dy.dtype, dev, "dy")
    xp, xn, xld, cols = _rows(x, x.dtype, dev, "x")
    if xn != n:
        raise ValueError("dy and x must have as many rows")
    ydt, xdt = _float_type(dy.dtype, "dy"), _float_type(x.dtype, "x")
    yp, yld = None, 0
    if y is not None:
        yp, yn, yld, yc = _rows(y, dy.dtype, dev, "y")
        if (yn, yc) != (n, outs):
            raise ValueError("y must have dy's shape")
    if out is None:
        dx = _new((n, cols), x.dtype, dev, stream) if want_dx else None
        dw, db = _new((outs, cols), torch.float32, dev, stream), \
            _new((outs,), torch.float32, dev, stream)
        out = dx, dw, db
        dxld = dwld = cols
    else:
        dx, dw, db = out
        if (dx is not None) != bool(want_dx):
            raise ValueError("out must hold a dx where it is wanted, and None where it is not")
        dxld = 0
        if want_dx:
            _, dn, dxld, dc = _rows(dx, x.dtype, dev, "dx")
            if (dn, dc) != (n, cols):
                raise ValueError("dx must have x's shape")
        _, wn, dwld, wc = _rows(dw, torch.float32, dev, "dw")
        if (wn, wc) != (outs, cols):
            raise ValueError("dw must be [outputs][inputs]")
    wtp, wtld, wtsp, wtsld = None, 0, None, 0
    if want_dx:
        if wtq is None or wtscale is None:
            raise ValueError("dx needs the weights' columns in 4 bits")
        wtp, wtld, wtsp, wtsld = _micro_rows(wtq, wtscale, cols, outs, dev, "wtq")
    drop, offset = _dropout_options(dropout, dev)
    dxp, dwp, dbp = dx.data_ptr() if want_dx else None, dw.data_ptr(), _vector(db, outs, dev, "db")
    if n == 0:  # what empty tensors point at
        dyp = xp = dwp
        yp = dxp = None
    g = _Gradients(n, cols, outs, dyp, yp, xp, dyld, yld, xld, ydt, xdt, wtp, wtsp, wtld, wtsld,
                   dxp, dwp, dbp, dxld, dwld, None if drop is None else ctypes.addressof(drop))
    lib = _lib()
    need = lib.oscars_linear_micro_backward_workspace(n, cols, outs, int(dxp is not None))
    ws = _workspace(need, dev, stream) if need else None
    with _on_device(dev):
        _check(lib.oscars_linear_micro_backward(
            ctypes.byref(g), ws.data_ptr() if need else None, need, _stream_handle(stream, dev)),
            "oscars_linear_micro_backward")
    _used_on(stream, dy, x, wtq, wtscale, y, offset, dx, dw, db)
    return out


def dropout(x, p: float, seed: int, offset=0, out=None, stream=None):
    """Dropout from a counter-based generator (oscars_dropout) of ``x`` (fp32 or bf16
    matrix, any row stride): entries are 0 with probability ``p`` (to 16 bits),
    multiplied by 1 / (1 - p) otherwise.  The mask is a function of ``seed``,
    ``offset`` (the call's number in a training run; an int64 tensor of one element
    on the device is read when the call runs) and the place, so the gradient is
    ``dropout(dy, p, seed, offset)``, which the program calls itself: autograd does not
    follow.  ``out``: ``x`` itself is allowed."""
    dev = x.device
    xp, n, ld, cols = _rows(x, x.dtype, dev, "x")
    dt = _float_type(x.dtype, "x")
    out, op, old, _ = _result(out, n, cols, x.dtype, x.dtype, dev, stream)
    options, more = _dropout_options((p, seed, offset), dev)
    if n == 0:
        return out
    with _on_device(dev):
        _check(_lib().oscars_dropout(op, old, xp, ld, dt, options, n, cols,
                                     _stream_handle(stream, dev)), "oscars_dropout")
    _used_on(stream, x, more, out)
    return out


class Context:
    """K replicas of a ReLU MLP (dims = (d, h_1, ..., C)) and their workspace;
    or, with ``cnn = (image, conv)``, of the convolutional model: image =
    (H, W, C), conv = ((out channels, stride[, shortcut]), ...), dims =
    (H W C, classes), fp32 (oscars_create_cnn; shortcut: the layer adds the
    output of the layer two before it)."""

    def __init__(self, dims: Sequence[int], dtype: int, K: int, max_batch: int, stream=None,
                 cnn=None):
        self.dims = [int(v) for v in dims]
        self.dtype = int(dtype)
        self.K = int(K)
        h = _vp()
        if cnn is None:
            self._dims_arr, dp = _arr(self.dims, np.int32)
            model = _Model(len(self.dims) - 1, dp, self.dtype)
            self.shapes = [(o, i) for i, o in zip(self.dims[:-1], self.dims[1:])]
            _check(_lib().oscars_create(ctypes.byref(h), ctypes.byref(model), self.K,
                                        int(max_batch), _stream_handle(stream)), "oscars_create")
        else:
            image = [int(v) for v in cnn[0]]
            conv = [(int(c[0]), int(c[1]), int(c[2]) if len(c) > 2 else 0) for c in cnn[1]]
            if self.dtype != FP32 or len(self.dims) != 2 or len(image) != 3:
                raise ValueError("convolutional models are fp32 with dims (H W C, classes)")
            self._ch, chp = _arr([c[0] for c in conv], np.int32)
            self._st, stp = _arr([c[1] for c in conv], np.int32)
            skp = None
            if any(c[2] for c in conv):
                self._sk, skp = _arr([c[2] for c in conv], np.int32)
            model = _CnnModel(image[0], image[1], image[2], len(conv), chp, stp, self.dims[-1], skp)
            self.shapes, cin = [], image[2]
            for o, *_ in conv:
                self.shapes.append((o, 3, 3, cin))
                cin = o
            self.shapes.append((self.dims[-1], cin))
            _check(_lib().oscars_create_cnn(ctypes.byref(h), ctypes.byref(model), self.K,
                                            int(max_batch), _stream_handle(stream)),
                   "oscars_create_cnn")
        self._h = h
        self._bind_stream(stream)
        self.n_pad = int(_lib().oscars_num_params(h))

    def close(self):
        if getattr(self, "_h", None):
            _lib().oscars_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_stream(self, stream=None):
        _check(_lib().oscars_set_stream(self._h, _stream_handle(stream)), "oscars_set_stream")
        self._bind_stream(stream)

    def _bind_stream(self, stream):
        import torch
        self._stream = stream if stream is not None else torch.cuda.current_stream()

    def layer_offsets(self, l: int) -> Tuple[int, int]:
        w, b = _i64(0), _i64(0)
        _check(_lib().oscars_layer_offsets(self._h, int(l), ctypes.byref(w), ctypes.byref(b)),
               "oscars_layer_offsets")
        return int(w.value), int(b.value)

    def pack(self, layers) -> np.ndarray:
        """Flat padded float32 vector from [(W, b), ...] in this model's layout."""
        flat = np.zeros(self.n_pad, np.float32)
        for l, (W, b) in enumerate(layers, start=1):
            wo, bo = self.layer_offsets(l)
            flat[wo:wo + W.size] = np.asarray(W, np.float32).ravel()
            flat[bo:bo + b.size] = np.asarray(b, np.float32)
        return flat

    def unpack(self, flat: np.ndarray):
        out = []
        for l, shape in enumerate(self.shapes, start=1):
            wo, bo = self.layer_offsets(l)
            size = int(np.prod(shape))
            out.append((flat[wo:wo + size].reshape(shape), flat[bo:bo + shape[0]]))
        return out

    def _step_args(self, replicas, x, y, offsets, seed, tau):
        import torch
        rp = _dev_ptr(replicas, torch.float32, "replicas")
        if replicas.numel() < self.K * self.n_pad:
            raise ValueError("replicas must hold K * n_pad floats")
        xdt = torch.bfloat16 if self.dtype == BF16 else torch.float32
        if x.dtype == torch.int16 or x.dtype == torch.uint16:
            xdt = x.dtype  # bf16 bit patterns
        xp = _dev_ptr(x, xdt, "x")
        yp = _dev_ptr(y, torch.int32, "y")
        if x.dim() != 2 or x.shape[1] != self.dims[0] or y.numel() != x.shape[0]:
            raise ValueError("x must be [n_rows][d] and y [n_rows]")
        sh, keep = _shards(xp, yp, x.shape[0], offsets, seed)
        t, tp = _arr(tau, np.int32)
        if len(t) != self.K or len(offsets) != self.K + 1:
            raise ValueError("tau needs K entries and offsets K + 1")
        return rp, sh, (keep, t), tp

    def local_steps(self, replicas, x, y, offsets: Sequence[int], seed: int, tau: Sequence[int],
                    lr: float, batch: int):
        rp, sh, keep, tp = self._step_args(replicas, x, y, offsets, seed, tau)
        _check(_lib().oscars_local_steps(self._h, rp, ctypes.byref(sh), tp, float(lr), int(batch)),
               "oscars_local_steps")

    def round(self, global_, replicas, x, y, offsets: Sequence[int], seed: int,
              tau: Sequence[int], lr: float, batch: int, weights: Sequence[float]):
        """One round of Eq. 4 from the global model (oscars_round)."""
        import torch
        gp = _dev_ptr(global_, torch.float32, "global")
        if global_.numel() < self.n_pad:
            raise ValueError("global must hold n_pad floats")
        rp, sh, keep, tp = self._step_args(replicas, x, y, offsets, seed, tau)
        w, wp = _arr(weights, np.float32)
        if len(w) != self.K:
            raise ValueError("one weight per worker")
        _check(_lib().oscars_round(self._h, gp, rp, ctypes.byref(sh), tp, float(lr), int(batch),
                                   wp), "oscars_round")

    def round_losses(self) -> np.ndarray:
        out = np.zeros(self.K, np.float32)
        _check(_lib().oscars_round_losses(self._h, out.ctypes.data_as(_P(_f32))),
               "oscars_round_losses")
        return out

    def evaluate(self, params, x, y, n_rows: Optional[int] = None, noalloc: bool = False):
        """Held-out (summed loss, correct count) of the flat model ``params``
        (device tensor [n_pad] fp32) on rows 0..n_rows-1 of x / y
        (oscars_evaluate, or with ``noalloc`` oscars_evaluate_noalloc)."""
        import torch
        n = int(x.shape[0] if n_rows is None else n_rows)
        if n > x.shape[0] or n > y.shape[0]:
            raise ValueError("n_rows exceeds the rows of x or y")
        loss = ctypes.c_double(0.0)
        hits = _i64(0)
        name = "oscars_evaluate_noalloc" if noalloc else "oscars_evaluate"
        _check(getattr(_lib(), name)(self._h, _dev_ptr(params, torch.float32, "params"),
                                     _dev_ptr(x, None, "x"), _dev_ptr(y, torch.int32, "y"), n,
                                     ctypes.byref(loss), ctypes.byref(hits)), name)
        return float(loss.value), int(hits.value)

    def _quantize_model(self, name, need, params, out):
        pp = _dev_ptr(params, torch.float32, "params")
        if params.numel() < self.n_pad:
            raise ValueError("params must hold n_pad floats")
        if out is None:
            out = _workspace(max(need, 1), params.device, self._stream)
        op = _dev_ptr(out, torch.uint8, "out")
        if out.numel() < need:
            raise ValueError(f"a quantised model takes {need} bytes")
        _check(getattr(_lib(), name)(self._h, pp, op), name)
        _used_on(self._stream, params, out)
        return out

    def _evaluate_quantized(self, name, need, model, x, y, n_rows):
        n = int(x.shape[0] if n_rows is None else n_rows)
        if n > x.shape[0] or n > y.shape[0]:
            raise ValueError("n_rows exceeds the rows of x or y")
        mp = _dev_ptr(model, torch.uint8, "model")
        if model.numel() < need:
            raise ValueError("model is not a quantised model of this context")
        xdt = x.dtype if self.dtype == BF16 and x.dtype in (torch.int16, torch.uint16) else (
            torch.bfloat16 if self.dtype == BF16 else torch.float32)
        if x.dim() != 2 or x.shape[1] != self.dims[0]:
            raise ValueError("x must be [n_rows][d]")
        loss = ctypes.c_double(0.0)
        hits = _i64(0)
        _check(getattr(_lib(), name)(self._h, mp, _dev_ptr(x, xdt, "x"),
                                     _dev_ptr(y, torch.int32, "y"), n, ctypes.byref(loss),
                                     ctypes.byref(hits)), name)
        return float(loss.value), int(hits.value)

    def quantize_model(self, params, out=None):
        """The flat model ``params`` (device tensor [n_pad] fp32) in 8-bit integers,
        a scale per output channel (oscars_quantize_model): one device tensor
        for evaluate_i8.  Fully connected models only."""
        return self._quantize_model("oscars_quantize_model",
                                    int(_lib().oscars_quantized_model_bytes(self._h)), params, out)

    def evaluate_i8(self, model, x, y, n_rows: Optional[int] = None):
        """``evaluate`` with the products of the quantised ``model``
        (oscars_evaluate_quantized)."""
        return self._evaluate_quantized("oscars_evaluate_quantized",
                                        int(_lib().oscars_quantized_model_bytes(self._h)), model,
                                        x, y, n_rows)

    def quantize_model_mx4(self, params, out=None):
        """``quantize_model`` in microscaled 4-bit floating point
        (oscars_quantize_model_micro), for evaluate_mx4."""
        return self._quantize_model("oscars_quantize_model_micro",
                                    int(_lib().oscars_micro_model_bytes(self._h)), params, out)

    def evaluate_mx4(self, model, x, y, n_rows: Optional[int] = None):
        """``evaluate`` with the products of the 4-bit ``model`` (oscars_evaluate_micro)."""
        return self._evaluate_quantized("oscars_evaluate_micro",
                                        int(_lib().oscars_micro_model_bytes(self._h)), model, x,
                                        y, n_rows)

    def server_step(self, global_, replicas, weights: Sequence[float], momentum, lr: float,
                    beta: float = 0.9, nesterov: bool = True, weight_decay: float = 0.0,
                    plain_lr: float = 1.0, plain_layers: Sequence[int] = (),
                    coeffs=NEWTON_SCHULZ, out=None):
        """The server's step with a momentum and orthogonalised updates
        (oscars_server_step) in the place of ``aggregate``: from the global model
        before the round and the workers' models at its barrier.  ``out``:
        (new global model, new momentum), by default in place.  Layers
        ``plain_layers`` (1..L) and all biases take the momentum as it is,
        times ``plain_lr``.  Returns ``out``."""
        import torch
        g_out, m_out = (global_, momentum) if out is None else out
        n = self.n_pad
        ptrs = []
        for t, size, what in ((global_, n, "global"), (replicas, self.K * n, "replicas"),
                              (momentum, n, "momentum"), (g_out, n, "global out"),
                              (m_out, n, "momentum out")):
            ptrs.append(_dev_ptr(t, torch.float32, what))
            if t.numel() < size:
                raise ValueError(f"{what} is smaller than the model needs")
        w, wp = _arr(weights, np.float32)
        if len(w) != self.K:
            raise ValueError("one weight per worker")
        mask = 0
        for l in plain_layers:
            if not 1 <= int(l) <= len(self.shapes):
                raise ValueError("plain_layers are layers 1 .. L")
            mask |= 1 << (int(l) - 1)
        ca, steps = _coeffs(tuple(map(tuple, coeffs)))
        o = _ServerOptions(lr, beta, weight_decay, plain_lr, int(bool(nesterov)), mask, ca, steps)
        need = _lib().oscars_server_workspace(self._h)
        ws = _workspace(need, global_.device, self._stream)
        _check(_lib().oscars_server_step(self._h, ptrs[0], ptrs[1], wp, ptrs[2], ptrs[3], ptrs[4],
                                         ctypes.byref(o), ws.data_ptr(), need),
               "oscars_server_step")
        _used_on(self._stream, global_, replicas, momentum, g_out, m_out)
        return g_out, m_out

    def cursors(self) -> List[int]:
        out = np.zeros(self.K, np.int64)
        _check(_lib().oscars_get_cursors(self._h, out.ctypes.data_as(_P(_i64))),
               "oscars_get_cursors")
        return out.tolist()

    def set_cursors(self, steps_done: Sequence[int]):
        a, ap = _arr(steps_done, np.int64)
        _check(_lib().oscars_set_cursors(self._h, ap), "oscars_set_cursors")

    def set_gemm_tiling(self, tiling: int):
        """Tiling of this context's forward / backward-data GEMMs (AUTO: tuned
        online per configuration, fastest kept); restarts the tuning."""
        _check(_lib().oscars_set_gemm_tiling(self._h, int(tiling)), "oscars_set_gemm_tiling")

    def tuning_pending(self) -> int:
        """This context's GEMM configurations whose AUTO tiling is still being
        tuned."""
        n = ctypes.c_int32(0)
        _check(_lib().oscars_tuning_pending(self._h, ctypes.byref(n)), "oscars_tuning_pending")
        return int(n.value)

    def set_backward(self, mode: int):
        """Backward of this context's hidden bf16 layers: AUTO (timed per
        configuration), SEPARATE, FUSED, FUSED_SPLIT."""
        _check(_lib().oscars_set_backward(self._h, int(mode)), "oscars_set_backward")

    def backward_path(self, layer: int, batch: int, replicas: int) -> int:
        """Backward of `layer` (1..L) with `replicas` active replicas: 1 fused,
        0 separate launches, -1 not timed yet (AUTO)."""
        out = _i32(0)
        _check(_lib().oscars_backward_path(self._h, int(layer), int(batch), int(replicas),
                                           ctypes.byref(out)), "oscars_backward_path")
        return int(out.value)

    def profile_begin(self, kinds: Sequence[int]):
        mask = 0
        for k in kinds:
            mask |= 1 << int(k)
        _check(_lib().oscars_profile_begin(self._h, mask), "oscars_profile_begin")

    def profile_end(self):
        k = len(KERNEL_NAMES)
        ms = (ctypes.c_double * k)()
        n = (_i64 * k)()
        _check(_lib().oscars_profile_end(self._h, ms, n), "oscars_profile_end")
        return {KERNEL_NAMES[i]: (ms[i], n[i]) for i in range(k)}
