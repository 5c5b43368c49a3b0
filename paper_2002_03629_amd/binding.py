"""ctypes binding of libjacobi_made.so: argument marshalling only.

Function names and argument order follow include/jacobi_made.h.  Device buffers are torch
tensors (torch is used for device memory and streams, nothing else); host arrays are numpy.
There is no fallback: if the shared library is missing, `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libjacobi_made.so")

MADE_OK, MADE_ERR_ARG, MADE_ERR_NOMEM, MADE_ERR_HIP, MADE_ERR_NOT_CONVERGED = 0, -1, -2, -3, -4
MADE_F32, MADE_BF16 = 0, 1

EXPORTS = ["made_init", "made_conv_init", "made_free", "made_forward_logits", "made_forward_logits_noalloc", "made_layer_activations", "sequential_sample", "jacobi_sample",
           "gs_jacobi_sample", "jacobi_gs_sample", "made_forward_params", "sequential_sample_real",
           "jacobi_sample_real", "gs_jacobi_sample_real", "made_last_stats", "made_set_profiling", "made_last_profile", "made_set_option",
           "made_layer_nnz",
           "rnn_forward", "rnn_backward_sequential", "rnn_backward_jacobi", "rnn_jacobi_max_steps", "rnn_param_grads",
           "linattn_workspace_bytes", "linattn_forward", "linattn_backward", "linattn_step",
           "adamw_step", "adamw_unpack",
           "made_last_error"]


class MadeError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"libjacobi_made status {code}: {message}")
        self.code = code


class made_config(C.Structure):
    _fields_ = [("D", C.c_int32), ("C", C.c_int32), ("n_hidden", C.c_int32),
                ("hidden", C.POINTER(C.c_int32)), ("dtype", C.c_int32), ("real", C.c_int32), ("onehot", C.c_int32)]


class made_conv_config(C.Structure):
    _fields_ = [("H", C.c_int32), ("W", C.c_int32), ("C", C.c_int32), ("F", C.c_int32), ("k", C.c_int32),
                ("n_conv", C.c_int32), ("dtype", C.c_int32)]


class linattn_config(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("Dk", C.c_int32),
                ("Dv", C.c_int32), ("dtype", C.c_int32), ("scale", C.c_float), ("ld_q", C.c_int64), ("ld_k", C.c_int64),
                ("ld_v", C.c_int64), ("ld_o", C.c_int64), ("offsets", C.c_void_p)]


class adamw_config(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("weight_decay", C.c_double), ("grad_scale", C.c_double), ("step", C.c_int32), ("param_dtype", C.c_int32),
                ("grad_dtype", C.c_int32), ("moment_bits", C.c_int32)]


ADAMW_BLOCK = 256

_lib = None


def lib() -> C.CDLL:
    """Load the HIP library (once).  Fails loudly when it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2002_03629_amd.build` "
                               "(there is no CPU fallback)")
        # Device pointers and streams come from torch, so the library must run on the very HIP runtime
        # torch has loaded: import torch first, then the loader resolves libamdhip64.so.7 to that copy.
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        vp, i32, i64p = C.c_void_p, C.c_int32, C.POINTER(C.c_int64)
        L.made_init.argtypes = [C.POINTER(made_config), C.POINTER(C.POINTER(C.c_int32)),
                                C.POINTER(C.POINTER(C.c_float)), C.POINTER(C.POINTER(C.c_float)), C.POINTER(vp)]
        L.made_conv_init.argtypes = [C.POINTER(made_conv_config), C.POINTER(C.POINTER(C.c_float)),
                                     C.POINTER(C.POINTER(C.c_float)), C.POINTER(vp)]
        L.made_free.argtypes = [vp]
        L.made_forward_logits.argtypes = [vp, vp, i32, vp, vp]
        L.made_forward_logits_noalloc.argtypes = [vp, vp, i32, vp, vp]
        L.made_layer_activations.argtypes = [vp, vp, i32, i32, vp, vp]
        L.sequential_sample.argtypes = [vp, vp, i32, i32, vp, vp]
        L.jacobi_sample.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp]
        L.gs_jacobi_sample.argtypes = [vp, vp, i32, vp, i32, vp, vp, vp]
        L.jacobi_gs_sample.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, vp]
        L.made_forward_params.argtypes = [vp, vp, i32, vp, vp]
        L.sequential_sample_real.argtypes = [vp, vp, i32, i32, vp, vp]
        L.jacobi_sample_real.argtypes = [vp, vp, i32, vp, C.c_float, i32, vp, vp, vp]
        L.gs_jacobi_sample_real.argtypes = [vp, vp, i32, vp, i32, C.c_float, vp, vp, vp]
        L.made_last_stats.argtypes = [vp, i64p, i32]
        L.made_set_profiling.argtypes = [vp, i32]
        L.made_last_profile.argtypes = [vp, C.POINTER(C.c_double), i64p, i32]
        L.made_layer_nnz.argtypes = [vp, i64p, i32]
        L.made_set_option.argtypes = [vp, i32, i32]
        L.rnn_forward.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]
        L.rnn_backward_sequential.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp]
        L.rnn_backward_jacobi.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, C.c_float, vp, vp, vp, vp]
        L.rnn_jacobi_max_steps.argtypes = [i32]
        L.rnn_param_grads.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]
        cfg = C.POINTER(linattn_config)
        L.linattn_workspace_bytes.argtypes = [cfg, i32, i64p]
        L.linattn_forward.argtypes = [cfg] + [vp] * 8 + [C.c_int64, vp]
        L.linattn_backward.argtypes = [cfg] + [vp] * 12 + [C.c_int64, vp]
        L.linattn_step.argtypes = [cfg] + [vp] * 5 + [i32, vp, vp, vp]
        vpp = C.POINTER(vp)
        L.adamw_step.argtypes = [C.POINTER(adamw_config), i32, i64p] + [vpp] * 7 + [vp, vp]
        L.adamw_unpack.argtypes = [i32, i64p] + [vpp] * 6 + [vp]
        L.made_last_error.argtypes = []
        L.made_last_error.restype = C.c_char_p
        for name in EXPORTS[:-1]:
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def made_last_error() -> str:
    return lib().made_last_error().decode()


def _check(code: int) -> None:
    if code != MADE_OK:
        raise MadeError(code, made_last_error())


def _ptr(t, dtype=None) -> Optional[int]:
    """Device pointer of a contiguous torch tensor (or None)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("device tensors must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected {dtype}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


def made_init(D: int, Cn: int, hidden: Sequence[int], dtype: int, degrees: Sequence[np.ndarray],
              W: Sequence[np.ndarray], b: Optional[Sequence[Optional[np.ndarray]]] = None, real: bool = False,
              onehot: bool = False) -> int:
    """Returns the opaque model handle (an integer address)."""
    L = len(hidden)
    hid = np.ascontiguousarray(hidden, dtype=np.int32)
    cfg = made_config(int(D), int(Cn), L, hid.ctypes.data_as(C.POINTER(C.c_int32)), int(dtype), 1 if real else 0,
                      1 if onehot else 0)
    keep = []
    deg_arr = (C.POINTER(C.c_int32) * L)()
    for l in range(L):
        a = np.ascontiguousarray(degrees[l], dtype=np.int32)
        if a.shape != (hidden[l],):
            raise ValueError("degrees[%d] has shape %s" % (l, a.shape))
        keep.append(a)
        deg_arr[l] = a.ctypes.data_as(C.POINTER(C.c_int32))
    dims = [D * Cn if onehot else D] + list(hidden) + [D * Cn]
    W_arr = (C.POINTER(C.c_float) * (L + 1))()
    b_arr = (C.POINTER(C.c_float) * (L + 1))()
    for l in range(L + 1):
        a = np.ascontiguousarray(W[l], dtype=np.float32)
        if a.shape != (dims[l + 1], dims[l]):
            raise ValueError("W[%d] has shape %s, expected %s" % (l, a.shape, (dims[l + 1], dims[l])))
        keep.append(a)
        W_arr[l] = a.ctypes.data_as(C.POINTER(C.c_float))
        bl = None if b is None else b[l]
        if bl is not None:
            bb = np.ascontiguousarray(bl, dtype=np.float32)
            if bb.shape != (dims[l + 1],):
                raise ValueError("b[%d] has shape %s" % (l, bb.shape))
            keep.append(bb)
            b_arr[l] = bb.ctypes.data_as(C.POINTER(C.c_float))
    out = C.c_void_p()
    _check(lib().made_init(C.byref(cfg), deg_arr, W_arr, b_arr, C.byref(out)))
    return out.value


def made_conv_init(H: int, W: int, Cn: int, F: int, k: int, n_conv: int, dtype: int, Wts: Sequence[np.ndarray],
                   b: Optional[Sequence[Optional[np.ndarray]]] = None) -> int:
    """Returns the opaque handle of a masked convolutional model (see include/jacobi_made.h)."""
    cfg = made_conv_config(int(H), int(W), int(Cn), int(F), int(k), int(n_conv), int(dtype))
    shapes = [(F, k, k, 3)] + [(F, k, k, F)] * (n_conv - 1) + [(3 * Cn, 1, 1, F)]
    keep = []
    W_arr = (C.POINTER(C.c_float) * (n_conv + 1))()
    b_arr = (C.POINTER(C.c_float) * (n_conv + 1))()
    for l, shp in enumerate(shapes):
        a = np.ascontiguousarray(Wts[l], dtype=np.float32)
        if a.shape != shp and a.shape != (shp[0], shp[3]):
            raise ValueError("W[%d] has shape %s, expected %s" % (l, a.shape, shp))
        keep.append(a)
        W_arr[l] = a.ctypes.data_as(C.POINTER(C.c_float))
        bl = None if b is None else b[l]
        if bl is not None:
            bb = np.ascontiguousarray(bl, dtype=np.float32)
            if bb.shape != (shp[0],):
                raise ValueError("b[%d] has shape %s" % (l, bb.shape))
            keep.append(bb)
            b_arr[l] = bb.ctypes.data_as(C.POINTER(C.c_float))
    out = C.c_void_p()
    _check(lib().made_conv_init(C.byref(cfg), W_arr, b_arr, C.byref(out)))
    return out.value


def conv_model_from_network(net) -> int:
    """made_conv_init from a synth.ConvNetwork description."""
    n_conv = len(net.W_) - 1
    return made_conv_init(net.H, net.W, net.C, net.F, net.k, n_conv, MADE_BF16 if net.dtype == "bf16" else MADE_F32,
                          net.W_, net.b)


def made_free(model: Optional[int]) -> None:
    _check(lib().made_free(model))


def made_forward_logits(model: int, x, N: int, logits, stream=None) -> None:
    import torch
    _check(lib().made_forward_logits(model, _ptr(x, torch.uint8), N, _ptr(logits, torch.float32), _stream(stream)))


def made_forward_logits_noalloc(model: int, x, N: int, logits, stream=None) -> None:
    import torch
    _check(lib().made_forward_logits_noalloc(model, _ptr(x, torch.uint8), N, _ptr(logits, torch.float32),
                                             _stream(stream)))


def made_layer_activations(model: int, x, N: int, layer: int, out, stream=None) -> None:
    import torch
    _check(lib().made_layer_activations(model, _ptr(x, torch.uint8), N, layer, _ptr(out, torch.float32),
                                        _stream(stream)))


def sequential_sample(model: int, noise, N: int, mode: int, x_out, stream=None) -> None:
    import torch
    _check(lib().sequential_sample(model, _ptr(noise, torch.float32), N, mode, _ptr(x_out, torch.uint8),
                                   _stream(stream)))


def jacobi_sample(model: int, noise, N: int, x_init, max_iters: int, x_out, iters_out=None, stream=None) -> None:
    import torch
    _check(lib().jacobi_sample(model, _ptr(noise, torch.float32), N, _ptr(x_init, torch.uint8), max_iters,
                               _ptr(x_out, torch.uint8), _ptr(iters_out, torch.int32), _stream(stream)))


class PreparedJacobi:
    """jacobi_sample with its arguments marshalled once, for loops that call it again and again on the same buffers
    (a call of cfg2's size takes ~90 us, of which checking and converting eight arguments costs ~2.5): calling the
    object runs the call.  The tensors are kept alive; their contents may change between calls."""

    def __init__(self, model: int, noise, N: int, x_init, max_iters: int, x_out, iters_out=None, stream=None):
        import torch
        self._keep = (noise, x_init, x_out, iters_out, stream)
        self._fn = lib().jacobi_sample
        self._args = (C.c_void_p(model), C.c_void_p(_ptr(noise, torch.float32)), C.c_int32(N),
                      C.c_void_p(_ptr(x_init, torch.uint8)), C.c_int32(max_iters), C.c_void_p(_ptr(x_out, torch.uint8)),
                      C.c_void_p(_ptr(iters_out, torch.int32)), C.c_void_p(_stream(stream)))

    def __call__(self) -> None:
        code = self._fn(*self._args)
        if code != MADE_OK:
            raise MadeError(code, made_last_error())


def gs_jacobi_sample(model: int, noise, N: int, x_init, block: int, x_out, iters_out=None, stream=None) -> None:
    import torch
    _check(lib().gs_jacobi_sample(model, _ptr(noise, torch.float32), N, _ptr(x_init, torch.uint8), block,
                                  _ptr(x_out, torch.uint8), _ptr(iters_out, torch.int32), _stream(stream)))


def jacobi_gs_sample(model: int, noise, N: int, x_init, block: int, max_iters: int, x_out, iters_out=None,
                     stream=None) -> None:
    import torch
    _check(lib().jacobi_gs_sample(model, _ptr(noise, torch.float32), N, _ptr(x_init, torch.uint8), block, max_iters,
                                  _ptr(x_out, torch.uint8), _ptr(iters_out, torch.int32), _stream(stream)))


def made_forward_params(model: int, x, N: int, params, stream=None) -> None:
    import torch
    _check(lib().made_forward_params(model, _ptr(x, torch.float32), N, _ptr(params, torch.float32), _stream(stream)))


def sequential_sample_real(model: int, noise, N: int, mode: int, x_out, stream=None) -> None:
    import torch
    _check(lib().sequential_sample_real(model, _ptr(noise, torch.float32), N, mode, _ptr(x_out, torch.float32),
                                        _stream(stream)))


def jacobi_sample_real(model: int, noise, N: int, x_init, eps: float, max_iters: int, x_out, iters_out=None,
                       stream=None) -> None:
    import torch
    _check(lib().jacobi_sample_real(model, _ptr(noise, torch.float32), N, _ptr(x_init, torch.float32), float(eps),
                                    max_iters, _ptr(x_out, torch.float32), _ptr(iters_out, torch.int32),
                                    _stream(stream)))


def gs_jacobi_sample_real(model: int, noise, N: int, x_init, block: int, eps: float, x_out, iters_out=None,
                          stream=None) -> None:
    import torch
    _check(lib().gs_jacobi_sample_real(model, _ptr(noise, torch.float32), N, _ptr(x_init, torch.float32), block,
                                       float(eps), _ptr(x_out, torch.float32), _ptr(iters_out, torch.int32),
                                       _stream(stream)))


def made_last_stats(model: int) -> dict:
    buf = (C.c_int64 * 8)()
    _check(lib().made_last_stats(model, buf, 8))
    return {"passes": buf[0], "sample_passes": buf[1], "kernels": buf[2], "host_waits": buf[3],
            "conv_rows": buf[4], "tail_less_passes": buf[5], "output_weights_evaluated": buf[6],
            "output_draws_evaluated": buf[7]}


def made_set_profiling(model: int, enable: bool) -> None:
    _check(lib().made_set_profiling(model, 1 if enable else 0))


MADE_OPT_PERSISTENT = 1
MADE_OPT_FUSED_CATEGORICAL = 2
MADE_OPT_CHAINS = 3
MADE_OPT_BIG_TILE_BATCH = 4
MADE_OPT_CONV_ROWS = 5
MADE_OPT_PREFIX_CACHE = 6
MADE_OPT_RESIDENT = 7
MADE_OPT_RETIRE_SPLIT = 8
MADE_OPT_MID_TILE_BATCH = 9
MADE_OPT_PARTIAL_SUM_BATCH = 10
MADE_OPT_XCD_RESIDENT = 11
MADE_OPT_LAZY_STOP_TEST = 12
MADE_OPT_CALL_GRAPH = 14
MADE_OPT_ZERO_START = 15
MADE_OPT_WAIT_LIMIT = 16
MADE_OPT_FROZEN_POSITIONS = 13


def made_set_option(model: int, option: int, value: int) -> None:
    _check(lib().made_set_option(model, option, value))


def made_last_profile(model: int, n_slots: int):
    """(ms[n_slots], launches[n_slots]) of the most recent *_sample call; n_slots = L + 2."""
    ms = (C.c_double * n_slots)()
    cnt = (C.c_int64 * n_slots)()
    _check(lib().made_last_profile(model, ms, cnt, n_slots))
    return list(ms), list(cnt)


def made_layer_nnz(model: int, n_layers: int) -> List[int]:
    buf = (C.c_int64 * n_layers)()
    _check(lib().made_layer_nnz(model, buf, n_layers))
    return list(buf)


def model_from_network(net) -> int:
    """made_init from a synth.Network description."""
    return made_init(net.D, net.C, net.hidden, MADE_BF16 if net.dtype == "bf16" else MADE_F32, net.degrees, net.W,
                     net.b, getattr(net, "real", False), getattr(net, "onehot", False))


# ------------------------------------------------------------------------------------------------
# recurrent network: backward pass by Jacobi iteration (include/jacobi_rnn.h); all tensors are float32 on the device
# ------------------------------------------------------------------------------------------------
def rnn_forward(W, U, b, x, h0, B: int, T: int, H: int, I: int, z, h, stream=None) -> None:
    import torch
    f = torch.float32
    _check(lib().rnn_forward(_ptr(W, f), _ptr(U, f), _ptr(b, f), _ptr(x, f), _ptr(h0, f), B, T, H, I, _ptr(z, f), _ptr(h, f),
                             _stream(stream)))


def rnn_backward_sequential(W, z, g, B: int, T: int, H: int, d, stream=None) -> None:
    import torch
    f = torch.float32
    _check(lib().rnn_backward_sequential(_ptr(W, f), _ptr(z, f), _ptr(g, f), B, T, H, _ptr(d, f), _stream(stream)))


def rnn_backward_jacobi(W, z, g, d_init, B: int, T: int, H: int, n_iters: int, eps: float, d, iters_out=None,
                        converged_out=None, stream=None) -> None:
    import torch
    f = torch.float32
    _check(lib().rnn_backward_jacobi(_ptr(W, f), _ptr(z, f), _ptr(g, f), _ptr(d_init, f), B, T, H, int(n_iters), float(eps),
                                     _ptr(d, f), _ptr(iters_out, torch.int32), _ptr(converged_out, torch.int32),
                                     _stream(stream)))


def rnn_jacobi_max_steps(H: int) -> int:
    return int(lib().rnn_jacobi_max_steps(int(H)))


def rnn_param_grads(z, h, x, d, h0, B: int, T: int, H: int, I: int, dW, dU, db, stream=None) -> None:
    import torch
    f = torch.float32
    _check(lib().rnn_param_grads(_ptr(z, f), _ptr(h, f), _ptr(x, f), _ptr(d, f), _ptr(h0, f), B, T, H, I, _ptr(dW, f),
                                 _ptr(dU, f), _ptr(db, f), _stream(stream)))


# ------------------------------------------------------------------------------------------------
# linear attention with a decay for each head (include/jacobi_linattn.h).  q, k, v, o and their gradients are float32 or
# bfloat16 (all the same), [B, T, heads, D] or, packed (offsets given), [T, heads, D]; the heads of a step are contiguous,
# the steps may lie further apart (parts of a wider tensor).  States and log_decay are float32.
# ------------------------------------------------------------------------------------------------
def _on_device(t, what: str, stream=None):
    """A tensor that a kernel on the current device may be handed, on `stream` if one is given."""
    import torch
    if not t.is_cuda:
        raise ValueError(f"{what} is not on the GPU")
    device = torch.cuda.current_device()
    if stream is not None and stream.device.index != device:
        raise ValueError(f"the stream is of cuda:{stream.device.index}, the current device is cuda:{device}")
    if t.device.index != device:
        raise ValueError(f"{what} is on cuda:{t.device.index}, the call is for cuda:{device}")
    return t


def _dense(t, what: str, shape, dtype, stream=None) -> Optional[int]:
    """Device pointer of a contiguous tensor of that shape and type (or None)."""
    if t is None:
        return None
    _on_device(t, what, stream)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return _ptr(t, dtype)


def _rows(t, what: str, lead, heads: int, D: int, dtype, stream=None):
    """(device pointer, elements from row to row) of [*lead, heads, D] whose rows are contiguous and equally far apart."""
    _on_device(t, what, stream)
    if tuple(t.shape) != tuple(lead) + (heads, D):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(lead) + (heads, D)}")
    if t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.numel() == 0:
        return None, 0
    st = t.stride()
    if (D > 1 and st[-1] != 1) or (heads > 1 and st[-2] != D):
        raise ValueError(f"{what}: the heads of a row must be contiguous")
    wide = heads * D
    if len(lead) == 1:
        ld = st[0] if lead[0] > 1 else wide
    elif lead[1] > 1:
        ld = st[1]
        if lead[0] > 1 and st[0] != ld * lead[1]:
            raise ValueError(f"{what}: the rows must be equally far apart")
    else:
        ld = st[0] if lead[0] > 1 else wide
    if ld < wide:
        raise ValueError(f"{what}: rows overlap")
    return t.data_ptr(), ld


def _linattn_dtype(dtype) -> int:
    import torch
    if dtype == torch.float32:
        return MADE_F32
    if dtype == torch.bfloat16:
        return MADE_BF16
    raise ValueError(f"expected torch.float32 or torch.bfloat16, got {dtype}")


def linattn_workspace_bytes(B: int, T: int, heads: int, kv_heads: int, Dk: int, Dv: int, dtype, packed: bool = False,
                            backward: bool = False) -> int:
    """dtype: torch.float32 or torch.bfloat16."""
    cfg = linattn_config(int(B), int(T), int(heads), int(kv_heads), int(Dk), int(Dv), _linattn_dtype(dtype), 1.0, 0, 0, 0, 0, 1 if packed else None)
    out = C.c_int64()
    _check(lib().linattn_workspace_bytes(C.byref(cfg), 1 if backward else 0, C.byref(out)))
    return out.value


def _linattn_args(q, k, v, log_decay, offsets, B, T, heads, kv_heads, Dk, Dv, scale, o, stream):
    import torch
    lead = (B, T) if offsets is None else (T,)
    dt = q.dtype
    code = _linattn_dtype(q.dtype)
    pq, lq = _rows(q, "q", lead, heads, Dk, dt, stream)
    pk, lk = _rows(k, "k", lead, kv_heads, Dk, dt, stream)
    pv, lv = _rows(v, "v", lead, kv_heads, Dv, dt, stream)
    po, lo = _rows(o, "o", lead, heads, Dv, dt, stream)
    cfg = linattn_config(int(B), int(T), int(heads), int(kv_heads), int(Dk), int(Dv), code, float(scale), lq, lk, lv, lo,
                         _dense(offsets, "offsets", (B + 1,), torch.int32, stream))
    return cfg, pq, pk, pv, po, _dense(log_decay, "log_decay", (kv_heads,), torch.float32, stream)


def _linattn_workspace(cfg, backward: bool, workspace, stream):
    """The workspace given, or one of torch's allocator's on the stream of the call."""
    import torch
    if workspace is None:
        need = C.c_int64()
        _check(lib().linattn_workspace_bytes(C.byref(cfg), 1 if backward else 0, C.byref(need)))
        if need.value == 0:
            return None, 0, None
        with torch.cuda.stream(stream):          # (None: the current one)
            workspace = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    else:
        _on_device(workspace, "workspace", stream)
    return _ptr(workspace, torch.uint8), workspace.numel(), workspace


def linattn_forward(q, k, v, log_decay, state_in, offsets, B: int, T: int, heads: int, kv_heads: int, Dk: int, Dv: int,
                    scale: float, o, state_out=None, workspace=None, stream=None) -> None:
    """workspace: uint8, of linattn_workspace_bytes(...) bytes, used by one call at a time; None: taken for the call."""
    import torch
    f = torch.float32
    cfg, pq, pk, pv, po, pd = _linattn_args(q, k, v, log_decay, offsets, B, T, heads, kv_heads, Dk, Dv, scale, o, stream)
    shape = (B, kv_heads, Dk, Dv)
    ws, ws_bytes, keep = _linattn_workspace(cfg, False, workspace, stream)
    _check(lib().linattn_forward(C.byref(cfg), pq, pk, pv, pd, _dense(state_in, "state_in", shape, f, stream), po,
                                 _dense(state_out, "state_out", shape, f, stream), ws, ws_bytes, _stream(stream)))


def linattn_backward(q, k, v, log_decay, state_in, offsets, d_o, d_state_out, B: int, T: int, heads: int, kv_heads: int,
                     Dk: int, Dv: int, scale: float, dq, dk, dv, d_state_in=None, workspace=None, stream=None) -> None:
    import torch
    f = torch.float32
    cfg, pq, pk, pv, pdo, pd = _linattn_args(q, k, v, log_decay, offsets, B, T, heads, kv_heads, Dk, Dv, scale, d_o, stream)
    lead = (B, T) if offsets is None else (T,)
    grads = []
    for t, what, n, D, ld in ((dq, "dq", heads, Dk, cfg.ld_q), (dk, "dk", kv_heads, Dk, cfg.ld_k), (dv, "dv", kv_heads, Dv, cfg.ld_v)):
        p, own = _rows(t, what, lead, n, D, q.dtype, stream)
        if own != ld:
            raise ValueError(f"{what} must have the row stride of {what[1:]} ({ld}), has {own}")
        grads.append(p)
    shape = (B, kv_heads, Dk, Dv)
    ws, ws_bytes, keep = _linattn_workspace(cfg, True, workspace, stream)
    _check(lib().linattn_backward(C.byref(cfg), pq, pk, pv, pd, _dense(state_in, "state_in", shape, f, stream), pdo,
                                  _dense(d_state_out, "d_state_out", shape, f, stream), *grads,
                                  _dense(d_state_in, "d_state_in", shape, f, stream), ws, ws_bytes, _stream(stream)))


class PreparedLinattnStep:
    """linattn_step with its arguments marshalled once, for loops that generate step after step on the same buffers: calling
    the object runs the step, on the stream given (None: the one that is current when the object is made).  The tensors are
    kept alive; their contents may change between calls."""

    def __init__(self, q, k, v, log_decay, state, slots, B: int, heads: int, kv_heads: int, Dk: int, Dv: int, scale: float, o,
                 stream=None):
        import torch
        code = _linattn_dtype(q.dtype)
        pq, lq = _rows(q, "q", (B,), heads, Dk, q.dtype, stream)
        pk, lk = _rows(k, "k", (B,), kv_heads, Dk, q.dtype, stream)
        pv, lv = _rows(v, "v", (B,), kv_heads, Dv, q.dtype, stream)
        po, lo = _rows(o, "o", (B,), heads, Dv, q.dtype, stream)
        n_slots = state.shape[0]
        self._device, self._current = q.device.index, torch.cuda.current_device
        self._keep = (q, k, v, log_decay, state, slots, o, stream)
        self._cfg = linattn_config(int(B), 1, int(heads), int(kv_heads), int(Dk), int(Dv), code, float(scale), lq, lk, lv, lo, None)
        self._fn = lib().linattn_step
        vp = C.c_void_p
        self._args = (C.byref(self._cfg), vp(pq), vp(pk), vp(pv), vp(_dense(log_decay, "log_decay", (kv_heads,), torch.float32, stream)),
                      vp(_dense(state, "state", (n_slots, kv_heads, Dk, Dv), torch.float32, stream)), C.c_int32(n_slots),
                      vp(_dense(slots, "slots", (B,), torch.int32, stream)), vp(po), vp(_stream(stream)))

    def __call__(self) -> None:
        if self._current() != self._device:      # (a launch goes to the current device whatever its tensors)
            raise ValueError(f"the tensors are on cuda:{self._device}, the current device is cuda:{self._current()}")
        code = self._fn(*self._args)
        if code != MADE_OK:
            raise MadeError(code, made_last_error())


def linattn_step(q, k, v, log_decay, state, slots, B: int, heads: int, kv_heads: int, Dk: int, Dv: int, scale: float, o,
                 stream=None) -> None:
    """state [n_slots, kv_heads, Dk, Dv] is updated in place; slots: int32 [B] or None (row b has place b)."""
    PreparedLinattnStep(q, k, v, log_decay, state, slots, B, heads, kv_heads, Dk, Dv, scale, o, stream)()


# ------------------------------------------------------------------------------------------------
# AdamW over many tensors (include/jacobi_adamw.h).  Weights and gradients are float32 or bfloat16 (each list of one type),
# moments float32, or int8 and uint8 with float32 scales (adamw_moments makes zeroed ones).
# ------------------------------------------------------------------------------------------------
def adamw_moments(params, bits: int = 32):
    """Zeroed moments for these tensors: (m, v, m_scale, v_scale), lists; the scales are None for 32 bits."""
    import torch
    if bits == 32:
        return [torch.zeros_like(p, dtype=torch.float32) for p in params], [torch.zeros_like(p, dtype=torch.float32) for p in params], None, None
    if bits != 8:
        raise ValueError(f"moments have 8 or 32 bits, not {bits}")
    scales = [[torch.zeros(-(-p.numel() // ADAMW_BLOCK), dtype=torch.float32, device=p.device) for p in params] for _ in range(2)]
    return ([torch.zeros_like(p, dtype=torch.int8) for p in params], [torch.zeros_like(p, dtype=torch.uint8) for p in params],
            scales[0], scales[1])


def _pointers(tensors, what: str, dtype, sizes, stream=None):
    """Host array of the device pointers of contiguous tensors of these sizes and one type."""
    if len(tensors) != len(sizes):
        raise ValueError(f"{len(tensors)} tensors in {what}, expected {len(sizes)}")
    out = (C.c_void_p * len(sizes))()
    for i, t in enumerate(tensors):
        _on_device(t, f"{what}[{i}]", stream)
        if t.numel() != sizes[i]:
            raise ValueError(f"{what}[{i}] has {t.numel()} elements, expected {sizes[i]}")
        out[i] = _ptr(t, dtype) or None
    return out


class PreparedAdamW:
    """adamw_step with its tensors checked and marshalled once, for loops that take step after step on the same buffers (a
    gradient that is allocated anew for every step needs a new object): calling the object runs a step.  The tensors are kept
    alive; their contents may change between calls."""

    def __init__(self, params, grads, m, v, m_scale=None, v_scale=None, copies=None):
        import torch
        if not params:
            raise ValueError("no tensors")
        sizes = [p.numel() for p in params]
        blocks = [-(-n // ADAMW_BLOCK) for n in sizes]
        eight = m_scale is not None
        if eight != (v_scale is not None):
            raise ValueError("m_scale and v_scale go together")
        for what, ts in (("params", params), ("grads", grads)):
            if ts[0].dtype not in (torch.float32, torch.bfloat16):
                raise ValueError(f"{what}: expected torch.float32 or torch.bfloat16, got {ts[0].dtype}")
        f = torch.float32
        self._device = params[0].device
        self._n = C.c_int32(len(sizes))
        self._sizes = (C.c_int64 * len(sizes))(*sizes)
        self._arrays = [_pointers(params, "params", params[0].dtype, sizes), _pointers(grads, "grads", grads[0].dtype, sizes),
                        _pointers(m, "m", torch.int8 if eight else f, sizes), _pointers(v, "v", torch.uint8 if eight else f, sizes),
                        _pointers(m_scale, "m_scale", f, blocks) if eight else None,
                        _pointers(v_scale, "v_scale", f, blocks) if eight else None,
                        _pointers(copies, "copies", torch.bfloat16, sizes) if copies is not None else None]
        written = [t for ts in (params, m, v, m_scale, v_scale, copies) if ts is not None for t in ts if t.numel()]
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in written)
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("two of the tensors that are written overlap (is one listed twice?)")
        self._types = (MADE_BF16 if params[0].dtype == torch.bfloat16 else MADE_F32,
                       MADE_BF16 if grads[0].dtype == torch.bfloat16 else MADE_F32, 8 if eight else 32)
        self._keep = (params, grads, m, v, m_scale, v_scale, copies)
        self._fn = lib().adamw_step

    def __call__(self, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, step: int, grad_scale: float = 1.0,
                 scalars=None, stream=None) -> None:
        """scalars: float64 [4] on the device, {lr, 1 / (1 - beta1^step), 1 / (1 - beta2^step), grad_scale}, read when the step
        runs in place of lr, step and grad_scale (a recorded step then follows them), or None."""
        import torch
        c = adamw_config(lr, beta1, beta2, eps, weight_decay, grad_scale, step, *self._types)     # (the call's own: threads may share the object)
        if any(self._device.index != d for d in (torch.cuda.current_device(), *([] if stream is None else [stream.device.index]))):
            raise ValueError(f"the tensors are on {self._device}, the call is for another device")
        _check(self._fn(C.byref(c), self._n, self._sizes, *self._arrays, _dense(scalars, "scalars", (4,), torch.float64, stream),
                        _stream(stream)))


def adamw_step(params, grads, m, v, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, step: int, m_scale=None,
               v_scale=None, copies=None, grad_scale: float = 1.0, scalars=None, stream=None) -> None:
    PreparedAdamW(params, grads, m, v, m_scale, v_scale, copies)(lr, beta1, beta2, eps, weight_decay, step, grad_scale, scalars, stream)


def adamw_unpack(m, v, m_scale, v_scale, m_out, v_out, stream=None) -> None:
    """The float32 values that 8-bit moments stand for (lists of tensors)."""
    import torch
    sizes = [t.numel() for t in m]
    blocks = [-(-n // ADAMW_BLOCK) for n in sizes]
    f = torch.float32
    _check(lib().adamw_unpack(len(sizes), (C.c_int64 * len(sizes))(*sizes), _pointers(m, "m", torch.int8, sizes, stream),
                              _pointers(v, "v", torch.uint8, sizes, stream), _pointers(m_scale, "m_scale", f, blocks, stream),
                              _pointers(v_scale, "v_scale", f, blocks, stream), _pointers(m_out, "m_out", f, sizes, stream),
                              _pointers(v_out, "v_out", f, sizes, stream), _stream(stream)))
