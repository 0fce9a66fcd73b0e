"""Python binding of libmhlmoe, the MI355X (gfx950) hot path of Multi-Head
LatentMoE: IO-aware routing and IO-aware expert computation.

The functions carry the C ABI's names (see include/mhlmoe.h) and only
marshal arguments: every step of the computation runs in the HIP kernels of
libmhlmoe.so.  PyTorch supplies device memory (outputs and workspaces the
caller did not pass) and the current HIP stream.  There is no CPU fallback:
if the library is not built, or a tensor is not on the GPU, the call raises.
"""
from __future__ import annotations

import ctypes
import os
import re
from typing import Optional

import torch

__all__ = [
    "MhlmoeError", "load_library", "library_path", "declared_functions",
    "MHLMOE_F32", "MHLMOE_BF16",
    "MHLMOE_OP_ROUTE", "MHLMOE_OP_BUCKET", "MHLMOE_OP_EXPERTS", "MHLMOE_OP_LAYER",
    "MHLMOE_OP_LAYER_BACKWARD",
    "mhlmoe_version", "mhlmoe_last_error", "mhlmoe_workspace_size",
    "mhlmoe_route", "mhlmoe_route_static", "mhlmoe_bucket", "mhlmoe_experts", "mhlmoe_layer",
    "mhlmoe_experts_gelu", "mhlmoe_layer_gelu",
    "mhlmoe_layer_backward", "workspace",
    "mhlmoe_rmsnorm", "mhlmoe_rmsnorm_backward", "mhlmoe_rmsnorm_backward_workspace",
    "mhlmoe_quantize", "mhlmoe_gemm_scaled", "mhlmoe_latent_layer_scaled",
    "mhlmoe_latent_layer_scaled_workspace",
    "mhlmoe_layernorm", "mhlmoe_layernorm_backward", "mhlmoe_layernorm_backward_workspace",
    "mhlmoe_expert_counts", "mhlmoe_balance_loss", "mhlmoe_balance_loss_workspace",
    "mhlmoe_balance_loss_backward", "mhlmoe_balance_loss_backward_workspace",
    "AdamWTensors", "mhlmoe_adamw",
    "mhlmoe_timing_enable", "mhlmoe_timing_query", "mhlmoe_timing_reset",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
HEADER = os.path.join(_ROOT, "include", "mhlmoe.h")

MHLMOE_OK, MHLMOE_EINVAL, MHLMOE_EUNSUPPORTED, MHLMOE_EWORKSPACE, MHLMOE_EHIP = range(5)
MHLMOE_F32, MHLMOE_BF16 = 0, 1
(MHLMOE_OP_ROUTE, MHLMOE_OP_BUCKET, MHLMOE_OP_EXPERTS, MHLMOE_OP_LAYER,
 MHLMOE_OP_LAYER_BACKWARD, MHLMOE_OP_LATENT_LAYER, MHLMOE_OP_LATENT_BACKWARD,
 MHLMOE_OP_ROUTE_BACKWARD) = range(8)
_STATUS = {0: "MHLMOE_OK", 1: "MHLMOE_EINVAL", 2: "MHLMOE_EUNSUPPORTED",
           3: "MHLMOE_EWORKSPACE", 4: "MHLMOE_EHIP"}

_P = ctypes.c_void_p
_I64 = ctypes.c_int64
_I = ctypes.c_int
_SZ = ctypes.c_size_t


class _AdamWTensor(ctypes.Structure):  # mhlmoe_adamw_tensor
    _fields_ = [("param", _P), ("master", _P), ("grad", _P), ("m", _P), ("v", _P),
                ("m_scale", _P), ("v_scale", _P), ("n", _I64), ("weight_decay", ctypes.c_float),
                ("seed", ctypes.c_uint32), ("param_dtype", _I), ("grad_dtype", _I)]


class _AdamWStep(ctypes.Structure):  # mhlmoe_adamw_step
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", _I64), ("grad_scale", _P)]


class MhlmoeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def library_path() -> str:
    return os.path.join(_PKG, "libmhlmoe.so")


_lib = None


def _declare(lib):
    lib.mhlmoe_version.restype = _I
    lib.mhlmoe_version.argtypes = []
    lib.mhlmoe_last_error.restype = ctypes.c_char_p
    lib.mhlmoe_last_error.argtypes = []
    lib.mhlmoe_workspace_size.argtypes = [_I, _I64, _I, _I, _I, _I, _I, _I, ctypes.POINTER(_SZ)]
    lib.mhlmoe_route.argtypes = [_P, _P, _P, _I64, _I, _I, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]
    lib.mhlmoe_route_static.argtypes = [_P, _P, _P, _I64, _I, _I, _I, _I, _I, _P, _P, _P, _P]
    lib.mhlmoe_route_backward.argtypes = [_P] * 5 + [_I64, _I, _I, _I, _I, _I] + [_P] * 3 + [_SZ, _P]
    lib.mhlmoe_bucket.argtypes = [_P, _I64, _I, _I, _I, _P, _P, _P, _P, _SZ, _P]
    lib.mhlmoe_experts.argtypes = [_P, _P, _P, _P, _P, _P, _I64, _I, _I, _I, _I, _I, _I, _P, _P, _SZ, _P]
    lib.mhlmoe_layer.argtypes = ([_P] * 6 + [_I64, _I, _I, _I, _I, _I, _I] + [_P] * 5 + [_SZ, _P])
    lib.mhlmoe_layer_backward.argtypes = ([_P] * 8 + [_I64, _I, _I, _I, _I, _I, _I] + [_P] * 6 + [_SZ, _P])
    lib.mhlmoe_experts_gelu.argtypes = [_P] * 5 + [_I64, _I, _I, _I, _I, _I, _I, _P, _P, _SZ, _P]
    lib.mhlmoe_layer_gelu.argtypes = ([_P] * 5 + [_I64, _I, _I, _I, _I, _I, _I] + [_P] * 5 + [_SZ, _P])
    lib.mhlmoe_layer_gelu_backward.argtypes = ([_P] * 7 + [_I64, _I, _I, _I, _I, _I, _I]
                                               + [_P] * 5 + [_SZ, _P])
    lib.mhlmoe_layer_routed.argtypes = ([_P] * 7 + [_I64, _I, _I, _I, _I, _I, _I] + [_P] * 5
                                        + [_SZ, _P])
    lib.mhlmoe_layer_backward_routed.argtypes = ([_P] * 9 + [_I64, _I, _I, _I, _I, _I, _I]
                                                 + [_P] * 7 + [_SZ, _P])
    lib.mhlmoe_latent_layer.argtypes = [_P] * 8 + [_I64] + [_I] * 8 + [_P] * 8 + [_SZ, _P]
    lib.mhlmoe_latent_layer_backward.argtypes = ([_P] * 13 + [_I64] + [_I] * 8 + [_P] * 8
                                                 + [_SZ, _P])
    lib.mhlmoe_bias_update.argtypes = [_P, _P, _I, _I, ctypes.c_float, _P]
    F = ctypes.c_float
    lib.mhlmoe_rmsnorm.argtypes = [_P] * 3 + [_I64, _I, F, _I] + [_P] * 5
    lib.mhlmoe_rmsnorm_backward_workspace.argtypes = [_I64, _I, ctypes.POINTER(_SZ)]
    lib.mhlmoe_rmsnorm_backward.argtypes = [_P] * 4 + [_I64, _I, F, _I] + [_P] * 3 + [_SZ, _P]
    lib.mhlmoe_quantize.argtypes = [_P, _I64, _I64, _I, _I, _I, _P, _P, _P]
    lib.mhlmoe_gemm_scaled.argtypes = [_P] * 4 + [_I64] * 3 + [_I, _I, _P, _P]
    lib.mhlmoe_latent_layer_scaled_workspace.argtypes = ([_I64] + [_I] * 7
                                                         + [ctypes.POINTER(_SZ)])
    lib.mhlmoe_latent_layer_scaled.argtypes = ([_P] * 3 + [F] + [_P] * 11 + [_I64] + [_I] * 7
                                               + [_P] * 9 + [_SZ, _P])
    lib.mhlmoe_layernorm.argtypes = [_P] * 4 + [_I64, _I, F, _I] + [_P] * 5
    lib.mhlmoe_layernorm_backward_workspace.argtypes = [_I64, _I, ctypes.POINTER(_SZ)]
    lib.mhlmoe_layernorm_backward.argtypes = ([_P] * 4 + [_I64, _I, F, _I] + [_P] * 4
                                              + [_SZ, _P])
    lib.mhlmoe_expert_counts.argtypes = [_P, _P, _I64, _I, _I, _I, _P, _P]
    lib.mhlmoe_balance_loss_workspace.argtypes = [_I64, _I, _I, _I, ctypes.POINTER(_SZ)]
    lib.mhlmoe_balance_loss.argtypes = [_P] * 4 + [_I64] + [_I] * 4 + [_P] * 3 + [_SZ, _P]
    lib.mhlmoe_balance_loss_backward_workspace.argtypes = [_I64, _I, _I, _I, ctypes.POINTER(_SZ)]
    lib.mhlmoe_balance_loss_backward.argtypes = ([_P] * 8 + [_I64] + [_I] * 4 + [_P] * 3
                                                 + [_SZ, _P])
    lib.mhlmoe_adamw.argtypes = [_P, _I, _P, _P]
    lib.mhlmoe_timing_enable.argtypes = [_I]
    lib.mhlmoe_timing_query.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                        ctypes.POINTER(_I64)]
    lib.mhlmoe_timing_reset.argtypes = []
    for name in ("mhlmoe_workspace_size", "mhlmoe_route", "mhlmoe_bucket", "mhlmoe_experts",
                 "mhlmoe_layer", "mhlmoe_layer_backward", "mhlmoe_experts_gelu",
                 "mhlmoe_layer_gelu", "mhlmoe_timing_enable",
                 "mhlmoe_timing_query", "mhlmoe_timing_reset", "mhlmoe_rmsnorm",
                 "mhlmoe_rmsnorm_backward", "mhlmoe_rmsnorm_backward_workspace",
                 "mhlmoe_quantize", "mhlmoe_gemm_scaled", "mhlmoe_latent_layer_scaled",
                 "mhlmoe_latent_layer_scaled_workspace", "mhlmoe_layernorm",
                 "mhlmoe_layernorm_backward", "mhlmoe_layernorm_backward_workspace",
                 "mhlmoe_expert_counts", "mhlmoe_balance_loss", "mhlmoe_balance_loss_workspace",
                 "mhlmoe_balance_loss_backward", "mhlmoe_balance_loss_backward_workspace",
                 "mhlmoe_adamw"):
        getattr(lib, name).restype = _I
    return lib


def load_library():
    """Load the in-tree libmhlmoe.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(
                f"{path} is missing: build it with `python -m paper_2602_04870_amd.build` "
                "(there is no fallback implementation)")
        _lib = _declare(ctypes.CDLL(path))
    return _lib


def declared_functions(header: str = HEADER):
    """Names of the functions include/mhlmoe.h declares."""
    text = open(header).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(mhlmoe_[a-z_]+)\s*\(", text)))


def _check(status: int):
    if status != MHLMOE_OK:
        msg = load_library().mhlmoe_last_error().decode(errors="replace")
        raise MhlmoeError(status, msg)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return MHLMOE_F32
    if t.dtype == torch.bfloat16:
        return MHLMOE_BF16
    raise TypeError(f"unsupported activation/weight dtype {t.dtype}")


def _dev(t: Optional[torch.Tensor], name: str, dtype=None, shape=None):
    """Device pointer of a contiguous GPU tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device}); libmhlmoe has no CPU path")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def mhlmoe_version() -> int:
    return load_library().mhlmoe_version()


def mhlmoe_last_error() -> str:
    return load_library().mhlmoe_last_error().decode(errors="replace")


def mhlmoe_workspace_size(op: int, T: int, n_heads: int, d_head: int, n_experts: int,
                          top_k: int, d_ff: int = 0, dtype: int = MHLMOE_BF16) -> int:
    out = _SZ(0)
    _check(load_library().mhlmoe_workspace_size(op, T, n_heads, d_head, n_experts, top_k,
                                                d_ff, dtype, ctypes.byref(out)))
    return out.value


def workspace(op: int, T: int, n_heads: int, d_head: int, n_experts: int, top_k: int,
              d_ff: int = 0, dtype: int = MHLMOE_BF16, device="cuda") -> torch.Tensor:
    """Allocate a workspace tensor for entry point `op` (at least 1 byte)."""
    n = mhlmoe_workspace_size(op, T, n_heads, d_head, n_experts, top_k, d_ff, dtype)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def _ws(ws, op, *shape):
    if ws is None:
        ws = workspace(op, *shape)
    return _dev(ws, "workspace", torch.uint8), ws.numel()


def mhlmoe_route(X, W_router, bias, top_k, *, idx=None, gate=None, counts=None,
                 workspace=None, stream=None):
    """Algorithm 1: returns (idx [T,Nh,k] int32, gate [T,Nh,k] f32,
    counts [Nh,Ne] int32)."""
    T, Nh, dh = X.shape
    Ne = W_router.shape[1]
    dt = _dtype_code(X)
    dev = X.device
    idx = idx if idx is not None else torch.empty((T, Nh, top_k), dtype=torch.int32, device=dev)
    gate = gate if gate is not None else torch.empty((T, Nh, top_k), dtype=torch.float32, device=dev)
    counts = counts if counts is not None else torch.empty((Nh, Ne), dtype=torch.int32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_ROUTE, T, Nh, dh, Ne, top_k, 0, dt)
    _check(load_library().mhlmoe_route(
        _dev(X, "X"), _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)), T, Nh, dh, Ne, top_k, dt,
        _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), wsp, wsn, _stream(stream)))
    return idx, gate, counts


def mhlmoe_route_static(X, W_router, bias, top_k, *, idx, gate, counts, stream=None):
    """mhlmoe_route without a workspace (the library's static scratch):
    the caller passes the outputs idx [T,Nh,k] int32, gate [T,Nh,k] f32 and
    counts [Nh,Ne] int32, so the call allocates nothing."""
    T, Nh, dh = X.shape
    Ne = W_router.shape[1]
    _check(load_library().mhlmoe_route_static(
        _dev(X, "X"), _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)), T, Nh, dh, Ne, top_k, _dtype_code(X),
        _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), _stream(stream)))
    return idx, gate, counts


def mhlmoe_route_backward(X, W_router, idx, gate, dgate, *, dX=None, dW_router=None,
                          workspace=None, stream=None):
    """Algorithm 2 from the gate gradient: returns (dX, dW_router)."""
    T, Nh, dh = X.shape
    Ne = W_router.shape[1]
    k = idx.shape[2]
    dt = _dtype_code(X)
    f32 = torch.float32
    dX = dX if dX is not None else torch.empty_like(X)
    dW_router = dW_router if dW_router is not None else torch.empty((Nh, Ne, dh), dtype=f32,
                                                                    device=X.device)
    wsp, wsn = _ws(workspace, MHLMOE_OP_ROUTE_BACKWARD, T, Nh, dh, Ne, k, 0, dt)
    _check(load_library().mhlmoe_route_backward(
        _dev(X, "X"), _dev(W_router, "W_router", f32, (Nh, Ne, dh)),
        _dev(idx, "idx", torch.int32, (T, Nh, k)), _dev(gate, "gate", f32, (T, Nh, k)),
        _dev(dgate, "dgate", f32, (T, Nh, k)), T, Nh, dh, Ne, k, dt,
        _dev(dX, "dX", X.dtype, (T, Nh, dh)), _dev(dW_router, "dW_router", f32, (Nh, Ne, dh)),
        wsp, wsn, _stream(stream)))
    return dX, dW_router


def mhlmoe_bucket(idx, n_experts, *, counts=None, offsets=None, perm=None, workspace=None,
                  stream=None):
    """Token clustering: returns (counts [Nh,Ne], offsets [Nh,Ne+1], perm [Nh,T*k])."""
    T, Nh, k = idx.shape
    Ne = n_experts
    dev = idx.device
    counts = counts if counts is not None else torch.empty((Nh, Ne), dtype=torch.int32, device=dev)
    offsets = offsets if offsets is not None else torch.empty((Nh, Ne + 1), dtype=torch.int32, device=dev)
    perm = perm if perm is not None else torch.empty((Nh, T * k), dtype=torch.int32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_BUCKET, T, Nh, 64, Ne, k, 0, MHLMOE_BF16)
    _check(load_library().mhlmoe_bucket(
        _dev(idx, "idx", torch.int32), T, Nh, Ne, k,
        _dev(counts, "counts", torch.int32, (Nh, Ne)),
        _dev(offsets, "offsets", torch.int32, (Nh, Ne + 1)),
        _dev(perm, "perm", torch.int32, (Nh, T * k)), wsp, wsn, _stream(stream)))
    return counts, offsets, perm


def mhlmoe_experts(X, idx, gate, W1, W3, W2, *, Y=None, workspace=None, stream=None):
    """Grouped SwiGLU experts + gate-weighted combine: returns Y [T,Nh,dh]."""
    T, Nh, dh = X.shape
    k = idx.shape[2]
    Ne, dff = W1.shape[1], W1.shape[2]
    dt = _dtype_code(X)
    Y = Y if Y is not None else torch.empty_like(X)
    wsp, wsn = _ws(workspace, MHLMOE_OP_EXPERTS, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_experts(
        _dev(X, "X"), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", torch.float32, (T, Nh, k)),
        _dev(W1, "W1", X.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", X.dtype, (Nh, Ne, dh, dff)), T, Nh, dh, Ne, k, dff, dt,
        _dev(Y, "Y", X.dtype, (T, Nh, dh)), wsp, wsn, _stream(stream)))
    return Y


def mhlmoe_layer(X, W_router, bias, W1, W3, W2, top_k, *, Y=None, idx=None, gate=None,
                 counts=None, workspace=None, stream=None, return_routing=True):
    """Routing + experts.  Returns Y, or (Y, idx, gate, counts) when
    return_routing (routing outputs are then allocated if not passed)."""
    T, Nh, dh = X.shape
    Ne, dff = W1.shape[1], W1.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    Y = Y if Y is not None else torch.empty_like(X)
    if return_routing:
        idx = idx if idx is not None else torch.empty((T, Nh, top_k), dtype=torch.int32, device=dev)
        gate = gate if gate is not None else torch.empty((T, Nh, top_k), dtype=torch.float32, device=dev)
        counts = counts if counts is not None else torch.empty((Nh, Ne), dtype=torch.int32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER, T, Nh, dh, Ne, top_k, dff, dt)
    _check(load_library().mhlmoe_layer(
        _dev(X, "X"), _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)),
        _dev(W1, "W1", X.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", X.dtype, (Nh, Ne, dh, dff)), T, Nh, dh, Ne, top_k, dff, dt,
        _dev(Y, "Y", X.dtype, (T, Nh, dh)), _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), wsp, wsn, _stream(stream)))
    return (Y, idx, gate, counts) if return_routing else Y


def mhlmoe_experts_gelu(X, idx, gate, W_in, W_out, *, Y=None, workspace=None, stream=None):
    """Grouped two-matrix GELU experts (Sec. 3.4) + gate-weighted combine:
    returns Y [T,Nh,dh]."""
    T, Nh, dh = X.shape
    k = idx.shape[2]
    Ne, dff = W_in.shape[1], W_in.shape[2]
    dt = _dtype_code(X)
    Y = Y if Y is not None else torch.empty_like(X)
    wsp, wsn = _ws(workspace, MHLMOE_OP_EXPERTS, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_experts_gelu(
        _dev(X, "X"), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", torch.float32, (T, Nh, k)),
        _dev(W_in, "W_in", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W_out, "W_out", X.dtype, (Nh, Ne, dh, dff)), T, Nh, dh, Ne, k, dff, dt,
        _dev(Y, "Y", X.dtype, (T, Nh, dh)), wsp, wsn, _stream(stream)))
    return Y


def mhlmoe_layer_gelu(X, W_router, bias, W_in, W_out, top_k, *, Y=None, idx=None, gate=None,
                      counts=None, workspace=None, stream=None, return_routing=True):
    """Routing + the GELU experts.  Returns Y, or (Y, idx, gate, counts)."""
    T, Nh, dh = X.shape
    Ne, dff = W_in.shape[1], W_in.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    Y = Y if Y is not None else torch.empty_like(X)
    if return_routing:
        idx = idx if idx is not None else torch.empty((T, Nh, top_k), dtype=torch.int32, device=dev)
        gate = gate if gate is not None else torch.empty((T, Nh, top_k), dtype=torch.float32, device=dev)
        counts = counts if counts is not None else torch.empty((Nh, Ne), dtype=torch.int32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER, T, Nh, dh, Ne, top_k, dff, dt)
    _check(load_library().mhlmoe_layer_gelu(
        _dev(X, "X"), _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)),
        _dev(W_in, "W_in", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W_out, "W_out", X.dtype, (Nh, Ne, dh, dff)), T, Nh, dh, Ne, top_k, dff, dt,
        _dev(Y, "Y", X.dtype, (T, Nh, dh)), _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), wsp, wsn, _stream(stream)))
    return (Y, idx, gate, counts) if return_routing else Y


def mhlmoe_layer_backward(X, W_router, W1, W3, W2, idx, gate, dY, *, dX=None, dW_router=None,
                          dW1=None, dW3=None, dW2=None, workspace=None, stream=None):
    """Backward of mhlmoe_layer: returns (dX, dW_router, dW1, dW3, dW2)."""
    T, Nh, dh = X.shape
    k = idx.shape[2]
    Ne, dff = W1.shape[1], W1.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    f32 = torch.float32
    dX = dX if dX is not None else torch.empty_like(X)
    dW_router = dW_router if dW_router is not None else torch.empty((Nh, Ne, dh), dtype=f32, device=dev)
    dW1 = dW1 if dW1 is not None else torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev)
    dW3 = dW3 if dW3 is not None else torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev)
    dW2 = dW2 if dW2 is not None else torch.empty((Nh, Ne, dh, dff), dtype=f32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER_BACKWARD, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_layer_backward(
        _dev(X, "X"), _dev(W_router, "W_router", f32, (Nh, Ne, dh)),
        _dev(W1, "W1", X.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", X.dtype, (Nh, Ne, dh, dff)), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", f32, (T, Nh, k)), _dev(dY, "dY", X.dtype, (T, Nh, dh)),
        T, Nh, dh, Ne, k, dff, dt, _dev(dX, "dX", X.dtype, (T, Nh, dh)),
        _dev(dW_router, "dW_router", f32, (Nh, Ne, dh)), _dev(dW1, "dW1", f32, (Nh, Ne, dff, dh)),
        _dev(dW3, "dW3", f32, (Nh, Ne, dff, dh)), _dev(dW2, "dW2", f32, (Nh, Ne, dh, dff)),
        wsp, wsn, _stream(stream)))
    return dX, dW_router, dW1, dW3, dW2


def mhlmoe_layer_routed(X, R, W_router, bias, W1, W3, W2, top_k, *, Y=None, idx=None,
                        gate=None, counts=None, workspace=None, stream=None,
                        return_routing=True):
    """Separate routing sub-tokens (Sec. 4.4): routes by R, computes the
    experts on X.  W3=None selects the two-matrix GELU expert (W1 = W_in,
    W2 = W_out).  Returns Y, or (Y, idx, gate, counts)."""
    T, Nh, dh = X.shape
    Ne, dff = W1.shape[1], W1.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    Y = Y if Y is not None else torch.empty_like(X)
    if return_routing:
        idx = idx if idx is not None else torch.empty((T, Nh, top_k), dtype=torch.int32, device=dev)
        gate = gate if gate is not None else torch.empty((T, Nh, top_k), dtype=torch.float32, device=dev)
        counts = counts if counts is not None else torch.empty((Nh, Ne), dtype=torch.int32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER, T, Nh, dh, Ne, top_k, dff, dt)
    _check(load_library().mhlmoe_layer_routed(
        _dev(X, "X"), _dev(R, "R", X.dtype, (T, Nh, dh)),
        _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)),
        _dev(W1, "W1", X.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", X.dtype, (Nh, Ne, dh, dff)), T, Nh, dh, Ne, top_k, dff, dt,
        _dev(Y, "Y", X.dtype, (T, Nh, dh)), _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), wsp, wsn, _stream(stream)))
    return (Y, idx, gate, counts) if return_routing else Y


def mhlmoe_layer_backward_routed(X, R, W_router, W1, W3, W2, idx, gate, dY, *, dX=None,
                                 dR=None, dW_router=None, dW1=None, dW3=None, dW2=None,
                                 workspace=None, stream=None):
    """Backward of mhlmoe_layer_routed: returns (dX, dR, dW_router, dW1, dW3, dW2).
    W3=None selects the GELU expert (W1 = W_in, W2 = W_out); dW3 is then None."""
    T, Nh, dh = X.shape
    k = idx.shape[2]
    Ne, dff = W1.shape[1], W1.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    f32 = torch.float32
    dX = dX if dX is not None else torch.empty_like(X)
    dR = dR if dR is not None else torch.empty_like(X)
    dW_router = dW_router if dW_router is not None else torch.empty((Nh, Ne, dh), dtype=f32, device=dev)
    dW1 = dW1 if dW1 is not None else torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev)
    if W3 is None:
        dW3 = None
    elif dW3 is None:
        dW3 = torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev)
    dW2 = dW2 if dW2 is not None else torch.empty((Nh, Ne, dh, dff), dtype=f32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER_BACKWARD, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_layer_backward_routed(
        _dev(X, "X"), _dev(R, "R", X.dtype, (T, Nh, dh)),
        _dev(W_router, "W_router", f32, (Nh, Ne, dh)),
        _dev(W1, "W1", X.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", X.dtype, (Nh, Ne, dh, dff)), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", f32, (T, Nh, k)), _dev(dY, "dY", X.dtype, (T, Nh, dh)),
        T, Nh, dh, Ne, k, dff, dt, _dev(dX, "dX", X.dtype, (T, Nh, dh)),
        _dev(dR, "dR", X.dtype, (T, Nh, dh)),
        _dev(dW_router, "dW_router", f32, (Nh, Ne, dh)), _dev(dW1, "dW1", f32, (Nh, Ne, dff, dh)),
        _dev(dW3, "dW3", f32, (Nh, Ne, dff, dh)), _dev(dW2, "dW2", f32, (Nh, Ne, dh, dff)),
        wsp, wsn, _stream(stream)))
    return dX, dR, dW_router, dW1, dW3, dW2


def mhlmoe_latent_layer(x, W_in, W_router, bias, W1, W3, W2, W_out, n_heads, top_k, *,
                        routing_tokens=False, out=None, X_lat=None, R_lat=None, Y_lat=None,
                        idx=None, gate=None, counts=None, workspace=None, stream=None):
    """The layer with its projections (Eq. (5)-(6); Eq. (9) with
    routing_tokens).  x [T, d_model]; W_in [(1 + routing_tokens) N, d_model];
    W_out [d_model, N].  Returns a dict with out, X_lat, R_lat (routing
    tokens only), Y_lat, idx, gate, counts."""
    T, d_model = x.shape
    Ne, dff, dh = W1.shape[1], W1.shape[2], W1.shape[3]
    Nh = n_heads
    N = Nh * dh
    rt = 1 if routing_tokens else 0
    dt = _dtype_code(x)
    dev = x.device

    def alloc(t, shape, dtype):
        return t if t is not None else torch.empty(shape, dtype=dtype, device=dev)

    out = alloc(out, (T, d_model), x.dtype)
    X_lat = alloc(X_lat, (T, Nh, dh), x.dtype)
    R_lat = alloc(R_lat, (T, Nh, dh), x.dtype) if rt else R_lat
    Y_lat = alloc(Y_lat, (T, Nh, dh), x.dtype)
    idx = alloc(idx, (T, Nh, top_k), torch.int32)
    gate = alloc(gate, (T, Nh, top_k), torch.float32)
    counts = alloc(counts, (Nh, Ne), torch.int32)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LATENT_LAYER, T, Nh, dh, Ne, top_k, dff, dt)
    _check(load_library().mhlmoe_latent_layer(
        _dev(x, "x"), _dev(W_in, "W_in", x.dtype, ((1 + rt) * N, d_model)),
        _dev(W_router, "W_router", torch.float32, (Nh, Ne, dh)),
        _dev(bias, "bias", torch.float32, (Nh, Ne)),
        _dev(W1, "W1", x.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", x.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", x.dtype, (Nh, Ne, dh, dff)), _dev(W_out, "W_out", x.dtype, (d_model, N)),
        T, d_model, Nh, dh, Ne, top_k, dff, rt, dt, _dev(out, "out", x.dtype, (T, d_model)),
        _dev(X_lat, "X_lat", x.dtype, (T, Nh, dh)),
        _dev(R_lat, "R_lat", x.dtype, (T, Nh, dh)) if rt else None,
        _dev(Y_lat, "Y_lat", x.dtype, (T, Nh, dh)), _dev(idx, "idx", torch.int32, (T, Nh, top_k)),
        _dev(gate, "gate", torch.float32, (T, Nh, top_k)),
        _dev(counts, "counts", torch.int32, (Nh, Ne)), wsp, wsn, _stream(stream)))
    res = {"out": out, "X_lat": X_lat, "Y_lat": Y_lat, "idx": idx, "gate": gate, "counts": counts}
    if rt:
        res["R_lat"] = R_lat
    return res


def mhlmoe_latent_layer_backward(x, W_in, W_router, W1, W3, W2, W_out, X_lat, R_lat, Y_lat, idx,
                                 gate, dout, *, routing_tokens=False, workspace=None,
                                 stream=None):
    """Backward of mhlmoe_latent_layer: returns a dict with dx, dW_in,
    dW_router, dW1, dW3, dW2, dW_out (W3=None: the GELU expert, dW3 None)."""
    T, d_model = x.shape
    Nh, Ne, dff, dh = W1.shape
    k = idx.shape[2]
    N = Nh * dh
    rt = 1 if routing_tokens else 0
    dt = _dtype_code(x)
    dev = x.device
    f32 = torch.float32
    g = {"dx": torch.empty_like(x),
         "dW_in": torch.empty(((1 + rt) * N, d_model), dtype=f32, device=dev),
         "dW_router": torch.empty((Nh, Ne, dh), dtype=f32, device=dev),
         "dW1": torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev),
         "dW3": None if W3 is None else torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev),
         "dW2": torch.empty((Nh, Ne, dh, dff), dtype=f32, device=dev),
         "dW_out": torch.empty((d_model, N), dtype=f32, device=dev)}
    wsp, wsn = _ws(workspace, MHLMOE_OP_LATENT_BACKWARD, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_latent_layer_backward(
        _dev(x, "x"), _dev(W_in, "W_in", x.dtype, ((1 + rt) * N, d_model)),
        _dev(W_router, "W_router", f32, (Nh, Ne, dh)),
        _dev(W1, "W1", x.dtype, (Nh, Ne, dff, dh)), _dev(W3, "W3", x.dtype, (Nh, Ne, dff, dh)),
        _dev(W2, "W2", x.dtype, (Nh, Ne, dh, dff)), _dev(W_out, "W_out", x.dtype, (d_model, N)),
        _dev(X_lat, "X_lat", x.dtype, (T, Nh, dh)),
        _dev(R_lat, "R_lat", x.dtype, (T, Nh, dh)) if rt else None,
        _dev(Y_lat, "Y_lat", x.dtype, (T, Nh, dh)), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", f32, (T, Nh, k)), _dev(dout, "dout", x.dtype, (T, d_model)),
        T, d_model, Nh, dh, Ne, k, dff, rt, dt,
        _dev(g["dx"], "dx"), _dev(g["dW_in"], "dW_in"), _dev(g["dW_router"], "dW_router"),
        _dev(g["dW1"], "dW1"), _dev(g["dW3"], "dW3"), _dev(g["dW2"], "dW2"),
        _dev(g["dW_out"], "dW_out"), wsp, wsn, _stream(stream)))
    return g


def mhlmoe_bias_update(counts, bias, rate: float, *, stream=None):
    """Aux-free load balancing (Sec. 2.2): bias += rate * sign(mean - count),
    per head, in place on the GPU.  Returns bias."""
    Nh, Ne = counts.shape
    _check(load_library().mhlmoe_bias_update(
        _dev(counts, "counts", torch.int32, (Nh, Ne)), _dev(bias, "bias", torch.float32, (Nh, Ne)),
        Nh, Ne, float(rate), _stream(stream)))
    return bias


def mhlmoe_layer_gelu_backward(X, W_router, W_in, W_out, idx, gate, dY, *, dX=None,
                               dW_router=None, dW_in=None, dW_out=None, workspace=None,
                               stream=None):
    """Backward of mhlmoe_layer_gelu: returns (dX, dW_router, dW_in, dW_out)."""
    T, Nh, dh = X.shape
    k = idx.shape[2]
    Ne, dff = W_in.shape[1], W_in.shape[2]
    dt = _dtype_code(X)
    dev = X.device
    f32 = torch.float32
    dX = dX if dX is not None else torch.empty_like(X)
    dW_router = dW_router if dW_router is not None else torch.empty((Nh, Ne, dh), dtype=f32, device=dev)
    dW_in = dW_in if dW_in is not None else torch.empty((Nh, Ne, dff, dh), dtype=f32, device=dev)
    dW_out = dW_out if dW_out is not None else torch.empty((Nh, Ne, dh, dff), dtype=f32, device=dev)
    wsp, wsn = _ws(workspace, MHLMOE_OP_LAYER_BACKWARD, T, Nh, dh, Ne, k, dff, dt)
    _check(load_library().mhlmoe_layer_gelu_backward(
        _dev(X, "X"), _dev(W_router, "W_router", f32, (Nh, Ne, dh)),
        _dev(W_in, "W_in", X.dtype, (Nh, Ne, dff, dh)),
        _dev(W_out, "W_out", X.dtype, (Nh, Ne, dh, dff)), _dev(idx, "idx", torch.int32, (T, Nh, k)),
        _dev(gate, "gate", f32, (T, Nh, k)), _dev(dY, "dY", X.dtype, (T, Nh, dh)),
        T, Nh, dh, Ne, k, dff, dt, _dev(dX, "dX", X.dtype, (T, Nh, dh)),
        _dev(dW_router, "dW_router", f32, (Nh, Ne, dh)),
        _dev(dW_in, "dW_in", f32, (Nh, Ne, dff, dh)), _dev(dW_out, "dW_out", f32, (Nh, Ne, dh, dff)),
        wsp, wsn, _stream(stream)))
    return dX, dW_router, dW_in, dW_out


# The operators around the heads.  Their tensors must all be on one GPU, and
# the call is enqueued there: on `stream`, or on that GPU's current stream.

E4M3 = torch.float8_e4m3fn


def _at(t, name, dtype, shape, device):
    """Address of a contiguous tensor on `device` (None -> NULL); the small
    calls' time is the host's, so everything is looked at once."""
    if t is None:
        return None
    try:
        if (t.dtype is dtype and t.shape == shape and t.get_device() == device and device >= 0
                and t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        pass
    _dev(t, name, dtype, shape)  # says what is wrong, but for the device's number
    raise ValueError(f"{name} is on {t.device}: all tensors must be on one GPU")


def _launch(device, stream, fn, *args):
    """fn(*args, stream) with GPU number `device` as the current one."""
    if stream is not None and getattr(stream, "device_index", device) != device:
        raise ValueError(f"stream is on GPU {stream.device_index}, the tensors are on {device}")
    if device == torch.cuda.current_device():
        s = torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)
        _check(fn(*args, s))
        return
    with torch.cuda.device(device):
        _check(fn(*args, _stream(stream)))


def _int(v, name):
    """v, where the C ABI takes an int: ctypes would pass on its low 32 bits."""
    if not -(1 << 31) <= v < 1 << 31:
        raise ValueError(f"{name} must fit 32 bits (got {v})")
    return v


def _rows_cols(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions (got {t.dim()})")
    return t.shape


def _new(t, shape, dtype, like, stream):
    """t, or a new tensor that belongs to the stream of the call, as one made
    under torch.cuda.stream does: its memory goes back to that stream's work,
    also where the caller drops it at once."""
    if t is not None:
        return t
    if stream is None or not like.is_cuda:
        return torch.empty(shape, dtype=dtype, device=like.device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(stream).value or 0, like.device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def mhlmoe_rmsnorm(x, weight, eps, *, residual=None, quantized=False, sum=None, y=None, q=None,
                   scales=None, stream=None):
    """h = x + residual and its RMS norm.  x [T, d_model]; weight [d_model]
    float.  quantized: the norm in 8 bits (q e4m3 and scales per 128 columns)
    instead of y; pass y as well to have both.  Returns a dict with sum (with
    residual), y, q and scales."""
    T, d = shape = _rows_cols(x, "x")
    _int(d, "d_model")
    dt, dtype, dev, f32 = _dtype_code(x), x.dtype, x.get_device(), torch.float32
    grid = (T, -(-d // 128))
    if residual is not None:
        sum = _new(sum, shape, dtype, x, stream)
    if quantized:
        q = _new(q, shape, E4M3, x, stream)
        scales = _new(scales, grid, f32, x, stream)
    else:
        if q is not None or scales is not None:
            raise ValueError("q and scales are outputs of quantized=True")
        y = _new(y, shape, dtype, x, stream)
    _launch(dev, stream, load_library().mhlmoe_rmsnorm, _at(x, "x", dtype, shape, dev),
            _at(residual, "residual", dtype, shape, dev), _at(weight, "weight", f32, (d,), dev), T, d,
            eps, dt, _at(sum, "sum", dtype, shape, dev), _at(y, "y", dtype, shape, dev),
            _at(q, "q", E4M3, shape, dev), _at(scales, "scales", f32, grid, dev))
    res = {}
    if sum is not None:
        res["sum"] = sum
    if y is not None:
        res["y"] = y
    if quantized:
        res["q"], res["scales"] = q, scales
    return res


def mhlmoe_rmsnorm_backward_workspace(T: int, d_model: int) -> int:
    """Workspace bytes of mhlmoe_rmsnorm_backward."""
    out = _SZ(0)
    _check(load_library().mhlmoe_rmsnorm_backward_workspace(T, _int(d_model, "d_model"),
                                                            ctypes.byref(out)))
    return out.value


def mhlmoe_rmsnorm_backward(h, weight, eps, dy, *, dsum=None, dx=None, dweight=None,
                            workspace=None, stream=None):
    """Backward of mhlmoe_rmsnorm from h, the forward's sum (x where there was
    no residual): returns (dx, dweight).  dsum: the gradient that reaches h
    past the norm; dx is the gradient of x and of residual."""
    T, d = shape = _rows_cols(h, "h")
    _int(d, "d_model")
    dt, dtype, dev, f32 = _dtype_code(h), h.dtype, h.get_device(), torch.float32
    dx = _new(dx, shape, dtype, h, stream)
    dweight = _new(dweight, (d,), f32, h, stream)
    if workspace is None:
        n = mhlmoe_rmsnorm_backward_workspace(T, d)
        workspace = _new(None, (max(n, 256),), torch.uint8, h, stream)
    _launch(dev, stream, load_library().mhlmoe_rmsnorm_backward, _at(h, "h", dtype, shape, dev),
            _at(weight, "weight", f32, (d,), dev), _at(dy, "dy", dtype, shape, dev),
            _at(dsum, "dsum", dtype, shape, dev), T, d, eps, dt, _at(dx, "dx", dtype, shape, dev),
            _at(dweight, "dweight", f32, (d,), dev),
            _at(workspace, "workspace", torch.uint8, (workspace.numel(),), dev), workspace.numel())
    return dx, dweight


def mhlmoe_quantize(x, *, block_rows=1, transpose=False, q=None, scales=None, stream=None):
    """x [rows, cols] in 8 bits with a scale per block_rows (1 or 128) x 128
    block; with transpose, x's transpose, its rows padded with zeros to a
    multiple of 16.  Returns (q, scales)."""
    rows, cols = _rows_cols(x, "x")
    dt, dev, f32 = _dtype_code(x), x.get_device(), torch.float32
    _int(block_rows, "block_rows")
    a, k = shape = (cols, -(-rows // 16) * 16) if transpose else (rows, cols)
    grid = (-(-a // block_rows) if block_rows in (1, 128) else a, -(-k // 128))
    q = _new(q, shape, E4M3, x, stream)
    scales = _new(scales, grid, f32, x, stream)
    _launch(dev, stream, load_library().mhlmoe_quantize, _at(x, "x", x.dtype, x.shape, dev), rows,
            cols, dt, block_rows, 1 if transpose else 0, _at(q, "q", E4M3, shape, dev),
            _at(scales, "scales", f32, grid, dev))
    return q, scales


def mhlmoe_gemm_scaled(A, scale_a, B, scale_b, *, b_block_rows=128, dtype=torch.bfloat16, C=None,
                       stream=None):
    """C [M, N] (dtype) = A [M, K] B [N, K]^T of e4m3 operands with scales per
    block of 128 along K: scale_a [M, KB], scale_b [ceil(N / b_block_rows), KB].
    float32 results are sums in fp32; bfloat16 ones lose, of products in a group
    of eight, what lies below 2^-13 of the largest."""
    M, K = _rows_cols(A, "A")
    N = _rows_cols(B, "B")[0]
    KB, dev, f32 = -(-K // 128), A.get_device(), torch.float32
    _int(b_block_rows, "b_block_rows")
    nb = -(-N // b_block_rows) if b_block_rows in (1, 128) else N
    C = _new(C, (M, N), dtype, A, stream)
    _launch(dev, stream, load_library().mhlmoe_gemm_scaled, _at(A, "A", E4M3, A.shape, dev),
            _at(scale_a, "scale_a", f32, (M, KB), dev), _at(B, "B", E4M3, (N, K), dev),
            _at(scale_b, "scale_b", f32, (nb, KB), dev), M, N, K, b_block_rows, _dtype_code(C),
            _at(C, "C", dtype, (M, N), dev))
    return C


def mhlmoe_latent_layer_scaled_workspace(T: int, d_model: int, n_heads: int, d_head: int,
                                         n_experts: int, top_k: int, d_ff: int,
                                         dtype: int = MHLMOE_BF16) -> int:
    """Workspace bytes of mhlmoe_latent_layer_scaled."""
    out = _SZ(0)
    shape = dict(d_model=d_model, n_heads=n_heads, d_head=d_head, n_experts=n_experts,
                 top_k=top_k, d_ff=d_ff)
    _check(load_library().mhlmoe_latent_layer_scaled_workspace(
        T, *(_int(v, name) for name, v in shape.items()), dtype, ctypes.byref(out)))
    return out.value


def mhlmoe_latent_layer_scaled(x, norm_weight, eps, W_in, scale_in, W_router, bias, W1, W3, W2,
                               W_out, scale_out, n_heads, top_k, *, residual=None, W_r=None,
                               scale_r=None, out=None, sum=None, X_lat=None, R_lat=None,
                               Y_lat=None, idx=None, gate=None, counts=None, workspace=None,
                               stream=None):
    """The latent layer behind its norm, with its projections in 8 bits (W_in
    [N, d_model], W_out [d_model, N] and, for separate routing sub-tokens, W_r
    [N, d_model]: e4m3 with scales per 128 x 128 tile).  Returns a dict with
    out, sum (with residual), X_lat, R_lat (with W_r), Y_lat, idx, gate,
    counts."""
    T, dm = _rows_cols(x, "x")
    Ne, dff, dh = W1.shape[1], W1.shape[2], W1.shape[3]
    Nh, N = n_heads, n_heads * dh
    for v, name in ((dm, "d_model"), (Nh, "n_heads"), (Ne, "n_experts"), (top_k, "top_k"),
                    (dff, "d_ff"), (dh, "d_head")):
        _int(v, name)
    dt, dtype, dev = _dtype_code(x), x.dtype, x.get_device()
    f32, i32 = torch.float32, torch.int32
    out = _new(out, (T, dm), dtype, x, stream)
    if residual is not None:
        sum = _new(sum, (T, dm), dtype, x, stream)
    X_lat = _new(X_lat, (T, Nh, dh), dtype, x, stream)
    if W_r is not None:
        R_lat = _new(R_lat, (T, Nh, dh), dtype, x, stream)
    Y_lat = _new(Y_lat, (T, Nh, dh), dtype, x, stream)
    idx = _new(idx, (T, Nh, top_k), i32, x, stream)
    gate = _new(gate, (T, Nh, top_k), f32, x, stream)
    counts = _new(counts, (Nh, Ne), i32, x, stream)
    if workspace is None:
        n = mhlmoe_latent_layer_scaled_workspace(T, dm, Nh, dh, Ne, top_k, dff, dt)
        workspace = _new(None, (max(n, 256),), torch.uint8, x, stream)
    grid = (-(-N // 128), -(-dm // 128))

    def at(t, name, dtype, *shape):
        return _at(t, name, dtype, shape, dev)

    _launch(dev, stream, load_library().mhlmoe_latent_layer_scaled,
            at(x, "x", dtype, T, dm), at(residual, "residual", dtype, T, dm),
            at(norm_weight, "norm_weight", f32, dm), eps,
            at(W_in, "W_in", E4M3, N, dm), at(scale_in, "scale_in", f32, *grid),
            at(W_r, "W_r", E4M3, N, dm), at(scale_r, "scale_r", f32, *grid),
            at(W_router, "W_router", f32, Nh, Ne, dh), at(bias, "bias", f32, Nh, Ne),
            at(W1, "W1", dtype, Nh, Ne, dff, dh), at(W3, "W3", dtype, Nh, Ne, dff, dh),
            at(W2, "W2", dtype, Nh, Ne, dh, dff), at(W_out, "W_out", E4M3, dm, N),
            at(scale_out, "scale_out", f32, *grid[::-1]), T, dm, Nh, dh, Ne, top_k, dff, dt,
            at(out, "out", dtype, T, dm), at(sum, "sum", dtype, T, dm),
            at(X_lat, "X_lat", dtype, T, Nh, dh), at(R_lat, "R_lat", dtype, T, Nh, dh),
            at(Y_lat, "Y_lat", dtype, T, Nh, dh), at(idx, "idx", i32, T, Nh, top_k),
            at(gate, "gate", f32, T, Nh, top_k), at(counts, "counts", i32, Nh, Ne),
            at(workspace, "workspace", torch.uint8, workspace.numel()), workspace.numel())
    res = {"out": out, "X_lat": X_lat, "Y_lat": Y_lat, "idx": idx, "gate": gate, "counts": counts}
    if residual is not None:
        res["sum"] = sum
    if W_r is not None:
        res["R_lat"] = R_lat
    return res


# What a training step has around the layer besides.  Devices and streams as above.

def mhlmoe_layernorm(x, weight, eps, *, bias=None, residual=None, quantized=False, sum=None, y=None,
                     q=None, scales=None, stream=None):
    """h = x + residual and its layer norm.  x [T, d_model]; weight and bias
    [d_model] float.  quantized: the norm in 8 bits (q e4m3 and scales per 128
    columns) instead of y; pass y as well to have both.  Returns a dict with sum
    (with residual), y, q and scales."""
    T, d = shape = _rows_cols(x, "x")
    _int(d, "d_model")
    dt, dtype, dev, f32 = _dtype_code(x), x.dtype, x.get_device(), torch.float32
    grid = (T, -(-d // 128))
    if residual is not None:
        sum = _new(sum, shape, dtype, x, stream)
    if quantized:
        q = _new(q, shape, E4M3, x, stream)
        scales = _new(scales, grid, f32, x, stream)
    else:
        if q is not None or scales is not None:
            raise ValueError("q and scales are outputs of quantized=True")
        y = _new(y, shape, dtype, x, stream)
    _launch(dev, stream, load_library().mhlmoe_layernorm, _at(x, "x", dtype, shape, dev),
            _at(residual, "residual", dtype, shape, dev), _at(weight, "weight", f32, (d,), dev),
            _at(bias, "bias", f32, (d,), dev), T, d, eps, dt, _at(sum, "sum", dtype, shape, dev),
            _at(y, "y", dtype, shape, dev), _at(q, "q", E4M3, shape, dev),
            _at(scales, "scales", f32, grid, dev))
    res = {}
    if sum is not None:
        res["sum"] = sum
    if y is not None:
        res["y"] = y
    if quantized:
        res["q"], res["scales"] = q, scales
    return res


def mhlmoe_layernorm_backward_workspace(T: int, d_model: int) -> int:
    """Workspace bytes of mhlmoe_layernorm_backward."""
    out = _SZ(0)
    _check(load_library().mhlmoe_layernorm_backward_workspace(T, _int(d_model, "d_model"),
                                                              ctypes.byref(out)))
    return out.value


def mhlmoe_layernorm_backward(h, weight, eps, dy, *, dsum=None, dx=None, dweight=None, dbias=None,
                              workspace=None, stream=None):
    """Backward of mhlmoe_layernorm from h, the forward's sum (x where there was
    no residual): returns (dx, dweight, dbias).  dsum: the gradient that reaches h
    past the norm; dx is the gradient of x and of residual."""
    T, d = shape = _rows_cols(h, "h")
    _int(d, "d_model")
    dt, dtype, dev, f32 = _dtype_code(h), h.dtype, h.get_device(), torch.float32
    dx = _new(dx, shape, dtype, h, stream)
    dweight = _new(dweight, (d,), f32, h, stream)
    dbias = _new(dbias, (d,), f32, h, stream)
    if workspace is None:
        n = mhlmoe_layernorm_backward_workspace(T, d)
        workspace = _new(None, (max(n, 256),), torch.uint8, h, stream)
    _launch(dev, stream, load_library().mhlmoe_layernorm_backward, _at(h, "h", dtype, shape, dev),
            _at(weight, "weight", f32, (d,), dev), _at(dy, "dy", dtype, shape, dev),
            _at(dsum, "dsum", dtype, shape, dev), T, d, eps, dt, _at(dx, "dx", dtype, shape, dev),
            _at(dweight, "dweight", f32, (d,), dev), _at(dbias, "dbias", f32, (d,), dev),
            _at(workspace, "workspace", torch.uint8, (workspace.numel(),), dev), workspace.numel())
    return dx, dweight, dbias


def _mask(mask, T, device):
    """Address of a mask [T] of truth values (None -> NULL)."""
    return _at(mask, "mask", torch.bool, (T,), device)


def _tokens_heads(t, name):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dim() != 3:
        raise ValueError(f"{name} must have 3 dimensions (got {t.dim()})")
    return t.shape


def mhlmoe_expert_counts(idx, n_experts, *, mask=None, counts=None, stream=None):
    """How often each head's experts are in idx [T, Nh, k], over the tokens of mask
    ([T] bool; None: all): returns counts [Nh, Ne] int32."""
    T, Nh, k = shape = _tokens_heads(idx, "idx")
    _int(n_experts, "n_experts")
    dev, i32 = idx.get_device(), torch.int32
    if n_experts < 1:
        raise ValueError(f"n_experts must be >= 1 (got {n_experts})")
    counts = _new(counts, (Nh, n_experts), i32, idx, stream)
    _launch(dev, stream, load_library().mhlmoe_expert_counts, _at(idx, "idx", i32, shape, dev),
            _mask(mask, T, dev), T, Nh, n_experts, k,
            _at(counts, "counts", i32, (Nh, n_experts), dev))
    return counts


def mhlmoe_balance_loss_workspace(T: int, n_heads: int, d_head: int, n_experts: int) -> int:
    """Workspace bytes of mhlmoe_balance_loss."""
    out = _SZ(0)
    _check(load_library().mhlmoe_balance_loss_workspace(
        T, _int(n_heads, "n_heads"), _int(d_head, "d_head"), _int(n_experts, "n_experts"),
        ctypes.byref(out)))
    return out.value


def mhlmoe_balance_loss(X, W_router, counts, *, mask=None, loss=None, stats=None, workspace=None,
                        stream=None):
    """The loss that balances the experts: X [T, Nh, dh], counts [Nh, Ne] as
    mhlmoe_expert_counts gives them.  Returns (loss [Nh], stats [T + 1, Nh, 2]),
    the latter for mhlmoe_balance_loss_backward."""
    T, Nh, dh = shape = _tokens_heads(X, "X")
    Ne = _rows_cols(counts, "counts")[1]
    dt, dev, f32 = _dtype_code(X), X.get_device(), torch.float32
    loss = _new(loss, (Nh,), f32, X, stream)
    stats = _new(stats, (T + 1, Nh, 2), f32, X, stream)
    if workspace is None:
        n = mhlmoe_balance_loss_workspace(T, Nh, dh, Ne)
        workspace = _new(None, (max(n, 256),), torch.uint8, X, stream)
    _launch(dev, stream, load_library().mhlmoe_balance_loss, _at(X, "X", X.dtype, shape, dev),
            _at(W_router, "W_router", f32, (Nh, Ne, dh), dev),
            _at(counts, "counts", torch.int32, (Nh, Ne), dev), _mask(mask, T, dev), T, Nh, dh, Ne, dt,
            _at(loss, "loss", f32, (Nh,), dev), _at(stats, "stats", f32, (T + 1, Nh, 2), dev),
            _at(workspace, "workspace", torch.uint8, (workspace.numel(),), dev), workspace.numel())
    return loss, stats


def mhlmoe_balance_loss_backward_workspace(T: int, n_heads: int, d_head: int,
                                           n_experts: int) -> int:
    """Workspace bytes of mhlmoe_balance_loss_backward."""
    out = _SZ(0)
    _check(load_library().mhlmoe_balance_loss_backward_workspace(
        T, _int(n_heads, "n_heads"), _int(d_head, "d_head"), _int(n_experts, "n_experts"),
        ctypes.byref(out)))
    return out.value


def mhlmoe_balance_loss_backward(X, W_router, counts, stats, dloss, *, mask=None, dX_add=None,
                                 dW_add=None, dX=None, dW_router=None, workspace=None, stream=None):
    """Backward of mhlmoe_balance_loss from its stats and dloss [Nh]: returns (dX,
    dW_router), added to the gradients dX_add and dW_add (the layer's, say), which
    they may replace."""
    T, Nh, dh = shape = _tokens_heads(X, "X")
    Ne = _rows_cols(counts, "counts")[1]
    dt, dtype, dev, f32 = _dtype_code(X), X.dtype, X.get_device(), torch.float32
    dX = _new(dX, shape, dtype, X, stream)
    dW_router = _new(dW_router, (Nh, Ne, dh), f32, X, stream)
    if workspace is None:
        n = mhlmoe_balance_loss_backward_workspace(T, Nh, dh, Ne)
        workspace = _new(None, (max(n, 256),), torch.uint8, X, stream)
    w = (Nh, Ne, dh)
    _launch(dev, stream, load_library().mhlmoe_balance_loss_backward, _at(X, "X", dtype, shape, dev),
            _at(W_router, "W_router", f32, w, dev),
            _at(counts, "counts", torch.int32, (Nh, Ne), dev),
            _at(stats, "stats", f32, (T + 1, Nh, 2), dev), _at(dloss, "dloss", f32, (Nh,), dev),
            _mask(mask, T, dev), _at(dX_add, "dX_add", dtype, shape, dev),
            _at(dW_add, "dW_add", f32, w, dev), T, Nh, dh, Ne, dt, _at(dX, "dX", dtype, shape, dev),
            _at(dW_router, "dW_router", f32, w, dev),
            _at(workspace, "workspace", torch.uint8, (workspace.numel(),), dev), workspace.numel())
    return dX, dW_router


class AdamWTensors:
    """The tensors of mhlmoe_adamw, looked over once and kept for every step.

    tensors: a list of dicts with the tensors param (float32 or bfloat16), grad
    (float32 or bfloat16), m and v (float32, or float8_e4m3fn together with m_scale
    and v_scale [ceil(n / 128)] float32, where v is the root of v), all of one
    shape, and, with a bfloat16 param, master (float32) if there is one; and the
    numbers weight_decay (0 if left out) and seed (of the 8-bit states' rounding;
    the tensor's place in the list if left out).  The memory that they have now is what
    every step reads and writes, also after a tensor was given other memory (.data)
    or let go: it is held here, and a new gradient tensor needs a new AdamWTensors."""

    _KEYS = {"param", "master", "grad", "m", "v", "m_scale", "v_scale", "weight_decay", "seed"}

    def __init__(self, tensors):
        # aliases, which keep the memory
        self.tensors = [{k: v.detach() if isinstance(v, torch.Tensor) else v for k, v in t.items()}
                        for t in tensors]
        self.array = (_AdamWTensor * max(len(self.tensors), 1))()
        self.device = None
        f32 = torch.float32
        for i, (t, c) in enumerate(zip(self.tensors, self.array)):
            unknown = set(t) - self._KEYS
            if unknown:
                raise ValueError(f"tensor {i}: unknown {', '.join(sorted(unknown))}")
            for name in ("param", "grad", "m", "v"):
                if not isinstance(t.get(name), torch.Tensor):
                    raise TypeError(f"tensor {i}: {name} must be a torch.Tensor")
            param, scaled = t["param"], t.get("m_scale") is not None
            dev, shape, n = param.get_device(), param.shape, param.numel()
            if self.device is None:
                self.device = dev
            state = E4M3 if scaled else f32
            grid = (-(-n // 128),)
            c.param_dtype, c.grad_dtype = _dtype_code(param), _dtype_code(t["grad"])
            for name, dtype, dims in (
                    ("param", param.dtype, shape), ("master", f32, shape),
                    ("grad", t["grad"].dtype, shape), ("m", state, shape), ("v", state, shape),
                    ("m_scale", f32, grid), ("v_scale", f32, grid)):
                setattr(c, name, _at(t.get(name), f"tensor {i}: {name}", dtype, dims, self.device))
            c.n = n
            c.weight_decay = t.get("weight_decay", 0.0)
            seed = t.get("seed", i)
            if not 0 <= seed < 1 << 32:
                raise ValueError(f"tensor {i}: seed must fit 32 bits (got {seed})")
            c.seed = seed


def mhlmoe_adamw(tensors, lr, *, beta1=0.9, beta2=0.999, eps=1e-8, step, grad_scale=None,
                 stream=None):
    """One AdamW step, the step-th from 1, over tensors: an AdamWTensors, or a list
    of what it takes.  grad_scale: [1] float32 on the GPU that the gradients are
    multiplied with (of clipping by their norm, say).  Everything is updated in
    place; lr and step are numbers of the host, which a captured call repeats."""
    if not isinstance(tensors, AdamWTensors):
        tensors = AdamWTensors(tensors)
    n = len(tensors.tensors)
    if n == 0:
        return
    dev = tensors.device
    s = _AdamWStep(lr, beta1, beta2, eps, step,
                   _at(grad_scale, "grad_scale", torch.float32, (1,), dev))
    _launch(dev, stream, load_library().mhlmoe_adamw, ctypes.addressof(tensors.array), n,
            ctypes.addressof(s))


def mhlmoe_timing_enable(on: bool = True) -> None:
    _check(load_library().mhlmoe_timing_enable(1 if on else 0))


def mhlmoe_timing_query(kernel: str):
    """(total_ms, launches) recorded for `kernel` since the last reset."""
    ms = ctypes.c_double(0.0)
    n = _I64(0)
    _check(load_library().mhlmoe_timing_query(kernel.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value


def mhlmoe_timing_reset() -> None:
    _check(load_library().mhlmoe_timing_reset())
