"""Binding of libaet_ops.so (include/aet_ops.h): a linear layer with bias, activation, dropout and
residual in its epilogue, group normalisation with an activation on channels-last maps, layer
normalisation of rows, and dropout from the counter generator, each with its gradient; values held in
microscaled 4-bit floating point, and the linear layer of such values; the orthogonalised update of
weight matrices.  Argument marshalling only, compiled
(csrc/ops/ops_torch.cpp); PyTorch supplies device memory and the stream, there is no CPU fallback.
Names follow the C entry points, whose records are here as ctypes structures too.

Tensors: one type a call, float32 or bfloat16, the last axis with stride 1, any other strides.  A
leading axis of clients may be left out everywhere (one client).  Outputs are allocated unless they
are given.  Calls enqueue on `stream`, the current stream where it is None.  Where it is another one,
outputs and workspaces are allocated on it, and tensors are kept from being given out again before both
are done with them (Tensor.record_stream); waiting for one another is the caller's (Stream.wait_stream).
Seeds are taken modulo 2^64.  Automatic differentiation does not know the calls: tensors that require a
gradient are refused while gradients are on (torch.no_grad, or detach, says that it is meant).
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import warnings
from typing import Optional, Tuple

import torch

from . import build as _build

AET_F32, AET_BF16 = 0, 1
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_U64 = (1 << 64) - 1

EXPORTS = [
    "aet_linear_workspace_bytes", "aet_linear_forward", "aet_linear_backward_workspace_bytes",
    "aet_linear_backward", "aet_group_norm_workspace_bytes", "aet_group_norm_forward",
    "aet_group_norm_backward_workspace_bytes", "aet_group_norm_backward", "aet_layer_norm_forward",
    "aet_layer_norm_backward_workspace_bytes", "aet_layer_norm_backward", "aet_orthogonalise_workspace_bytes",
    "aet_orthogonalise", "aet_mx4_quantise", "aet_mx4_dequantise",
    "aet_mx4_linear_workspace_bytes", "aet_mx4_linear_forward", "aet_mx4_linear_backward_workspace_bytes",
    "aet_mx4_linear_backward", "aet_dropout_forward",
    "aet_dropout_backward", "aet_ops_last_error",
]

_i32, _i64, _vp = C.c_int32, C.c_int64, C.c_void_p
# aet_in, aet_out: a pointer, the clients' stride, the rows'; maps: a pointer and three strides.  Their fields
# stand in the records one after another (a struct of 8-byte fields lies as its fields do).


def _mat(name):
    return [(name + "_p", _vp), (name + "_client", _i64), (name + "_row", _i64)]


def _maps(name):
    return [(name + "_p", _vp), (name + "_client", _i64), (name + "_sample", _i64), (name + "_row", _i64)]


_DROP = [("p", C.c_double), ("seed", C.c_uint64), ("first_row", _i64)]
_LINEAR = [(f, _i32) for f in ("dtype", "act", "n", "rows", "in", "out")] + _DROP
_NORM = [(f, _i32) for f in ("dtype", "act", "n", "batch", "positions", "groups", "width")]


class aet_linear(C.Structure):
    _fields_ = _LINEAR + _mat("x") + _mat("w") + _mat("bias") + _mat("residual") + _mat("y") + _mat("pre")


class aet_linear_grad(C.Structure):
    _fields_ = _LINEAR + _mat("dy") + _mat("x") + _mat("w") + _mat("pre") + _mat("dx") + _mat("dw") + _mat("db")


class aet_group_norm(C.Structure):
    _fields_ = _NORM + [("eps", C.c_float)] + _maps("x") + _mat("gamma") + _mat("beta") + _maps("y") + [
        ("mean", _vp), ("rstd", _vp)]


class aet_group_norm_grad(C.Structure):
    _fields_ = _NORM + _maps("dy") + _maps("x") + [("mean", _vp), ("rstd", _vp)] + _mat("gamma") + _mat(
        "beta") + _maps("dx") + _mat("dgamma") + _mat("dbeta")


class aet_layer_norm(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + [("eps", C.c_float)] + _mat("x") + _mat("residual") + _mat(
        "gamma") + _mat("beta") + _mat("y") + _mat("h") + [("mean", _vp), ("rstd", _vp)]


class aet_layer_norm_grad(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + _mat("dy") + _mat("x") + _mat("dh") + _mat("gamma") + [
        ("mean", _vp), ("rstd", _vp)] + _mat("dx") + _mat("dgamma") + _mat("dbeta")


class aet_orthogonal(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols", "steps")] + [(f, C.c_double) for f in ("a", "b", "c", "eps", "keep", "scale")] + _mat(
        "g") + _mat("w") + _mat("y")


class aet_mx4_values(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + _mat("x") + _mat("codes") + _mat("scales")


class aet_mx4_codes(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + _mat("codes") + _mat("scales") + _mat("y")


class aet_mx4_linear(C.Structure):
    _fields_ = _LINEAR + _mat("x") + _mat("x_scales") + _mat("w") + _mat("w_scales") + _mat("bias") + _mat("residual") + _mat("y") + _mat("pre")


class aet_mx4_linear_grad(C.Structure):
    _fields_ = _LINEAR + _mat("dy") + _mat("x") + _mat("x_scales") + _mat("w") + _mat("w_scales") + _mat("pre") + _mat("dx") + _mat("dw") + _mat("db")


class aet_dropout(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + _DROP + _mat("x") + _mat("residual") + _mat("y")


_LIB = None
_EXT = None


def load_library():
    """Load the in-tree library (building it only if it has never been built; one that is older than its sources is
    loaded with a warning)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not (os.path.exists(_build.OPS_LIB) and os.path.exists(_build.OPS_TORCH)):
        _build.build_ops()
    elif _build.needs_build_ops():
        warnings.warn(f"{os.path.basename(_build.OPS_LIB)} or its binding is older than its sources: build.build_ops() makes them anew",
                      RuntimeWarning, stacklevel=2)
    lib = C.CDLL(_build.OPS_LIB)
    for name in ("aet_linear", "aet_linear_backward", "aet_group_norm", "aet_group_norm_backward", "aet_layer_norm_backward",
                 "aet_mx4_linear", "aet_mx4_linear_backward", "aet_orthogonalise"):
        f = getattr(lib, name + "_workspace_bytes")
        f.restype, f.argtypes = C.c_size_t, [_vp]
    for name in ("aet_linear_forward", "aet_linear_backward", "aet_group_norm_forward", "aet_group_norm_backward",
                 "aet_layer_norm_backward", "aet_mx4_linear_forward", "aet_mx4_linear_backward", "aet_orthogonalise"):
        f = getattr(lib, name)
        f.restype, f.argtypes = C.c_int, [_vp, _vp, C.c_size_t, _vp]
    for name in ("aet_dropout_forward", "aet_dropout_backward", "aet_layer_norm_forward", "aet_mx4_quantise", "aet_mx4_dequantise"):
        f = getattr(lib, name)
        f.restype, f.argtypes = C.c_int, [_vp, _vp]
    lib.aet_ops_last_error.restype = C.c_char_p
    lib.aet_ops_last_error.argtypes = []
    _LIB = lib
    return lib


def _tensors():
    """The compiled marshalling of tensors (csrc/ops/ops_torch.cpp)."""
    global _EXT
    if _EXT is None:
        load_library()
        spec = importlib.util.spec_from_file_location("_ops_torch", _build.OPS_TORCH)
        _EXT = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_EXT)
    return _EXT


def _on(x: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    """The stream's handle and, where it is not the current one, what identifies it."""
    index = x.get_device()
    here = torch._C._cuda_getCurrentRawStream(index) if index >= 0 else 0
    if stream is None or stream.cuda_stream == here:
        return here, None
    return stream.cuda_stream, (stream.stream_id, stream.device_index, stream.device_type)


def _act(act: str) -> int:
    if act not in ACTS:
        raise ValueError(f"act is one of {', '.join(ACTS)}: got {act!r}")
    return ACTS[act]


def aet_linear_forward(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None, *,
                       residual: Optional[torch.Tensor] = None, act: str = "none", p: float = 0.0, seed: int = 0,
                       first_row: int = 0, keep_pre: bool = False, out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None):
    """residual + dropout(act(x w^T + bias)) and, with keep_pre, what act was given (else None).
    x: [n, rows, in] or [rows, in]; w: [n, out, in], or [out, in] for all clients; bias likewise
    [n, out] or [out]; residual and out (which may be the residual): as the result."""
    return (_EXT or _tensors()).linear_forward(x, w, bias, residual, _act(act), p, seed & _U64, first_row, keep_pre, out,
                                               *_on(x, stream))


def aet_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor] = None, *,
                        act: str = "none", p: float = 0.0, seed: int = 0, first_row: int = 0,
                        need: Tuple[bool, bool, bool] = (True, True, True), out=(None, None, None),
                        stream: Optional[torch.cuda.Stream] = None):
    """(dx, dw, db) of aet_linear_forward, None where `need` says so; dw and db have w's clients: with
    w [out, in] for several clients they are sums over them.  out: places for the three, of any strides,
    or None."""
    return (_EXT or _tensors()).linear_backward(dy, x, w, pre, _act(act), p, seed & _U64, first_row, need, out,
                                                *_on(x, stream))


def aet_group_norm_forward(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None,
                           beta: Optional[torch.Tensor] = None, *, eps: float = 1e-5, act: str = "none",
                           out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(y, mean, rstd): act of the normalised x * gamma + beta, and each group's statistics (float32).
    x: [n, batch, positions, channels] or [batch, positions, channels]; gamma, beta: [n, channels], or
    [channels] for all clients; out (which may be x): as x."""
    return (_EXT or _tensors()).group_norm_forward(x, groups, gamma, beta, eps, _act(act), out, *_on(x, stream))


def aet_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, *,
                            act: str = "none", need: Tuple[bool, bool] = (True, True), out=(None, None, None),
                            stream: Optional[torch.cuda.Stream] = None):
    """(dx, dgamma, dbeta) of aet_group_norm_forward from its inputs and statistics.  `need`: dx; dgamma and dbeta (None
    where they are not wanted, or have no parameter).  A gamma or beta for all clients gets the sum over them.  out:
    places for the three, of any strides, or None; dx may be dy."""
    return (_EXT or _tensors()).group_norm_backward(dy, x, mean, rstd, gamma, beta, _act(act), need, out, *_on(x, stream))


def aet_layer_norm_forward(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, *,
                           residual: Optional[torch.Tensor] = None, eps: float = 1e-5, out=(None, None),
                           stream: Optional[torch.cuda.Stream] = None):
    """(y, h, mean, rstd): h = x + residual (None where there is no residual), its normalised rows * gamma + beta, and each
    row's statistics (float32).  x: [n, rows, cols] or [rows, cols]; residual: as x; gamma, beta: [n, cols], or [cols] for all
    clients.  out: places for y and h, or None; either may be x or the residual."""
    return (_EXT or _tensors()).layer_norm_forward(x, gamma, beta, residual, eps, out, *_on(x, stream))


def aet_layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, *, dh: Optional[torch.Tensor] = None,
                            need: Tuple[bool, bool] = (True, True), out=(None, None, None),
                            stream: Optional[torch.cuda.Stream] = None):
    """(dx, dgamma, dbeta) of aet_layer_norm_forward, x being what it normalised (its h where it had a residual), dh what
    comes to h from behind, which is added to dx.  `need`: dx; dgamma and dbeta (made in gamma's shape: None without
    gamma).  A gamma for all clients gets the sum over them.  out: places for the three, of any strides, or None; dx may be
    dy or dh."""
    return (_EXT or _tensors()).layer_norm_backward(dy, x, mean, rstd, gamma, dh, need, out, *_on(x, stream))


def aet_orthogonalise(g: torch.Tensor, *, steps: int = 5, polynomial: Tuple[float, float, float] = (3.4445, -4.7750, 2.0315),
                      eps: float = 1e-7, w: Optional[torch.Tensor] = None, keep: float = 1.0, scale: float = 1.0,
                      out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """keep * w + scale * X (scale * X without w), X being g / (|g| + eps) after `steps` times X = a X + (b A + c A A) X, A = X X^T,
    (a, b, c) the polynomial, which takes each singular value s to a s + b s^3 + c s^5.  g: [n, rows, cols] or [rows, cols]; w and
    out, which may be w or g: as g."""
    return (_EXT or _tensors()).orthogonalise(g, steps, polynomial, eps, w, keep, scale, out, *_on(g, stream))


def _bf16(dtype: torch.dtype) -> bool:
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"dtype is torch.float32 or torch.bfloat16: got {dtype}")
    return dtype == torch.bfloat16


def aet_mx4_quantise(x: torch.Tensor, *, out=(None, None), stream: Optional[torch.cuda.Stream] = None):
    """(codes, scales), uint8, [..., ceil(cols / 2)] and [..., ceil(cols / 32)]: x, [n, rows, cols] or [rows, cols], in
    microscaled 4-bit floating point, blocks along the last axis.  out: places for the two, or None."""
    return (_EXT or _tensors()).mx4_quantise(x, out, *_on(x, stream))


def aet_mx4_dequantise(codes: torch.Tensor, scales: torch.Tensor, *, cols: Optional[int] = None, dtype: torch.dtype = torch.bfloat16,
                       out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """What codes and scales stand for.  cols: of the rows, where it is odd (else twice the bytes)."""
    return (_EXT or _tensors()).mx4_dequantise(codes, scales, cols, _bf16(dtype), out, *_on(codes, stream))


def aet_mx4_linear_forward(x: torch.Tensor, x_scales: torch.Tensor, w: torch.Tensor, w_scales: torch.Tensor,
                           bias: Optional[torch.Tensor] = None, *, cols: Optional[int] = None, residual: Optional[torch.Tensor] = None,
                           act: str = "none", p: float = 0.0, seed: int = 0, first_row: int = 0, keep_pre: bool = False,
                           dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None):
    """aet_linear_forward where x and w are held in 4 bits (aet_mx4_quantise's codes and scales).  cols: of x and w, where
    it is odd; dtype: of bias, residual, and the result."""
    return (_EXT or _tensors()).mx4_linear_forward(x, x_scales, w, w_scales, bias, cols, residual, _act(act), p, seed & _U64, first_row,
                                                   keep_pre, _bf16(dtype), out, *_on(x, stream))


def aet_mx4_linear_backward(dy: torch.Tensor, x: torch.Tensor, x_scales: torch.Tensor, w: torch.Tensor, w_scales: torch.Tensor,
                            pre: Optional[torch.Tensor] = None, *, cols: Optional[int] = None, act: str = "none", p: float = 0.0,
                            seed: int = 0, first_row: int = 0, need: Tuple[bool, bool, bool] = (True, True, True),
                            out=(None, None, None), stream: Optional[torch.cuda.Stream] = None):
    """(dx, dw, db) of aet_mx4_linear_forward with regard to what the codes stand for, in dy's type, as
    aet_linear_backward has them."""
    return (_EXT or _tensors()).mx4_linear_backward(dy, x, x_scales, w, w_scales, pre, cols, _act(act), p, seed & _U64, first_row, need, out,
                                                    *_on(dy, stream))


def aet_dropout_forward(x: torch.Tensor, *, p: float, seed: int, first_row: int = 0,
                        residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """residual + dropout(x).  x: [n, rows, cols] or [rows, cols]; out may be x or the residual."""
    return (_EXT or _tensors()).dropout(False, x, p, seed & _U64, first_row, residual, out, *_on(x, stream))


def aet_dropout_backward(dy: torch.Tensor, *, p: float, seed: int, first_row: int = 0,
                         out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The gradient of x: the forward call's mask and scale on dy; out may be dy."""
    return (_EXT or _tensors()).dropout(True, dy, p, seed & _U64, first_row, None, out, *_on(dy, stream))
