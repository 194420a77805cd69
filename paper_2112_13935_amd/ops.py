"""Thin ctypes binding of libaet_ops.so (include/aet_ops.h): a linear layer with bias, activation,
dropout and residual in its epilogue, group normalisation with an activation on channels-last maps,
and dropout from the counter generator, each with its gradient.  Argument marshalling only; PyTorch
supplies device memory and the stream, there is no CPU fallback.  Names follow the C entry points.

Tensors: one type a call, float32 or bfloat16, the last axis with stride 1, any other strides.  A
leading axis of clients may be left out everywhere (one client).  Outputs are allocated unless they
are given.  Calls enqueue on `stream`, the current stream where it is None; tensors used there are
kept from being given out again before it is done with them (Tensor.record_stream).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence, Tuple

import torch

from . import build as _build
from .binding import AET_OK, AetError

AET_F32, AET_BF16 = 0, 1
ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_DTYPES = {torch.float32: AET_F32, torch.bfloat16: AET_BF16}

EXPORTS = [
    "aet_linear_workspace_bytes", "aet_linear_forward", "aet_linear_backward_workspace_bytes",
    "aet_linear_backward", "aet_group_norm_workspace_bytes", "aet_group_norm_forward",
    "aet_group_norm_backward_workspace_bytes", "aet_group_norm_backward", "aet_dropout_forward",
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


class aet_dropout(C.Structure):
    _fields_ = [(f, _i32) for f in ("dtype", "n", "rows", "cols")] + _DROP + _mat("x") + _mat("residual") + _mat("y")


_LIB = None


def load_library():
    """Load the in-tree library (building it only if it has never been built)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(_build.OPS_LIB):
        _build.build_ops()
    lib = C.CDLL(_build.OPS_LIB)
    for name in ("aet_linear", "aet_linear_backward", "aet_group_norm", "aet_group_norm_backward"):
        f = getattr(lib, name + "_workspace_bytes")
        f.restype, f.argtypes = C.c_size_t, [_vp]
    for name in ("aet_linear_forward", "aet_linear_backward", "aet_group_norm_forward", "aet_group_norm_backward"):
        f = getattr(lib, name)
        f.restype, f.argtypes = C.c_int, [_vp, _vp, C.c_size_t, _vp]
    for name in ("aet_dropout_forward", "aet_dropout_backward"):
        f = getattr(lib, name)
        f.restype, f.argtypes = C.c_int, [_vp, _vp]
    lib.aet_ops_last_error.restype = C.c_char_p
    lib.aet_ops_last_error.argtypes = []
    _LIB = lib
    return lib


def _check(lib, rc: int):
    if rc != AET_OK:
        raise AetError(rc, lib.aet_ops_last_error().decode())


def _same(first: torch.Tensor, *others: Tuple[str, Optional[torch.Tensor], Sequence[int]]):
    """The other tensors' type and device are the first one's, their shapes as they are said to be."""
    if first.dtype not in _DTYPES or not first.is_cuda:
        raise ValueError(f"float32 or bfloat16 on a GPU is wanted, got {first.dtype} on {first.device}")
    for name, t, shape in others:
        if t is None:
            continue
        if t.dtype != first.dtype or t.device != first.device:
            raise ValueError(f"{name} is {t.dtype} on {t.device}, the others are {first.dtype} on {first.device}")
        if tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _dense_last(name: str, t: torch.Tensor):
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last axis has stride {t.stride(-1)}, 1 is wanted")


def _m(name: str, t: Optional[torch.Tensor], clients: bool):
    """Pointer and strides of a matrix per client."""
    if t is None:
        return None, 0, 0
    _dense_last(name, t)
    st = t.stride()
    return (t.data_ptr(), st[0], st[1]) if clients else (t.data_ptr(), t.shape[0] * st[0], st[0])


def _v(name: str, t: Optional[torch.Tensor]):
    """Pointer and strides of a vector per client, or of one for all."""
    if t is None:
        return None, 0, 0
    _dense_last(name, t)
    return t.data_ptr(), t.stride(0) if t.dim() == 2 else 0, 0


class _On:
    """The call's device and stream; keeps the tensors' memory while the stream uses it."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream], tensors):
        self.current = torch.cuda.current_stream(device)
        self.handle = (self.current if stream is None else stream).cuda_stream
        if self.handle != self.current.cuda_stream:
            for t in tensors:
                if t is not None:
                    t.record_stream(stream)
        self.device = device

    def call(self, fn, record, nbytes: int):
        ws = None
        if nbytes:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            if self.handle != self.current.cuda_stream:
                ws.record_stream(torch.cuda.ExternalStream(self.handle, device=self.device))
        return fn(C.addressof(record), None if ws is None else ws.data_ptr(), nbytes, self.handle)


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
    lib = load_library()
    clients = x.dim() == 3
    n, rows, inp = x.shape if clients else (1, *x.shape)
    outs = w.shape[-2]
    shape = (n, rows, outs) if clients else (rows, outs)
    per = w.dim() == 3
    _same(x, ("w", w, (n, outs, inp) if per else (outs, inp)), ("residual", residual, shape), ("out", out, shape),
          ("bias", bias, (n, outs) if bias is not None and bias.dim() == 2 else (outs,)))
    y = x.new_empty(shape) if out is None else out
    pre = x.new_empty(shape) if keep_pre else None
    _dense_last("w", w)
    a = aet_linear(_DTYPES[x.dtype], _act(act), n, rows, inp, outs, p, seed, first_row, *_m("x", x, clients),
                   w.data_ptr(), w.stride(0) if per else 0, w.stride(-2), *_v("bias", bias),
                   *_m("residual", residual, clients), *_m("out", y, clients), *_m("pre", pre, clients))
    with torch.cuda.device(x.device):
        on = _On(x.device, stream, (x, w, bias, residual, y, pre))
        _check(lib, on.call(lib.aet_linear_forward, a, lib.aet_linear_workspace_bytes(C.addressof(a))))
    return y, pre


def aet_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor] = None, *,
                        act: str = "none", p: float = 0.0, seed: int = 0, first_row: int = 0,
                        need: Tuple[bool, bool, bool] = (True, True, True),
                        stream: Optional[torch.cuda.Stream] = None):
    """(dx, dw, db) of aet_linear_forward, None where `need` says so; dw and db have w's clients: with
    w [out, in] for several clients they are sums over them."""
    lib = load_library()
    clients = x.dim() == 3
    n, rows, inp = x.shape if clients else (1, *x.shape)
    outs = w.shape[-2]
    shape = (n, rows, outs) if clients else (rows, outs)
    per = w.dim() == 3
    _same(x, ("dy", dy, shape), ("w", w, (n, outs, inp) if per else (outs, inp)), ("pre", pre, shape))
    if pre is None and act != "none":
        raise ValueError("pre, as the forward call gave it, is wanted where there is an activation")
    dx = x.new_empty(x.shape) if need[0] else None
    dw = x.new_empty(w.shape) if need[1] else None
    db = x.new_empty(w.shape[:-1]) if need[2] else None
    _dense_last("w", w)
    a = aet_linear_grad(_DTYPES[x.dtype], _act(act), n, rows, inp, outs, p, seed, first_row, *_m("dy", dy, clients),
                        *_m("x", x, clients), w.data_ptr(), w.stride(0) if per else 0, w.stride(-2),
                        *_m("pre", pre, clients), *_m("dx", dx, clients),
                        None if dw is None else dw.data_ptr(), dw.stride(0) if per and dw is not None else 0, inp,
                        *_v("db", db))
    with torch.cuda.device(x.device):
        on = _On(x.device, stream, (dy, x, w, pre, dx, dw, db))
        _check(lib, on.call(lib.aet_linear_backward, a, lib.aet_linear_backward_workspace_bytes(C.addressof(a))))
    return dx, dw, db


def _m3(name: str, t: Optional[torch.Tensor], clients: bool):
    if t is None:
        return None, 0, 0, 0
    _dense_last(name, t)
    st = t.stride()
    return (t.data_ptr(), *st[:3]) if clients else (t.data_ptr(), t.shape[0] * st[0], st[0], st[1])


def aet_group_norm_forward(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None,
                           beta: Optional[torch.Tensor] = None, *, eps: float = 1e-5, act: str = "none",
                           out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(y, mean, rstd): act of the normalised x * gamma + beta, and each group's statistics (float32).
    x: [n, batch, positions, channels] or [batch, positions, channels]; gamma, beta: [n, channels], or
    [channels] for all clients; out (which may be x): as x."""
    lib = load_library()
    clients = x.dim() == 4
    n, batch, positions, ch = x.shape if clients else (1, *x.shape)
    if groups < 1 or ch % groups:
        raise ValueError(f"{ch} channels cannot be parted into {groups} groups")
    _same(x, ("gamma", gamma, (n, ch) if gamma is not None and gamma.dim() == 2 else (ch,)),
          ("beta", beta, (n, ch) if beta is not None and beta.dim() == 2 else (ch,)), ("out", out, x.shape))
    y = x.new_empty(x.shape) if out is None else out
    stats = (n, batch, groups) if clients else (batch, groups)
    mean = torch.empty(stats, dtype=torch.float32, device=x.device)
    rstd = torch.empty(stats, dtype=torch.float32, device=x.device)
    a = aet_group_norm(_DTYPES[x.dtype], _act(act), n, batch, positions, groups, ch // groups, eps,
                       *_m3("x", x, clients), *_v("gamma", gamma), *_v("beta", beta), *_m3("out", y, clients),
                       mean.data_ptr(), rstd.data_ptr())
    with torch.cuda.device(x.device):
        on = _On(x.device, stream, (x, gamma, beta, y, mean, rstd))
        _check(lib, on.call(lib.aet_group_norm_forward, a, lib.aet_group_norm_workspace_bytes(C.addressof(a))))
    return y, mean, rstd


def aet_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, *,
                            act: str = "none", need: Tuple[bool, bool] = (True, True),
                            stream: Optional[torch.cuda.Stream] = None):
    """(dx, dgamma, dbeta) of aet_group_norm_forward from its inputs and statistics.  `need`: dx; dgamma and dbeta (None
    where they are not wanted, or have no parameter).  A gamma or beta for all clients gets the sum over them."""
    lib = load_library()
    clients = x.dim() == 4
    n, batch, positions, ch = x.shape if clients else (1, *x.shape)
    groups = mean.shape[-1]
    stats = (n, batch, groups) if clients else (batch, groups)
    if groups < 1 or ch % groups:
        raise ValueError(f"{ch} channels cannot be parted into {groups} groups")
    _same(x, ("dy", dy, x.shape), ("gamma", gamma, (n, ch) if gamma is not None and gamma.dim() == 2 else (ch,)),
          ("beta", beta, (n, ch) if beta is not None and beta.dim() == 2 else (ch,)))
    if gamma is not None and beta is not None and gamma.dim() != beta.dim():
        raise ValueError("gamma and beta: either both or none have an axis of clients")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or t.device != x.device or tuple(t.shape) != stats or not t.is_contiguous():
            raise ValueError(f"{name} has to be as the forward call gave it: float32, contiguous, {stats}")
    dx = x.new_empty(x.shape) if need[0] else None
    dgamma = x.new_empty(gamma.shape) if need[1] and gamma is not None else None
    dbeta = x.new_empty(beta.shape) if need[1] and beta is not None else None
    a = aet_group_norm_grad(_DTYPES[x.dtype], _act(act), n, batch, positions, groups, ch // groups,
                            *_m3("dy", dy, clients), *_m3("x", x, clients), mean.data_ptr(), rstd.data_ptr(),
                            *_v("gamma", gamma), *_v("beta", beta), *_m3("dx", dx, clients), *_v("dgamma", dgamma),
                            *_v("dbeta", dbeta))
    with torch.cuda.device(x.device):
        on = _On(x.device, stream, (dy, x, mean, rstd, gamma, beta, dx, dgamma, dbeta))
        _check(lib, on.call(lib.aet_group_norm_backward, a,
                            lib.aet_group_norm_backward_workspace_bytes(C.addressof(a))))
    return dx, dgamma, dbeta


def _dropout(fn: str, x, p, seed, first_row, residual, out, stream):
    lib = load_library()
    if x.dim() not in (2, 3):
        raise ValueError("[n, rows, cols] or [rows, cols] is wanted")
    clients = x.dim() == 3
    n, rows, cols = x.shape if clients else (1, *x.shape)
    _same(x, ("residual", residual, x.shape), ("out", out, x.shape))
    y = x.new_empty(x.shape) if out is None else out
    a = aet_dropout(_DTYPES[x.dtype], n, rows, cols, p, seed, first_row, *_m("x", x, clients),
                    *_m("residual", residual, clients), *_m("out", y, clients))
    with torch.cuda.device(x.device):
        on = _On(x.device, stream, (x, residual, y))
        _check(lib, getattr(lib, fn)(C.addressof(a), on.handle))
    return y


def aet_dropout_forward(x: torch.Tensor, *, p: float, seed: int, first_row: int = 0,
                        residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """residual + dropout(x).  x: [n, rows, cols] or [rows, cols]; out may be x or the residual."""
    return _dropout("aet_dropout_forward", x, p, seed, first_row, residual, out, stream)


def aet_dropout_backward(dy: torch.Tensor, *, p: float, seed: int, first_row: int = 0,
                         out: Optional[torch.Tensor] = None,
                         stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The gradient of x: the forward call's mask and scale on dy; out may be dy."""
    return _dropout("aet_dropout_backward", dy, p, seed, first_row, None, out, stream)
