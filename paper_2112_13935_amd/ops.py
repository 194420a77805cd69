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
import struct
from typing import Optional, Tuple

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


def _packer(record):
    """The record's fields in its C layout, as bytes: several times faster than to fill the ctypes structure."""
    code, end = "", 0
    letters = {_i32: "i", _i64: "q", _vp: "Q", C.c_uint64: "Q", C.c_double: "d", C.c_float: "f"}
    for name, kind in record._fields_:
        field = getattr(record, name)
        code += "x" * (field.offset - end) + letters[kind]
        end = field.offset + field.size
    packer = struct.Struct("=" + code + "x" * (C.sizeof(record) - end))
    assert packer.size == C.sizeof(record)
    return packer.pack


_pack_linear, _pack_linear_grad = _packer(aet_linear), _packer(aet_linear_grad)
_pack_norm, _pack_norm_grad, _pack_dropout = _packer(aet_group_norm), _packer(aet_group_norm_grad), _packer(aet_dropout)

_U64 = (1 << 64) - 1
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


class _Call:
    """The type, device and stream of a call, by its first tensor; marshals the others, which have to agree with it."""

    __slots__ = ("dtype", "index", "code", "handle", "stream")

    def __init__(self, x: torch.Tensor, stream: Optional[torch.cuda.Stream]):
        self.dtype, self.index = x.dtype, x.get_device()
        self.code = _DTYPES.get(x.dtype, -1)
        if self.code < 0 or self.index < 0:
            raise ValueError(f"float32 or bfloat16 on a GPU is wanted, got {x.dtype} on {x.device}")
        self.stream = None
        self.handle = torch._C._cuda_getCurrentRawStream(self.index)
        if stream is not None and stream.cuda_stream != self.handle:
            self.stream, self.handle = stream, stream.cuda_stream

    def _strides(self, name: str, t: torch.Tensor, shape):
        if t.dtype is not self.dtype or t.get_device() != self.index:
            raise ValueError(f"{name} is {t.dtype} on {t.device}, the others are {self.dtype} on GPU {self.index}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        st = t.stride()
        if st[-1] != 1 and shape[-1] > 1:
            raise ValueError(f"{name}: the last axis has stride {st[-1]}, 1 is wanted")
        if self.stream is not None:   # its memory is not given out again before that stream is done with it
            t.record_stream(self.stream)
        return st

    def mat(self, name: str, t: Optional[torch.Tensor], shape):
        """Pointer and strides of a matrix per client, or of one (two axes)."""
        if t is None:
            return 0, 0, 0
        st = self._strides(name, t, shape)
        return (t.data_ptr(), st[0], st[1]) if len(st) == 3 else (t.data_ptr(), shape[0] * st[0], st[0])

    def weights(self, name: str, t: Optional[torch.Tensor], shape):
        """The same, of one for all clients where there are two axes."""
        if t is None:
            return 0, 0, 0
        st = self._strides(name, t, shape)
        return (t.data_ptr(), st[0], st[1]) if len(st) == 3 else (t.data_ptr(), 0, st[0])

    def vec(self, name: str, t: Optional[torch.Tensor], n: int, cols: int):
        """Pointer and strides of a vector per client, or of one for all."""
        if t is None:
            return 0, 0, 0
        per = t.dim() == 2
        st = self._strides(name, t, (n, cols) if per else (cols,))
        return t.data_ptr(), st[0] if per else 0, 0

    def maps(self, name: str, t: Optional[torch.Tensor], shape):
        if t is None:
            return 0, 0, 0, 0
        st = self._strides(name, t, shape)
        return (t.data_ptr(), st[0], st[1], st[2]) if len(st) == 4 else (t.data_ptr(), shape[0] * st[0], st[0], st[1])

    def new_mat(self, x: torch.Tensor, wanted: bool, shape):
        """A new matrix per client (three axes) or one (two), without gaps: it, and as mat gives it."""
        if not wanted:
            return None, (0, 0, 0)
        t = x.new_empty(shape)
        if self.stream is not None:
            t.record_stream(self.stream)
        return t, (t.data_ptr(), shape[-2] * shape[-1], shape[-1])

    def stats(self, name: str, t: torch.Tensor, shape) -> int:
        if t.dtype is not torch.float32 or t.get_device() != self.index or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} has to be as the forward call gave it: float32, contiguous, {tuple(shape)}")
        if self.stream is not None:
            t.record_stream(self.stream)
        return t.data_ptr()

    def run(self, fn, record: bytes, workspace_bytes=None):
        """fn(record, workspace, its size, stream) on the tensors' device; its workspace from workspace_bytes(record)."""
        if torch.cuda.current_device() != self.index:
            with torch.cuda.device(self.index):
                return self.run(fn, record, workspace_bytes)
        if workspace_bytes is None:
            rc = fn(record, self.handle)
        elif size := workspace_bytes(record):
            ws = torch.empty(size, dtype=torch.uint8, device=torch.device("cuda", self.index))
            if self.stream is not None:
                ws.record_stream(self.stream)
            rc = fn(record, ws.data_ptr(), size, self.handle)
        else:
            rc = fn(record, None, 0, self.handle)
        if rc != AET_OK:
            raise AetError(rc, _LIB.aet_ops_last_error().decode())


def _axes(x: torch.Tensor, most: int):
    """x's sizes with a leading axis of clients (1 where x has none)."""
    shape = x.shape
    if len(shape) == most:
        return shape
    if len(shape) != most - 1:
        raise ValueError(f"a tensor of {most - 1} or {most} axes is wanted, got {tuple(shape)}")
    return (1, *shape)


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
    lib = _LIB or load_library()
    call = _Call(x, stream)
    n, rows, inp = _axes(x, 3)
    outs, per = w.shape[-2], w.dim() == 3
    shape = (n, rows, outs) if x.dim() == 3 else (rows, outs)
    y, ym = (out, call.mat("out", out, shape)) if out is not None else call.new_mat(x, True, shape)
    pre, prem = call.new_mat(x, keep_pre, shape)
    a = _pack_linear(call.code, _act(act), n, rows, inp, outs, p, seed & _U64, first_row, *call.mat("x", x, x.shape),
                   *call.weights("w", w, (n, outs, inp) if per else (outs, inp)), *call.vec("bias", bias, n, outs),
                   *call.mat("residual", residual, shape), *ym, *prem)
    call.run(lib.aet_linear_forward, a, lib.aet_linear_workspace_bytes)
    return y, pre


def aet_linear_backward(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, pre: Optional[torch.Tensor] = None, *,
                        act: str = "none", p: float = 0.0, seed: int = 0, first_row: int = 0,
                        need: Tuple[bool, bool, bool] = (True, True, True),
                        stream: Optional[torch.cuda.Stream] = None):
    """(dx, dw, db) of aet_linear_forward, None where `need` says so; dw and db have w's clients: with
    w [out, in] for several clients they are sums over them."""
    lib = _LIB or load_library()
    call = _Call(x, stream)
    n, rows, inp = _axes(x, 3)
    outs, per = w.shape[-2], w.dim() == 3
    shape = (n, rows, outs) if x.dim() == 3 else (rows, outs)
    wshape = (n, outs, inp) if per else (outs, inp)
    if pre is None and act != "none":
        raise ValueError("pre, as the forward call gave it, is wanted where there is an activation")
    dx, dxm = call.new_mat(x, need[0], x.shape)
    dw = x.new_empty(wshape) if need[1] else None
    db = x.new_empty(wshape[:-1]) if need[2] else None
    a = _pack_linear_grad(call.code, _act(act), n, rows, inp, outs, p, seed & _U64, first_row, *call.mat("dy", dy, shape),
                        *call.mat("x", x, x.shape), *call.weights("w", w, wshape), *call.mat("pre", pre, shape),
                        *dxm, *call.weights("dw", dw, wshape), *call.vec("db", db, n, outs))
    call.run(lib.aet_linear_backward, a, lib.aet_linear_backward_workspace_bytes)
    return dx, dw, db


def aet_group_norm_forward(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None,
                           beta: Optional[torch.Tensor] = None, *, eps: float = 1e-5, act: str = "none",
                           out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
    """(y, mean, rstd): act of the normalised x * gamma + beta, and each group's statistics (float32).
    x: [n, batch, positions, channels] or [batch, positions, channels]; gamma, beta: [n, channels], or
    [channels] for all clients; out (which may be x): as x."""
    lib = _LIB or load_library()
    n, batch, positions, ch = _axes(x, 4)
    if groups < 1 or ch % groups:
        raise ValueError(f"{ch} channels cannot be parted into {groups} groups")
    call = _Call(x, stream)
    y = x.new_empty(x.shape) if out is None else out
    stats = (n, batch, groups) if x.dim() == 4 else (batch, groups)
    mean, rstd = x.new_empty(stats, dtype=torch.float32), x.new_empty(stats, dtype=torch.float32)
    a = _pack_norm(call.code, _act(act), n, batch, positions, groups, ch // groups, eps,
                       *call.maps("x", x, x.shape), *call.vec("gamma", gamma, n, ch), *call.vec("beta", beta, n, ch),
                       *call.maps("out", y, x.shape), call.stats("mean", mean, stats), call.stats("rstd", rstd, stats))
    call.run(lib.aet_group_norm_forward, a, lib.aet_group_norm_workspace_bytes)
    return y, mean, rstd


def aet_group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                            gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, *,
                            act: str = "none", need: Tuple[bool, bool] = (True, True),
                            stream: Optional[torch.cuda.Stream] = None):
    """(dx, dgamma, dbeta) of aet_group_norm_forward from its inputs and statistics.  `need`: dx; dgamma and dbeta (None
    where they are not wanted, or have no parameter).  A gamma or beta for all clients gets the sum over them."""
    lib = _LIB or load_library()
    call = _Call(x, stream)
    n, batch, positions, ch = _axes(x, 4)
    groups = mean.shape[-1]
    stats = (n, batch, groups) if x.dim() == 4 else (batch, groups)
    if groups < 1 or ch % groups:
        raise ValueError(f"{ch} channels cannot be parted into {groups} groups")
    if gamma is not None and beta is not None and gamma.dim() != beta.dim():
        raise ValueError("gamma and beta: either both or none have an axis of clients")
    dx = x.new_empty(x.shape) if need[0] else None
    dgamma = x.new_empty(gamma.shape) if need[1] and gamma is not None else None
    dbeta = x.new_empty(beta.shape) if need[1] and beta is not None else None
    a = _pack_norm_grad(call.code, _act(act), n, batch, positions, groups, ch // groups,
                            *call.maps("dy", dy, x.shape), *call.maps("x", x, x.shape),
                            call.stats("mean", mean, stats), call.stats("rstd", rstd, stats),
                            *call.vec("gamma", gamma, n, ch), *call.vec("beta", beta, n, ch),
                            *call.maps("dx", dx, x.shape), *call.vec("dgamma", dgamma, n, ch),
                            *call.vec("dbeta", dbeta, n, ch))
    call.run(lib.aet_group_norm_backward, a, lib.aet_group_norm_backward_workspace_bytes)
    return dx, dgamma, dbeta


def _dropout(fn: str, x, p, seed, first_row, residual, out, stream):
    lib = _LIB or load_library()
    call = _Call(x, stream)
    n, rows, cols = _axes(x, 3)
    y, ym = (out, call.mat("out", out, x.shape)) if out is not None else call.new_mat(x, True, x.shape)
    a = _pack_dropout(call.code, n, rows, cols, p, seed & _U64, first_row, *call.mat("x", x, x.shape),
                    *call.mat("residual", residual, x.shape), *ym)
    call.run(getattr(lib, fn), a)
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
