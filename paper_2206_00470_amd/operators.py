"""Operators on gradients and on quantised tables: the global gradient norm
with clipping, and rows in microscaled 4-bit floating point.

As in ``store``, only argument marshalling happens here; the computation runs
in the HIP kernels of ``libadapm_hip.so``.
"""
from __future__ import annotations

import ctypes as C
import threading

import torch

from . import _lib
from ._lib import check, lib
from .store import _dev, _On, _pad, _rows, _type


# ---------------------------------------------------------------------------- norm and clipping
def _dense(t: torch.Tensor, device, name: str):
    if not t.is_cuda or t.device != device:
        raise TypeError(f"{name} must be CUDA tensors of one device")
    if not t.is_contiguous():
        raise TypeError(f"{name} must be contiguous")
    return t


class _Tensors:
    """Gradients and where clipped ones go, checked and marshalled."""

    def __init__(self, grads, out=None):
        grads = list(grads)
        out = grads if out is None else list(out)
        if len(out) != len(grads):
            raise ValueError("out must have one tensor per gradient")
        if not grads:
            raise ValueError("need at least one gradient")
        self.grads, self.out, self.device = grads, out, grads[0].device
        for g, o in zip(grads, out):
            _dense(g, self.device, "grads")
            _dense(o, self.device, "out")
            if o.dtype != g.dtype or o.shape != g.shape:
                raise ValueError("an output must have its gradient's type and shape")
        self.n = k = len(grads)
        self.types = (C.c_int32 * k)(*(_type(g.dtype, "grads") for g in grads))
        self.numel = (C.c_int64 * k)(*(g.numel() for g in grads))
        self.at = [g.data_ptr() for g in grads]
        self.out_at = self.at if out is grads else [o.data_ptr() for o in out]
        self.ins, self.outs = (C.c_void_p * k)(*self.at), (C.c_void_p * k)(*self.out_at)


def _buffers(count: int, device):
    """The norm, and a workspace of the call's own (a captured call keeps it)."""
    words = int(lib().ps_clip_workspace_bytes(count)) // 8
    buf = torch.empty(1 + words, dtype=torch.float64, device=device)
    return buf[:1], buf.data_ptr() + 8, 8 * words


class ClipPlan:
    """The gradients of a model as one list, for its global norm and for
    clipping by it: checked once and listed on the device, for buffers that stay
    where they are from step to step.  The plan keeps the tensors; a call after
    one was moved raises.  A program that makes its gradients anew each step
    (and so would go on clipping the old ones, which the plan holds) takes
    clip_grads.  Made before a capture; a captured call needs the plan as long
    as its graph.

    grads: contiguous CUDA tensors (float32, bfloat16, float16, mixed, of any
    size) of one device.  out: where clipped gradients go, one tensor of the
    same type and size for each (each its gradient itself, or apart from all
    others); None: in place."""

    def __init__(self, grads, out=None):
        t = _Tensors(grads, out)
        with torch.cuda.device(t.device):
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a plan copies its list and waits for it: make it before a capture")
        self.grads, self.out, self.device, self._at = t.grads, t.out, t.device, t.at
        self._out_at = t.out_at if t.out is not t.grads else None
        host = torch.empty(int(lib().ps_clip_plan_bytes(t.n, t.numel)), dtype=torch.uint8)
        apart = C.c_int64()
        check(lib().ps_clip_plan(t.n, t.ins, t.outs, t.numel, t.types, host.data_ptr(), host.numel(), C.byref(apart)))
        self._apart = apart.value
        self._list = host.to(self.device)
        torch.cuda.current_stream(self.device).synchronize()   # there for calls on every stream
        self._list_at, self._list_bytes = self._list.data_ptr(), host.numel()

    def _run(self, scaling: int, max_norm: float, stream):
        if list(map(torch.Tensor.data_ptr, self.grads)) != self._at or (
                scaling and self._out_at is not None and list(map(torch.Tensor.data_ptr, self.out)) != self._out_at):
            raise RuntimeError("a tensor of the plan has moved: make a new one")
        with _On(self.device, stream, (*self.grads, *self.out, self._list) if stream is not None else ()) as st:
            norm, ws, wsb = _buffers(1, self.device)
            check(lib().ps_clip_run(self._list_at, self._list_bytes, self._apart, scaling, max_norm, norm.data_ptr(), ws,
                                    wsb, st))
        return norm

    def norm(self, stream=None) -> torch.Tensor:
        """The global norm of the gradients, float64[1]."""
        return self._run(0, 0.0, stream)

    def clip(self, max_norm: float, stream=None) -> torch.Tensor:
        """Write the gradients, scaled by max_norm / norm where the norm is
        larger, to the outputs; returns the norm before, float64[1]."""
        return self._run(1, max_norm, stream)


def grad_norm(grads, stream=None) -> torch.Tensor:
    """The global norm of a list of gradients, float64[1] (tensors as in
    ClipPlan, which is quicker where they stay the same)."""
    t = _Tensors(grads)
    with _On(t.device, stream, t.grads) as st:
        norm, ws, wsb = _buffers(t.n, t.device)
        check(lib().ps_grad_norm(t.n, t.ins, t.numel, t.types, norm.data_ptr(), ws, wsb, st))
    return norm


def clip_grads(grads, max_norm: float, out=None, stream=None) -> torch.Tensor:
    """Clip a list of gradients by their global norm, in place or into out;
    returns the norm before, float64[1] (as ClipPlan.clip)."""
    t = _Tensors(grads, out)
    with _On(t.device, stream, (*t.grads, *t.out)) as st:
        norm, ws, wsb = _buffers(t.n, t.device)
        check(lib().ps_clip_grads(t.n, t.ins, t.outs, t.numel, t.types, max_norm, norm.data_ptr(), ws, wsb, st))
    return norm


# ---------------------------------------------------------------------------- microscaled 4-bit rows
MX_BLOCK = 32
_FLAGS = threading.Lock()   # held while a table's error flag is made (of all tables: one that held its own could not be copied)


class MX4:
    """Rows of dim values in microscaled 4-bit floating point: codes
    uint8[rows, ceil(dim/32)*16] (two to a byte, the first in the low half) and
    scales uint8[rows, ceil(dim/32)], contiguous CUDA tensors.  A read-only
    copy of a table at 4.25 bits a value; see mx4_quantize.  Where dim is no
    multiple of 32 the codes behind a row are zero (products read them)."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, dim: int):
        _dev(codes, torch.uint8, "codes")
        _dev(scales, torch.uint8, "scales")
        nb = -(-dim // MX_BLOCK)
        if codes.dim() != 2 or scales.dim() != 2 or dim < 1:
            raise ValueError("codes and scales must be [rows, ...] and dim at least 1")
        if codes.shape[0] != scales.shape[0] or scales.shape[1] != nb or codes.shape[1] != 16 * nb:
            raise ValueError(f"rows of {dim} values have {16 * nb} bytes of codes and {nb} scales")
        if codes.device != scales.device:
            raise TypeError("codes and scales must be on one device")
        self._set(codes, scales, dim)

    def _set(self, codes, scales, dim):
        self.codes, self.scales, self.dim = codes, scales, dim
        self.rows, self.device = codes.shape[0], codes.device
        self._err = None
        return self

    def _make_flag(self, stream):
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the first embed of a table makes its error flag: call it before a capture")
        with _FLAGS:
            if self._err is None:
                flag = torch.zeros(2, dtype=torch.int32, device=self.device)
                torch.cuda.current_stream(self.device).synchronize()
                self._err = flag   # seen by other threads from now on: zero for calls on every stream
        if stream is not None:
            self._err.record_stream(stream)

    def embed(self, ids: torch.Tensor, scale: float = 1.0, dtype: torch.dtype = torch.float32, pad: int | None = None,
              out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
        """Store.embed from these rows; an id outside them gives zeros and
        raises the sticky error that error() reports.  The first call waits for
        that error's flag to be cleared, and is refused during a capture."""
        _dev(ids, torch.int64, "ids")
        if ids.device != self.device:
            raise TypeError(f"ids must be on {self.device}")
        return self._lookup(ids, ids.numel(), ids.shape, scale, dtype, pad, out, stream)

    def dequantize(self, dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
        """The values of all rows, [rows, dim] of dtype."""
        return self._lookup(None, self.rows, (self.rows,), 1.0, dtype, None, out, stream)

    def _lookup(self, ids, n, shape, scale, dtype, pad, out, stream):
        with _On(self.device, stream, (self.codes, self.scales, ids, out, self._err)) as st:
            if ids is not None and self._err is None:
                self._make_flag(stream)
            ld = self.dim
            if out is None:
                out = torch.empty((*shape, ld), dtype=dtype, device=self.device)
            else:
                rows, ld = _rows(out, ld, self.device, "out")
                if rows != n:
                    raise ValueError("out must have one row per id")
            at, err = (ids.data_ptr(), self._err.data_ptr()) if ids is not None else (None, None)
            check(lib().ps_mx4_embed(self.codes.data_ptr(), self.scales.data_ptr(), self.rows, self.dim, at, n, _pad(pad),
                                     scale, _type(out.dtype, "out"), out.data_ptr(), ld, err, st))
        return out

    def error(self) -> int:
        """Synchronize, then return and clear the sticky status of embed."""
        torch.cuda.synchronize(self.device)
        if self._err is None or not int(self._err[0].item()):
            return _lib.PS_OK
        self._err.zero_()
        torch.cuda.synchronize(self.device)
        return _lib.PS_ERR_KEY_RANGE


def mx4_quantize(x: torch.Tensor, stream=None) -> MX4:
    """Quantise the rows of x ([rows, dim], float32, bfloat16 or float16, unit
    column stride; a store's value table W as it is)."""
    if x.dim() != 2:
        raise ValueError("x must be [rows, dim]")
    rows, dim = x.shape
    _, ld = _rows(x, dim, x.device, "x")
    nb = -(-dim // MX_BLOCK)
    with _On(x.device, stream, (x,)) as st:
        codes = torch.empty((rows, 16 * nb), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, nb), dtype=torch.uint8, device=x.device)
        check(lib().ps_mx4_quantize(rows, dim, _type(x.dtype, "x"), x.data_ptr(), ld, codes.data_ptr(),
                                    scales.data_ptr(), st))
    return MX4.__new__(MX4)._set(codes, scales, dim)


def mx4_product(a: MX4, b: MX4, scale: float = 1.0, dtype: torch.dtype = torch.float32,
                out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Scores of quantised queries against quantised rows, scale * a b^T as
    [a.rows, b.rows] of dtype."""
    if a.dim != b.dim:
        raise ValueError(f"rows of {a.dim} and of {b.dim} values")
    if a.device != b.device:
        raise TypeError("the operands must be on one device")
    with _On(a.device, stream, (a.codes, a.scales, b.codes, b.scales, out)) as st:
        if out is None:
            out = torch.empty((a.rows, b.rows), dtype=dtype, device=a.device)
        if tuple(out.shape) != (a.rows, b.rows):
            raise ValueError(f"out must be [{a.rows}, {b.rows}]")
        _, ld = _rows(out, b.rows, a.device, "out")
        check(lib().ps_mx4_product(a.rows, b.rows, a.dim, a.codes.data_ptr(), a.scales.data_ptr(), b.codes.data_ptr(),
                                   b.scales.data_ptr(), scale, _type(out.dtype, "out"), out.data_ptr(), ld, st))
    return out
