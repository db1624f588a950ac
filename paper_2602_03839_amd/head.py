"""ctypes binding to libpulse.so's operators at a model's output end (C ABI in
include/pulse_head.h).

Argument marshalling only, like ``pulse``: every call takes torch tensors that
already live on the GPU, passes their device pointers and the current HIP
stream to the C entry point, and raises ``pulse.PulseError`` on a non-zero
status.  A class holds what a program keeps beside its weights (the weight
itself and the call's workspace); one object's calls must be ordered on one
stream.  Matrices are two-dimensional with rows of adjacent elements; rows may
lie further apart than their length (a view's stride), weights may not.

Outputs are allocated on the stream that the call runs on unless they are given.
"""
from __future__ import annotations

import ctypes
import threading
from typing import Optional

import torch

from . import pulse
from .pulse import PulseError, _check, _f32, _p, _stream

F32, BF16 = 3, 4  # PULSE_DTYPE_F32, PULSE_DTYPE_BF16
NORM_RMS = 1      # PULSE_NORM_RMS
NORM_MAX_COLS = 16384
CE_MAX_HIDDEN = 65536
MAX_SIZE = (1 << 31) - 1  # of a vocabulary, a weight's rows or columns, tokens

EXPORTS = ("pulse_layer_norm_workspace_bytes", "pulse_layer_norm_forward",
           "pulse_layer_norm_backward", "pulse_linear_ce_workspace_bytes", "pulse_linear_ce_forward",
           "pulse_linear_ce_backward", "pulse_lowp_matmul")

_lock = threading.Lock()
_lib = None


def lib():
    """libpulse.so with this module's entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = pulse.lib()
    with _lock:
        if _lib is None:
            vp, u64, u32, f32, i32 = (ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32,
                                      ctypes.c_float, ctypes.c_int)
            sz = ctypes.c_size_t
            L.pulse_layer_norm_workspace_bytes.argtypes = [u32]
            L.pulse_layer_norm_forward.argtypes = [i32, vp, u64, i32, vp, vp, vp, u64, vp, vp, u64,
                                                   u32, f32, u32, vp]
            L.pulse_layer_norm_backward.argtypes = [i32, vp, u64, vp, u64, i32, vp, vp, vp, vp, u64,
                                                    vp, vp, u64, u32, u32, vp, sz, vp]
            L.pulse_lowp_matmul.argtypes = [i32, vp, vp, f32, u32, u32, vp, u64, u32, i32, vp, u64, vp]
            L.pulse_linear_ce_workspace_bytes.argtypes = [u32, u32, u32]
            L.pulse_linear_ce_forward.argtypes = [vp, u64, vp, vp, u32, u32, u32, f32, vp, vp, vp, sz, vp]
            L.pulse_linear_ce_backward.argtypes = [vp, u64, vp, vp, u32, u32, u32, f32, vp, vp, vp, u64,
                                                   vp, vp, sz, vp]
            for name in EXPORTS:
                getattr(L, name).restype = sz if name.endswith("_workspace_bytes") else i32
            _lib = L
    return _lib


_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


def _dtype(t: torch.Tensor, name: str) -> int:
    code = _DTYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
    if code is None:
        raise PulseError(f"{name} must be float32 or bfloat16, got {getattr(t, 'dtype', type(t).__name__)}")
    return code


def _matrix(t: torch.Tensor, name: str, cols: int, rows: Optional[int] = None, dtype=None, device=None):
    """(pointer, row stride) of a device matrix whose rows are adjacent elements."""
    # one chain of cheap tests, as in pulse._p; a failing one is named below
    if isinstance(t, torch.Tensor) and t.dim() == 2 and t.is_cuda:
        r, c = t.shape
        if (c == cols and (rows is None or r == rows) and (dtype is None or t.dtype is dtype)
                and (device is None or t.device == device)):
            if t.is_contiguous():
                return t.data_ptr(), cols
            if t.stride(1) == 1 and t.stride(0) >= cols:
                return t.data_ptr(), t.stride(0)
    if not isinstance(t, torch.Tensor):
        raise PulseError(f"{name} must be a torch.Tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise PulseError(f"{name} must be a device tensor (got {t.device})")
    if t.dim() != 2 or t.shape[1] != cols or (rows is not None and t.shape[0] != rows):
        want = f"[{'rows' if rows is None else rows}, {cols}]"
        raise PulseError(f"{name} must have the shape {want}, got {list(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise PulseError(f"{name} must be {dtype}, got {t.dtype}")
    if device is not None and t.device != device:
        raise PulseError(f"{name} is on {t.device}, the call's other tensors on {device}")
    raise PulseError(f"{name} must have rows of adjacent elements that do not overlap "
                     f"(strides {t.stride()})")


def _new(shape, dtype, device, stream):
    """An output on the stream that will write it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _out(t, name, cols, rows, dtype, device, stream):
    """A matrix to write: the caller's, checked, or a new one; with pointer and row stride."""
    if t is None:
        t = _new((rows, cols), dtype, device, stream)
        return t, t.data_ptr(), cols
    return (t, *_matrix(t, name, cols, rows, dtype, device))


def _vec(t, name, n, device, stream):
    """A float32 vector to write: the caller's, checked, or a new one; with its pointer."""
    if t is None:
        t = _new((n,), torch.float32, device, stream)
        return t, t.data_ptr()
    return t, _f32(t, name, n, device)


class LayerNorm:
    """Layer norm, or RMS norm with ``rms``, over the last axis.

    ``weight`` and ``bias`` (may be None) are [cols], both float32 or both
    bfloat16; activations are float32 or bfloat16 of their own.
    """

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, rms: bool = False):
        self._dt = _dtype(weight, "weight")
        self.device, self.cols = weight.device, weight.numel()
        self._pw = _p(weight, "weight", optional=False)
        self._pb = _p(bias, "bias", dtype=weight.dtype, numel=self.cols, device=self.device)
        if not 1 <= self.cols <= NORM_MAX_COLS:
            raise PulseError(f"weight has {self.cols} elements, 1 to {NORM_MAX_COLS} are handled")
        self.weight, self.bias, self.eps, self.rms = weight, bias, float(eps), bool(rms)
        self._flags, self._lib = NORM_RMS if rms else 0, lib()
        self._nws = int(self._lib.pulse_layer_norm_workspace_bytes(self.cols))
        self.ws = None  # of the gradient: allocated by the first call that asks for one

    def __call__(self, x: torch.Tensor, y: Optional[torch.Tensor] = None,
                 mean: Optional[torch.Tensor] = None, rstd: Optional[torch.Tensor] = None, stream=None):
        """(y, mean, rstd) of x [rows, cols]; mean is None for the RMS form."""
        dev, cols, dt = self.device, self.cols, _dtype(x, "x")
        px, sx = _matrix(x, "x", cols, device=dev)
        rows = x.shape[0]
        if y is None and stream is None and sx == cols:
            y = torch.empty_like(x)
            py, sy = y.data_ptr(), cols
        else:
            y, py, sy = _out(y, "y", cols, rows, x.dtype, dev, stream)
        mean, pm = (None, None) if self.rms else _vec(mean, "mean", rows, dev, stream)
        rstd, pr = _vec(rstd, "rstd", rows, dev, stream)
        rc = self._lib.pulse_layer_norm_forward(dt, px, sx, self._dt, self._pw, self._pb, py, sy, pm, pr,
                                                rows, cols, self.eps, self._flags, _stream(stream, dev))
        if rc:
            _check(rc, "pulse_layer_norm_forward")
        return y, mean, rstd

    def backward(self, dy: torch.Tensor, x: torch.Tensor, mean: Optional[torch.Tensor],
                 rstd: torch.Tensor, dx: Optional[torch.Tensor] = None,
                 dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                 stream=None):
        """(dx, dweight, dbias) for the upstream gradient dy and the forward
        pass's x, mean and rstd; dbias is None where there is no bias."""
        dev, cols, dt = self.device, self.cols, _dtype(x, "x")
        px, sx = _matrix(x, "x", cols, device=dev)
        rows = x.shape[0]
        pdy, sdy = _matrix(dy, "dy", cols, rows, x.dtype, dev)
        pm = None if self.rms else _f32(mean, "mean", rows, dev)
        pr = _f32(rstd, "rstd", rows, dev)
        if dx is None and stream is None and sx == cols:
            dx = torch.empty_like(x)
            pdx, sdx = dx.data_ptr(), cols
        else:
            dx, pdx, sdx = _out(dx, "dx", cols, rows, x.dtype, dev, stream)
        if self.ws is None:
            self.ws = _new((self._nws,), torch.uint8, dev, stream)
        dweight, pdw = _vec(dweight, "dweight", cols, dev, stream)
        dbias, pdb = (None, None) if self.bias is None else _vec(dbias, "dbias", cols, dev, stream)
        rc = self._lib.pulse_layer_norm_backward(dt, pdy, sdy, px, sx, self._dt, self._pw, pm, pr, pdx, sdx,
                                                 pdw, pdb, rows, cols, self._flags, self.ws.data_ptr(), self._nws,
                                                 _stream(stream, dev))
        if rc:
            _check(rc, "pulse_layer_norm_backward")
        return dx, dweight, dbias


class LinearCE:
    """Softmax cross entropy of logits = logit_scale * x weight^T that are never
    stored, per token, and its gradient.

    ``weight`` is bfloat16 [vocab, hidden] and may change in place between
    calls; the workspace serves up to ``max_tokens`` tokens a call.
    """

    def __init__(self, weight: torch.Tensor, max_tokens: int, logit_scale: float = 1.0):
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise PulseError("weight must be a tensor [vocab, hidden]")
        self.device, (self.vocab, self.hidden) = weight.device, weight.shape
        if not 1 <= self.vocab <= MAX_SIZE:
            raise PulseError(f"vocabulary of {self.vocab}, 1 to {MAX_SIZE} are handled")
        if not 1 <= self.hidden <= CE_MAX_HIDDEN:
            raise PulseError(f"hidden size {self.hidden}, 1 to {CE_MAX_HIDDEN} are handled")
        _p(weight, "weight", dtype=torch.bfloat16, optional=False)
        if not 0 <= max_tokens <= MAX_SIZE:
            raise PulseError(f"max_tokens {max_tokens} is out of range")
        self.weight, self.max_tokens, self.logit_scale = weight, max_tokens, float(logit_scale)
        self._lib, self._pw = lib(), weight.data_ptr()
        need = int(self._lib.pulse_linear_ce_workspace_bytes(max_tokens, self.vocab, self.hidden))
        self._nws = max(need, 1)
        self.ws = torch.empty(self._nws, dtype=torch.uint8, device=self.device)
        self._pws = self.ws.data_ptr()

    def _tokens(self, x, targets):
        px, sx = _matrix(x, "x", self.hidden, dtype=torch.bfloat16, device=self.device)
        n = x.shape[0]
        if n > self.max_tokens:
            raise PulseError(f"{n} tokens, this object was built for {self.max_tokens}")
        return px, sx, _p(targets, "targets", dtype=torch.int64, numel=n, device=self.device,
                          optional=False), n

    def forward(self, x: torch.Tensor, targets: torch.Tensor, loss: Optional[torch.Tensor] = None,
                lse: Optional[torch.Tensor] = None, stream=None):
        """(loss, lse), float32 [tokens], of x [tokens, hidden] and int64 targets;
        a target outside [0, vocab) is ignored and has loss 0."""
        dev = self.device
        px, sx, pt, n = self._tokens(x, targets)
        loss, pl = _vec(loss, "loss", n, dev, stream)
        lse, ps = _vec(lse, "lse", n, dev, stream)
        rc = self._lib.pulse_linear_ce_forward(px, sx, self._pw, pt, n, self.vocab, self.hidden,
                                               self.logit_scale, pl, ps, self._pws, self._nws,
                                               _stream(stream, dev))
        if rc:
            _check(rc, "pulse_linear_ce_forward")
        return loss, lse

    def backward(self, x: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor,
                 dloss: torch.Tensor, dx: Optional[torch.Tensor] = None,
                 dweight: Optional[torch.Tensor] = None, stream=None):
        """(dx, dweight), bfloat16, for the upstream gradient dloss [tokens] of
        each token's loss and the forward pass's lse."""
        dev = self.device
        px, sx, pt, n = self._tokens(x, targets)
        ps, pd = _f32(lse, "lse", n, dev), _f32(dloss, "dloss", n, dev)
        dx, pdx, sdx = _out(dx, "dx", self.hidden, n, torch.bfloat16, dev, stream)
        if dweight is None:
            dweight = _new((self.vocab, self.hidden), torch.bfloat16, dev, stream)
        pdw = _p(dweight, "dweight", dtype=torch.bfloat16, numel=self.vocab * self.hidden, device=dev,
                 optional=False)
        rc = self._lib.pulse_linear_ce_backward(px, sx, self._pw, pt, n, self.vocab, self.hidden,
                                                self.logit_scale, ps, pd, pdx, sdx, pdw, self._pws,
                                                self._nws, _stream(stream, dev))
        if rc:
            _check(rc, "pulse_linear_ce_backward")
        return dx, dweight


class LowpLinear:
    """Products with a [rows, cols] weight that a receiver holds as MXFP4 or FP8
    codes (the tensors that ``pulse.ApplyLowpBatch`` patches in place)."""

    def __init__(self, dtype: int, codes: torch.Tensor, scales: Optional[torch.Tensor], rows: int,
                 cols: int, inv_scale: float = 1.0):
        if not (1 <= rows <= MAX_SIZE and 1 <= cols <= MAX_SIZE):
            raise PulseError(f"a weight of {rows} x {cols}, 1 to {MAX_SIZE} of each are handled")
        nc, ns = pulse.lowp_sizes(dtype, rows * cols)
        self._codes = _p(codes, "codes", esize=1, min_numel=nc, optional=False)
        self.device = codes.device
        self._scales = _p(scales, "scales", esize=1, min_numel=ns, device=self.device,
                          optional=dtype != pulse.MXFP4)
        self.dtype, self.rows, self.cols, self.inv_scale = dtype, rows, cols, float(inv_scale)
        self.keep, self._lib = (codes, scales), lib()

    def __call__(self, x: torch.Tensor, out: Optional[torch.Tensor] = None,
                 out_dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
        """x W^T for BF16 x [tokens, cols]: [tokens, rows], float32 or bfloat16."""
        dev = self.device
        px, sx = _matrix(x, "x", self.cols, dtype=torch.bfloat16, device=dev)
        n = x.shape[0]
        if out is None:
            dt = _DTYPES.get(out_dtype)
            if dt is None:
                raise PulseError(f"out_dtype must be float32 or bfloat16, got {out_dtype}")
            out = _new((n, self.rows), out_dtype, dev, stream)
            py, sy = out.data_ptr(), self.rows
        else:
            dt = _dtype(out, "out")
            py, sy = _matrix(out, "out", self.rows, n, device=dev)
        rc = self._lib.pulse_lowp_matmul(self.dtype, self._codes, self._scales, self.inv_scale, self.rows,
                                         self.cols, px, sx, n, dt, py, sy, _stream(stream, dev))
        if rc:
            _check(rc, "pulse_lowp_matmul")
        return out
