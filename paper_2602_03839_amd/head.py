"""ctypes binding to libpulse.so's operators at a model's output end and between its
blocks (C ABI in include/pulse_head.h).

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

import contextlib
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
VERIFY_MAX_DRAFTS = 128
LINEAR_MAX_WIDTH = 1 << 20  # of a weight's rows and columns, and tokens
LINEAR_FEW_TOKENS = 16  # up to which Linear's forward pass needs no workspace
# PULSE_ACT_*
ACTIVATIONS = {None: 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
MAX_SIZE = (1 << 31) - 1  # of a vocabulary, a weight's rows or columns, tokens

EXPORTS = ("pulse_layer_norm_workspace_bytes", "pulse_layer_norm_forward",
           "pulse_layer_norm_backward", "pulse_block_norm_workspace_bytes", "pulse_block_norm_forward",
           "pulse_block_norm_backward", "pulse_linear_ce_workspace_bytes", "pulse_linear_ce_forward",
           "pulse_linear_ce_backward", "pulse_verify_drafts_workspace_bytes", "pulse_verify_drafts",
           "pulse_lowp_matmul", "pulse_lowp_linear", "pulse_linear_workspace_bytes",
           "pulse_linear_forward", "pulse_linear_backward")

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
            sz, f64 = ctypes.c_size_t, ctypes.c_double
            L.pulse_layer_norm_workspace_bytes.argtypes = [u32]
            L.pulse_layer_norm_forward.argtypes = [i32, vp, u64, i32, vp, vp, vp, u64, vp, vp, u64,
                                                   u32, f32, u32, vp]
            L.pulse_layer_norm_backward.argtypes = [i32, vp, u64, vp, u64, i32, vp, vp, vp, vp, u64,
                                                    vp, vp, u64, u32, u32, vp, sz, vp]
            L.pulse_block_norm_workspace_bytes.argtypes = [u32]
            L.pulse_block_norm_forward.argtypes = [i32, vp, u64, vp, u64, f32, i32, vp, vp, vp, vp, vp, vp, u64,
                                                   vp, u64, vp, u64, u64, u32, f32, u32, vp]
            L.pulse_block_norm_backward.argtypes = [i32, vp, u64, vp, u64, vp, u64, vp, u64, f32, i32, vp, vp, vp,
                                                    vp, vp, u64, vp, u64, vp, u64, vp, vp, vp, vp, vp, u64, u32,
                                                    u32, vp, sz, vp]
            L.pulse_verify_drafts_workspace_bytes.argtypes = [u32, u32, u32]
            L.pulse_verify_drafts.argtypes = [i32, vp, u64, vp, u64, vp, vp, vp, u32, u32, u32, f64, f64, vp,
                                              vp, vp, vp, sz, vp]
            L.pulse_lowp_matmul.argtypes = [i32, vp, vp, f32, u32, u32, vp, u64, u32, i32, vp, u64, vp]
            L.pulse_lowp_linear.argtypes = [i32, vp, vp, f32, u32, u32, vp, u64, u32, i32, vp, i32, vp, u64, vp, u64,
                                            i32, vp, u64, vp]
            L.pulse_linear_workspace_bytes.argtypes = [u32, u32, u32]
            L.pulse_linear_forward.argtypes = [vp, u64, vp, u32, u32, u32, i32, vp, i32, vp, u64, vp, u64, i32, vp,
                                               u64, vp, u64, vp, sz, vp]
            L.pulse_linear_backward.argtypes = [i32, vp, u64, vp, u64, vp, vp, u64, i32, vp, u64, u32, u32, u32, vp,
                                                u64, vp, vp, vp, u64, vp, sz, vp]
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


def _like(t, like, stride, name, stream):
    """A matrix of `like`'s shape and type to write, as _out; `stride`: of its rows."""
    rows, cols = like.shape
    if t is None and stream is None and stride == cols:
        t = torch.empty_like(like)  # the cheapest of allocations
        return t, t.data_ptr(), cols
    return _out(t, name, cols, rows, like.dtype, like.device, stream)


def _vec(t, name, n, device, stream):
    """A float32 vector to write: the caller's, checked, or a new one; with its pointer."""
    if t is None:
        t = _new((n,), torch.float32, device, stream)
        return t, t.data_ptr()
    return t, _f32(t, name, n, device)


_NOTHING = contextlib.nullcontext()


def _on(device):
    """The device of a call's tensors as the current one, which a launch goes by."""
    return _NOTHING if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


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


class BlockNorm:
    """What joins two blocks: a block's output b is added to the residual stream h
    and the stream is normalised for the next block,

        h_out = residual_scale * h + gate * post_norm(b),    y = norm(h_out),

    in one pass.  ``weight`` and ``bias`` (may be None) are the norm's, [cols];
    ``post_weight``, ``post_bias`` those of the norm of the block's output, None for
    none; ``gate`` a factor per column, None for none.  All parameters are float32 or
    all bfloat16; activations are float32 or bfloat16 of their own.  Both norms are
    RMS norms with ``rms``, layer norms without.
    """

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, residual_scale: float = 1.0, eps: float = 1e-6,
                 rms: bool = True):
        self._dt = _dtype(weight, "weight")
        self.device, self.cols = weight.device, weight.numel()
        if not 1 <= self.cols <= NORM_MAX_COLS:
            raise PulseError(f"weight has {self.cols} elements, 1 to {NORM_MAX_COLS} are handled")
        if post_bias is not None and post_weight is None:
            raise PulseError("post_bias needs post_weight")
        self._params = [_p(t, name, dtype=weight.dtype, numel=self.cols, device=self.device, optional=k > 0)
                        for k, (t, name) in enumerate(((weight, "weight"), (bias, "bias"),
                                                       (post_weight, "post_weight"), (post_bias, "post_bias"),
                                                       (gate, "gate")))]
        self.weight, self.bias, self.post_weight, self.post_bias, self.gate = weight, bias, post_weight, post_bias, gate
        self.residual_scale, self.eps, self.rms = float(residual_scale), float(eps), bool(rms)
        self._flags, self._nstats, self._lib = (NORM_RMS, 2, lib()) if rms else (0, 4, lib())
        self._nws = int(self._lib.pulse_block_norm_workspace_bytes(self.cols))
        self.ws = None  # of the gradient: allocated by the first call that asks for one

    def __call__(self, b: torch.Tensor, h: torch.Tensor, y: Optional[torch.Tensor] = None,
                 h_out: Optional[torch.Tensor] = None, stats: Optional[torch.Tensor] = None,
                 keep_stats: bool = True, stream=None):
        """(y, h_out, stats) for b and h [rows, cols].  ``h_out`` may be h itself, which
        is then brought up to date in place.  stats, float32 [2 or 4, rows], is what the
        gradient asks for: rstd, post_rstd and, for layer norms, mean, post_mean (post:
        only with post_weight); None with ``keep_stats`` false."""
        dev, cols, dt = self.device, self.cols, _dtype(b, "b")
        pb, sb = _matrix(b, "b", cols, device=dev)
        rows = b.shape[0]
        ph, sh = _matrix(h, "h", cols, rows, b.dtype, dev)
        y, py, sy = _like(y, b, sb, "y", stream)
        if h_out is h:
            po, so = ph, sh
        else:
            h_out, po, so = _like(h_out, b, sb, "h_out", stream)
        if not keep_stats:
            stats, ps, ss = None, None, 0
        else:
            stats, ps, ss = _out(stats, "stats", rows, self._nstats, torch.float32, dev, stream)
        pw, pwb, pp, ppb, pg = self._params
        with _on(dev):
            rc = self._lib.pulse_block_norm_forward(dt, pb, sb, ph, sh, self.residual_scale, self._dt, pw, pwb, pp,
                                                    ppb, pg, py, sy, po, so, ps, ss, rows, cols, self.eps,
                                                    self._flags, _stream(stream, dev))
        if rc:
            _check(rc, "pulse_block_norm_forward")
        return y, h_out, stats

    def backward(self, dy: torch.Tensor, dh_out: Optional[torch.Tensor], b: Optional[torch.Tensor],
                 h_out: torch.Tensor, stats: torch.Tensor, db: Optional[torch.Tensor] = None,
                 dh: Optional[torch.Tensor] = None, stream=None):
        """(db, dh, dweight, dbias, dpost_weight, dpost_bias, dgate) for the upstream
        gradients of y and of h_out (None: zeros) and the forward pass's b (None will do
        with neither post norm nor gate), h_out and stats; None for a parameter that is
        not there, float32 for the others."""
        dev, cols, dt = self.device, self.cols, _dtype(h_out, "h_out")
        po, so = _matrix(h_out, "h_out", cols, device=dev)
        rows, typ = h_out.shape[0], h_out.dtype
        py, sy = _matrix(dy, "dy", cols, rows, typ, dev)
        pd, sd = (None, 0) if dh_out is None else _matrix(dh_out, "dh_out", cols, rows, typ, dev)
        if b is None and self.post_weight is None and self.gate is None:
            pb, sb = None, 0
        else:
            pb, sb = _matrix(b, "b", cols, rows, typ, dev)
        ps, ss = _matrix(stats, "stats", rows, self._nstats, torch.float32, dev)
        db, pdb, sdb = _like(db, h_out, so, "db", stream)
        dh, pdh, sdh = _like(dh, h_out, so, "dh", stream)
        if self.ws is None:
            self.ws = _new((self._nws,), torch.uint8, dev, stream)
        pw, pwb, pp, ppb, pg = self._params
        # one allocation for all parameters' gradients: a call of few rows is bound by the host
        there = [k for k, p in enumerate(self._params) if p is not None]
        sums, to = _new((len(there), cols), torch.float32, dev, stream), [None] * 5
        out, at = [None] * 5, sums.data_ptr()
        for k, g in zip(there, sums.unbind()):
            out[k], to[k] = g, at
            at += 4 * cols
        with _on(dev):
            rc = self._lib.pulse_block_norm_backward(dt, py, sy, pd, sd, pb, sb, po, so, self.residual_scale,
                                                     self._dt, pw, pp, ppb, pg, ps, ss, pdb, sdb, pdh, sdh, *to,
                                                     rows, cols, self._flags, self.ws.data_ptr(), self._nws,
                                                     _stream(stream, dev))
        if rc:
            _check(rc, "pulse_block_norm_backward")
        return (db, dh, *out)


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


class VerifyDrafts:
    """Which drafted tokens a target model keeps, and the token that follows them:
    drafts are taken while u q(x) < p(x), then one token is drawn from max(p - q, 0),
    or from p where all drafts were taken.  With p and q the softmax of logit_scale
    times the target's and draft_scale times the draft's logits, the tokens are
    distributed as the target's own.  Without drafts it samples.

    One object serves up to ``max_batch`` sequences of up to ``max_drafts`` drafts a call,
    which are ordered on one stream.  The scales are from 1e-100 to 1e100.
    """

    def __init__(self, vocab: int, max_batch: int, max_drafts: int = 0, logit_scale: float = 1.0,
                 draft_scale: Optional[float] = None, device=None):
        if not 1 <= vocab <= MAX_SIZE:
            raise PulseError(f"vocabulary of {vocab}, 1 to {MAX_SIZE} are handled")
        if not 0 <= max_drafts <= VERIFY_MAX_DRAFTS:
            raise PulseError(f"{max_drafts} drafts, 0 to {VERIFY_MAX_DRAFTS} are handled")
        if not 1 <= max_batch <= MAX_SIZE // (2 * max_drafts + 1):
            raise PulseError(f"batch of {max_batch} is out of range")
        self.vocab, self.max_batch, self.max_drafts = vocab, max_batch, max_drafts
        self.logit_scale = float(logit_scale)
        self.draft_scale = self.logit_scale if draft_scale is None else float(draft_scale)
        self._lib = lib()
        self._nws = int(self._lib.pulse_verify_drafts_workspace_bytes(max_batch, max_drafts, vocab))
        self.ws = torch.empty(self._nws, dtype=torch.uint8, device=device or "cuda")
        self.device, self._pws = self.ws.device, self.ws.data_ptr()

    def _rows(self, t, name, n, k, dtype):
        if isinstance(t, torch.Tensor) and t.dim() == 3:
            if t.shape[:2] != (n, k):
                raise PulseError(f"{name} must be [{n}, {k}, {self.vocab}], got {tuple(t.shape)}")
            try:
                t = t.view(-1, t.shape[2])
            except RuntimeError:
                raise PulseError(f"{name}'s rows must be equally far apart (strides {t.stride()})") from None
        return _matrix(t, name, self.vocab, n * k, dtype, self.device)

    def __call__(self, target: torch.Tensor, drafts: Optional[torch.Tensor], uniform: torch.Tensor,
                 draft_logits: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                 tokens: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
                 logprob: Optional[torch.Tensor] = None, stream=None):
        """(tokens, count, logprob) for B sequences of K drafts: ``target`` logits
        [B * (K + 1), V] or [B, K + 1, V], float32 or bfloat16; ``drafts`` int64 [B, K]
        (None for K = 0); ``uniform`` float32 [B, K + 1] in [0, 1), a sequence's last for
        the token that is drawn; ``draft_logits`` [B * K, V] or [B, K, V] (None: the draft
        was certain of its tokens); ``lengths`` int32 [B], the drafts a sequence has (None:
        K).  tokens, int64 [B, K + 1], holds the drafts taken, the token drawn, then -1;
        count, int32 [B], how many were taken; logprob, float32 [B, K + 1], each token's
        log p, 0 past them.  Where p is empty the token is -1, its logprob -inf."""
        dev = self.device
        if not isinstance(uniform, torch.Tensor) or uniform.dim() != 2 or uniform.shape[1] < 1:
            raise PulseError("uniform must be a tensor [batch, drafts + 1]")
        n, k = uniform.shape[0], uniform.shape[1] - 1
        if n > self.max_batch or k > self.max_drafts:
            raise PulseError(f"{n} sequences of {k} drafts, this object was built for {self.max_batch} of "
                             f"{self.max_drafts}")
        pu = _f32(uniform, "uniform", device=dev)
        dt = _dtype(target, "target")
        pt, st = self._rows(target, "target", n, k + 1, target.dtype)
        pd, sd = (None, 0) if draft_logits is None else self._rows(draft_logits, "draft_logits", n, k, target.dtype)
        px = _p(drafts, "drafts", dtype=torch.int64, numel=n * k, device=dev, optional=k == 0)
        if px and drafts.dim() == 2 and drafts.shape != (n, k):
            raise PulseError(f"drafts must be [{n}, {k}], got {tuple(drafts.shape)}")
        pl = _p(lengths, "lengths", dtype=torch.int32, numel=n, device=dev)
        if tokens is None:
            tokens = _new((n, k + 1), torch.int64, dev, stream)
            po = tokens.data_ptr()
        else:
            po = _p(tokens, "tokens", dtype=torch.int64, numel=n * (k + 1), device=dev)
        if count is None:
            count = _new((n,), torch.int32, dev, stream)
            pc = count.data_ptr()
        else:
            pc = _p(count, "count", dtype=torch.int32, numel=n, device=dev)
        if logprob is None:
            logprob = _new((n, k + 1), torch.float32, dev, stream) if stream is not None else torch.empty_like(uniform)
            pp = logprob.data_ptr()
        else:
            pp = _f32(logprob, "logprob", n * (k + 1), dev)
        with _on(dev):
            rc = self._lib.pulse_verify_drafts(dt, pt, st, pd, sd, px, pl, pu, n, k, self.vocab, self.logit_scale,
                                               self.draft_scale, po, pc, pp, self._pws, self._nws,
                                               _stream(stream, dev))
        if rc:
            _check(rc, "pulse_verify_drafts")
        return tokens, count, logprob


def _activation(name) -> int:
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise PulseError(f"activation must be one of {list(ACTIVATIONS)}, got {name!r}") from None


def linear_workspace_bytes(max_tokens: int, rows: int, cols: int) -> int:
    """What a Linear of a [rows, cols] weight and so many tokens needs, 0 for sizes that no
    call handles: the largest of several is a workspace for all of them."""
    if not all(0 <= v <= LINEAR_MAX_WIDTH for v in (max_tokens, rows, cols)):
        return 0
    return int(lib().pulse_linear_workspace_bytes(max_tokens, rows, cols))


class Linear:
    """y = act(x W^T + bias) * times + residual for a BF16 weight [rows, cols], from one
    token to many, and its gradient.

    ``weight`` may change in place between calls.  ``bias`` is [rows], float32 or
    bfloat16, or None; ``activation`` None, "relu", "silu", "gelu" or "gelu_tanh".  One
    object serves up to ``max_tokens`` tokens a call.  Its workspace is allocated by the
    first call that needs one (forward, more than LINEAR_FEW_TOKENS tokens), or given: a
    uint8 tensor of at least ``linear_workspace_bytes`` of its sizes, which objects whose
    calls are ordered on one stream may share.
    """

    def __init__(self, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 activation: Optional[str] = None, max_tokens: int = 32,
                 workspace: Optional[torch.Tensor] = None):
        if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
            raise PulseError("weight must be a tensor [rows, cols]")
        self._pw = _p(weight, "weight", dtype=torch.bfloat16, optional=False)
        self.device, (self.rows, self.cols) = weight.device, weight.shape
        if not (1 <= self.rows <= LINEAR_MAX_WIDTH and 1 <= self.cols <= LINEAR_MAX_WIDTH):
            raise PulseError(f"a weight of {self.rows} x {self.cols}, 1 to {LINEAR_MAX_WIDTH} of each are handled")
        if not 0 <= max_tokens <= LINEAR_MAX_WIDTH:
            raise PulseError(f"max_tokens {max_tokens} is out of range")
        self._act, self._bias = _activation(activation), _p(bias, "bias", numel=self.rows, device=self.device)
        self._bias_dt = 0 if bias is None else _dtype(bias, "bias")
        self.weight, self.bias, self.activation, self.max_tokens = weight, bias, activation, max_tokens
        self._lib = lib()
        self.workspace_bytes = linear_workspace_bytes(max_tokens, self.rows, self.cols)
        self.ws = workspace
        if workspace is not None:
            _p(workspace, "workspace", dtype=torch.uint8, min_numel=self.workspace_bytes, device=self.device)

    def _tokens(self, x, few, stream):
        px, sx = _matrix(x, "x", self.cols, dtype=torch.bfloat16, device=self.device)
        n = x.shape[0]
        if n > self.max_tokens:
            raise PulseError(f"{n} tokens, this object was built for {self.max_tokens}")
        if n <= few:
            return px, sx, n, None, 0
        if self.ws is None:
            self.ws = _new((self.workspace_bytes,), torch.uint8, self.device, stream)
        return px, sx, n, self.ws.data_ptr(), self.ws.numel()

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 times: Optional[torch.Tensor] = None, keep_pre: bool = False,
                 out: Optional[torch.Tensor] = None, out_dtype: torch.dtype = torch.bfloat16,
                 pre: Optional[torch.Tensor] = None, stream=None):
        """y, or (y, pre) with ``keep_pre`` (or a ``pre`` to write), for BF16 x [tokens,
        cols]: y, pre = x W^T + bias, residual and times are [tokens, rows], all float32
        or all bfloat16.  ``out`` may be the residual or the multiplier."""
        dev = self.device
        px, sx, n, pws, nws = self._tokens(x, LINEAR_FEW_TOKENS, stream)
        if out is None:
            dt, typ = _DTYPES.get(out_dtype), out_dtype
            if dt is None:
                raise PulseError(f"out_dtype must be float32 or bfloat16, got {out_dtype}")
        else:
            dt, typ = _dtype(out, "out"), out.dtype
        pt, st = (None, 0) if times is None else _matrix(times, "times", self.rows, n, typ, dev)
        pr, sr = (None, 0) if residual is None else _matrix(residual, "residual", self.rows, n, typ, dev)
        out, py, sy = _out(out, "out", self.rows, n, typ, dev, stream)
        pp, sp = None, 0
        if keep_pre or pre is not None:
            pre, pp, sp = _out(pre, "pre", self.rows, n, typ, dev, stream)
        with _on(dev):
            rc = self._lib.pulse_linear_forward(px, sx, self._pw, n, self.rows, self.cols, self._bias_dt, self._bias,
                                                self._act, pt, st, pr, sr, dt, py, sy, pp, sp, pws, nws,
                                                _stream(stream, dev))
        if rc:
            _check(rc, "pulse_linear_forward")
        return out if pp is None and pre is None else (out, pre)

    def backward(self, dy: torch.Tensor, x: torch.Tensor, pre: Optional[torch.Tensor] = None,
                 times: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                 dweight: Optional[torch.Tensor] = None, dbias: Optional[torch.Tensor] = None,
                 dtimes: Optional[torch.Tensor] = None, stream=None):
        """(dx, dweight, dbias, dtimes) for the upstream gradient dy [tokens, rows] and
        the forward pass's x, pre (needed with an activation or a multiplier) and times,
        all of dy's type but x.  dx and dweight are bfloat16, dbias float32, dtimes of
        dy's type; None where there is no bias or multiplier.  The residual's gradient is
        dy itself.  What is multiplied with weight and x, dy * times * act'(pre), keeps 16
        bits, which costs twice the products (a bfloat16 dy without a multiplier, with no
        activation or relu, once)."""
        dev = self.device
        px, sx, n, pws, nws = self._tokens(x, 0, stream)
        dt, typ = _dtype(dy, "dy"), dy.dtype
        py, sy = _matrix(dy, "dy", self.rows, n, typ, dev)
        pp, sp = None, 0
        if self._act or times is not None:
            pp, sp = _matrix(pre, "pre", self.rows, n, typ, dev)
        pt, st = (None, 0) if times is None else _matrix(times, "times", self.rows, n, typ, dev)
        dx, pdx, sdx = _out(dx, "dx", self.cols, n, torch.bfloat16, dev, stream)
        if dweight is None:
            dweight = _new((self.rows, self.cols), torch.bfloat16, dev, stream)
        pdw = _p(dweight, "dweight", dtype=torch.bfloat16, numel=self.rows * self.cols, device=dev)
        dbias, pdb = (None, None) if self.bias is None else _vec(dbias, "dbias", self.rows, dev, stream)
        pdt, sdt = None, 0
        if times is None:
            dtimes = None
        else:
            dtimes, pdt, sdt = _out(dtimes, "dtimes", self.rows, n, typ, dev, stream)
        with _on(dev):
            rc = self._lib.pulse_linear_backward(dt, py, sy, px, sx, self._pw, pp, sp, self._act, pt, st, n, self.rows,
                                                 self.cols, pdx, sdx, pdw, pdb, pdt, sdt, pws, nws,
                                                 _stream(stream, dev))
        if rc:
            _check(rc, "pulse_linear_backward")
        return dx, dweight, dbias, dtimes


class LowpLinear:
    """Products with a [rows, cols] weight that a receiver holds as MXFP4 or FP8
    codes (the tensors that ``pulse.ApplyLowpBatch`` patches in place), with what
    follows them in a block: y = act(x W^T + bias) * times + residual.

    ``bias`` is [rows], float32 or bfloat16, or None; ``activation`` None, "relu",
    "silu", "gelu" or "gelu_tanh".
    """

    def __init__(self, dtype: int, codes: torch.Tensor, scales: Optional[torch.Tensor], rows: int,
                 cols: int, inv_scale: float = 1.0, bias: Optional[torch.Tensor] = None,
                 activation: Optional[str] = None):
        if not (1 <= rows <= MAX_SIZE and 1 <= cols <= MAX_SIZE):
            raise PulseError(f"a weight of {rows} x {cols}, 1 to {MAX_SIZE} of each are handled")
        nc, ns = pulse.lowp_sizes(dtype, rows * cols)
        self._codes = _p(codes, "codes", esize=1, min_numel=nc, optional=False)
        self.device = codes.device
        self._scales = _p(scales, "scales", esize=1, min_numel=ns, device=self.device,
                          optional=dtype != pulse.MXFP4)
        self.dtype, self.rows, self.cols, self.inv_scale = dtype, rows, cols, float(inv_scale)
        self._act, self._bias = _activation(activation), _p(bias, "bias", numel=rows, device=self.device)
        self._bias_dt = 0 if bias is None else _dtype(bias, "bias")
        self.bias, self.activation = bias, activation
        self.keep, self._lib = (codes, scales), lib()

    def __call__(self, x: torch.Tensor, out: Optional[torch.Tensor] = None,
                 out_dtype: torch.dtype = torch.float32, stream=None, times: Optional[torch.Tensor] = None,
                 residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """act(x W^T + bias) * times + residual for BF16 x [tokens, cols]: [tokens,
        rows], float32 or bfloat16.  times and residual are of the same shape and type;
        ``out`` may be either of them."""
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
        if times is None and residual is None and self._bias is None and not self._act:
            rc = self._lib.pulse_lowp_matmul(self.dtype, self._codes, self._scales, self.inv_scale, self.rows,
                                             self.cols, px, sx, n, dt, py, sy, _stream(stream, dev))
            if rc:
                _check(rc, "pulse_lowp_matmul")
            return out
        pt, st = (None, 0) if times is None else _matrix(times, "times", self.rows, n, out.dtype, dev)
        pr, sr = (None, 0) if residual is None else _matrix(residual, "residual", self.rows, n, out.dtype, dev)
        with _on(dev):
            rc = self._lib.pulse_lowp_linear(self.dtype, self._codes, self._scales, self.inv_scale, self.rows,
                                             self.cols, px, sx, n, self._bias_dt, self._bias, self._act, pt, st,
                                             pr, sr, dt, py, sy, _stream(stream, dev))
        if rc:
            _check(rc, "pulse_lowp_linear")
        return out
