"""C ABI checks of include/pulse_head.h that need no GPU: every declared function
is exported and bound, and bad arguments are rejected on the host before any
launch (the pointers below are never dereferenced)."""
import os
import re

import pytest
import torch

from paper_2602_03839_amd import head, pulse

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EALIGN = 0, -1, -3
A = 1 << 20  # fake, aligned "device" address
F32, BF16, FP8, MX, RMS = head.F32, head.BF16, pulse.FP8_E4M3, pulse.MXFP4, head.NORM_RMS
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(pulse.LIB_PATH):
        from paper_2602_03839_amd import build
        build.build()
    return head.lib()


def test_exports_every_declared_function(L):
    text = open(os.path.join(ROOT, "include", "pulse_head.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(pulse_[a-z0-9_]+)\s*\(", text))
    assert names == set(head.EXPORTS)
    for name in names:
        assert getattr(L, name).argtypes is not None, name
    for macro, value in (("PULSE_NORM_MAX_COLS", head.NORM_MAX_COLS), ("PULSE_DTYPE_F32", F32),
                         ("PULSE_DTYPE_BF16", BF16), ("PULSE_CE_MAX_HIDDEN", head.CE_MAX_HIDDEN)):
        assert re.search(rf"#define {macro} {value}\b", text), macro


def refused(rc, status, L, word):
    assert rc == status, (rc, L.pulse_last_error())
    assert word in L.pulse_last_error(), L.pulse_last_error()


def test_layer_norm_validation(L):
    good = dict(dtype=BF16, x=A, xs=64, pd=F32, w=A, b=A, y=A, ys=64, mean=A, rstd=A, rows=4, cols=64,
                eps=1e-6, flags=0, stream=None)

    def fwd(**k):
        return L.pulse_layer_norm_forward(*{**good, **k}.values())

    assert fwd(rows=0, x=None, y=None, mean=None, rstd=None) == OK
    for k, status, word in ((dict(dtype=FP8), EINVAL, b"dtype"), (dict(pd=0), EINVAL, b"param_dtype"),
                            (dict(flags=2), EINVAL, b"flags"), (dict(cols=0), EINVAL, b"columns"),
                            (dict(cols=16385, xs=20000, ys=20000), EINVAL, b"columns"),
                            (dict(rows=1 << 31), EINVAL, b"rows"), (dict(x=None), EINVAL, b"x is NULL"),
                            (dict(y=None), EINVAL, b"y is NULL"), (dict(w=None), EINVAL, b"weight"),
                            (dict(mean=None), EINVAL, b"mean"), (dict(rstd=None), EINVAL, b"rstd"),
                            (dict(xs=63), EINVAL, b"stride"), (dict(ys=1 << 41), EINVAL, b"stride"),
                            (dict(eps=-1.0), EINVAL, b"eps"), (dict(eps=NAN), EINVAL, b"eps"),
                            (dict(x=A + 8), EALIGN, b"x not"), (dict(y=A + 2), EALIGN, b"y not"),
                            (dict(w=A + 4), EALIGN, b"weight"), (dict(b=A + 4), EALIGN, b"bias"),
                            (dict(mean=A + 2), EALIGN, b"mean"), (dict(rstd=A + 1), EALIGN, b"rstd")):
        refused(fwd(**k), status, L, word)

    size = L.pulse_layer_norm_workspace_bytes(64)
    good = dict(dtype=F32, dy=A, dys=64, x=A, xs=64, pd=BF16, w=A, mean=A, rstd=A, dx=A, dxs=64, dw=A, db=A,
                rows=4, cols=64, flags=0, ws=A, wsb=size, stream=None)

    def bwd(**k):
        return L.pulse_layer_norm_backward(*{**good, **k}.values())

    for k, status, word in ((dict(dy=None), EINVAL, b"dy"), (dict(dx=None), EINVAL, b"dx"),
                            (dict(dw=None), EINVAL, b"dweight"), (dict(mean=None), EINVAL, b"mean"),
                            (dict(dys=5), EINVAL, b"dy stride"), (dict(dxs=5), EINVAL, b"dx stride"),
                            (dict(ws=None), EINVAL, b"workspace"), (dict(wsb=size - 1), EINVAL, b"workspace"),
                            (dict(ws=A + 16), EALIGN, b"workspace"), (dict(dw=A + 2), EALIGN, b"dweight"),
                            (dict(dy=A + 4), EALIGN, b"dy not"), (dict(dtype=7), EINVAL, b"dtype")):
        refused(bwd(**k), status, L, word)


def test_linear_ce_validation(L):
    assert L.pulse_linear_ce_workspace_bytes(0, 100, 64) == 0
    size = L.pulse_linear_ce_workspace_bytes(8, 100, 64)
    assert 0 < size <= L.pulse_linear_ce_workspace_bytes(9, 100, 64)
    good = dict(x=A, xs=64, w=A, y=A, tokens=8, vocab=100, hidden=64, scale=1.0, loss=A, lse=A, ws=A, wsb=size,
                stream=None)

    def fwd(**k):
        return L.pulse_linear_ce_forward(*{**good, **k}.values())

    assert fwd(tokens=0, x=None, y=None, ws=None, wsb=0) == OK
    shared = ((dict(vocab=0), EINVAL, b"vocabulary"), (dict(vocab=1 << 31), EINVAL, b"vocabulary"),
              (dict(tokens=1 << 31), EINVAL, b"tokens"), (dict(hidden=0), EINVAL, b"hidden"),
              (dict(hidden=65537), EINVAL, b"hidden"), (dict(scale=INF), EINVAL, b"logit_scale"),
              (dict(scale=NAN), EINVAL, b"logit_scale"), (dict(x=None), EINVAL, b"x is NULL"),
              (dict(xs=60), EINVAL, b"stride"), (dict(w=None), EINVAL, b"weight"), (dict(y=None), EINVAL, b"targets"),
              (dict(x=A + 8), EALIGN, b"x not"), (dict(w=A + 2), EALIGN, b"weight"), (dict(y=A + 4), EALIGN, b"targets"),
              (dict(ws=None), EINVAL, b"workspace"), (dict(wsb=size - 1), EINVAL, b"workspace"),
              (dict(ws=A + 128), EALIGN, b"workspace"))
    for k, status, word in shared + ((dict(loss=None), EINVAL, b"loss"), (dict(lse=A + 2), EALIGN, b"lse")):
        refused(fwd(**k), status, L, word)
    good = dict(x=A, xs=64, w=A, y=A, tokens=8, vocab=100, hidden=64, scale=1.0, lse=A, dloss=A, dx=A, dxs=64, dw=A,
                ws=A, wsb=size, stream=None)

    def bwd(**k):
        return L.pulse_linear_ce_backward(*{**good, **k}.values())

    for k, status, word in shared + ((dict(lse=None), EINVAL, b"lse"), (dict(dloss=A + 1), EALIGN, b"dloss"),
                                     (dict(dx=None), EINVAL, b"dx"), (dict(dxs=63), EINVAL, b"dx stride"),
                                     (dict(dw=None), EINVAL, b"dweight"), (dict(dw=A + 8), EALIGN, b"dweight")):
        refused(bwd(**k), status, L, word)


def test_linear_ce_workspace_of_sizes_out_of_range(L):
    """Sizes that every call refuses have no workspace; the largest handled ones have."""
    top = (1 << 31) - 1
    for sizes in ((1, 100, 0), (1, 100, 65537), (1, 100, 0xFFFFFFF9), (1, 100, 0xFFFFFFFF), (1, 0, 64), (1, 1 << 31, 64),
                  (1, 0xFFFFFFFF, 64), (1 << 31, 100, 64), (0xFFFFFFFF, 100, 64), (0xFFFFFFFF,) * 3):
        assert L.pulse_linear_ce_workspace_bytes(*sizes) == 0, sizes
    for sizes in ((1, top, 1), (top, 1, 1), (1, 1, 65536), (top, top, 65536)):
        assert L.pulse_linear_ce_workspace_bytes(*sizes) > 0, sizes


def test_linear_ce_workspace_serves_fewer_tokens(L):
    """The size for n tokens covers every call of fewer: each such call gets past the
    workspace check (and stops at the missing loss, before any launch)."""
    for vocab, hidden in ((1000, 64), (152064, 3584), (5003, 203), (40, 5120), (3_000_000, 128)):
        for most in (1, 64, 100, 128, 129, 300, 513, 2000, 5000, 40000):
            size = L.pulse_linear_ce_workspace_bytes(most, vocab, hidden)
            for n in {1, 2, 33, 64, 65, 127, 128, 129, 200, 511, 512, 513, 700, 1023, 1999, 3333, 4097, 20011, most}:
                if n > most:
                    continue
                rc = L.pulse_linear_ce_forward(A, hidden, A, A, n, vocab, hidden, 1.0, None, A, A, size, None)
                refused(rc, EINVAL, L, b"loss")


def test_lowp_matmul_validation(L):
    good = dict(dtype=MX, codes=A, scales=A, inv=1.0, rows=16, cols=64, x=A, xs=64, tokens=2, yd=F32, y=A, ys=16,
                stream=None)

    def f(**k):
        return L.pulse_lowp_matmul(*{**good, **k}.values())

    assert f(tokens=0, x=None, y=None) == OK
    for k, status, word in ((dict(dtype=F32), EINVAL, b"dtype"), (dict(yd=MX), EINVAL, b"y_dtype"),
                            (dict(rows=0), EINVAL, b"weight"), (dict(cols=1 << 31), EINVAL, b"weight"),
                            (dict(tokens=(1 << 20) + 1), EINVAL, b"tokens"), (dict(codes=None), EINVAL, b"codes"),
                            (dict(scales=None), EINVAL, b"scales"), (dict(codes=A + 2), EALIGN, b"codes"),
                            (dict(dtype=FP8, codes=A + 4), EALIGN, b"codes"),
                            (dict(dtype=FP8, inv=0.0), EINVAL, b"inv_scale"),
                            (dict(dtype=FP8, inv=NAN), EINVAL, b"inv_scale"), (dict(x=None), EINVAL, b"x is NULL"),
                            (dict(xs=63), EINVAL, b"x stride"), (dict(y=A + 4), EALIGN, b"y not"),
                            (dict(ys=15), EINVAL, b"y stride")):
        refused(f(**k), status, L, word)


def test_binding_rejects_host_tensors(L):
    w = torch.zeros(4, 8, dtype=torch.bfloat16)
    for call in (lambda: head.LayerNorm(torch.ones(8)), lambda: head.LinearCE(w, 4),
                 lambda: head.LowpLinear(MX, torch.zeros(16, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8), 4, 8)):
        with pytest.raises(pulse.PulseError, match="device tensor"):
            call()


def test_binding_rejects_sizes_past_32_bits():
    """Sizes that the C calls take as 32 bits: no call computes with what is left of a
    larger one.  The sizes are looked at before the tensors are."""
    byte = torch.zeros(1, dtype=torch.uint8)
    for dtype in (MX, FP8):
        for rows, cols in (((1 << 32) + 16, 1), (1, (1 << 32) + 16), (1 << 31, 1), (1, 1 << 31), (0, 64), (64, 0), (-4, -8)):
            with pytest.raises(pulse.PulseError, match="weight of"):
                head.LowpLinear(dtype, byte, byte, rows, cols)
    for shape in (((1 << 32) + 1, 1), (1 << 31, 8), (0, 8)):
        with pytest.raises(pulse.PulseError, match="vocabulary"):
            head.LinearCE(torch.empty(shape, dtype=torch.bfloat16, device="meta"), 4)
    for shape in ((8, 1 << 32), (8, 65537), (8, 0)):
        with pytest.raises(pulse.PulseError, match="hidden size"):
            head.LinearCE(torch.empty(shape, dtype=torch.bfloat16, device="meta"), 4)


def test_binding_rejects_what_is_no_tensor():
    one = torch.zeros(16, dtype=torch.uint8)
    for call in (lambda: head.LowpLinear(MX, None, one, 4, 8), lambda: head.LowpLinear(FP8, [1] * 32, None, 4, 8),
                 lambda: head.LayerNorm(None), lambda: head.LinearCE(None, 4)):
        with pytest.raises(pulse.PulseError):
            call()
