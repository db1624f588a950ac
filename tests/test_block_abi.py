"""C ABI checks that need no GPU for the operators between blocks (include/pulse_head.h):
bad arguments are rejected on the host before any launch (the pointers below are never
dereferenced)."""
import os

import pytest

from paper_2602_03839_amd import head, pulse

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


def refused(call, good, L, cases):
    for change, status, word in cases:
        rc = call(*{**good, **change}.values())
        assert rc == status, (change, rc, L.pulse_last_error())
        assert word in L.pulse_last_error(), (change, L.pulse_last_error())


def test_block_norm_forward_validation(L):
    good = dict(dtype=BF16, b=A, bs=64, h=A, hs=64, scale=1.0, pd=F32, w=A, bias=A, pw=A, pb=A, gate=A, y=A, ys=64,
                ho=A + 4096, hos=64, stats=A, ss=4, rows=4, cols=64, eps=1e-6, flags=0, stream=None)
    empty = dict(rows=0, b=None, h=None, y=None, ho=None, stats=None)
    assert L.pulse_block_norm_forward(*{**good, **empty}.values()) == OK
    refused(L.pulse_block_norm_forward, good, L, (
        (dict(dtype=FP8), EINVAL, b"dtype"), (dict(pd=0), EINVAL, b"param_dtype"), (dict(flags=2), EINVAL, b"flags"),
        (dict(cols=0), EINVAL, b"columns"), (dict(cols=16385), EINVAL, b"columns"), (dict(rows=1 << 31), EINVAL, b"rows"),
        (dict(scale=NAN), EINVAL, b"residual_scale"), (dict(scale=-INF), EINVAL, b"residual_scale"),
        (dict(b=None), EINVAL, b"b is NULL"), (dict(h=None), EINVAL, b"h is NULL"), (dict(y=None), EINVAL, b"y is NULL"),
        (dict(ho=None), EINVAL, b"h_out is NULL"), (dict(w=None), EINVAL, b"weight"),
        (dict(pw=None), EINVAL, b"post_bias without"), (dict(bs=63), EINVAL, b"b stride"),
        (dict(hs=1), EINVAL, b"h stride"), (dict(ys=1 << 41), EINVAL, b"y stride"), (dict(hos=5), EINVAL, b"h_out stride"),
        (dict(ss=3), EINVAL, b"stats stride"), (dict(ho=A, hos=72), EINVAL, b"another stride"),
        (dict(eps=-1.0), EINVAL, b"eps"), (dict(eps=NAN), EINVAL, b"eps"), (dict(b=A + 2), EALIGN, b"b not"),
        (dict(h=A + 8), EALIGN, b"h not"), (dict(ho=A + 4), EALIGN, b"h_out not"), (dict(w=A + 4), EALIGN, b"weight"),
        (dict(pw=A + 4), EALIGN, b"post_weight"), (dict(pb=A + 8), EALIGN, b"post_bias"), (dict(gate=A + 2), EALIGN, b"gate"),
        (dict(bias=A + 4), EALIGN, b"bias"), (dict(stats=A + 2), EALIGN, b"stats")))


def test_block_norm_backward_validation(L):
    size = L.pulse_block_norm_workspace_bytes(64)
    assert size > 0
    good = dict(dtype=F32, dy=A, dys=64, dho=A, dhos=64, b=A, bs=64, ho=A, hos=64, scale=1.0, pd=BF16, w=A, pw=A, pb=A,
                gate=A, stats=A, ss=4, db=A, dbs=64, dh=A, dhs=64, dw=A, dbias=A, dpw=A, dpb=A, dgate=A, rows=4, cols=64,
                flags=0, ws=A, wsb=size, stream=None)
    refused(L.pulse_block_norm_backward, good, L, (
        (dict(dy=None), EINVAL, b"dy is NULL"), (dict(b=None), EINVAL, b"b is NULL"), (dict(ho=None), EINVAL, b"h_out"),
        (dict(db=None), EINVAL, b"db is NULL"), (dict(dh=None), EINVAL, b"dh is NULL"), (dict(dw=None), EINVAL, b"dweight"),
        (dict(stats=None), EINVAL, b"stats is NULL"), (dict(ss=1), EINVAL, b"stats stride"),
        (dict(pw=None, pb=None), EINVAL, b"dpost_weight"), (dict(gate=None), EINVAL, b"dgate"),
        (dict(pw=None), EINVAL, b"post_bias without"), (dict(dhos=3), EINVAL, b"dh_out stride"),
        (dict(scale=INF), EINVAL, b"residual_scale"), (dict(dys=5), EINVAL, b"dy stride"), (dict(dhs=5), EINVAL, b"dh stride"),
        (dict(ws=None), EINVAL, b"workspace"), (dict(wsb=size - 1), EINVAL, b"workspace"),
        (dict(ws=A + 16), EALIGN, b"workspace"), (dict(dgate=A + 2), EALIGN, b"gradient"),
        (dict(dy=A + 4), EALIGN, b"dy not"), (dict(dtype=7), EINVAL, b"dtype")))


def test_verify_drafts_validation(L):
    need = L.pulse_verify_drafts_workspace_bytes
    size = need(4, 3, 1000)
    assert 0 < size <= min(need(5, 3, 1000), need(4, 4, 1000), need(4, 3, 3000))
    for sizes in ((0, 3, 1000), (4, 129, 1000), (4, 3, 0), (4, 3, 1 << 31), (1 << 31, 0, 10), (0xFFFFFFFF, 128, 10)):
        assert need(*sizes) == 0, sizes
    good = dict(dtype=BF16, z=A, zs=1000, d=A, ds=1000, x=A, lengths=A, u=A, batch=4, drafts=3, vocab=1000, scale=1.0,
                dscale=1.0, out=A, count=A, lp=A, ws=A, wsb=size, stream=None)
    assert L.pulse_verify_drafts(*{**good, **dict(batch=0, z=None, x=None, u=None, out=None, count=None, lp=None, ws=None,
                                                  wsb=0)}.values()) == OK
    refused(L.pulse_verify_drafts, good, L, (
        (dict(dtype=FP8), EINVAL, b"dtype"), (dict(drafts=129), EINVAL, b"drafts"), (dict(vocab=0), EINVAL, b"vocabulary"),
        (dict(vocab=1 << 31), EINVAL, b"vocabulary"), (dict(batch=1 << 31), EINVAL, b"sequences"),
        (dict(scale=0.0), EINVAL, b"scale"), (dict(scale=INF), EINVAL, b"scale"), (dict(scale=NAN), EINVAL, b"scale"),
        (dict(dscale=-1.0), EINVAL, b"scale"), (dict(z=None), EINVAL, b"target"), (dict(x=None), EINVAL, b"tokens"),
        (dict(u=None), EINVAL, b"uniform"), (dict(out=None), EINVAL, b"out"), (dict(count=None), EINVAL, b"count"),
        (dict(lp=None), EINVAL, b"logprob"), (dict(zs=999), EINVAL, b"stride"), (dict(ds=1), EINVAL, b"stride"),
        (dict(zs=1 << 41), EINVAL, b"stride"), (dict(z=A + 1), EALIGN, b"aligned"), (dict(x=A + 4), EALIGN, b"aligned"),
        (dict(out=A + 4), EALIGN, b"aligned"), (dict(lp=A + 2), EALIGN, b"aligned"), (dict(lengths=A + 2), EALIGN, b"aligned"),
        (dict(dtype=F32, z=A + 2), EALIGN, b"aligned"), (dict(ws=None), EINVAL, b"workspace"),
        (dict(wsb=size - 1), EINVAL, b"workspace"), (dict(ws=A + 64), EALIGN, b"workspace")))
