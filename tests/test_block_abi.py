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
        (dict(dscale=-1.0), EINVAL, b"scale"), (dict(scale=9e-101), EINVAL, b"scale"),
        (dict(dscale=1.1e100), EINVAL, b"scale"), (dict(z=None), EINVAL, b"target"), (dict(x=None), EINVAL, b"tokens"),
        (dict(u=None), EINVAL, b"uniform"), (dict(out=None), EINVAL, b"out"), (dict(count=None), EINVAL, b"count"),
        (dict(lp=None), EINVAL, b"logprob"), (dict(zs=999), EINVAL, b"stride"), (dict(ds=1), EINVAL, b"stride"),
        (dict(zs=1 << 41), EINVAL, b"stride"), (dict(z=A + 1), EALIGN, b"aligned"), (dict(x=A + 4), EALIGN, b"aligned"),
        (dict(out=A + 4), EALIGN, b"aligned"), (dict(lp=A + 2), EALIGN, b"aligned"), (dict(lengths=A + 2), EALIGN, b"aligned"),
        (dict(dtype=F32, z=A + 2), EALIGN, b"aligned"), (dict(ws=None), EINVAL, b"workspace"),
        (dict(wsb=size - 1), EINVAL, b"workspace"), (dict(ws=A + 64), EALIGN, b"workspace")))


def test_lowp_linear_validation(L):
    good = dict(dtype=MX, codes=A, scales=A, inv=1.0, rows=64, cols=128, x=A, xs=128, tokens=4, bd=F32, bias=A, act=2,
                times=A, ts=64, res=A, rs=64, yd=BF16, y=A + 4096, ys=64, stream=None)
    assert L.pulse_lowp_linear(*{**good, **dict(tokens=0, x=None, y=None, codes=None, times=None, res=None)}.values()) == OK
    refused(L.pulse_lowp_linear, good, L, (
        (dict(dtype=9), EINVAL, b"dtype"), (dict(yd=FP8), EINVAL, b"y_dtype"), (dict(rows=0), EINVAL, b"weight of"),
        (dict(cols=1 << 31), EINVAL, b"weight of"), (dict(tokens=(1 << 20) + 1), EINVAL, b"tokens"),
        (dict(codes=None), EINVAL, b"codes"), (dict(scales=None), EINVAL, b"scales"), (dict(codes=A + 2), EALIGN, b"codes"),
        (dict(dtype=FP8, inv=0.0), EINVAL, b"inv_scale"), (dict(dtype=FP8, inv=NAN), EINVAL, b"inv_scale"),
        (dict(x=None), EINVAL, b"x is NULL"), (dict(xs=100), EINVAL, b"x stride"), (dict(y=None), EINVAL, b"y is NULL"),
        (dict(ys=63), EINVAL, b"y stride"), (dict(bd=0), EINVAL, b"bias_dtype"), (dict(bias=A + 4), EALIGN, b"bias"),
        (dict(act=5), EINVAL, b"activation"), (dict(act=-1), EINVAL, b"activation"), (dict(ts=3), EINVAL, b"times stride"),
        (dict(rs=3), EINVAL, b"residual stride"), (dict(times=A + 8), EALIGN, b"times"), (dict(res=A + 2), EALIGN, b"residual"),
        (dict(y=A, ys=72), EINVAL, b"another stride")))


def test_linear_validation(L):
    need = L.pulse_linear_workspace_bytes
    top = 1 << 20
    assert need(0, 64, 128) == 0
    for sizes in ((1, 0, 8), (1, 8, 0), (top + 1, 8, 8), (1, top + 1, 8), (1, 8, top + 1), (0xFFFFFFFF,) * 3):
        assert need(*sizes) == 0, sizes
    for sizes in ((1, 1, 1), (top, 1, 1), (1, top, 1), (1, 1, top), (top, top, top), (4096, 18944, 3584)):
        assert need(*sizes) > 0, sizes
    size = need(100, 64, 128)
    good = dict(x=A, xs=128, w=A, tokens=100, rows=64, cols=128, bd=BF16, bias=A, act=1, times=A, ts=64, res=A, rs=64,
                yd=F32, y=A + (1 << 16), ys=64, pre=A, ps=64, ws=A, wsb=size, stream=None)
    assert L.pulse_linear_forward(*{**good, **dict(tokens=0, x=None, w=None, y=None, ws=None, wsb=0)}.values()) == OK
    shared = ((dict(rows=0), EINVAL, b"weight of"), (dict(cols=top + 1), EINVAL, b"weight of"),
              (dict(tokens=top + 1), EINVAL, b"tokens"), (dict(x=None), EINVAL, b"x is NULL"), (dict(xs=9), EINVAL, b"x stride"),
              (dict(w=None), EINVAL, b"weight is NULL"), (dict(w=A + 8), EALIGN, b"weight"), (dict(ws=None), EINVAL, b"workspace"),
              (dict(ws=A + 8), EALIGN, b"workspace"), (dict(wsb=64), EINVAL, b"workspace"),
              (dict(act=7), EINVAL, b"activation"), (dict(times=A + 4), EALIGN, b"times"), (dict(ts=1), EINVAL, b"times stride"))
    refused(L.pulse_linear_forward, good, L, shared + (
        (dict(yd=0), EINVAL, b"y_dtype"), (dict(y=None), EINVAL, b"y is NULL"), (dict(ys=8), EINVAL, b"y stride"),
        (dict(bd=1), EINVAL, b"bias_dtype"), (dict(res=A + 4), EALIGN, b"residual"), (dict(pre=A + 8), EALIGN, b"pre"),
        (dict(ps=63), EINVAL, b"pre stride"), (dict(y=A, ys=65), EINVAL, b"another stride")))
    good = dict(dtype=BF16, dy=A, dys=64, x=A, xs=128, w=A, pre=A, ps=64, act=2, times=A, ts=64, tokens=100, rows=64,
                cols=128, dx=A, dxs=128, dw=A, db=A, dt=A, dts=64, ws=A, wsb=size, stream=None)
    refused(L.pulse_linear_backward, good, L, shared + (
        (dict(dtype=1), EINVAL, b"dtype"), (dict(dy=None), EINVAL, b"dy is NULL"), (dict(dys=3), EINVAL, b"dy stride"),
        (dict(pre=None), EINVAL, b"pre is NULL"), (dict(pre=None, act=0), EINVAL, b"pre is NULL"),
        (dict(times=None, ts=0), EINVAL, b"dtimes without"), (dict(dts=3), EINVAL, b"dtimes stride"),
        (dict(dx=None), EINVAL, b"dx is NULL"), (dict(dxs=1), EINVAL, b"dx stride"), (dict(dw=None), EINVAL, b"dweight"),
        (dict(dw=A + 2), EALIGN, b"dweight"), (dict(db=A + 2), EALIGN, b"dbias")))


def test_linear_workspace_serves_fewer_tokens(L):
    """What a call asks for is within the workspace of any larger number of tokens."""
    for rows, cols in ((64, 128), (1003, 203), (18944, 3584), (3584, 18944), (64, 64), (1, 1), (7, 27648)):
        for most in (40, 700, 9000):
            size = L.pulse_linear_workspace_bytes(most, rows, cols)
            for tokens in range(33, most + 1, max(1, most // 50)):
                # a wrong pointer at the end: the workspace is looked at before
                rc = L.pulse_linear_forward(A, cols, A, tokens, rows, cols, 0, None, 0, None, 0, None, 0, BF16, None,
                                            rows, None, 0, A, size, None)
                assert rc == EINVAL and b"y is NULL" in L.pulse_last_error(), (rows, cols, most, tokens, L.pulse_last_error())


def test_linear_workspace_of_padded_sums(L):
    """8,191 columns are padded to 8,192, which may be split in 32 by 256 (8,191 in 31 at
    most): the workspace has to hold the splits that are run.  512 rows and 32 tokens: the
    padded weight and tokens, d, one chunk's sums and 32 splits' FP32 sums, 256-byte
    multiples all."""
    rows, tokens, ld = 512, 32, 8192
    least = 2 * rows * ld + 2 * tokens * ld + 2 * tokens * rows + 4 * rows + 32 * 4 * tokens * rows
    assert L.pulse_linear_workspace_bytes(tokens, rows, ld - 1) >= least

    def forward(size):  # a NULL y at the end: nothing is launched
        rc = L.pulse_linear_forward(A, ld, A, tokens, rows, ld - 1, 0, None, 0, None, 0, None, 0, BF16, None, rows, None, 0,
                                    A, size, None)
        assert rc == EINVAL
        return L.pulse_last_error()
    assert b"workspace" in forward(least - 1)
    assert b"y is NULL" in forward(least)


def test_constants(L):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pulse_head.h")).read()
    for macro, value in (("PULSE_VERIFY_MAX_DRAFTS", head.VERIFY_MAX_DRAFTS), ("PULSE_LINEAR_MAX_WIDTH", head.LINEAR_MAX_WIDTH),
                         ("PULSE_LINEAR_FEW_TOKENS", head.LINEAR_FEW_TOKENS),
                         *((f"PULSE_ACT_{(name or 'none').upper()}", v) for name, v in head.ACTIVATIONS.items())):
        assert f"#define {macro} {value}\n" in text, macro
    # up to so many tokens no workspace is asked for
    n = head.LINEAR_FEW_TOKENS
    for tokens, status in ((n, b"y is NULL"), (n + 1, b"workspace")):
        assert L.pulse_linear_forward(A, 64, A, tokens, 64, 64, 0, None, 0, None, 0, None, 0, BF16, None, 64, None, 0, None, 0,
                                      None) == EINVAL
        assert status in L.pulse_last_error()
