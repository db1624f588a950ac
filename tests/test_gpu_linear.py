"""Linear layers with their epilogue on the GPU, BF16 weights and receivers' codes, against
the definition in 64 bits.

Tolerances.  A product's sum: each matrix instruction adds 32 products to an FP32 sum, so
with k values at most k / 32 roundings follow each other in a wave, and some 80 more
where parts are added (16 in a block, 64 splits): (k / 32 + 80) 2^-24 of the sum of
the products' magnitudes, which for random signs is far above what occurs.  An
activation's exponential and reciprocal are good to 1 ulp, its argument v log2(e) to
half an ulp, so its relative error is at most (6 + 2 |v|) 2^-24; its slope is at most
1.13, that of its derivative below 1.  A BF16 result adds half a step, 2^-8 of it.  In
the gradient d is rounded to BF16 as well, 2^-8 of each term.  Besides, over a whole
BF16 result the roundings are independent: the root mean square of each is at most
2^-8 / sqrt 3 of the result's, of two 0.0032.
"""
import math

import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]
RMS = 2.0 ** -8 / math.sqrt(3) * math.sqrt(2)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def act64(name, v):
    """An activation and its derivative in 64 bits."""
    if name is None:
        return v, torch.ones_like(v)
    if name == "relu":
        return v.clamp(min=0), (v > 0).double()
    if name == "silu":
        s = torch.sigmoid(v)
        return v * s, s + v * s * (1 - s)
    if name == "gelu":
        c = torch.special.ndtr(v)
        return v * c, c + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
    y = math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    s = torch.sigmoid(2 * y)
    return v * s, s + v * 2 * s * (1 - s) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v * v)


def within(got, want, bound, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: off by {off[bad].max().item():.3g} at {bad.nonzero()[0].tolist()}"


def rms_within(got, want, share, what):
    if want.numel() >= 4096:
        assert (got.double() - want).norm() <= share * want.norm(), what


def product64(x, w):
    """x w^T and the sum of magnitudes."""
    x, w = x.double(), w.double()
    return x @ w.t(), x.abs() @ w.abs().t()


def forward64(x, w, bias, act, times, residual, typ):
    """y and pre, each with its bound."""
    pre, size = product64(x, w)
    err = (w.shape[1] / 32 + 80) * U * size
    if bias is not None:
        pre = pre + bias.double()
        err = err + U * pre.abs() + 2 * U * size
    a, _ = act64(act, pre)
    y, yerr = a, 1.13 * err + (0 if act is None else (6 + 2 * pre.abs()) * U * pre.abs())
    if times is not None:
        y, yerr = y * times.double(), (yerr + 2 * U * y.abs()) * times.double().abs()
    if residual is not None:
        y, yerr = y + residual.double(), yerr + 2 * U * (y.abs() + residual.double().abs())
    return y, yerr + HALF[typ] * y.abs() * 1.01 + 1e-37, pre, err + HALF[typ] * pre.abs() * 1.01 + 1e-37


def make(tokens, rows, cols, typ, seed, bias=True, times=True, residual=True, bias_type=torch.float32):
    g = gen(seed)
    x = normal(g, tokens, cols).bfloat16()
    w = (normal(g, rows, cols) / math.sqrt(cols)).bfloat16()
    return (x, w, (0.3 * normal(g, rows)).to(bias_type) if bias else None,
            normal(g, tokens, rows).to(typ) if times else None, normal(g, tokens, rows).to(typ) if residual else None,
            normal(g, tokens, rows).to(typ))


def check_forward(tokens, rows, cols, typ, seed, act, bias=True, times=True, residual=True):
    x, w, b, t, r, _ = make(tokens, rows, cols, typ, seed, bias, times, residual)
    h = head.Linear(w, b, activation=act, max_tokens=tokens)
    y, pre = h(x, residual=r, times=t, keep_pre=True, out_dtype=typ)
    ey, yerr, epre, perr = forward64(x, w, b, act, t, r, typ)
    assert y.dtype is typ and pre.dtype is typ
    within(y, ey, yerr, "y")
    within(pre, epre, perr, "pre")
    return h, x, w, b, t, r, y, pre


def check_backward(h, x, w, b, t, dy, pre, act):
    typ = dy.dtype
    needs = act is not None or t is not None
    dx, dw, db, dt = h.backward(dy, x, pre=pre if needs else None, times=t)
    a, slope = act64(act, pre.double())
    d, tt = dy.double(), 1 if t is None else t.double()
    exact = d * tt * slope
    derr = (20 + 4 * pre.double().abs()) * U * (d * tt).abs()
    rounded = needs or typ is torch.float32
    each = derr + (HALF[torch.bfloat16] * exact.abs() * 1.01 if rounded else 0)
    tokens, rows = dy.shape
    want, size = exact @ w.double(), exact.abs() @ w.double().abs()
    within(dx, want, each @ w.double().abs() + (rows / 32 + 80) * U * size + HALF[torch.bfloat16] * want.abs() * 1.01 + 1e-37,
           "dx")
    rms_within(dx, want, RMS if rounded else RMS / math.sqrt(2), "dx")
    xd = x.double()
    want, size = exact.t() @ xd, exact.abs().t() @ xd.abs()
    within(dw, want, each.t() @ xd.abs() + (tokens / 32 + 80) * U * size + HALF[torch.bfloat16] * want.abs() * 1.01 + 1e-37,
           "dweight")
    rms_within(dw, want, RMS if rounded else RMS / math.sqrt(2), "dweight")
    assert (db is None) == (b is None) and (dt is None) == (t is None)
    if b is not None:
        # chunks of tokens in a wave's turns, then the chunks' sums
        assert db.dtype is torch.float32
        within(db, exact.sum(0), derr.sum(0) + (tokens / 4 + 520) * U * exact.abs().sum(0), "dbias")
    if t is not None:
        v = pre.double().abs()
        within(dt, d * a, ((6 + 2 * v) * U * v + 2 * U * a.abs()) * d.abs() + HALF[typ] * (d * a).abs() * 1.01 + 1e-37, "dtimes")


SIZES = [
    (1, 16, 8), (1, 1, 1), (1, 3584, 3584), (2, 100, 129), (3, 64, 64), (5, 1003, 203), (8, 48, 5120), (16, 896, 4864),
    (17, 200, 640), (20, 4864, 896), (31, 77, 7), (32, 3584, 1024), (9, 130, 9216), (1, 520, 18944), (4, 33, 27648),
    (33, 128, 64), (33, 1, 1), (63, 65, 72), (64, 128, 3584), (65, 1003, 203), (100, 256, 18944), (129, 130, 8),
    (200, 896, 896), (257, 264, 136), (300, 1, 2000), (512, 64, 64), (700, 3000, 320), (1000, 7, 5), (2048, 512, 256),
    (1025, 2056, 1096), (4097, 64, 72),
]


@pytest.mark.parametrize("tokens,rows,cols", SIZES)
def test_sizes(tokens, rows, cols):
    """Every path: few tokens from slabs and by chunks, each tile, splits, padded copies."""
    for k, typ in enumerate((torch.bfloat16, torch.float32)):
        act = ACTS[(tokens + rows + cols + k) % 5]
        h, x, w, b, t, r, y, pre = check_forward(tokens, rows, cols, typ, rows + k, act)
        check_backward(h, x, w, b, t, normal(gen(9), tokens, rows).to(typ), pre, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("typ", [torch.bfloat16, torch.float32])
def test_parts_of_the_epilogue(act, typ):
    for tokens in (3, 90):
        for mask in range(8):
            bias, times, residual = mask & 1, mask & 2, mask & 4
            h, x, w, b, t, r, y, pre = check_forward(tokens, 136, 200, typ, mask, act, bias, times, residual)
            plain = h(x, residual=r, times=t, out_dtype=typ)
            assert torch.equal(plain, y)
            check_backward(h, x, w, b, t, normal(gen(9), tokens, 136).to(typ), pre, act)


@pytest.mark.parametrize("rows,cols", [(18944, 3584), (3584, 18944)])
def test_large(rows, cols):
    h, x, w, b, t, r, y, pre = check_forward(2048, rows, cols, torch.bfloat16, 1, "silu", bias=False, residual=False)
    check_backward(h, x, w, b, t, normal(gen(9), 2048, rows).bfloat16(), pre, "silu")


def test_gradient_against_differences():
    """x W^T kept small, d's and the results' roundings as everywhere: the gradient along
    random directions against central differences of the definition (step 1e-4 of the
    directions, whose own error is 1e-8), to the roundings' share of the terms."""
    tokens, rows, cols = 70, 40, 64
    for act in ACTS:
        x, w, b, t, r, _ = make(tokens, rows, cols, torch.float32, 3)
        h = head.Linear(w, b, activation=act, max_tokens=tokens)
        _, pre = h(x, residual=r, times=t, keep_pre=True, out_dtype=torch.float32)
        dy = normal(gen(4), tokens, rows)
        grads = h.backward(dy, x, pre=pre, times=t)

        def loss(x, w, b, t):
            return ((act64(act, x @ w.t() + b)[0] * t + r.double()) * dy.double()).sum()

        base = [v.double() for v in (x, w, b, t)]
        for k, (v, grad) in enumerate(zip(base, grads)):
            d = normal(gen(5 + k), *v.shape).double()
            if act == "relu" and k < 3:  # away from the corner: entries whose sign would change are rare
                step = 1e-7
            else:
                step = 1e-4
            side = [loss(*(u + s * step * d if i == k else u for i, u in enumerate(base))) for s in (1, -1)]
            want = ((side[0] - side[1]) / (2 * step)).item()
            terms = grad.double() * d
            assert abs(terms.sum().item() - want) <= 2.0 ** -7 * terms.abs().sum().item() / math.sqrt(terms.numel()) * 8 + 1e-3


def test_strides_and_given_outputs():
    tokens, rows, cols = 50, 136, 264
    for n in (5, tokens):
        for typ in (torch.bfloat16, torch.float32):
            for wide in (16, 13):  # rows of 16-byte groups, and not
                x, w, b, t, r, dy = make(n, rows, cols, typ, 6)
                h = head.Linear(w, b, activation="silu", max_tokens=tokens)
                want_y, want_pre = h(x, residual=r, times=t, keep_pre=True, out_dtype=typ)
                want = h.backward(dy, x, pre=want_pre, times=t)

                def view(like):
                    buf = torch.full((n, like.shape[1] + wide), 7.0, dtype=like.dtype, device="cuda")
                    buf[:, :like.shape[1]] = like
                    return buf[:, :like.shape[1]], buf

                (xv, _), (tv, _), (rv, rb), (dv, _) = map(view, (x, t, r, dy))
                (pv, pb), (dxv, dxb), (dtv, dtb) = map(view, (torch.zeros_like(dy), torch.zeros_like(x), torch.zeros_like(dy)))
                y, pre = h(xv, residual=rv, times=tv, pre=pv, out=rv)  # the stream in place
                assert y.data_ptr() == rv.data_ptr() and pre.data_ptr() == pv.data_ptr()
                tol = 2.0 ** -7 if typ is torch.bfloat16 else 1e-5
                within(y, want_y.double(), tol * (1 + want_y.double().abs()), "y")
                within(pre, want_pre.double(), tol * (1 + want_pre.double().abs()), "pre")
                got = h.backward(dv, xv, pre=want_pre, times=tv, dx=dxv, dtimes=dtv)
                for a, e in zip(got, want):
                    within(a, e.double(), 2.0 ** -7 * (e.double().abs() + e.double().abs().mean()), "gradient")
                for buf, like in ((rb, r), (pb, dy), (dxb, x), (dtb, dy)):
                    assert (buf[:, like.shape[1]:] == 7).all()


def test_no_tokens():
    x, w, b, t, r, dy = make(4, 24, 40, torch.bfloat16, 7)
    h = head.Linear(w, b, activation="relu", max_tokens=64)
    y, pre = h(x[:0], keep_pre=True)
    assert y.shape == (0, 24) and pre.shape == (0, 24)
    dx, dw, db, dt = h.backward(dy[:0], x[:0], pre=pre)
    assert dx.shape == (0, 40) and (dw == 0).all() and (db == 0).all() and dt is None


def test_bfloat16_bias_and_a_weight_changed_in_place():
    for tokens in (4, 80):
        x, w, b, t, r, _ = make(tokens, 64, 128, torch.float32, 8, bias_type=torch.bfloat16)
        h = head.Linear(w, b, activation="gelu", max_tokens=tokens)
        for k in range(2):
            y = h(x, out_dtype=torch.float32)
            ey, err, _, _ = forward64(x, w, b, "gelu", None, None, torch.float32)
            within(y, ey, err, "y")
            w.mul_(-0.5)


def test_infinities_stay_in_their_place():
    """An infinite weight or a NaN token reaches its row's features or its own token only."""
    for tokens in (3, 100):
        for cols in (200, 264):
            x, w, b, t, r, _ = make(tokens, 96, cols, torch.bfloat16, 9)
            x = x.abs().clamp(min=0.1)
            h = head.Linear(w, max_tokens=tokens)
            clean = h(x)
            w[17, cols - 1], x[1, 5] = math.inf, math.nan
            y = h(x)
            assert y[1].isnan().all()
            for k in range(tokens):
                if k != 1:
                    assert y[k, 17] == math.inf
                    keep = [i for i in range(96) if i != 17]
                    assert torch.equal(y[k, keep], clean[k, keep])


def test_activations_over_their_range():
    """A weight of one: the activations themselves, from the smallest to the largest values."""
    v = torch.cat([s * torch.logspace(-30, 4, 200) for s in (1, -1)]).cuda().bfloat16()[:, None]
    w = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    for act in ACTS:
        h = head.Linear(w, activation=act, max_tokens=len(v))
        y, pre = h(v, keep_pre=True, out_dtype=torch.float32)
        assert torch.equal(pre, v.float())
        e, slope = act64(act, v.double())
        # below -16 or so the FP32 sum 1 + erf has lost what is left of gelu
        within(y, e, (6 + 2 * v.double().abs().clamp(max=20)) * U * v.double().abs() + 1e-37, f"{act}")
        ones = torch.ones_like(pre)
        dx, _, _, _ = h.backward(ones, v, pre=pre)
        within(dx, slope, 2.0 ** -7 * 1.01 * slope.abs() + 1e-5, f"{act}'")


def test_activations_far_from_zero():
    """The largest BF16 values, where a cube or an exponential overflows, and NaN."""
    top = torch.finfo(torch.bfloat16).max
    v = torch.tensor([top, -top, 1e30, -1e30, 1e20, -1e20, 1e13, -1e13]).cuda().bfloat16()[:, None]
    w = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    for act in ACTS[1:]:
        for tokens in (8, 40):
            x = v.repeat(tokens // 8, 1)
            h = head.Linear(w, activation=act, max_tokens=tokens)
            y, pre = h(x, keep_pre=True)
            assert torch.equal(y, x.clamp(min=0)), act
            assert torch.equal(h.backward(torch.ones_like(pre), x, pre=pre)[0], (x > 0).bfloat16()), act
            x[3] = math.nan
            y, pre = h(x, keep_pre=True)
            dx = h.backward(torch.ones_like(pre), x, pre=pre)[0]
            assert y[3].isnan().all() and dx[3].isnan().all() and y.isnan().sum() == 1 and dx.isnan().sum() == 1


@pytest.mark.parametrize("form", [pulse.MXFP4, pulse.FP8_E4M3])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 3584, 3584), (1, 40, 96), (2, 100, 129), (5, 1003, 203), (16, 300, 5120),
                                              (17, 256, 640), (33, 4100, 512), (64, 512, 1024), (90, 72, 256),
                                              (1, 512, 18944), (9, 64, 27648), (3, 7, 31)])
def test_codes(form, tokens, rows, cols):
    g = gen(rows)
    w = (normal(g, rows * cols) / math.sqrt(cols))
    inv_scale = 64.0 * math.sqrt(cols) if form == pulse.FP8_E4M3 else 1.0
    codes, scales = pulse.cast_lowp(form, w, inv_scale)
    if form == pulse.FP8_E4M3:
        wd = codes.view(torch.float8_e4m3fn).double()[:rows * cols] / inv_scale
    else:
        table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        nib = torch.stack((codes & 15, codes >> 4), 1).flatten()[:rows * cols].int()
        wd = torch.where(nib > 7, -1.0, 1.0) * table[nib & 7]
        wd = wd * torch.exp2(scales.double() - 127).repeat_interleave(32)[:rows * cols]
    wd = wd.view(rows, cols)
    for typ, act, mask in ((torch.bfloat16, "silu", 7), (torch.float32, "gelu", 1), (torch.float32, None, 4),
                           (torch.bfloat16, "relu", 2), (torch.float32, "gelu_tanh", 6)):
        x, _, b, t, r, _ = make(tokens, rows, cols, typ, mask, mask & 1, mask & 2, mask & 4)
        h = head.LowpLinear(form, codes, scales, rows, cols, inv_scale, bias=b, activation=act)
        y = h(x, out_dtype=typ, times=t, residual=r)
        # FP8's scale is divided out of the sum: one more rounding
        ey, err, _, _ = forward64(x, wd, b, act, t, r, typ)
        within(y, ey, err + 4 * U * (1 + ey.abs()), "y")
        if r is not None:
            out = r.clone()
            assert torch.equal(h(x, out=out, times=t, residual=out), y) and torch.equal(out, y)
    # without any of it the product as before
    x = make(tokens, rows, cols, torch.float32, 1)[0]
    plain = head.LowpLinear(form, codes, scales, rows, cols, inv_scale)
    y, err = plain(x), forward64(x, wd, None, None, None, None, torch.float32)
    within(y, err[0], err[1] + 4 * U * (1 + err[0].abs()), "plain")


def test_shared_workspace_and_fewer_tokens():
    """One workspace for two layers, and calls of fewer tokens than it was sized for."""
    x, w, b, t, r, dy = make(700, 300, 264, torch.bfloat16, 12)
    w2 = (normal(gen(13), 264, 300) / 17).bfloat16()
    a = head.Linear(w, b, activation="silu", max_tokens=700)
    need = max(a.workspace_bytes, head.Linear(w2, max_tokens=700).workspace_bytes)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    a = head.Linear(w, b, activation="silu", max_tokens=700, workspace=ws)
    c = head.Linear(w2, max_tokens=700, workspace=ws)
    for n in (700, 1, 33, 64, 200, 699):
        y, pre = a(x[:n], keep_pre=True)
        z = c(y)
        dz = normal(gen(14), n, 264).bfloat16()
        dy1, dw2, _, _ = c.backward(dz, y)
        dx, dw, db, _ = a.backward(dy1, x[:n], pre=pre)
        own_a, own_c = head.Linear(w, b, activation="silu", max_tokens=n), head.Linear(w2, max_tokens=n)
        assert torch.equal(own_a(x[:n]), y) and torch.equal(own_c(y), z)
        for p, q in zip((dy1, dw2), own_c.backward(dz, y)):
            assert torch.equal(p, q)
        for p, q in zip((dx, dw, db), own_a.backward(dy1, x[:n], pre=pre)):
            assert torch.equal(p, q)


def test_a_graph_replays_it():
    for tokens in (4, 90, 600):
        x, w, b, t, r, dy = make(tokens, 264, 520, torch.bfloat16, 15)
        h = head.Linear(w, b, activation="gelu_tanh", max_tokens=tokens)

        def step():
            y, pre = h(x, residual=r, times=t, keep_pre=True)
            return [y, pre, *h.backward(dy, x, pre=pre, times=t)]

        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for turn in range(3):
            x.copy_(torch.randn(x.shape, device="cuda"))
            want = step()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, e) for a, e in zip(out, want)), turn


def test_another_stream():
    x, w, b, t, r, dy = make(200, 264, 520, torch.bfloat16, 16)
    h, other = (head.Linear(w, b, activation="relu", max_tokens=200) for _ in range(2))
    want = h(x, residual=r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = other(x, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    x, w, b, t, r, dy = make(6, 24, 40, torch.bfloat16, 17)
    for bad, word in ((dict(weight=w[0]), "rows, cols"), (dict(weight=w.float()), "weight"),
                      (dict(weight=w, bias=b[:3]), "bias"), (dict(weight=w, bias=b.half()), "bias"),
                      (dict(weight=w, activation="tanh"), "activation"), (dict(weight=w, max_tokens=-1), "max_tokens"),
                      (dict(weight=w, max_tokens=(1 << 20) + 1), "max_tokens"),
                      (dict(weight=w, max_tokens=64, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), "workspace")):
        with pytest.raises(pulse.PulseError, match=word):
            head.Linear(**bad)
    h = head.Linear(w, b, activation="silu", max_tokens=6)
    for call, word in ((dict(x=x.float()), "x must"), (dict(x=x[:, :39]), "x must"), (dict(x=x, times=t[:5]), "times"),
                       (dict(x=x, times=t.float()), "times"), (dict(x=x, residual=r[:, :8]), "residual"),
                       (dict(x=x, out_dtype=torch.half), "out_dtype"), (dict(x=x, out=r.half()), "out"),
                       (dict(x=torch.cat((x, x))), "built for"), (dict(x=x, pre=t.float()), "pre")):
        with pytest.raises(pulse.PulseError, match=word):
            h(**call)
    for call, word in ((dict(dy=dy, x=x), "pre"), (dict(dy=dy.half(), x=x, pre=t), "dy"), (dict(dy=dy, x=x, pre=t.float()), "pre"),
                       (dict(dy=dy, x=x, pre=t, times=t.float()), "times"), (dict(dy=dy[:2], x=x, pre=t), "dy")):
        with pytest.raises(pulse.PulseError, match=word):
            h.backward(**call)
    codes = torch.zeros(24 * 40, dtype=torch.uint8, device="cuda")
    with pytest.raises(pulse.PulseError, match="activation"):
        head.LowpLinear(pulse.FP8_E4M3, codes, None, 24, 40, activation="swish")
    low = head.LowpLinear(pulse.FP8_E4M3, codes, None, 24, 40, activation="silu")
    with pytest.raises(pulse.PulseError, match="times"):
        low(x, times=t)  # bfloat16 beside a float32 result
    with pytest.raises(pulse.PulseError, match="residual"):
        low(x, out_dtype=torch.bfloat16, residual=r[:1])
