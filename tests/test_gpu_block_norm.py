"""The block norm on the GPU against its definition in 64 bits.

Tolerances, relative to the size of the terms that a value is made of (of x - mean: |x| and
|mean|, since the mean's own rounding is a share of those however small their difference): an FP32 value
is a few dozen FP32 roundings (sums are trees of at most 16 terms a lane and 1,024
lanes), for which 1e-5 leaves a factor of five (two norms in a row); a BF16 one adds
its own rounding, half a step: 2^-8.  A sum down the columns adds at most some 70
roundings in a row (a lane's rows, the blocks' slices) to those of its terms: 80 times
2^-24, 5e-6 of the sum of its terms' magnitudes.
"""
import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -8 + 1e-5}
SUM_TOL = 5e-6
EPS = 1e-5
NAMES = ("weight", "bias", "post_weight", "post_bias", "gate")


def make(rows, cols, dtype, seed, rms=True, post=True, gate=True, param_dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g)

    b = (normal(rows, cols) * (0.3 + torch.rand(rows, 1, generator=g)) + 0.2).to(dtype)
    h = (normal(rows, cols) * (0.5 + torch.rand(rows, 1, generator=g)) - 0.3).to(dtype)
    dy, dh = normal(rows, cols).to(dtype), (0.7 * normal(rows, cols)).to(dtype)
    p = {"weight": 1 + 0.2 * normal(cols), "bias": None if rms else 0.3 * normal(cols),
         "post_weight": 1 + 0.2 * normal(cols) if post else None,
         "post_bias": 0.3 * normal(cols) if post and not rms else None,
         "gate": 0.5 + 0.3 * normal(cols) if gate else None}
    p = {k: None if v is None else v.to(param_dtype) for k, v in p.items()}
    return b, h, dy, dh, p


def handle(p, rms, scale):
    return head.BlockNorm(**{k: None if v is None else v.cuda() for k, v in p.items()}, residual_scale=scale,
                          eps=EPS, rms=rms)


def norm64(v, w, bias, rms):
    mean = torch.zeros_like(v[:, 0]) if rms else v.mean(1)
    c = v - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(1) + EPS)
    y = c * rstd[:, None] * w
    return y if bias is None else y + bias, mean, rstd


def forward64(b, h, p, rms, scale):
    """y, h_out and the statistics; p in float64 (its entries may want gradients)."""
    u, pm, pr = b, None, None
    if p["post_weight"] is not None:
        u, pm, pr = norm64(b, p["post_weight"], p["post_bias"], rms)
    if p["gate"] is not None:
        u = u * p["gate"]
    h_out = scale * h + u
    y, mean, rstd = norm64(h_out, p["weight"], p["bias"], rms)
    return y, h_out, [rstd, pr, mean, pm]


def double(p):
    return {k: None if v is None else v.double() for k, v in p.items()}


def near(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: off by {off[bad].max().item():.3g} at {bad.nonzero()[0].tolist()}"


def backward64(dy, dh_out, b, h_out, stats, p, rms, scale):
    """The formulas, each result with the magnitude of its terms."""
    st = [None if s is None else s.double()[:, None] for s in stats]
    one = torch.ones_like(p["weight"])

    def rows(v, mean, rstd):
        return (v if rms else v - mean) * rstd, (v.abs() if rms else v.abs() + mean.abs()) * rstd

    def through(a, size, xh, xs, rstd):
        t = a - xh * (a * xh).mean(1, keepdim=True)
        size = (size + xs * (size * xs).mean(1, keepdim=True) + size.mean(1, keepdim=True)) * rstd
        return (t if rms else t - a.mean(1, keepdim=True)) * rstd, size

    xh, xs = rows(h_out, st[2], st[0])
    a = dy * p["weight"]
    g, size = through(a, a.abs(), xh, xs, st[0])
    g, size = g + dh_out, size + dh_out.abs()
    out = {"dh": (scale * g, abs(scale) * size), "dweight": ((dy * xh).sum(0), (dy.abs() * xs).sum(0)),
           "dbias": (dy.sum(0), dy.abs().sum(0))}
    gate = one if p["gate"] is None else p["gate"]
    t, ts = g * gate, size * gate.abs()
    n, bs = b, b.abs()
    if p["post_weight"] is None:
        out["db"] = t, ts
    else:
        bh, bs = rows(b, st[3], st[1])
        out["db"] = through(t * p["post_weight"], ts * p["post_weight"].abs(), bh, bs, st[1])
        out["dpost_weight"] = (t * bh).sum(0), (ts * bs).sum(0)
        out["dpost_bias"] = t.sum(0), ts.sum(0)
        n = bh * p["post_weight"]
        if p["post_bias"] is not None:
            n = n + p["post_bias"]
    if p["gate"] is not None:
        ns = bs * (1 if p["post_weight"] is None else p["post_weight"].abs())
        if p["post_bias"] is not None:
            ns = ns + p["post_bias"].abs()
        out["dgate"] = (g * n).sum(0), (size * ns).sum(0)
    return out


def check(b, h, dy, dh, p, rms, scale, dtype):
    """One forward and one backward pass against 64 bits."""
    post = p["post_weight"] is not None
    norm = handle(p, rms, scale)
    y, h_out, stats = norm(b.cuda(), h.cuda())
    pd, tol = double(p), TOL[dtype]
    ey, eh, es = forward64(b.double(), h.double(), pd, rms, scale)
    us = b.double().abs()
    if post:
        us = (us + us.mean(1, keepdim=True)) * es[1][:, None] * pd["post_weight"].abs()
        us = us + (0 if p["post_bias"] is None else pd["post_bias"].abs())
    size = abs(scale) * h.double().abs() + us * (1 if p["gate"] is None else pd["gate"].abs())
    near(h_out, eh, tol * size, "h_out")
    bias = 0 if p["bias"] is None else pd["bias"].abs()
    near(y, ey, tol * ((size + size.mean(1, keepdim=True)) * es[0][:, None] * pd["weight"].abs() + bias), "y")
    assert stats.shape == (2 if rms else 4, b.shape[0])
    near(stats[0], es[0], 1e-5 * es[0], "rstd")
    if not rms:
        near(stats[2], es[2], 1e-5 * size.mean(1), "mean")
    if post:
        near(stats[1], es[1], 1e-5 * es[1], "post_rstd")
        if not rms:
            near(stats[3], es[3], 1e-5 * b.double().abs().mean(1), "post_mean")
    got = norm.backward(dy.cuda(), dh.cuda(), b.cuda(), h_out, stats)
    s = [v.cpu() for v in stats] if not rms else [stats[0].cpu(), stats[1].cpu(), None, None]
    want = backward64(dy.double(), dh.double(), b.double(), h_out.cpu().double(), s, pd, rms, scale)
    for name, v in zip(("db", "dh", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"), got):
        if name not in ("db", "dh") and p[name[1:]] is None:
            assert v is None, name
            continue
        exact, size = want[name]
        near(v, exact, (tol if name in ("db", "dh") else SUM_TOL) * size + 1e-30, name)


# every form of the kernels: lanes a row and elements a lane, and their edges
COLS = [1, 7, 8, 64, 511, 512, 520, 896, 1024, 1025, 2048, 2056, 3584, 4097, 5120, 8192, 8200, 16383, 16384]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("cols", COLS)
def test_both_directions(cols, rms, dtype):
    rows = 7 if cols > 2048 else 37
    b, h, dy, dh, p = make(rows, cols, dtype, cols, rms)
    check(b, h, dy, dh, p, rms, 0.75, dtype)


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("cols", [200, 3584])
def test_parts(cols, post, gate, rms):
    """With and without the norm of the block's output and the gate; BF16 parameters."""
    for scale, param_dtype in ((1.0, torch.float32), (-0.5, torch.bfloat16), (0.0, torch.float32)):
        b, h, dy, dh, p = make(19, cols, torch.float32, 3, rms, post, gate, param_dtype)
        check(b, h, dy, dh, p, rms, scale, torch.float32)


@pytest.mark.parametrize("rows", [1, 2, 511, 513, 2049, 4097, 20000])
@pytest.mark.parametrize("cols", [40, 700])
def test_row_counts(rows, cols):
    """Fewer, as many and more rows than blocks; two rows a group forward."""
    for dtype, rms in ((torch.float32, False), (torch.bfloat16, True)):
        b, h, dy, dh, p = make(rows, cols, dtype, rows, rms)
        check(b, h, dy, dh, p, rms, 0.5, dtype)


@pytest.mark.parametrize("cols", [2304, 5120, 5121])
def test_many_wide_rows(cols):
    for dtype, rms in ((torch.float32, False), (torch.bfloat16, True)):
        b, h, dy, dh, p = make(4099, cols, dtype, cols, rms)
        check(b, h, dy, dh, p, rms, 0.5, dtype)


def test_gradient_against_differences():
    """The FP32 gradient along random directions against central differences of the
    definition in 64 bits: step 1e-5, whose own error is of the order 1e-10."""
    rows, cols, scale = 9, 130, 0.6
    for rms in (True, False):
        b, h, dy, dh, p = make(rows, cols, torch.float32, 11, rms)
        norm = handle(p, rms, scale)
        y, h_out, stats = norm(b.cuda(), h.cuda())
        got = norm.backward(dy.cuda(), dh.cuda(), b.cuda(), h_out, stats)
        grads = dict(zip(("b", "h") + NAMES, got))
        pd = double(p)

        def loss(b, h, p):
            y, h_out, _ = forward64(b, h, p, rms, scale)
            return (y * dy.double()).sum() + (h_out * dh.double()).sum()

        g = torch.Generator().manual_seed(5)
        for name, grad in grads.items():
            if grad is None:
                continue
            base = {"b": b.double(), "h": h.double()}.get(name, pd.get(name))
            d = torch.randn(base.shape, generator=g, dtype=torch.float64)
            step, side = 1e-5, []
            for sign in (1, -1):
                moved = base + sign * step * d
                q = {**pd, name: moved} if name in pd else pd
                side.append(loss(moved if name == "b" else b.double(), moved if name == "h" else h.double(), q))
            want = ((side[0] - side[1]) / (2 * step)).item()
            terms = (grad.cpu().double() * d)
            assert abs(terms.sum().item() - want) <= 1e-5 * terms.abs().sum().item() + 1e-7, name


def test_strides_and_outputs():
    """Views with wider rows, given outputs, the stream in place, and what lies between
    the rows left as it was."""
    rows, cols = 33, 640
    for dtype in (torch.bfloat16, torch.float32):
        for wide in (648, 643):  # rows of 16-byte groups, and not
            b, h, dy, dh, p = make(rows, cols, dtype, 4)
            norm = handle(p, True, 0.5)
            want = norm(b.cuda(), h.cuda())
            bufs = [torch.full((rows, wide), 7.0, dtype=dtype, device="cuda") for _ in range(6)]
            views = [t[:, :cols] for t in bufs]
            views[0].copy_(b)
            views[1].copy_(h)
            stats = torch.full((2, rows + 5), -1.0, device="cuda")
            y, h_out, st = norm(views[0], views[1], y=views[2], h_out=views[1], stats=stats[:, :rows])
            assert y.data_ptr() == views[2].data_ptr() and h_out.data_ptr() == views[1].data_ptr()
            for got, exp in zip((y, h_out, st), want):
                near(got, exp.cpu().double(), 1e-6 if dtype is torch.float32 else 2.0 ** -6, "strided")
            views[3].copy_(dy)
            got = norm.backward(views[3], dh.cuda(), views[0], h_out, st, db=views[4], dh=views[5])
            exp = norm.backward(dy.cuda(), dh.cuda(), b.cuda(), want[1], want[2])
            for x, e in zip(got, exp):
                assert (x is None) == (e is None)
                if e is not None:
                    near(x, e.cpu().double(), 1e-5 * e.abs().max().item() if x.dtype is torch.float32 else 2.0 ** -5, "strided gradient")
            for t in bufs:
                assert (t[:, cols:] == 7).all()
            assert (stats[:, rows:] == -1).all()


def test_without_statistics_and_without_rows():
    b, h, dy, dh, p = make(5, 96, torch.bfloat16, 6)
    norm = handle(p, True, 1.0)
    a, c = norm(b.cuda(), h.cuda()), norm(b.cuda(), h.cuda(), keep_stats=False)
    assert c[2] is None and torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    e = torch.empty(0, 96, dtype=torch.bfloat16, device="cuda")
    y, h_out, stats = norm(e, e)
    assert y.shape == (0, 96) and stats.shape == (2, 0)
    got = norm.backward(e, None, e, h_out, stats)
    assert got[0].shape == (0, 96)
    for v in got[2:]:
        assert v is None or (v == 0).all()


def test_no_upstream_of_the_stream():
    """dh_out None is dh_out of zeros; without post norm and gate b may be None."""
    b, h, dy, dh, p = make(13, 260, torch.float32, 8)
    norm = handle(p, True, 0.5)
    y, h_out, stats = norm(b.cuda(), h.cuda())
    zero = torch.zeros_like(h_out)
    for x, e in zip(norm.backward(dy.cuda(), None, b.cuda(), h_out, stats),
                    norm.backward(dy.cuda(), zero, b.cuda(), h_out, stats)):
        assert (x is None and e is None) or torch.equal(x, e)
    plain = head.BlockNorm(p["weight"].cuda())
    y, h_out, stats = plain(b.cuda(), h.cuda())
    for x, e in zip(plain.backward(dy.cuda(), dh.cuda(), None, h_out, stats),
                    plain.backward(dy.cuda(), dh.cuda(), b.cuda(), h_out, stats)):
        assert (x is None and e is None) or torch.equal(x, e)


def test_what_a_row_holds_stays_in_it():
    """An infinity or a NaN in a row reaches no other row forward; rows of zeros."""
    b, h, dy, dh, p = make(12, 384, torch.float32, 9)
    norm = handle(p, True, 0.5)
    clean = norm(b.cuda(), h.cuda())
    b[3, 5], h[7, 9] = float("nan"), float("inf")
    b[5], h[5] = 0, 0
    got = norm(b.cuda(), h.cuda())
    keep = [k for k in range(12) if k not in (3, 5, 7)]
    for x, e in zip(got[:2], clean[:2]):
        assert torch.equal(x[keep], e[keep])
        assert x[3].isnan().all() and not x[7].isfinite().all() and (x[5] == 0).all()


def test_results_repeat_and_a_graph_replays_them():
    b, h, dy, dh, p = (t.cuda() if isinstance(t, torch.Tensor) else t for t in make(1500, 1024, torch.bfloat16, 10))
    norm = handle(p, True, 0.5)

    def step():
        y, h_out, stats = norm(b, h)
        return [y, h_out, stats, *norm.backward(dy, dh, b, h_out, stats)]

    first = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for turn in range(3):
        b.copy_(torch.randn_like(b))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for x, e in zip(out, want):
            assert (x is None and e is None) or torch.equal(x, e), turn
    again = step()
    assert all((x is None and e is None) or torch.equal(x, e) for x, e in zip(again, want))
    assert not torch.equal(first[0], again[0])


def test_another_stream():
    b, h, dy, dh, p = make(64, 512, torch.bfloat16, 12)
    norm = handle(p, True, 0.5)
    want = norm(b.cuda(), h.cuda())
    side = torch.cuda.Stream()
    bd, hd = b.cuda(), h.cuda()
    side.wait_stream(torch.cuda.current_stream())
    got = norm(bd, hd, stream=side)
    side.synchronize()
    assert all(torch.equal(x, e) for x, e in zip(got, want))


def test_refusals():
    w = torch.ones(64, device="cuda")
    x = torch.zeros(3, 64, device="cuda")
    with pytest.raises(pulse.PulseError, match="post_bias"):
        head.BlockNorm(w, post_bias=w)
    with pytest.raises(pulse.PulseError, match="gate"):
        head.BlockNorm(w, gate=torch.ones(63, device="cuda"))
    with pytest.raises(pulse.PulseError, match="post_weight"):
        head.BlockNorm(w, post_weight=w.bfloat16())
    with pytest.raises(pulse.PulseError, match="residual_scale"):
        head.BlockNorm(w, residual_scale=float("inf"))(x, x)
    with pytest.raises(pulse.PulseError, match="1 to"):
        head.BlockNorm(torch.ones(16385, device="cuda"))
    norm = head.BlockNorm(w)
    with pytest.raises(pulse.PulseError, match="h must"):
        norm(x, x.bfloat16())
    with pytest.raises(pulse.PulseError, match="h must"):
        norm(x, x[:2])
    with pytest.raises(pulse.PulseError, match="b must"):
        norm(x.half(), x)
    with pytest.raises(pulse.PulseError, match="stats"):
        norm(x, x, stats=torch.zeros(4, 3, device="cuda"))
    with pytest.raises(pulse.PulseError, match="stride"):
        wide = torch.zeros(3, 128, device="cuda")
        norm(x, wide[:, :64], h_out=torch.as_strided(wide, (3, 64), (64, 1)))
    y, h_out, stats = norm(x, x)
    with pytest.raises(pulse.PulseError, match="dy must"):
        norm.backward(x.bfloat16(), None, x, h_out, stats)
    with pytest.raises(pulse.PulseError, match="stats"):
        norm.backward(x, None, x, h_out, stats[:1])
    with pytest.raises(pulse.PulseError, match="must be"):
        head.BlockNorm(w, gate=w).backward(x, None, None, h_out, stats)


@pytest.mark.parametrize("cols", [4099, 8193, 12000])
@pytest.mark.parametrize("rows", [1, 63, 65, 1200])
def test_wide_rows(rows, cols):
    """Rows whose columns' sums are taken in a pass of their own."""
    for dtype, rms, post, gate in ((torch.float32, False, True, True), (torch.bfloat16, True, True, False),
                                   (torch.bfloat16, False, False, True), (torch.float32, True, False, False)):
        b, h, dy, dh, p = make(rows, cols, dtype, rows + cols, rms, post, gate)
        check(b, h, dy, dh, p, rms, 0.5, dtype)


def test_more_rows_than_a_launch_takes():
    """2^22 rows are one launch's; each of few elements."""
    rows = (1 << 22) + 5
    w = torch.ones(8, device="cuda")
    norm = head.BlockNorm(w, gate=2 * w)
    b = torch.ones(rows, 8, dtype=torch.bfloat16, device="cuda")
    h = torch.full_like(b, -1.0)
    h[-1], b[-2] = 3.0, 0.5
    y, h_out, stats = norm(b, h)
    assert (h_out[:-2] == 1).all() and (h_out[-1] == 5).all() and (h_out[-2] == 0).all()
    assert (y[:-2] == 1).all() and (y[-1] == 1).all() and (y[-2] == 0).all()
    got = norm.backward(y, h_out, b, h_out, stats)
    # y is constant along a row, so nothing comes through the norm: g = dh_out
    assert (got[1][:-2] == 1).all() and (got[1][-1] == 5).all() and (got[0][:-2] == 2).all()
    assert abs(got[6][0].item() / (rows - 2 + 5) - 1) < 1e-4
