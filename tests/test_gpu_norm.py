"""Layer norm and RMS norm on the GPU against the definition in 64 bits.

Tolerances (relative to the largest magnitude of the exact result): an FP32
output is a few dozen FP32 roundings of the exact one (the sums are trees of at
most 16 terms a lane and 1,024 lanes), 1e-5 leaves a factor of ten; a BF16
output adds its own rounding, half a step: 2^-8 of a value just above a power
of two (a significand of 8 bits).
"""
import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

TOL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -8 + 1e-5}


def rows_of(rows, cols, dtype, seed, offset=0.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * (0.5 + torch.rand(rows, 1, generator=g)) + offset
    return x.to(dtype)


def params(cols, dtype, seed, bias):
    g = torch.Generator().manual_seed(seed)
    w = (1 + 0.2 * torch.randn(cols, generator=g)).to(dtype)
    b = (0.3 * torch.randn(cols, generator=g)).to(dtype) if bias else None
    return w, b


def exact_forward(x, w, b, eps, rms):
    x, w = x.double(), w.double()
    mean = torch.zeros(x.shape[0], dtype=torch.float64) if rms else x.mean(1)
    c = x - mean[:, None]
    rstd = 1 / torch.sqrt((c * c).mean(1) + eps)
    y = c * rstd[:, None] * w
    return (y if b is None else y + b.double()), mean, rstd


def exact_backward(dy, x, w, mean, rstd, rms):
    dy, x, r = dy.double(), x.double(), rstd.double()[:, None]
    xh = (x if rms else x - mean.double()[:, None]) * r
    a = dy * w.double()
    dx = a - xh * (a * xh).mean(1, keepdim=True)
    if not rms:
        dx = dx - a.mean(1, keepdim=True)
    return dx * r, (dy * xh).sum(0), dy.sum(0)


def near(got, want, tol, what):
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, what
    if want.numel():
        bound = tol * max(want.abs().max().item(), 1e-30)
        off = (got - want).abs().max().item()
        assert off <= bound, f"{what}: off by {off:.3g}, {bound:.3g} allowed"


# every form of the kernel: lanes a row and elements a lane, and their edges
COLS = [1, 7, 8, 64, 511, 512, 520, 896, 1024, 1025, 2048, 2056, 3584, 4097, 5120, 8192, 8200,
        16383, 16384]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("cols", COLS)
def test_both_directions(cols, rms, dtype):
    rows = 7 if cols > 2048 else 37
    x, dy = rows_of(rows, cols, dtype, cols), rows_of(rows, cols, dtype, cols + 1, 0.0)
    w, b = params(cols, torch.float32, cols + 2, bias=not rms)
    n = head.LayerNorm(w.cuda(), None if b is None else b.cuda(), eps=1e-5, rms=rms)
    y, mean, rstd = n(x.cuda())
    ey, em, er = exact_forward(x, w, b, 1e-5, rms)
    near(y, ey, TOL[dtype], "y")
    near(rstd, er, 1e-5, "rstd")
    assert (mean is None) == rms
    if not rms:
        near(mean, em, 1e-5, "mean")
    dx, dw, db = n.backward(dy.cuda(), x.cuda(), mean, rstd)
    m, r = (None if rms else mean.cpu()), rstd.cpu()
    edx, edw, edb = exact_backward(dy, x, w, m, r, rms)
    # one column: dx cancels to nearly nothing, so it is held to its terms' size
    scale = (dy.double() * w.double() * r.double()[:, None]).abs().max()
    assert (dx.cpu().double() - edx).abs().max() <= TOL[dtype] * scale
    near(dw, edw, 1e-5, "dweight")
    assert (db is None) == rms
    if not rms:
        near(db, edb, 1e-5, "dbias")


@pytest.mark.parametrize("rows", [1, 2, 511, 512, 513, 1025, 3001])
def test_row_counts(rows):
    """Fewer, as many and more rows than the backward pass has blocks."""
    for cols in (40, 2304):
        x, dy = rows_of(rows, cols, torch.float32, rows), rows_of(rows, cols, torch.float32, 3, 0.1)
        w, b = params(cols, torch.float32, 5, True)
        n = head.LayerNorm(w.cuda(), b.cuda())
        y, mean, rstd = n(x.cuda())
        near(y, exact_forward(x, w, b, 1e-6, False)[0], 1e-5, "y")
        dx, dw, db = n.backward(dy.cuda(), x.cuda(), mean, rstd)
        edx, edw, edb = exact_backward(dy, x, w, mean.cpu(), rstd.cpu(), False)
        near(dx, edx, 1e-5, "dx")
        near(dw, edw, 1e-5, "dweight")
        near(db, edb, 1e-5, "dbias")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("cols", [7, 40, 700, 1000, 1025, 2000, 3584, 5120, 8199, 16384])
@pytest.mark.parametrize("rows", [1281, 3001])
def test_many_rows_backward(rows, cols, rms, dtype):
    """The kernel for more than 1,280 rows, whose blocks keep the columns' sums of their
    rows, in every form; into outputs of NaN."""
    x, dy = rows_of(rows, cols, dtype, cols).cuda(), rows_of(rows, cols, dtype, cols + 1, 0.1).cuda()
    w, b = params(cols, torch.float32, cols + 2, bias=not rms)
    w, b = w.cuda(), None if b is None else b.cuda()
    xd = x.double()
    mean = None if rms else xd.mean(1).float()
    rstd = (1 / torch.sqrt((xd if rms else xd - mean.double()[:, None]).square().mean(1) + 1e-5)).float()
    none = [torch.full((rows, cols), float("nan"), dtype=dtype, device="cuda")]
    none += [torch.full((cols,), float("nan"), device="cuda") for _ in range(1 if rms else 2)]
    dx, dw, db = head.LayerNorm(w, b, eps=1e-5, rms=rms).backward(dy, x, mean, rstd, *none)
    edx, edw, edb = exact_backward(dy, x, w, mean, rstd, rms)
    near(dx, edx.cpu(), TOL[dtype], "dx")
    # a column's sum has 3,001 terms of either sign: 1e-5 of the largest of their magnitudes
    xh = (xd if rms else xd - mean.double()[:, None]) * rstd.double()[:, None]
    assert (dw.double() - edw).abs().max() <= 1e-5 * (dy.double() * xh).abs().sum(0).max()
    assert (db is None) == rms
    if not rms:
        assert (db.double() - edb).abs().max() <= 1e-5 * dy.double().abs().sum(0).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [7, 700, 896, 1500, 2500, 5120, 8200, 16383])
def test_two_rows_a_group(cols, dtype):
    """The forward kernel that takes two rows at a time, in every form, with an odd last row."""
    rows = 16387 if cols <= 1024 else 4099
    x = rows_of(rows, cols, dtype, cols).cuda()
    w, b = params(cols, torch.float32, 5, True)
    w, b = w.cuda(), b.cuda()
    y, mean, rstd = head.LayerNorm(w, b)(x, y=torch.full_like(x, float("nan")))
    ey, em, er = exact_forward(x, w, b, 1e-6, False)
    near(y, ey.cpu(), TOL[dtype], "y")
    near(mean, em.cpu(), 1e-5, "mean")
    near(rstd, er.cpu(), 1e-5, "rstd")


@pytest.mark.parametrize("rows", [16383, 16385, 4097, 2049])
def test_many_rows_forward(rows):
    """Two rows a group of lanes, and an odd last one."""
    for cols in (24, 700, 2000, 2500):
        if rows * cols > 40_000_000:
            continue
        x = rows_of(rows, cols, torch.bfloat16, rows)
        w, b = params(cols, torch.float32, 5, True)
        y, mean, rstd = head.LayerNorm(w.cuda(), b.cuda())(x.cuda())
        ey, em, er = exact_forward(x, w, b, 1e-6, False)
        near(y, ey, TOL[torch.bfloat16], "y")
        near(mean, em, 1e-5, "mean")
        near(rstd, er, 1e-5, "rstd")


@pytest.mark.parametrize("cols,dtype,rms", [(2, torch.bfloat16, True), (1, torch.float32, False)])
def test_more_rows_than_one_launch_has_threads(cols, dtype, rms):
    """2^27 rows and a few: with 32 threads a row, 2^32 threads and more."""
    rows = (1 << 27) + 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=dtype, device="cuda").normal_(generator=g)
    w, b = params(cols, torch.float32, 2, bias=not rms)
    y = torch.full((rows, cols), 77.0, dtype=dtype, device="cuda")
    y, mean, rstd = head.LayerNorm(w.cuda(), None if b is None else b.cuda(), eps=1e-3, rms=rms)(x, y=y)
    for first in (0, (1 << 22) - 3, (1 << 26) - 2, (1 << 27) - 4, rows - (1 << 20)):
        part = slice(first, first + (1 << 20))
        ey, em, er = exact_forward(x[part].cpu(), w, b, 1e-3, rms)
        near(y[part], ey, TOL[dtype], "y")
        near(rstd[part], er, 1e-5, "rstd")
        if not rms:
            near(mean[part], em, 1e-5, "mean")
    step = 1 << 24
    assert all((y[k:k + step] != 77.0).all() and torch.isfinite(rstd[k:k + step]).all() for k in range(0, rows, step))


def test_gradient_against_differences():
    """The formula's gradient against central differences of a 64-bit loss
    sum(dy * y): second order, so a step of 1e-4 leaves about 1e-7."""
    rows, cols = 3, 24
    x, dy = rows_of(rows, cols, torch.float32, 1), rows_of(rows, cols, torch.float32, 2, 0.0)
    w, b = params(cols, torch.float32, 3, True)
    n = head.LayerNorm(w.cuda(), b.cuda(), eps=1e-3)
    _, mean, rstd = n(x.cuda())
    got = dict(zip("xwb", n.backward(dy.cuda(), x.cuda(), mean, rstd)))
    args = {"x": x.double(), "w": w.double(), "b": b.double()}

    def loss():
        return (exact_forward(args["x"], args["w"], args["b"], 1e-3, False)[0] * dy.double()).sum()

    for key, t in args.items():
        flat, grad = t.view(-1), got[key].cpu().double().view(-1)
        for i in range(0, flat.numel(), 5):
            keep, h = flat[i].item(), 1e-4
            flat[i] = keep + h
            up = loss()
            flat[i] = keep - h
            down = loss()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - grad[i]) <= 1e-5 * grad.abs().max() + 1e-6, (key, i)


@pytest.mark.parametrize("cols", [96, 100])
def test_strided_rows_and_bf16_parameters(cols):
    """Views with rows apart, outputs into views; neighbours stay as they are."""
    rows, wide = 19, 160
    x, dy = rows_of(rows, wide, torch.bfloat16, 1), rows_of(rows, wide, torch.bfloat16, 2)
    w, b = params(cols, torch.bfloat16, 3, True)
    n = head.LayerNorm(w.cuda(), b.cuda())
    out = torch.full((rows, wide), 7.0, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = n(x.cuda()[:, :cols], y=out[:, :cols])
    ey, _, _ = exact_forward(x[:, :cols], w, b, 1e-6, False)
    near(out[:, :cols], ey, TOL[torch.bfloat16], "y")
    assert (out[:, cols:] == 7).all()
    g = torch.full((rows, wide), 7.0, dtype=torch.bfloat16, device="cuda")
    n.backward(dy.cuda()[:, :cols], x.cuda()[:, :cols], mean, rstd, dx=g[:, :cols])
    edx = exact_backward(dy[:, :cols], x[:, :cols], w, mean.cpu(), rstd.cpu(), False)[0]
    near(g[:, :cols], edx, TOL[torch.bfloat16], "dx")
    assert (g[:, cols:] == 7).all()


def test_no_rows():
    w, b = params(48, torch.float32, 1, True)
    n = head.LayerNorm(w.cuda(), b.cuda())
    x = torch.empty(0, 48, device="cuda")
    y, mean, rstd = n(x)
    assert y.shape == (0, 48) and mean.numel() == rstd.numel() == 0
    dw, db = torch.ones(48, device="cuda"), torch.ones(48, device="cuda")
    dx, dw, db = n.backward(x, x, mean, rstd, dweight=dw, dbias=db)
    assert dx.shape == (0, 48) and (dw == 0).all() and (db == 0).all()


def test_nan_and_infinity_stay_in_their_row():
    x = rows_of(8, 777, torch.float32, 4)
    x[2, 5], x[6, 700] = float("nan"), float("inf")
    w, b = params(777, torch.float32, 1, True)
    y, _, _ = head.LayerNorm(w.cuda(), b.cuda())(x.cuda())
    ey, _, _ = exact_forward(x, w, b, 1e-6, False)
    clean = [0, 1, 3, 4, 5, 7]
    near(y.cpu()[clean], ey[clean], 1e-5, "clean rows")
    assert not torch.isfinite(y.cpu()[2]).any() and not torch.isfinite(y.cpu()[6]).any()


def test_constant_rows_and_large_offsets():
    """A constant row has zero variance: eps alone sets rstd.  A row far from
    zero keeps its spread, since the mean is taken off before squaring."""
    x = torch.full((2, 640), 3.25)
    x[1] = 4096 + torch.arange(640) / 64
    w, b = params(640, torch.float32, 1, True)
    y, mean, rstd = head.LayerNorm(w.cuda(), b.cuda(), eps=1e-4)(x.cuda())
    ey, _, er = exact_forward(x, w, b, 1e-4, False)
    near(rstd, er, 1e-5, "rstd")
    # the mean of values near 4096 is itself rounded by up to 2^-12
    near(y, ey, 2.0 ** -12 * er[1].item() + 1e-5, "y")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [300, 700, 896, 1500, 3584, 5120, 12000])
@pytest.mark.parametrize("rows", [3, 1300])
def test_mean_times_rstd_past_the_range(rows, cols, dtype):
    """Constant rows of 2^120 and an rstd of 1,024: their product has no FP32 value,
    but no element is that far from its mean."""
    x = torch.full((rows, cols), 2.0 ** 120, dtype=dtype)
    dy = rows_of(rows, cols, dtype, 1, 0.0)
    w, b = params(cols, torch.float32, 2, True)
    mean, rstd = torch.full((rows,), 2.0 ** 120), torch.full((rows,), 1024.0)
    dx, dw, db = head.LayerNorm(w.cuda(), b.cuda()).backward(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda())
    edx, edw, edb = exact_backward(dy, x, w, mean, rstd, False)
    near(dx, edx, TOL[dtype], "dx")
    near(db, edb, 1e-5, "dbias")
    assert (dw == 0).all() and (edw == 0).all()


def test_same_bits_and_other_stream():
    x, dy = rows_of(1500, 1000, torch.bfloat16, 1).cuda(), rows_of(1500, 1000, torch.bfloat16, 2).cuda()
    w, b = params(1000, torch.float32, 1, True)
    n = head.LayerNorm(w.cuda(), b.cuda())
    y, mean, rstd = n(x)
    first = n.backward(dy, x, mean, rstd)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y2, m2, r2 = n(x, stream=s)
    second = n.backward(dy, x, m2, r2, stream=s)
    s.synchronize()
    for a, c in zip((y, mean, rstd) + first, (y2, m2, r2) + second):
        assert torch.equal(a, c)


def test_forward_takes_no_workspace():
    """The gradient's partial sums (67 MB at this width) are allocated when a gradient
    is asked for: a model that answers has a norm or two a layer and no gradient."""
    w = torch.ones(16384, device="cuda")
    x = torch.randn(3, 16384, device="cuda")
    before = torch.cuda.memory_allocated()
    norms = [head.LayerNorm(w, rms=True) for _ in range(8)]
    for n in norms:
        _, _, rstd = n(x)
    assert torch.cuda.memory_allocated() - before < 1 << 20
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dx, dw, _ = norms[0].backward(x, x, None, rstd, stream=s)
    s.synchronize()
    edx, edw, _ = exact_backward(x.cpu(), x.cpu(), w.cpu(), None, rstd.cpu(), True)
    # dy = x: dx cancels to its share of eps, so it is held to its terms' size
    assert (dx.cpu().double() - edx).abs().max() <= 1e-5 * (x * rstd[:, None]).abs().max().item()
    near(dw, edw, 1e-5, "dweight")


def test_refusals():
    w, b = params(64, torch.float32, 1, True)
    w, b = w.cuda(), b.cuda()
    n = head.LayerNorm(w, b)
    x = torch.zeros(4, 64, device="cuda")
    _, mean, rstd = n(x)
    bad = [lambda: head.LayerNorm(w.half()), lambda: head.LayerNorm(w, b.bfloat16()),
           lambda: head.LayerNorm(w, b[:32].clone()), lambda: head.LayerNorm(w.cpu()),
           lambda: head.LayerNorm(torch.ones(head.NORM_MAX_COLS + 1, device="cuda")),
           lambda: n(x.half()), lambda: n(x[:, :32]), lambda: n(x.t()), lambda: n(x.cpu()),
           lambda: n(x[0]), lambda: n(x, y=torch.zeros(3, 64, device="cuda")),
           lambda: n(x, y=torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16)),
           lambda: n(x.expand(4, 64)[:1].expand(4, 64)),
           lambda: n(torch.zeros(4 * 64 + 1, device="cuda")[1:].view(4, 64)),
           lambda: n.backward(x.bfloat16(), x, mean, rstd), lambda: n.backward(x, x, None, rstd),
           lambda: n.backward(x, x, mean[:2], rstd), lambda: n.backward(x, x, mean, rstd.double()),
           lambda: head.LayerNorm(w, b, eps=-1.0)(x), lambda: head.LayerNorm(w, b, eps=float("nan"))(x)]
    for k, call in enumerate(bad):
        with pytest.raises(pulse.PulseError):
            call()
            pytest.fail(f"call {k} was not refused")
