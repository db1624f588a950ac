"""The linear layers' gradient to the bits of its results: d = dy * times * act'(pre) goes
into both products as two BF16 values, against the definition in 64 bits.

Tolerances.  d's two parts leave 2^-16 of each d at most, independently of each other: over
a sum a root mean square of 2^-16 / sqrt 3 of the terms' (and six of it for the largest of
some 10^5 sums).  A sum of k products adds (k / 16 + 80) roundings of 2^-24 of the sum of
magnitudes at most (two steps for each 32 k, and parts); d itself is good to (20 + 4 |pre|)
2^-24.  A BF16 result adds half a step, 2^-8 of it, whose root mean square over many
is at most 2^-8 / sqrt 3.
"""
import math

import pytest
import torch

from paper_2602_03839_amd import head

from test_gpu_linear import ACTS, HALF, U, act64, gen, normal, within

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
REST = 2.0 ** -16 / math.sqrt(3)  # of a d, its root mean square at most
ONE = HALF[BF16] / math.sqrt(3)   # of a BF16 result


def d64(dy, pre, times, act):
    """d in 64 bits and how far an FP32 one may be off."""
    v = 0 if pre is None else pre.double()
    d = dy.double() * (1 if times is None else times.double())
    slope = 1.0 if act is None else act64(act, v)[1]
    size = 0 if pre is None else v.abs()
    return d * slope, (20 + 4 * size) * U * d.abs()


def check(h, x, w, dy, pre, times, act, exact=False):
    dx, dw, _, _ = h.backward(dy, x, pre=pre, times=times)
    d, off = d64(dy, pre, times, act)
    rest = 0.0 if exact else 6 * REST
    for got, a, b, e, what in ((dx, d, w.double(), off, "dx"), (dw, d.t(), x.double(), off.t(), "dweight")):
        a, e = a.contiguous(), e.contiguous()
        want, size = a @ b, a.abs() @ b.abs()
        bound = e @ b.abs() + rest * ((a * a) @ (b * b)).sqrt() + (a.shape[1] / 16 + 80) * U * size
        within(got, want, bound + HALF[BF16] * 1.01 * want.abs() + 1e-37, what)
    return dx, dw


FORMS = [(F32, None, False), (F32, "gelu", False), (F32, "relu", True), (BF16, "silu", True), (BF16, "gelu_tanh", False),
         (BF16, None, True), (BF16, "relu", False), (BF16, None, False)]


@pytest.mark.parametrize("typ,act,with_times", FORMS)
@pytest.mark.parametrize("tokens,rows,cols", [(5, 256, 136), (77, 1003, 203), (300, 130, 264), (700, 256, 72),
                                              (1100, 520, 896)])
def test_a_shared_direction_cancels(tokens, rows, cols, typ, act, with_times):
    """Weights and tokens that are 64 times as large in common as apart, and d whose sums
    over features and over tokens are nearly 0: of the common part nothing is left, but
    what a rounding of d would leave of it."""
    g = gen(tokens)
    w = (8 * normal(g, 1, cols) + 0.125 * normal(g, rows, cols)).bfloat16()
    x = (8 * normal(g, 1, cols) + 0.125 * normal(g, tokens, cols)).bfloat16()
    times = (1 + normal(g, tokens, rows).abs()).to(typ) if with_times else None
    pre = normal(g, tokens, rows).to(typ) if act or with_times else None
    d = normal(g, tokens, rows).double()
    if act:
        slope = act64(act, pre.double())[1]
        d = torch.where(slope.abs() < 0.2, 0.0, d)
    # centred where something is left, by turns
    for _ in range(20):
        for dim in (0, 1):
            n = (d != 0).sum(dim, keepdim=True).clamp(min=1)
            d = torch.where(d != 0, d - d.sum(dim, keepdim=True) / n, 0.0)
    dy = d
    if times is not None:
        dy = dy / times.double()
    if act:
        dy = torch.where(d != 0, dy / slope, 0.0)
    h = head.Linear(w, activation=act, max_tokens=tokens)
    check(h, x, w, dy.to(typ), pre, times, act, exact=typ is BF16 and act in (None, "relu") and not with_times)


@pytest.mark.parametrize("typ,act,with_times", FORMS)
@pytest.mark.parametrize("tokens,rows,cols", [(77, 1003, 203), (300, 520, 896), (2100, 1536, 520), (33, 9000, 640)])
def test_off_by_the_results_own_rounding(tokens, rows, cols, typ, act, with_times):
    """Over a whole result the root mean square of what it is off is that of its own
    rounding; 1% more for d's rest and the sums."""
    g = gen(rows)
    w = (normal(g, rows, cols) / math.sqrt(cols)).bfloat16()
    x = normal(g, tokens, cols).bfloat16()
    pre = normal(g, tokens, rows).to(typ) if act or with_times else None
    times = normal(g, tokens, rows).to(typ) if with_times else None
    dy = (0.01 * normal(g, tokens, rows)).to(typ)
    h = head.Linear(w, activation=act, max_tokens=tokens)
    dx, dw, _, _ = h.backward(dy, x, pre=pre, times=times)
    d, _ = d64(dy, pre, times, act)
    for got, want, what in ((dx, d @ w.double(), "dx"), (dw, d.t().contiguous() @ x.double(), "dweight")):
        off = (got.double() - want).norm() / want.norm()
        assert off <= 1.01 * ONE, (what, off.item())


@pytest.mark.parametrize("tokens", [5, 40, 200])
def test_the_ends_of_the_range(tokens):
    """d up to FP32's largest number, whose rounding to BF16 would be infinite; infinities and
    NaN; and an infinite weight or token, which gives infinities where d is exact too."""
    rows, cols = 96, 200
    g = gen(tokens)
    w = (2.0 ** -10 * (1 + normal(g, rows, cols).abs())).bfloat16()
    x = (2.0 ** -10 * (1 + normal(g, tokens, cols).abs())).bfloat16()
    h = head.Linear(w, max_tokens=tokens)
    top = torch.finfo(F32).max
    dy = torch.zeros(tokens, rows, device="cuda")
    for t in range(tokens):
        dy[t, t % rows] = top * (1 - 2.0 ** -24) if t % 2 else -top
    check(h, x, w, dy, None, None, None)
    # one token's d is infinite, another's NaN (its bits in the lower half alone)
    dy = normal(g, tokens, rows).abs()
    clean = h.backward(dy, x)
    dy[1, 3] = math.inf
    dy[2] = torch.tensor([0x7F800001], dtype=torch.int32, device="cuda").view(F32)
    dx, dw, _, _ = h.backward(dy, x)
    assert (dx[1] == math.inf).all() and dx[2].isnan().all() and dw.isnan().all()
    keep = [t for t in range(tokens) if t not in (1, 2)]
    assert torch.equal(dx[keep], clean[0][keep])
    # infinite weights and tokens: d > 0, exact in BF16 and not
    for dy in (torch.ones(tokens, rows, device="cuda"), 0.3 + normal(g, tokens, rows).abs(),
               torch.full((tokens, rows), 1e-30, device="cuda")):
        wi, xi = w.clone(), x.clone()
        wi[7, 11], xi[3, 13] = math.inf, math.inf
        dx, dw, _, _ = head.Linear(wi, max_tokens=tokens).backward(dy, xi)
        assert (dx[:, 11] == math.inf).all() and (dw[:, 13] == math.inf).all()
        dx[:, 11], dw[:, 13] = 0, 0
        assert dx.isfinite().all() and dw.isfinite().all()
        # a feature without a gradient has none
        dy = dy.clone()
        dy[:, 5] = 0
        dx, dw, _, _ = h.backward(dy, x)
        assert (dw[5] == 0).all()
        assert (h.backward(torch.zeros_like(dy), x)[0] == 0).all()


def test_small_values():
    """d down to FP32's smallest normal numbers: nothing is lost but what lies below them."""
    tokens, rows, cols = 40, 64, 72
    g = gen(3)
    w, x = normal(g, rows, cols).bfloat16(), normal(g, tokens, cols).bfloat16()
    h = head.Linear(w, max_tokens=tokens)
    for size in (1e-20, 1e-30, 1e-34):
        dy = size * normal(g, tokens, rows)
        dx, dw, _, _ = h.backward(dy, x)
        for got, a, b in ((dx, dy.double(), w.double()), (dw, dy.double().t().contiguous(), x.double())):
            want = a @ b
            bound = 6 * REST * ((a * a) @ (b * b)).sqrt() + 100 * U * (a.abs() @ b.abs()) + 2.0 ** -125 * b.abs().sum(0)
            within(got, want, bound + HALF[BF16] * 1.01 * want.abs(), size)


@pytest.mark.parametrize("tokens,rows", [(128, 8192), (128, 8193), (100, 18945), (17, 70001), (129, 8128), (1, 1 << 20)])
def test_wide_rows_of_few_tokens(tokens, rows):
    """On both sides of 2^20 values, where d, dtimes and dbias change their kernel: one launch's
    sums over tokens, or chunks of them."""
    for typ in (BF16, F32):
        g = gen(rows)
        w, x = normal(g, rows, 16).bfloat16(), normal(g, tokens, 16).bfloat16()
        pre, times = (normal(g, tokens, rows).to(typ) for _ in range(2))
        dy = normal(g, tokens, rows).to(typ)
        h = head.Linear(w, torch.zeros(rows, device="cuda"), activation="silu", max_tokens=tokens)
        check(h, x, w, dy, pre, times, "silu")
        _, _, db, dt = h.backward(dy, x, pre=pre, times=times)
        d, off = d64(dy, pre, times, "silu")
        within(db, d.sum(0), off.sum(0) + (tokens + 20) * U * d.abs().sum(0) + 1e-37, "dbias")
        value = act64("silu", pre.double())[0] * dy.double()
        within(dt, value, (8 + 2 * pre.double().abs()) * U * value.abs() + HALF[typ] * 1.01 * value.abs() + 1e-37, "dtimes")
