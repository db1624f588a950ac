"""The epilogue's activations and slopes relative to their own values, against 64 bits.

A weight of zeros leaves the bias, so a result is act(bias) and, in the gradient, dbias of one
token act'(pre) and dtimes act(pre), all of any FP32 number.

Tolerances, in units of 2^-24, the rounding of one operation.  An exponential's argument a
is off by a product's and a constant's rounding, 1.5 |a| units, which is the relative error
they make; the exponential and the reciprocal are good to 2 each, a sum and a product to 1.
So v s(v), s the logistic function, is off by 6 + 2 |v|; gelu_tanh, whose argument w = 2 y has
four roundings more, by 6 + 6 |w|; gelu, by erfc's 16 ulp and what its argument's 1.5 roundings
make of it, (v^2 + 0.8 |v|) 1.5, by 36 + 3 v^2.  A slope is a sum of two terms of the same
kind; 1 - s loses 1 unit of 1 where s is near 1.  A reciprocal or an exponential below 2^-126 may be
0, where |v| is up to 91: 2^-119 of a value; of gelu_tanh's slope, whose s gets there at
v = -10.1 and is multiplied by 1 + 10.1 * 1.6 (1 + 0.134 * 10.1^2) = 238, 2^-118.
"""
import math

import pytest
import torch

from paper_2602_03839_amd import head, pulse

import test_gpu_linear
from test_gpu_linear import U, within

pytestmark = pytest.mark.gpu

LEAST = 2.0 ** -119


def act64(name, v):
    """An activation and its derivative, gelu's tail without the cancellation of 1 + erf."""
    if name != "gelu":
        return test_gpu_linear.act64(name, v)
    c = 0.5 * torch.special.erfc(-v / math.sqrt(2))
    return v * c, c + v * torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)


def terms(name, v):
    """How far the activation and its slope may be off, v in 64 bits."""
    a = v.abs()
    value = act64(name, v)[0].abs()
    if name == "silu":
        s = torch.sigmoid(v)
        return (6 + 2 * a) * U * value, (10 + 2 * a) * U * (s + a * s * (1 - s)) + 2 * U * a * s
    if name == "gelu":
        cdf, pdf = 0.5 * torch.special.erfc(-v / math.sqrt(2)), torch.exp(-v * v / 2) / math.sqrt(2 * math.pi)
        return (36 + 3 * v * v) * U * value, (40 + 3 * v * v) * U * (cdf + a * pdf)
    u = v.clamp(-30, 30)
    w = 2 * math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)
    s, y = torch.sigmoid(w), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * u * u)
    return (6 + 6 * w.abs()) * U * value, (16 + 6 * w.abs()) * U * (s + u.abs() * y * s * (1 - s)) + 2 * U * u.abs() * y * s


def points():
    v = torch.cat([torch.linspace(-14, 14, 20001, dtype=torch.float64), torch.linspace(-95, 95, 4001, dtype=torch.float64),
                   torch.logspace(-30, 30, 2001, dtype=torch.float64), -torch.logspace(-30, 30, 2001, dtype=torch.float64)])
    return v.float().cuda()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("tokens", [1, 40])
def test_values_to_their_own_size(act, tokens):
    """The negative tail among them, where a gelu made of 1 + erf has lost everything."""
    v = points()
    n = len(v)
    want, _ = act64(act, v.double())
    bound, _ = terms(act, v.double())
    x = torch.ones(tokens, 8, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    y = head.Linear(w, v, activation=act, max_tokens=tokens)(x, out_dtype=torch.float32)
    for t in {0, tokens - 1}:
        within(y[t], want, bound + LEAST, act)
    codes = torch.zeros(n * 8, dtype=torch.uint8, device="cuda")
    y = head.LowpLinear(pulse.FP8_E4M3, codes, None, n, 8, bias=v, activation=act)(x)
    within(y[0], want, bound + LEAST, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_slopes_and_the_multipliers_gradient(act):
    v = points()
    n = len(v)
    value, slope = act64(act, v.double())
    vbound, sbound = terms(act, v.double())
    x = torch.ones(1, 8, dtype=torch.bfloat16, device="cuda")
    h = head.Linear(torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, device="cuda"), activation=act,
                    max_tokens=1)
    one = torch.ones(1, n, device="cuda")
    _, _, db, dt = h.backward(one, x, pre=v[None], times=one)
    within(dt[0], value, vbound + LEAST, act)
    within(db, slope, sbound + 2 * LEAST, act + "'")


@pytest.mark.parametrize("act", ["relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("typ", [torch.float32, torch.bfloat16])
def test_infinities_have_their_limits(act, typ):
    """A bias of -inf switches a feature off, one of inf gives inf; slopes are 0 and 1; a NaN
    stays one."""
    inf = math.inf
    v = torch.tensor([-inf, inf, math.nan, -1e38, 1e38, 1.0, -inf, inf]).cuda()
    want = torch.tensor([0, inf, math.nan, 0, 1e38, math.nan, 0, inf]).to(typ)
    slope = torch.tensor([0, 1, math.nan, 0, 1, math.nan, 0, 1])

    def same(got, want):
        for g, e in zip(got.cpu().tolist(), want.tolist()):
            if e == e:
                assert g == e, (act, got, want)
        assert got[2].isnan() and got[5].isfinite()

    w = torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda")
    codes = torch.zeros(8 * 16, dtype=torch.uint8, device="cuda")
    low = head.LowpLinear(pulse.FP8_E4M3, codes, None, 8, 16, bias=v, activation=act)
    for tokens in (1, 5, 40):
        x = torch.ones(tokens, 16, dtype=torch.bfloat16, device="cuda")
        h = head.Linear(w, v, activation=act, max_tokens=tokens)
        y, pre = h(x, out_dtype=typ, keep_pre=True)
        one = torch.ones(tokens, 8, dtype=typ, device="cuda")
        _, _, db, dt = h.backward(one, x, pre=pre, times=one)
        for t in range(tokens):
            same(y[t], want)
            same(dt[t], want)
        same(db / tokens, slope)
        same(low(x, out_dtype=typ)[0], want)
