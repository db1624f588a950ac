"""Cross entropy of a head's logits on the GPU against the definition in 64 bits.

Tolerances.  A logit is a sum of `hidden` exact products in FP32: off by at most
hidden * 2^-24 of the sum of their magnitudes; loss and lse add the rounding of
log and of a few sums (1e-6 of their terms).  A gradient is a sum whose terms
carry the BF16 rounding of G (2^-8 relative to each, and the error of the logits
and of lse in the exponent, which is relative to p) and is itself rounded to BF16:
at most 2^-8 of the sum of the terms' magnitudes, plus 2^-8 of the result.
"""
import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def inputs(tokens, vocab, hidden, seed, ignored=0.2, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(vocab, hidden, generator=g) * 2 / hidden ** 0.5).bfloat16()
    y = torch.randint(vocab, (tokens,), generator=g)
    x = (torch.randn(tokens, hidden, generator=g) + torch.rand(tokens, 1, generator=g) * w[y]).bfloat16()
    y[torch.rand(tokens, generator=g) < ignored] = -100
    return x, w, y, torch.randn(tokens, generator=g) / max(tokens, 1)


def exact(x, w, y, dloss, scale):
    """loss, lse, their error bound, G in 64 bits."""
    x, w = x.double(), w.double()
    z = scale * (x @ w.t())
    size = abs(scale) * (x.abs() @ w.abs().t())
    lse = torch.logsumexp(z, 1)
    kept = (y >= 0) & (y < w.shape[0])
    at = torch.where(kept, y, torch.zeros_like(y))
    hit = z.gather(1, at[:, None])[:, 0]
    loss = torch.where(kept, lse - hit, torch.zeros_like(lse))
    dz = (x.shape[1] + 2) * U * size.amax(1)
    g = torch.exp(z - lse[:, None])
    g[torch.arange(len(y)), at] -= 1
    g = torch.where(kept[:, None], g * dloss.double()[:, None] * scale, torch.zeros_like(g))
    return loss, lse, 2 * dz + 1e-6 * (1 + lse.abs() + hit.abs()), g


def check(tokens, vocab, hidden, seed=0, scale=1.0, data=None):
    x, w, y, dl = data or inputs(tokens, vocab, hidden, seed)
    ce = head.LinearCE(w.cuda(), max_tokens=tokens, logit_scale=scale)
    loss, lse = ce.forward(x.cuda(), y.cuda())
    el, es, bound, g = exact(x, w, y, dl, scale)
    assert ((loss.cpu().double() - el).abs() <= bound).all()
    assert ((lse.cpu().double() - es).abs() <= bound).all()
    kept = (y >= 0) & (y < vocab)
    assert (loss.cpu()[~kept] == 0).all()
    dx, dw = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
    xk = torch.where(kept[:, None], x.double(), torch.zeros((), dtype=torch.float64))
    # G's own relative error: its rounding, and twice the logits' error in the exponent
    rel = 2.0 ** -8 + 2 * bound.max().item()
    size = g.abs() + 2 * U * dl.double().abs()[:, None] * abs(scale)
    # at the target p's error is relative to p, up to 1, and not to p - 1
    at = torch.where(kept, y, torch.zeros_like(y))
    size[torch.arange(tokens), at] += 2 * bound / rel * dl.double().abs() * abs(scale)
    for got, want, terms in ((dx, g @ w.double(), size @ w.double().abs()),
                             (dw, g.t() @ xk, size.t() @ xk.abs())):
        off = (got.cpu().double() - want).abs()
        allowed = (rel + (vocab + tokens) * U) * terms + 2.0 ** -8 * want.abs() + 1e-38
        assert got.shape == want.shape
        assert (off <= allowed).all(), ((off - allowed).max(), off.max(), want.abs().max())
    assert (dx.cpu()[~kept] == 0).all()
    return dx, dw


# tokens through every tile shape and its edges
@pytest.mark.parametrize("tokens", [1, 2, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 600])
def test_tokens(tokens):
    check(tokens, 1500, 192, seed=tokens)


@pytest.mark.parametrize("vocab", [1, 2, 7, 63, 64, 255, 256, 257, 511, 1023, 5003])
@pytest.mark.parametrize("tokens", [5, 100, 300])
def test_vocabularies(vocab, tokens):
    check(tokens, vocab, 128, seed=vocab)


@pytest.mark.parametrize("hidden", [1, 3, 7, 8, 9, 56, 63, 64, 65, 72, 96, 100, 128, 203, 264, 520])
@pytest.mark.parametrize("tokens", [3, 70, 200])
def test_hidden_sizes(hidden, tokens):
    check(tokens, 700, hidden, seed=hidden)


@pytest.mark.parametrize("scale", [0.0, 0.5, 1 / 0.7, -1.0])
def test_scales(scale):
    check(33, 900, 64, seed=3, scale=scale)


def test_several_pieces():
    """More vocabulary than one piece of G holds, and a short last piece."""
    for tokens, vocab, hidden in ((40, 40000, 2048), (2100, 66000, 64), (2500, 70000, 520),
                                  (1, 90001, 776), (17, 66003, 1032), (64, 70000, 1024), (33, 300000, 264)):
        x, w, y, dl = inputs(tokens, vocab, hidden, 8)
        ce = head.LinearCE(w.cuda(), max_tokens=tokens)
        _, lse = ce.forward(x.cuda(), y.cuda())
        dx, dw = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
        # in FP32 on the GPU: the 64-bit definition piece by piece
        xd, wd = x.cuda().double(), w.cuda().double()
        z = xd @ wd.t()
        assert (lse.double() - torch.logsumexp(z, 1)).abs().max() < 1e-4
        g = torch.exp(z - torch.logsumexp(z, 1)[:, None])
        kept = (y >= 0).cuda()
        at = y.clamp(min=0).cuda()
        g[torch.arange(tokens), at] -= 1
        g *= torch.where(kept, dl.cuda().double(), torch.zeros((), dtype=torch.float64, device="cuda"))[:, None]
        for got, want in ((dx, g @ wd), (dw, g.t().contiguous() @ xd)):
            assert (got.double() - want).norm() <= 2.0 ** -8 * want.norm()


def check_on_gpu(tokens, vocab, hidden, seed=8, ignored=0.1):
    """``check`` in 64 bits on the GPU, into outputs of NaN and row by row: a row of dw
    is off by at most 2^-8 of each token's term (G's rounding) and 2^-8 of itself, a
    row of dx by the same over the entries; FP32 sums add (terms) * 2^-24 of the terms, and
    the logits in G's exponents 2 * (hidden + 2) * 2^-24 of their magnitudes."""
    x, w, y, dl = (t.cuda() for t in inputs(tokens, vocab, hidden, seed, ignored))
    nan = float("nan")
    ce = head.LinearCE(w, max_tokens=tokens)
    loss, lse = ce.forward(x, y, *[torch.full((tokens,), nan, device="cuda") for _ in range(2)])
    dx, dw = ce.backward(x, y, lse, dl, torch.full_like(x, nan), torch.full_like(w, nan))
    xd, wd, kept = x.double(), w.double(), y >= 0
    z, size = xd @ wd.t(), (xd.abs() @ wd.abs().t()).amax(1)
    want = torch.logsumexp(z, 1)
    dz = (hidden + 2) * U * size
    bound = 2 * dz + 1e-6 * (1 + want.abs() + z.abs().amax(1))
    hit = z.gather(1, y.clamp(min=0)[:, None])[:, 0]
    assert ((lse.double() - want).abs() <= bound).all()
    assert ((loss.double() - torch.where(kept, want - hit, 0.0)).abs() <= bound).all()
    p = torch.exp(z - want[:, None])
    by = torch.where(kept, dl.double(), 0.0)[:, None]
    g, terms = p * by, p * by.abs()
    rows = torch.arange(tokens, device="cuda")
    g[rows, y.clamp(min=0)] -= by[:, 0]
    # G's error: of its rounding, and of p through its exponent (relative to p, not to p - 1)
    err = g.abs() * 2.0 ** -8 + terms * 2 * bound[:, None] + (g.abs() + terms) * (vocab + tokens) * U
    xd = torch.where(kept[:, None], xd, 0.0)
    for got, want, allowed in ((dw, g.t() @ xd, err.t() @ xd.norm(dim=1)), (dx, g @ wd, err @ wd.norm(dim=1))):
        off = (got.double() - want).norm(dim=1)
        assert (off <= allowed + 2.0 ** -8 * want.norm(dim=1) + 1e-30).all(), (off - allowed).max()
    return g, (dx, g @ wd), (dw, g.t() @ xd)


# pieces, the running dw kernel, all tile shapes, a weight past the caches (61 x 40,003 x 4,096),
# odd hidden sizes, with ragged last tiles everywhere
@pytest.mark.parametrize("tokens,vocab,hidden", [(1, 90001, 776), (17, 66003, 1032), (33, 300000, 264), (40, 40000, 2048),
                                                 (61, 40003, 4096), (64, 70000, 1024), (64, 66003, 1032), (100, 66003, 1032),
                                                 (128, 20001, 1032), (129, 30011, 520), (500, 40003, 203), (600, 90001, 264),
                                                 (2100, 66000, 64), (2500, 70000, 520), (2500, 70001, 521)])
def test_rows_of_large_gradients(tokens, vocab, hidden):
    _, of_x, of_w = check_on_gpu(tokens, vocab, hidden, ignored=0.0 if tokens == 1 else 0.1)
    for got, want in (of_x, of_w):  # as exact as their own rounding
        assert (got.double() - want).norm() <= 0.002 * want.norm()


@pytest.mark.parametrize("most", [65, 129, 513, 3000])
def test_one_workspace_for_fewer_tokens(most):
    """Calls of fewer tokens than a workspace was sized for give the bits that an object of
    that number gives, and write nothing past its end."""
    vocab, hidden = 9000, 136
    w = inputs(1, vocab, hidden, 1)[1].cuda()
    L, size = head.lib(), head.lib().pulse_linear_ce_workspace_bytes(most, vocab, hidden)
    ws = torch.full((size + 65536,), 0xA5, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for tokens in (1, 64, 65, 128, 129, 512, 513, most):
        if tokens > most:
            continue
        x, _, y, dl = (t.cuda() for t in inputs(tokens, vocab, hidden, tokens))
        ce = head.LinearCE(w, max_tokens=tokens)
        loss, lse = ce.forward(x, y)
        dx, dw = ce.backward(x, y, lse, dl)
        got = [torch.full_like(t, float("nan")) for t in (loss, lse, dx, dw)]
        ws[:size] = 0xA5
        assert L.pulse_linear_ce_forward(x.data_ptr(), hidden, w.data_ptr(), y.data_ptr(), tokens, vocab, hidden, 1.0,
                                         got[0].data_ptr(), got[1].data_ptr(), ws.data_ptr(), size, stream) == 0
        assert L.pulse_linear_ce_backward(x.data_ptr(), hidden, w.data_ptr(), y.data_ptr(), tokens, vocab, hidden, 1.0,
                                          lse.data_ptr(), dl.data_ptr(), got[2].data_ptr(), hidden, got[3].data_ptr(),
                                          ws.data_ptr(), size, stream) == 0
        for a, b in zip(got, (loss, lse, dx, dw)):
            assert torch.equal(a, b), tokens
        assert (ws[size:] == 0xA5).all(), tokens


@pytest.mark.parametrize("tokens,vocab,hidden", [(300, 40, 72), (1000, 300, 203), (700, 3, 64)])
def test_many_tokens_share_a_target(tokens, vocab, hidden):
    """Far more tokens than entries, and half of them with the same target."""
    x, w, y, dl = inputs(tokens, vocab, hidden, 11)
    y[::2] = vocab - 1
    check(tokens, vocab, hidden, data=(x, w, y, dl))


def test_precision_of_few_and_many_tokens():
    """Every gradient is as exact as its own rounding to BF16: what G's rounding
    takes from the targets' entries is added back (a relative error, in the
    2-norm, of 0.0017 for the output's rounding alone; 0.0024 with G's)."""
    for tokens in (1, 5, 64, 65, 128, 129, 400):
        x, w, y, dl = inputs(tokens, 3000, 256, tokens, ignored=0.0)
        ce = head.LinearCE(w.cuda(), max_tokens=tokens)
        _, lse = ce.forward(x.cuda(), y.cuda())
        dx, dw = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
        g = exact(x, w, y, dl, 1.0)[3]
        for got, want in ((dx, g @ w.double()), (dw, g.t() @ x.double())):
            assert (got.cpu().double() - want).norm() <= 0.002 * want.norm(), tokens


@pytest.mark.parametrize("tokens,vocab,hidden", [(40, 20000, 256), (100, 5003, 203), (200, 20000, 256), (600, 9001, 320),
                                                 (2100, 9000, 256)])
@pytest.mark.parametrize("shared", [0, 3, 10])
@pytest.mark.parametrize("sure", [0, 3])
def test_precision_where_rows_share_a_direction(tokens, vocab, hidden, shared, sure):
    """Rows of the head that share a direction, several times as long as what they
    differ by, as trained ones do, and (`sure`) most of the probability on one
    entry that is not the target.  A row of G sums to zero, so the shared direction cancels in
    dx: what G's rounding loses must not bring it back.

    dx's own rounding to BF16 is off by up to 2^-8 of each value, 0.0017 in the
    2-norm and 0.0020 for a token's row.  What may be left of G's: entries that lose at most
    2^-12 of the token's dloss, so are at most an eighth of it, with uniform errors:
    in the 2-norm 2^-8 sqrt(1/8 / 3) = 0.0008 of a row's unshared part.  Together
    0.0019 over all, 0.0022 for a token."""
    g = torch.Generator().manual_seed(tokens + shared + sure)
    w = torch.randn(vocab, hidden, generator=g) * 2 / hidden ** 0.5
    d = torch.randn(hidden, generator=g)
    d /= d.norm()
    w = (w + 2 * shared * d).bfloat16()
    y, other = torch.randint(vocab, (tokens,), generator=g), torch.randint(vocab, (tokens,), generator=g)
    x = torch.randn(tokens, hidden, generator=g)
    x += 2 * torch.rand(tokens, 1, generator=g) * w[y] + sure * w[other]
    x = (x - (x @ d)[:, None] * d).bfloat16()  # along d it would only move the token's lse
    dl = torch.randn(tokens, generator=g) / tokens
    ce = head.LinearCE(w.cuda(), max_tokens=tokens)
    _, lse = ce.forward(x.cuda(), y.cuda())
    dx, _ = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
    want = exact(x, w, y, dl, 1.0)[3] @ w.double()
    assert torch.equal(dx, ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())[0])
    off = dx.cpu().double() - want
    each = off.norm(dim=1) / want.norm(dim=1)
    print(f"off by {(off.norm() / want.norm()).item():.5f}, a token by {each.max().item():.5f}")
    assert off.norm() <= 0.002 * want.norm() and each.max() <= 0.0025


@pytest.mark.parametrize("tokens", [20, 300])
def test_gradient_for_a_smaller_lse(tokens):
    """With an lse below the forward's the entries of G are no probabilities: any
    number of a token's may be large.  The definition holds, and the bits repeat."""
    x, w, y, dl = inputs(tokens, 900, 64, tokens, ignored=0.0)
    ce = head.LinearCE(w.cuda(), max_tokens=tokens)
    lse = ce.forward(x.cuda(), y.cuda())[1] - 5
    dx, dw = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
    for again, first in zip(ce.backward(x.cuda(), y.cuda(), lse, dl.cuda()), (dx, dw)):
        assert torch.equal(again, first)
    g = torch.exp(x.double() @ w.double().t() - lse.cpu().double()[:, None])
    g[torch.arange(tokens), y] -= 1
    g *= dl.double()[:, None]
    # G's and the result's roundings, each at most 2^-8; the exponents' errors are below 2^-16
    for got, want, size in ((dx, g @ w.double(), g.abs() @ w.double().abs()), (dw, g.t() @ x.double(), g.abs().t() @ x.double().abs())):
        assert ((got.cpu().double() - want).abs() <= (2.0 ** -8 + 2.0 ** -15) * size + 2.0 ** -8 * want.abs()).all()


def test_all_ignored_and_odd_targets():
    x, w, y, dl = inputs(50, 300, 64, 1)
    y[:] = -100
    dx, dw = check(50, 300, 64, data=(x, w, y, dl))
    assert (dx == 0).all() and (dw == 0).all()
    y = torch.tensor([0, 299, 300, -1, 2 ** 40, -2 ** 40, 5, 2 ** 32 + 5] * 6 + [1, 2])
    check(50, 300, 64, data=(x, w, y, dl))


def test_nothing_of_an_ignored_token_gets_out():
    """NaN and infinities in the rows and upstream gradients of ignored tokens."""
    for tokens in (40, 300):
        x, w, y, dl = inputs(tokens, 520, 96, 2)
        y[::3] = -100
        want = check(tokens, 520, 96, data=(x, w, y, dl))
        x, dl = x.clone(), dl.clone()
        bad = (y < 0).nonzero()[:, 0]
        x[bad[0::2]], x[bad[1::2], 5] = float("nan"), float("inf")
        dl[bad] = float("nan")
        ce = head.LinearCE(w.cuda(), max_tokens=tokens)
        loss, lse = ce.forward(x.cuda(), y.cuda())
        assert (loss.cpu()[bad] == 0).all() and torch.isfinite(lse.cpu()[y >= 0]).all()
        got = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_large_logits():
    """Logits of +-several hundred: no overflow, and a loss far below 1 and far
    above it keep their relative size."""
    x, w, y, dl = inputs(64, 400, 64, 4, ignored=0.0)
    y[0] = (x[0].double() @ w.double().t()).argmax()
    y[1] = (x[1].double() @ w.double().t()).argmin()
    check(64, 400, 64, scale=60.0, data=(x, w, y, dl))


def test_minus_infinite_logits():
    """A weight row of infinities on one side: a probability of zero."""
    x, w, y, dl = inputs(20, 300, 32, 5)
    x[:, 0] = x[:, 0].abs() + 1
    w[7, 0] = float("-inf")
    w[7, 1:] = 0
    y[y == 7] = 8
    ce = head.LinearCE(w.cuda(), max_tokens=20)
    loss, lse = ce.forward(x.cuda(), y.cuda())
    z = x.double() @ w.double().t()
    assert (lse.cpu().double() - torch.logsumexp(z, 1)).abs().max() < 1e-5
    assert torch.isfinite(loss.cpu()).all()


@pytest.mark.parametrize("tokens,vocab", [(20, 300), (100, 1300), (600, 5000)])
def test_infinite_logits(tokens, vocab):
    """lse is infinite with a logit, and the loss then infinite but at that very
    target, where it is undefined; minus infinite if every logit is."""
    x, w, y, _ = inputs(tokens, vocab, 32, 6, ignored=0.0)
    x[:, 0] = x[:, 0].abs() + 1
    x[1::2, 0] = 0  # zero times infinity: NaN
    w[vocab - 2, 0] = float("inf")
    w[5, 0] = float("-inf")
    y[y == 5] = 6
    y[0] = vocab - 2
    ce = head.LinearCE(w.cuda(), max_tokens=tokens)
    loss, lse = (t.cpu() for t in ce.forward(x.cuda(), y.cuda()))
    assert (lse[0::2] == float("inf")).all() and torch.isnan(lse[1::2]).all()
    there = y == vocab - 2
    assert torch.isnan(loss[there]).all() and (loss[0::2][~there[0::2]] == float("inf")).all()
    w[:, 0] = float("-inf")
    ce = head.LinearCE(w.cuda(), max_tokens=tokens)
    _, lse = ce.forward(x.cuda(), y.cuda())
    assert (lse.cpu()[0::2] == float("-inf")).all() and torch.isnan(lse.cpu()[1::2]).all()


def test_gradient_against_differences():
    """dx against central differences of the loss in 64 bits, for inputs that are
    exact in BF16; the gradient's own roundings allow 2^-7 of its largest entry."""
    x, w, y, dl = inputs(6, 40, 16, 6)
    ce = head.LinearCE(w.cuda(), max_tokens=6, logit_scale=1.25)
    _, lse = ce.forward(x.cuda(), y.cuda())
    dx, dw = ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())

    def total(xv, wv):
        z = 1.25 * xv @ wv.t()
        kept = y >= 0
        per = torch.logsumexp(z, 1) - z.gather(1, y.clamp(min=0)[:, None])[:, 0]
        return (per[kept] * dl.double()[kept]).sum()

    for which, grad in ((0, dx), (1, dw)):
        args = [x.double(), w.double()]
        flat, grad = args[which].view(-1), grad.cpu().double().view(-1)
        for i in range(0, flat.numel(), 7):
            keep, h = flat[i].item(), 1e-4
            flat[i] = keep + h
            up = total(*args)
            flat[i] = keep - h
            down = total(*args)
            flat[i] = keep
            assert abs((up - down) / (2 * h) - grad[i]) <= 2.0 ** -7 * grad.abs().max() + 1e-7, (which, i)


def test_views_streams_and_same_bits():
    tokens, vocab, hidden = 90, 1000, 128
    x, w, y, dl = inputs(tokens, vocab, hidden, 7)
    wide = torch.zeros(tokens, 200, dtype=torch.bfloat16, device="cuda")
    odd = torch.zeros(tokens, 133, dtype=torch.bfloat16, device="cuda")
    wide[:, :hidden] = x.cuda()
    odd[:, :hidden] = x.cuda()
    yd, dld = y.cuda(), dl.cuda()
    ce = head.LinearCE(w.cuda(), max_tokens=200)
    loss, lse = ce.forward(x.cuda(), yd)
    dx, dw = ce.backward(x.cuda(), yd, lse, dld)
    out = torch.full((tokens, 131), 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for view in (wide, odd):
        l2, s2 = ce.forward(view[:, :hidden], yd, stream=s)
        dx2, dw2 = ce.backward(view[:, :hidden], yd, s2, dld, dx=out[:, :hidden], stream=s)
        s.synchronize()
        assert torch.equal(loss, l2) and torch.equal(lse, s2)
        assert torch.equal(dx, out[:, :hidden]) and torch.equal(dw, dw2)
        assert (out[:, hidden:] == 7).all()


@pytest.mark.parametrize("most", [65, 129, 513, 3000])
def test_fewer_tokens_than_built_for(most):
    """One object's workspace serves every smaller call."""
    _, w, _, _ = inputs(1, 9000, 136, 1)
    ce = head.LinearCE(w.cuda(), max_tokens=most)
    for tokens in (1, 64, 65, 128, 129, 512, 513, most):
        if tokens > most:
            continue
        x, _, y, dl = inputs(tokens, 9000, 136, tokens)
        _, lse = ce.forward(x.cuda(), y.cuda())
        ce.backward(x.cuda(), y.cuda(), lse, dl.cuda())
    torch.cuda.synchronize()


def test_more_tokens_than_one_launch_has_threads():
    """2^26 tokens and a few forward (64 threads a token in the join) and 2^24 backward
    (256), most of them without a target."""
    hidden, vocab = 8, 100
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randn(vocab, hidden, generator=g, device="cuda").bfloat16()
    for tokens, backward in (((1 << 26) + 5, False), ((1 << 24) + 5, True)):
        x = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        y = torch.full((tokens,), -100, device="cuda")
        kept = torch.cat([torch.arange(300), (1 << 22) - 5 + torch.arange(10), tokens - 300 + torch.arange(300)]).cuda()
        y[kept] = torch.randint(vocab, (len(kept),), generator=g, device="cuda")
        ce = head.LinearCE(w, max_tokens=tokens)
        out = [torch.full((tokens,), 77.0, device="cuda") for _ in range(2)]
        loss, lse = ce.forward(x, y, *out)
        wd, step = w.double(), 1 << 22
        for k in range(0, tokens, step):
            z = x[k:k + step].double() @ wd.t()
            want = torch.logsumexp(z, 1)
            assert ((lse[k:k + step].double() - want).abs() < 1e-5).all(), k
            yk = y[k:k + step]
            want = torch.where(yk >= 0, want - z.gather(1, yk.clamp(min=0)[:, None])[:, 0], 0.0)
            assert ((loss[k:k + step].double() - want).abs() < 1e-5).all(), k
        if not backward:
            continue
        dl = torch.randn(tokens, generator=g, device="cuda")
        dx = torch.full_like(x, 77.0)
        dx, dw = ce.backward(x, y, lse, dl, dx=dx)
        p = torch.exp(x[kept].double() @ wd.t() - lse[kept].double()[:, None])
        p[torch.arange(len(kept)), y[kept]] -= 1
        p *= dl[kept].double()[:, None]
        xk = x[kept].double()
        for got, want, size in ((dx[kept], p @ wd, p.abs() @ wd.abs()), (dw, p.t() @ xk, p.abs().t() @ xk.abs())):
            assert ((got.double() - want).abs() <= 2.0 ** -8 * (want.abs() + size) + 1e-6).all()
        dx[kept] = 0
        assert (dx == 0).all()


def test_more_tiles_than_one_launch_has_threads():
    """2^23 tiles of 512 threads and more, in the forward pass."""
    tokens, vocab, hidden = 1_050_000, 524_500, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(vocab, hidden, generator=g, device="cuda").bfloat16()
    x = torch.randn(tokens, hidden, generator=g, device="cuda").bfloat16()
    y = torch.randint(vocab, (tokens,), generator=g, device="cuda")
    ce = head.LinearCE(w, max_tokens=tokens)
    loss, lse = ce.forward(x, y, *[torch.full((tokens,), 77.0, device="cuda") for _ in range(2)])
    assert torch.isfinite(lse).all() and (lse != 77).all() and (loss != 77).all()
    for first in (0, 255, 400_000, 524_200, 800_000, tokens - 500):
        part = slice(first, first + 500)
        z = x[part].double() @ w.double().t()
        want = torch.logsumexp(z, 1)
        assert ((lse[part].double() - want).abs() < 1e-4).all()
        hit = z[torch.arange(500), y[part]]
        assert ((loss[part].double() - (want - hit)).abs() < 1e-4).all()


def test_no_tokens():
    _, w, _, _ = inputs(1, 64, 32, 1)
    ce = head.LinearCE(w.cuda(), max_tokens=0)
    x, y = torch.empty(0, 32, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = ce.forward(x, y)
    assert loss.numel() == lse.numel() == 0
    dw = torch.ones(64, 32, dtype=torch.bfloat16, device="cuda")
    dx, dw = ce.backward(x, y, lse, loss, dweight=dw)
    assert dx.shape == (0, 32) and (dw == 0).all()


def test_refusals():
    x, w, y, dl = (t.cuda() for t in inputs(8, 64, 32, 1))
    ce = head.LinearCE(w, max_tokens=8)
    _, lse = ce.forward(x, y)
    bad = [lambda: head.LinearCE(w.float(), 8), lambda: head.LinearCE(w[0], 8), lambda: head.LinearCE(w.t(), 8),
           lambda: head.LinearCE(w.cpu(), 8), lambda: head.LinearCE(w, -1), lambda: head.LinearCE(w[:0], 8),
           lambda: head.LinearCE(torch.zeros(1, 65537, dtype=torch.bfloat16, device="cuda"), 1),
           lambda: ce.forward(x.float(), y), lambda: ce.forward(x[:, :16], y), lambda: ce.forward(x, y[:4]),
           lambda: ce.forward(x, y.int()), lambda: ce.forward(x, y.cpu()), lambda: ce.forward(x, None),
           lambda: ce.forward(torch.cat([x, x]), torch.cat([y, y])),
           lambda: ce.forward(x, y, loss=lse[:3]), lambda: ce.forward(x, y, lse=lse.double()),
           lambda: ce.backward(x, y, lse[:3], dl), lambda: ce.backward(x, y, lse, dl.double()),
           lambda: ce.backward(x, y, lse, dl, dx=x[:4]), lambda: ce.backward(x, y, lse, dl, dweight=w.t()),
           lambda: ce.backward(x, y, lse, dl, dweight=w[:8].clone()),
           lambda: head.LinearCE(w, 8, logit_scale=float("nan")).forward(x, y)]
    for k, call in enumerate(bad):
        with pytest.raises(pulse.PulseError):
            call()
            pytest.fail(f"call {k} was not refused")
