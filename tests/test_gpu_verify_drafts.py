"""Verification of drafted tokens on the GPU against the definition in 64 bits.

Tokens and counts have to be equal.  The kernel's probabilities are off by some 1e-12, so
a draw's border is met by chance once in 1e6 draws or so (150,000 borders); the tests
make some thousand.  logprob is FP32 of a value in 64 bits: half a step, 2^-24, and
1e-11 of the logits' size for the sums.
"""
import math

import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu


def probs(z, scale):
    """Probabilities of one row in 64 bits, all 0 where the row is empty, and their logs.
    Differences from the largest logit come first: added to a log-sum-exp of 1e38 its
    logarithm of the number of entries would be lost."""
    z = z.double() * scale
    if z.isnan().any() or (z == math.inf).any() or (z == -math.inf).all():
        return torch.zeros_like(z), torch.full_like(z, -math.inf)
    z = z - z.max()
    logs = z - torch.log(torch.exp(z).sum())
    return torch.exp(logs), logs


def oracle(target, drafts, uniform, draft_logits, lengths, scale, draft_scale):
    """Sequence by sequence, from the definition.  CPU tensors."""
    batch, more = uniform.shape
    k_all, vocab = more - 1, target.shape[-1]
    tokens = torch.full((batch, more), -1, dtype=torch.int64)
    count = torch.zeros(batch, dtype=torch.int32)
    logprob = torch.zeros(batch, more, dtype=torch.float64)
    for b in range(batch):
        length = k_all if lengths is None else min(max(int(lengths[b]), 0), k_all)
        for k in range(length + 1):
            z = target[b * more + k]
            p, logs = probs(z, scale)
            weights = p
            if k < length:
                x = int(drafts[b, k])
                known = 0 <= x < vocab
                if draft_logits is None:
                    q = torch.zeros(vocab, dtype=torch.float64)
                    if known:
                        q[x] = 1
                else:
                    q, _ = probs(draft_logits[b * k_all + k], draft_scale)
                if known and float(uniform[b, k]) * float(q[x]) < float(p[x]):
                    tokens[b, k], count[b] = x, k + 1
                    logprob[b, k] = logs[x]
                    continue
                weights = (p - q).clamp(min=0)
            c = weights.cumsum(0)
            if c[-1] > 0:
                over = (c > float(uniform[b, k_all]) * c[-1]).nonzero()
                v = int(over[0]) if len(over) else int((weights > 0).nonzero()[-1])
                tokens[b, k] = v
                logprob[b, k] = logs[v]
            else:
                logprob[b, k] = -math.inf
            break
    return tokens, count, logprob


def make(batch, drafts, vocab, dtype, seed, noise=0.5, sd=3.0):
    g = torch.Generator().manual_seed(seed)
    z = sd * torch.randn(batch * (drafts + 1), vocab, generator=g)
    zd = z.view(batch, drafts + 1, vocab)[:, :drafts].reshape(batch * drafts, vocab)
    zd = (zd + noise * torch.randn(zd.shape, generator=g)).to(dtype)
    pick = torch.softmax(zd.double(), 1)
    x = torch.multinomial(pick, 1, generator=g).view(batch, drafts) if drafts else torch.zeros(batch, 0, dtype=torch.int64)
    return z.to(dtype), x, torch.rand(batch, drafts + 1, generator=g), zd


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


def same(got, want, size=40.0):
    tokens, count, logprob = [t.cpu() for t in got]
    assert torch.equal(count, want[1]), (count, want[1])
    assert torch.equal(tokens, want[0]), (tokens[tokens != want[0]], want[0][tokens != want[0]])
    lp = want[2]
    assert torch.equal(logprob.isinf(), lp.isinf())
    fine = lp.isfinite()
    off = (logprob.double() - lp)[fine].abs()
    assert (off <= 2.0 ** -24 * lp[fine].abs() + 1e-11 * size).all(), off.max()


def check(z, x, u, zd, lengths=None, scale=1.0, draft_scale=1.0):
    batch, more = u.shape
    v = head.VerifyDrafts(z.shape[1], batch, more - 1, logit_scale=scale, draft_scale=draft_scale)
    zc, xc, uc, zdc, lc = cuda(z, x, u, zd, lengths)
    got = v(zc, xc, uc, draft_logits=zdc, lengths=lc)
    same(got, oracle(z, x, u, zd, lengths, scale, draft_scale))
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 255, 2047, 2048, 2049, 5003, 16385])
def test_vocabularies(vocab, dtype):
    for drafts in (0, 3):
        z, x, u, zd = make(5, drafts, vocab, dtype, vocab + drafts)
        check(z, x, u, zd if drafts else None)
        if drafts:
            check(z, x, u, None)


@pytest.mark.parametrize("drafts", [0, 1, 2, 7, 16, 128])
@pytest.mark.parametrize("draft", [False, True])
def test_numbers_of_drafts(drafts, draft):
    z, x, u, zd = make(4, drafts, 300, torch.float32, drafts, noise=0.1)
    check(z, x, u, zd if draft and drafts else None, scale=0.8, draft_scale=1.3)


@pytest.mark.parametrize("batch", [1, 33, 257])
def test_batches(batch):
    """Few tiles, and enough of them for the larger ones (257 * 7 * 2 of 8,192)."""
    z, x, u, zd = make(batch, 3, 9000, torch.bfloat16, batch)
    got = check(z, x, u, zd)
    if batch > 30:  # some of each
        assert set(got[1].cpu().tolist()) == {0, 1, 2, 3}


def test_large_vocabulary():
    z, x, u, zd = make(6, 2, 152064, torch.bfloat16, 1)
    check(z, x, u, zd, scale=1 / 0.7, draft_scale=1 / 0.9)
    check(z.float(), x, u, None)


def test_more_segments_than_are_kept():
    """Vocabularies whose sums a wave does not hold at once: 512 entries a sum, 320 sums."""
    for vocab in (163841, 400003):
        z, x, u, zd = make(3, 1, vocab, torch.bfloat16, vocab, sd=1.0)
        check(z, x, u, zd)
        # the draw in the last entries
        z[:, :-300] = -math.inf
        check(z, x.clamp(min=vocab - 300), u, None)


def test_more_sequences_than_a_launch_takes():
    """2^22 units of work are one launch's."""
    n = (1 << 22) + 3
    z = torch.zeros(n, 2, device="cuda")
    z[:, 0] = -math.inf
    z[0, 0], z[n - 1, 1], z[n - 1, 0] = 0.0, -math.inf, 1.0
    u = torch.full((n, 1), 0.25, device="cuda")
    tokens, count, logprob = head.VerifyDrafts(2, n)(z, None, u)
    assert (count == 0).all() and (tokens[1:n - 1] == 1).all() and tokens[0] == 0 and tokens[n - 1] == 0
    assert (logprob[1:] == 0).all() and abs(logprob[0].item() + math.log(2)) < 1e-6


def test_lengths():
    z, x, u, zd = make(9, 4, 400, torch.float32, 2, noise=0.05)
    lengths = torch.tensor([0, 1, 2, 3, 4, -5, 99, 2, 0], dtype=torch.int32)
    check(z, x, u, zd, lengths)
    # rows past a sequence's length are not looked at
    for b in range(9):
        n = min(max(int(lengths[b]), 0), 4)
        z.view(9, 5, -1)[b, n + 1:] = float("nan")
        zd.view(9, 4, -1)[b, n:] = float("nan")
        x[b, n:] = 1 << 40
    check(z, x, u, zd, lengths)


def test_masked_entries_and_empty_rows():
    z, x, u, zd = make(12, 2, 3000, torch.float32, 3)
    z[:, ::3] = -math.inf                       # the target's mask, at drafted tokens too
    zd[:, 1::5] = -math.inf
    lowest = torch.finfo(torch.float32).min
    z[4, 1::3] = lowest
    z[3] = -math.inf                            # first target row of sequence 1
    z[6, 5] = float("nan")                      # first target row of sequence 2
    z[9, 7] = math.inf                          # first target row of sequence 3
    z[14] = -math.inf                           # last target row of sequence 4
    zd[10] = -math.inf                          # first draft row of sequence 5
    zd[12, 0] = float("nan")                    # first draft row of sequence 6
    z[21] = lowest                              # the lowest value throughout is a flat row
    got = check(z, x, u, zd)
    tokens, count, logprob = [t.cpu() for t in got]
    for b in (1, 2, 3):
        assert count[b] == 0 and tokens[b].tolist() == [-1, -1, -1] and logprob[b, 0] == -math.inf


def test_bfloat16_masks_of_the_lowest_value():
    z, x, u, zd = make(8, 2, 3000, torch.bfloat16, 4)
    z[:, 100:] = torch.finfo(torch.bfloat16).min
    check(z, x, u, zd)
    check(z, x.clamp(max=99), u, None)


FLAT = [0.3, -5.0, 77.0, -1e9, 3e20, -1e30, "lowest", "largest"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [1.0, 0.7, 1.3, 1e-20, 1e20])
def test_flat_rows_of_any_value(scale, dtype):
    """Equal logits have equal weights, whatever their size: u = v / 4096 gives v, and each
    logprob is log(1 / 4096) in FP32; where others lie far below they do not count."""
    vocab = 4096
    info = torch.finfo(dtype)
    values = [{"lowest": info.min, "largest": info.max}.get(v, v) for v in FLAT]
    v = torch.arange(len(values)) * 511
    z = torch.tensor(values).to(dtype)[:, None].repeat(1, vocab)
    u = (v.double() / vocab).float()[:, None]
    h = head.VerifyDrafts(2 * vocab, len(v), logit_scale=scale)
    for mask in (-math.inf, info.min):
        if mask == info.min:  # 1e-20 * 3e20 is not far
            z, v, u = (t[[0, 1, 2, 7]] for t in (z, v, u))
            if scale < 1e-3:
                continue
        wide = torch.cat([z, torch.full_like(z, mask)], 1)
        tokens, count, logprob = h(wide.cuda(), None, u.cuda())
        assert torch.equal(tokens.cpu()[:, 0], v)
        assert torch.equal(logprob.cpu(), torch.full((len(v), 1), -math.log(4096)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_only_token_has_a_logprob_of_zero(dtype):
    z = torch.tensor(FLAT[:-2] + [0.1, 0.7, 11.3, -0.01], dtype=torch.float64).to(dtype)[:, None]
    for scale in (1.0, 0.7, 1.3):
        h = head.VerifyDrafts(1, len(z), logit_scale=scale)
        tokens, count, logprob = h(z.cuda(), None, torch.full((len(z), 1), 0.5).cuda())
        assert (tokens == 0).all() and (logprob == 0).all()


def test_drafts_out_of_range_are_refused():
    z, x, u, zd = make(6, 2, 500, torch.float32, 5, noise=0.01)
    x[0, 0], x[1, 1], x[2, 0], x[3, 1], x[4, 0] = -1, 500, 1 << 33, -(1 << 40), -100
    check(z, x, u, zd)
    got = check(z, x, u, None)
    assert (got[1].cpu()[torch.tensor([0, 2, 4])] == 0).all()


def test_equal_weights_at_exact_borders():
    """4,096 equal logits: weights and their sums are exact, so u = v / 4096 lies on the
    border of v - 1 and v and belongs to v."""
    vocab = 4096
    v = torch.tensor([0, 1, 2, 7, 8, 63, 64, 511, 2047, 2048, 2049, 4095])
    u = (v.double() / vocab).float()[:, None]
    z = torch.zeros(len(v), vocab)
    h = head.VerifyDrafts(vocab, len(v))
    tokens, count, logprob = h(z.cuda(), None, u.cuda())
    assert torch.equal(tokens.cpu()[:, 0], v) and (count == 0).all()
    assert torch.equal(logprob.cpu(), torch.full((len(v), 1), -math.log(4096)))


def test_ends_of_the_range():
    """u = 0 draws the first entry that has a weight, the largest u below 1 the last (equal
    weights, so that it has 2^-12 of the sum); u out of range still draws an entry."""
    vocab = 4099
    z = torch.full((4, vocab), -math.inf)
    z[:, 3:4096] = 0.0
    u = torch.tensor([[0.0], [1 - 2.0 ** -24], [1.0], [float("nan")]])
    tokens, _, _ = head.VerifyDrafts(vocab, 4)(z.cuda(), None, u.cuda())
    assert tokens.cpu()[:, 0].tolist() == [3, 4095, 4095, 4095]


def test_the_same_logits_keep_every_draft():
    z, x, u, _ = make(16, 5, 1000, torch.bfloat16, 6)
    zd = z.view(16, 6, -1)[:, :5].reshape(80, -1)
    u[0, :5] = 1 - 2.0 ** -24
    got = check(z, x, u, zd)
    assert (got[1] == 5).all()
    # u = 1 refuses where p = q, and leaves nothing of p - q: drawn from p
    u[:, 0] = 1.0
    h = head.VerifyDrafts(1000, 16, 5)
    tokens, count, _ = h(z.cuda(), x.cuda(), u.cuda(), draft_logits=zd.cuda())
    want = head.VerifyDrafts(1000, 16)(z.view(16, 6, -1)[:, 0].cuda(), None, u[:, 5:].contiguous().cuda())
    assert (count == 0).all() and torch.equal(tokens[:, 0], want[0][:, 0])


def test_the_tokens_are_distributed_as_the_target():
    """20,000 sequences of one draft from another distribution over 8 tokens: the first
    token's frequencies lie within 5 standard deviations of p."""
    n, vocab = 20000, 8
    g = torch.Generator().manual_seed(7)
    zt, zd = torch.randn(2 * vocab, generator=g), torch.randn(vocab, generator=g)
    target = zt.view(1, 2, vocab).expand(n, 2, vocab).contiguous()
    x = torch.multinomial(torch.softmax(zd, 0).expand(n, vocab), 1, generator=g)
    u = torch.rand(n, 2, generator=g)
    h = head.VerifyDrafts(vocab, n, 1)
    tokens, count, _ = h(target.cuda(), x.cuda(), u.cuda(), draft_logits=zd.expand(n, vocab).contiguous().cuda())
    p = torch.softmax(zt[:vocab].double(), 0)
    seen = torch.bincount(tokens[:, 0].cpu(), minlength=vocab).double() / n
    assert ((seen - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n)).all()
    assert 0 < count.sum() < n


def test_strides_shapes_and_outputs():
    z, x, u, zd = make(5, 3, 1001, torch.float32, 8)
    want = oracle(z, x, u, zd, None, 1.0, 1.0)
    h = head.VerifyDrafts(1001, 8, 5)  # built for more
    for dtype in (torch.float32, torch.bfloat16):
        z, zd = z.to(dtype), zd.to(dtype)
        want = oracle(z, x, u, zd, None, 1.0, 1.0)
        same(h(z.view(5, 4, -1).cuda(), x.cuda(), u.cuda(), draft_logits=zd.view(5, 3, -1).cuda()), want)
        wide = torch.full((20, 1030), float("nan"), dtype=dtype, device="cuda")
        wide[:, 5:1006] = z.cuda()
        out = (torch.full((5, 4), 9, device="cuda"), torch.full((5,), 9, dtype=torch.int32, device="cuda"),
               torch.full((5, 4), 9.0, device="cuda"))
        got = h(wide[:, 5:1006], x.cuda(), u.cuda(), draft_logits=zd.cuda(), tokens=out[0], count=out[1], logprob=out[2])
        assert all(a.data_ptr() == b.data_ptr() for a, b in zip(got, out))
        same(got, want)
    # no sequences
    e = head.VerifyDrafts(10, 1)(torch.empty(0, 10, device="cuda"), None, torch.empty(0, 1, device="cuda"))
    assert [t.shape[0] for t in e] == [0, 0, 0]


def test_calls_of_all_sizes_share_a_workspace():
    h = head.VerifyDrafts(20000, 40, 6)
    for batch, drafts in ((40, 6), (1, 0), (40, 0), (3, 6), (17, 2)):
        z, x, u, zd = make(batch, drafts, 20000, torch.bfloat16, batch)
        got = h(z.cuda(), x.cuda(), u.cuda(), draft_logits=zd.cuda() if drafts else None)
        same(got, oracle(z, x, u, zd if drafts else None, None, 1.0, 1.0))


def test_a_graph_replays_it():
    z, x, u, zd = make(7, 3, 5000, torch.bfloat16, 9)
    h = head.VerifyDrafts(5000, 7, 3)
    zc, xc, uc, zdc = cuda(z, x, u, zd)
    h(zc, xc, uc, draft_logits=zdc)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = h(zc, xc, uc, draft_logits=zdc)
    for seed in (10, 11, 12):
        z, x, u, zd = make(7, 3, 5000, torch.bfloat16, seed)
        for to, t in zip((zc, xc, uc, zdc), (z, x, u, zd)):
            to.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        same(out, oracle(z, x, u, zd, None, 1.0, 1.0))


def test_another_stream():
    z, x, u, zd = make(7, 3, 5000, torch.bfloat16, 13)
    h = head.VerifyDrafts(5000, 7, 3)
    zc, xc, uc, zdc = cuda(z, x, u, zd)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = h(zc, xc, uc, draft_logits=zdc, stream=side)
    side.synchronize()
    same(got, oracle(z, x, u, zd, None, 1.0, 1.0))


def test_drafts_before_sequences_are_refused():
    z, x, u, zd = cuda(*make(3, 1, 50, torch.float32, 15))
    h = head.VerifyDrafts(50, 3, 2)
    good = h(z.view(3, 2, 50), x, u, draft_logits=zd.view(3, 1, 50))
    assert all(torch.equal(a, b) for a, b in zip(good, h(z, x.view(-1), u, draft_logits=zd)))
    with pytest.raises(pulse.PulseError, match="target must"):
        h(z.view(2, 3, 50), x, u)
    with pytest.raises(pulse.PulseError, match="draft_logits must"):
        h(z, x, u, draft_logits=zd.view(1, 3, 50))
    with pytest.raises(pulse.PulseError, match="drafts must"):
        h(z, x.view(1, 3), u)


def test_refusals():
    z, x, u, zd = cuda(*make(3, 2, 50, torch.float32, 14))
    h = head.VerifyDrafts(50, 3, 2)
    for bad, word in ((dict(vocab=0, max_batch=1), "vocabulary"), (dict(vocab=5, max_batch=0), "batch"),
                      (dict(vocab=5, max_batch=1, max_drafts=129), "drafts"),
                      (dict(vocab=5, max_batch=1 << 31), "batch")):
        with pytest.raises(pulse.PulseError, match=word):
            head.VerifyDrafts(**bad)
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(pulse.PulseError, match="scale"):
            head.VerifyDrafts(50, 3, 2, logit_scale=scale)(z, x, u, draft_logits=zd)
    with pytest.raises(pulse.PulseError, match="built for"):
        head.VerifyDrafts(50, 2, 2)(z, x, u)
    with pytest.raises(pulse.PulseError, match="built for"):
        head.VerifyDrafts(50, 3, 1)(z, x, u)
    with pytest.raises(pulse.PulseError, match="target must"):
        h(z[:5], x, u)
    with pytest.raises(pulse.PulseError, match="target must"):
        h(z.half(), x, u)
    with pytest.raises(pulse.PulseError, match="draft_logits must"):
        h(z, x, u, draft_logits=zd.bfloat16())
    with pytest.raises(pulse.PulseError, match="drafts"):
        h(z, None, u)
    with pytest.raises(pulse.PulseError, match="drafts"):
        h(z, x.int(), u)
    with pytest.raises(pulse.PulseError, match="lengths"):
        h(z, x, u, lengths=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(pulse.PulseError, match="uniform"):
        h(z, x, u.view(-1))
    with pytest.raises(pulse.PulseError, match="uniform"):
        h(z, x, u.double())
    with pytest.raises(pulse.PulseError, match="equally"):
        h(torch.zeros(3, 6, 50, device="cuda")[:, :3], x, u)
