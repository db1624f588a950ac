"""The operators between blocks together, as a trainer and a receiver use them
(examples/block_loop.py): it runs, its gradients are the chain's, drafting and verifying
as one captured graph."""
import importlib.util
import os

import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "block_loop.py")


def example():
    spec = importlib.util.spec_from_file_location("block_loop", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("form", [pulse.MXFP4, pulse.FP8_E4M3])
def test_it_runs(form):
    log = example().run(form, steps=4)
    assert len(log) == 4
    assert all(0 < r["sent"] <= 1 and 0 <= r["taken"] <= 1 and r["loss"] == r["loss"] for r in log)


def rms(v, w):
    r = torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6)
    return v * r * w


@pytest.mark.parametrize("tokens", [16, 100, 700])
def test_gradients_of_the_chain(tokens):
    """Against autograd in 64 bits on the same BF16 weights.  On its way from the loss a
    gradient is rounded to BF16 at most a dozen times (each activation and gradient
    tensor and each product's operand once), each by at most 2^-8 / sqrt 3 of its root mean
    square and independently of the others: sqrt 12 times 0.00226, 0.008, of the whole;
    through the norms and the gate, whose other factors are rounded as well, up to twice
    that."""
    m = example()
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    vocab, hidden, inner = 500, 136, 264
    policy = m.Policy(m.masters(vocab, hidden, inner, g), tokens)
    here = torch.randint(vocab, (tokens,), generator=g, device="cuda")
    there = torch.randint(vocab, (tokens,), generator=g, device="cuda")
    there[::5] = -1  # ignored
    loss, grad = policy.gradients(here, there)

    p = {k: (policy.bf16[k] if v.dim() == 2 else v).double().requires_grad_() for k, v in policy.master.items()}
    h = p["embed"][here]
    x = rms(h, p["norm"])
    u = x @ p["gate"].t()
    b = (u * torch.sigmoid(u) * (x @ p["up"].t())) @ p["down"].t()
    y = rms(m.SCALE * h + rms(b, p["post"]), p["last"])
    kept = there >= 0
    logp = torch.log_softmax(y @ p["head"].t(), 1)
    want = -(logp.gather(1, there.clamp(min=0)[:, None])[:, 0] * kept).sum() / tokens
    want.backward()
    assert abs(loss.item() - want.item()) <= 0.004 * want.item()
    for k, v in p.items():
        off = (grad[k].double() - v.grad).norm() / v.grad.norm()
        assert off <= 0.016, (k, off.item())


def test_drafting_and_verifying_as_a_graph():
    """Three drafted tokens, each sampled from the one before, and their verification,
    captured once and replayed on new tokens and numbers."""
    m = example()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    vocab, batch, drafts = 1000, 8, 3
    policy = m.Policy(m.masters(vocab, 128, 256, g), 64)
    codes = {k: pulse.cast_lowp(pulse.MXFP4, policy.master[k].view(-1), 1.0) for k in m.MATRICES}
    drafter = m.Drafter(pulse.MXFP4, codes, policy, 1.0, batch)
    verify = head.VerifyDrafts(vocab, batch, drafts)
    last = torch.zeros(batch, dtype=torch.int64, device="cuda")
    uniform = torch.zeros(batch, 2 * drafts + 1, device="cuda")

    def answer():
        seen, zd = drafter.draft(last, drafts, uniform)
        z = policy.logits(seen.view(-1))
        return verify(z.view(batch, drafts + 1, vocab), seen[:, 1:].contiguous(), uniform[:, drafts:].contiguous(),
                      draft_logits=zd)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        answer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = answer()
    counts = set()
    for _ in range(5):
        last.copy_(torch.randint(vocab, (batch,), generator=g, device="cuda"))
        uniform.copy_(torch.rand(uniform.shape, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, answer()):
            assert torch.equal(a, b)
        counts.update(got[1].tolist())
    assert len(counts) > 1 and max(counts) <= drafts
