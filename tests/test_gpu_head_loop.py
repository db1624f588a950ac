"""The operators at a model's output end together, as a trainer and a receiver use
them: the loss falls, and the receiver answers from its patched codes."""
import importlib.util
import os

import pytest
import torch

from paper_2602_03839_amd import head, pulse

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "head_loop.py")


def example():
    spec = importlib.util.spec_from_file_location("head_loop", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("form", [pulse.MXFP4, pulse.FP8_E4M3])
def test_loop_learns_and_the_receiver_follows(form):
    log = example().run(form, steps=30)
    # 2,048 entries: ln 2048 = 7.6 at the start
    assert log[0]["loss"] > 6.5 and log[-1]["loss"] < 0.7 * log[0]["loss"], log
    assert all(0 < r["sent"] <= 1 for r in log)
    assert log[-1]["agree"] > 0.5, log[-1]


@pytest.mark.parametrize("tokens", [40, 300])
def test_a_step_as_a_graph(tokens):
    """Norm, loss and gradients captured once and replayed on new inputs, with eager calls
    between, give the eager calls' bits: nothing is left from one replay to the next.
    Half the probability lies beside the target, so that large entries of G are listed."""
    vocab, hidden = 3000, 192
    g = torch.Generator(device="cuda").manual_seed(tokens)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    w = (normal(vocab, hidden) / 4).bfloat16()
    norm, ce = head.LayerNorm(torch.ones(hidden, device="cuda"), rms=True), head.LinearCE(w, max_tokens=tokens)
    x, y = torch.zeros(tokens, hidden, dtype=torch.bfloat16, device="cuda"), torch.zeros(tokens, dtype=torch.int64, device="cuda")
    dl = torch.zeros(tokens, device="cuda")

    def new_inputs():
        x.copy_((normal(tokens, hidden) + 4 * w[torch.randint(vocab, (tokens,), generator=g, device="cuda")].float()).bfloat16())
        y.copy_(torch.randint(-1, vocab, (tokens,), generator=g, device="cuda"))
        dl.copy_(normal(tokens))

    def step():
        h, _, rstd = norm(x)
        loss, lse = ce.forward(h, y)
        dh, dw = ce.backward(h, y, lse, dl)
        dx, dgain, _ = norm.backward(dh, x, None, rstd)
        return loss, lse, dh, dw, dx, dgain

    new_inputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        new_inputs()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
        assert torch.isfinite(got[2]).all() and got[2].abs().max() > 0
