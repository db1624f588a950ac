"""A model's output end, trained on one side and answering on the other.

    python examples/head_loop.py [--form mxfp4|fp8] [--steps N]

The trainer holds FP32 masters of the last norm's gain and of the head.  Each
step it normalises the hidden states, takes the cross entropy of the head's
logits and its gradient (nothing of the size tokens x vocabulary is stored),
steps the masters, and sends the receiver the values whose FP8 or MXFP4 view
changed.  The receiver patches its codes in place and answers the same hidden
states from them.  Hidden states are synthetic: noisy copies of one random
direction per class.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_03839_amd import head, pulse  # noqa: E402


class Receiver:
    """Codes of the head and the norm's gain, brought up to date by patches."""

    def __init__(self, form, codes, scales, gain, vocab, hidden, inv_scale):
        self.codes, self.scales = codes.clone(), None if scales is None else scales.clone()
        self.norm = head.LayerNorm(gain.clone(), rms=True)
        self.head = head.LowpLinear(form, self.codes, self.scales, vocab, hidden, inv_scale)
        self.apply = pulse.ApplyLowpBatch(
            form, [pulse.LowpApplyTensor(self.codes, self.scales, vocab * hidden)])

    def patch(self, idx, val, seg, count, gain):
        self.apply(idx, val, seg, count)
        self.norm.weight.copy_(gain)

    def logits(self, x):
        return self.head(self.norm(x)[0])


def run(form=pulse.MXFP4, steps=20, vocab=2048, hidden=256, tokens=192, lr=0.5, seed=0):
    """Trains and answers; a list of {loss, sent, agree} per step: the mean loss, the
    share of the head's values that were sent, and the share of tokens where the
    receiver's best entry is the target."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    classes = torch.randn(vocab, hidden, generator=g, device="cuda")
    master = 0.02 * torch.randn(vocab, hidden, generator=g, device="cuda")
    gain = torch.ones(hidden, device="cuda")
    n = vocab * hidden
    inv_scale = 64.0 if form == pulse.FP8_E4M3 else 1.0

    bf16 = pulse.cast_bf16(master).view(torch.bfloat16)
    norm = head.LayerNorm(gain, rms=True)
    ce = head.LinearCE(bf16, max_tokens=tokens)
    codes, scales = pulse.cast_lowp(form, master, inv_scale)
    receiver = Receiver(form, codes, scales, gain, vocab, hidden, inv_scale)

    idx = torch.empty(n, dtype=torch.int32, device="cuda")
    val = torch.empty(n, dtype=torch.uint8 if form == pulse.FP8_E4M3 else torch.int16, device="cuda")
    count, seg = (torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2))
    ws = pulse.workspace()
    # the trainer's snapshot of the receiver: the codes it sent last
    encode = pulse.EncodeLowpBatch(form, [pulse.LowpTensor(master, codes, scales, inv_scale=inv_scale)])
    keep_up = pulse.ApplyLowpBatch(form, [pulse.LowpApplyTensor(codes, scales, n)])

    log = []
    for _ in range(steps):
        target = torch.randint(vocab // 8, (tokens,), generator=g, device="cuda")
        noise = torch.randn(tokens, hidden, generator=g, device="cuda")
        x = (classes[target] + 0.25 * noise).bfloat16()
        target[::16] = -100  # a prompt's tokens: no loss

        y, _, rstd = norm(x)
        loss, lse = ce.forward(y, target)
        kept = target >= 0
        dloss = kept.float() / kept.sum()
        dy, dhead = ce.backward(y, target, lse, dloss)
        _, dgain, _ = norm.backward(dy, x, None, rstd)

        master -= lr * dhead.float()
        gain -= 0.1 * lr * dgain
        pulse.cast_bf16(master, out=bf16)

        count.zero_()
        encode(idx, val, count, ws, seg_begin=seg)
        keep_up(idx, val, seg, count)
        receiver.patch(idx, val, seg, count, gain)

        best = receiver.logits(x).argmax(1)
        log.append({"loss": loss.sum().item() / int(kept.sum()), "sent": count.item() / n,
                    "agree": (best == target)[kept].float().mean().item()})
    pulse.check_workspace(ws)
    assert torch.equal(receiver.codes, codes)
    return log


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--form", choices=("mxfp4", "fp8"), default="mxfp4")
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    for k, r in enumerate(run(pulse.MXFP4 if a.form == "mxfp4" else pulse.FP8_E4M3, a.steps)):
        print(f"step {k:3d}  loss {r['loss']:7.4f}  sent {r['sent']:7.2%}  receiver right {r['agree']:7.2%}")
