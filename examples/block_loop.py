"""A block trained on one side, drafting from codes and verified on the other.

    python examples/block_loop.py [--form mxfp4|fp8] [--steps N]

The model is a gated MLP block over token embeddings, which learns a chain of
tokens: norm, gate and up projections, their product, down projection, the block's
output normalised and added to the stream, the stream normalised, head.  The
trainer takes the gradient of the next token's cross entropy, steps FP32 masters, and
sends the receiver the values whose FP8 or MXFP4 view changed.  The receiver drafts a
few tokens from its codes, one after the other; the BF16 policy looks at all of them
at once and keeps those that its own probabilities allow, with one more of its own.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2602_03839_amd import head, pulse  # noqa: E402

MATRICES = ("gate", "up", "down", "head")
SCALE = 0.7  # of the residual stream


class Policy:
    """The BF16 model and its gradient, from FP32 masters."""

    def __init__(self, master, max_tokens):
        self.master = master
        self.bf16 = {k: pulse.cast_bf16(v).view(torch.bfloat16).view(v.shape) for k, v in master.items() if v.dim() == 2}
        w = self.bf16
        self.norm = head.LayerNorm(master["norm"], rms=True)
        self.join = head.BlockNorm(master["last"], post_weight=master["post"], residual_scale=SCALE)
        # one workspace for all: their calls follow each other
        need = max(head.linear_workspace_bytes(max_tokens, *w[k].shape) for k in MATRICES)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.gate, self.up, self.down, self.head = (
            head.Linear(w[k], max_tokens=max_tokens, activation="silu" if k == "gate" else None, workspace=ws)
            for k in MATRICES)
        self.ce = head.LinearCE(w["head"], max_tokens=max_tokens)

    def hidden(self, tokens, keep=False):
        h = self.bf16["embed"][tokens]
        x, _, rstd = self.norm(h)
        up = self.up(x)
        g, pre = self.gate(x, times=up, keep_pre=True)
        b = self.down(g)
        y, h_out, stats = self.join(b, h)
        return (y, (h, x, rstd, up, g, pre, b, h_out, stats)) if keep else y

    def logits(self, tokens):
        return self.head(self.hidden(tokens))

    def gradients(self, tokens, targets):
        """(mean loss, {name: gradient}) of the next tokens' cross entropy."""
        y, (h, x, rstd, up, g, pre, b, h_out, stats) = self.hidden(tokens, keep=True)
        loss, lse = self.ce.forward(y, targets)
        dloss = torch.full_like(loss, 1.0 / len(tokens))
        grad = {}
        dy, grad["head"] = self.ce.backward(y, targets, lse, dloss)
        db, dh, grad["last"], _, grad["post"], _, _ = self.join.backward(dy, None, b, h_out, stats)
        dg, grad["down"], _, _ = self.down.backward(db, g)
        dx, grad["gate"], _, dup = self.gate.backward(dg, x, pre=pre, times=up)
        dx_up, grad["up"], _, _ = self.up.backward(dup, x)
        dh_norm, grad["norm"], _ = self.norm.backward(dx + dx_up, h, None, rstd)
        grad["embed"] = torch.zeros_like(self.master["embed"])
        grad["embed"].index_add_(0, tokens, dh.float() + dh_norm.float())
        return loss.mean(), grad

    def step(self, grad, lr):
        for k, v in self.master.items():
            v -= lr * grad[k].float()
            if v.dim() == 2:
                pulse.cast_bf16(v, out=self.bf16[k])


class Drafter:
    """The receiver: the block's matrices as codes, brought up to date by patches."""

    def __init__(self, form, codes, policy, inv_scale, batch):
        self.codes = {k: (c.clone(), None if s is None else s.clone()) for k, (c, s) in codes.items()}
        self.small = {k: policy.master[k].clone() for k in ("norm", "last", "post")}
        self.embed = policy.bf16["embed"].clone()
        self.norm = head.LayerNorm(self.small["norm"], rms=True)
        self.join = head.BlockNorm(self.small["last"], post_weight=self.small["post"], residual_scale=SCALE)
        for k in MATRICES:
            rows, cols = policy.master[k].shape
            setattr(self, k, head.LowpLinear(form, *self.codes[k], rows, cols, inv_scale,
                                             activation="silu" if k == "gate" else None))
        self.sample = head.VerifyDrafts(policy.master["head"].shape[0], max_batch=batch)
        self.apply = pulse.ApplyLowpBatch(form, [pulse.LowpApplyTensor(*self.codes[k], policy.master[k].numel())
                                                 for k in MATRICES])

    def patch(self, idx, val, seg, count, policy):
        self.apply(idx, val, seg, count)
        for k, v in self.small.items():
            v.copy_(policy.master[k])
        self.embed.copy_(policy.bf16["embed"])

    def logits(self, tokens):
        h = self.embed[tokens]
        x, _, _ = self.norm(h)
        up = self.up(x, out_dtype=torch.bfloat16)
        g = self.gate(x, out=up, times=up)  # in place of the multiplier
        b = self.down(g, out_dtype=torch.bfloat16)
        y, _, _ = self.join(b, h, h_out=h, keep_stats=False)
        return self.head(y, out_dtype=torch.bfloat16)

    def draft(self, last, count, uniform):
        """`count` tokens after `last` [batch], and the logits they were drawn from."""
        tokens, logits = [last], []
        for k in range(count):
            z = self.logits(tokens[-1])
            tokens.append(self.sample(z, None, uniform[:, k:k + 1].contiguous())[0][:, 0])
            logits.append(z)
        return torch.stack(tokens, 1), torch.stack(logits, 1)


def masters(vocab, hidden, inner, g):
    def normal(rows, cols):
        return torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5

    return {"embed": torch.randn(vocab, hidden, generator=g, device="cuda"), "gate": normal(inner, hidden),
            "up": normal(inner, hidden), "down": normal(hidden, inner), "head": normal(vocab, hidden),
            "norm": torch.ones(hidden, device="cuda"), "post": torch.ones(hidden, device="cuda"),
            "last": torch.ones(hidden, device="cuda")}


def run(form=pulse.MXFP4, steps=20, vocab=512, hidden=256, inner=512, tokens=192, batch=16, drafts=4, lr=1.0, seed=0):
    """Trains, sends, drafts and verifies; a list of {loss, sent, taken} per step: the
    mean loss, the share of the matrices' values that were sent, and the drafts that the
    policy kept, of those it was shown."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    policy = Policy(masters(vocab, hidden, inner, g), tokens)
    follows = torch.randperm(vocab, generator=g, device="cuda")  # the chain that is learnt
    inv_scale = 64.0 if form == pulse.FP8_E4M3 else 1.0
    codes = {k: pulse.cast_lowp(form, policy.master[k].view(-1), inv_scale) for k in MATRICES}
    drafter = Drafter(form, codes, policy, inv_scale, batch)
    verify = head.VerifyDrafts(vocab, batch, drafts)

    n = sum(policy.master[k].numel() for k in MATRICES)
    idx = torch.empty(n, dtype=torch.int32, device="cuda")
    val = torch.empty(n, dtype=torch.uint8 if form == pulse.FP8_E4M3 else torch.int16, device="cuda")
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    seg = torch.zeros(len(MATRICES), dtype=torch.int64, device="cuda")
    ws = pulse.workspace()
    encode = pulse.EncodeLowpBatch(form, [pulse.LowpTensor(policy.master[k].view(-1), *codes[k], inv_scale=inv_scale)
                                          for k in MATRICES])
    keep_up = pulse.ApplyLowpBatch(form, [pulse.LowpApplyTensor(*codes[k], policy.master[k].numel()) for k in MATRICES])

    log = []
    for _ in range(steps):
        here = torch.randint(vocab, (tokens,), generator=g, device="cuda")
        loss, grad = policy.gradients(here, follows[here])
        policy.step(grad, lr)
        count.zero_()
        encode(idx, val, count, ws, seg_begin=seg)
        keep_up(idx, val, seg, count)
        drafter.patch(idx, val, seg, count, policy)

        last = torch.randint(vocab, (batch,), generator=g, device="cuda")
        uniform = torch.rand(batch, 2 * drafts + 1, generator=g, device="cuda")
        seen, zd = drafter.draft(last, drafts, uniform[:, :drafts])
        z = policy.logits(seen.view(-1))  # the policy's rows for the last token and all drafts at once
        out, taken, logprob = verify(z.view(batch, drafts + 1, vocab), seen[:, 1:].contiguous(),
                                     uniform[:, drafts:].contiguous(), draft_logits=zd)
        assert (out.gather(1, taken.long()[:, None]) >= 0).all() and (logprob <= 0).all()
        log.append({"loss": loss.item(), "sent": count.item() / n, "taken": taken.float().mean().item() / drafts})
    pulse.check_workspace(ws)
    for k in MATRICES:
        assert torch.equal(drafter.codes[k][0], codes[k][0])
    return log


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--form", choices=("mxfp4", "fp8"), default="mxfp4")
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    for k, r in enumerate(run(pulse.MXFP4 if a.form == "mxfp4" else pulse.FP8_E4M3, a.steps)):
        print(f"step {k:3d}  loss {r['loss']:7.4f}  sent {r['sent']:7.2%}  drafts kept {r['taken']:7.2%}")
