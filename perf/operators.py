"""Timed cases of the operators at a model's output end, on both sides of a patch.

The trainer normalises the last hidden states, takes the cross entropy of the
head's logits and its gradient; a receiver multiplies its few current tokens
with weights it holds as FP8 or MXFP4 codes.  A case is

  op       "norm_fwd"   head.LayerNorm forward        (y, mean, rstd)
           "norm_bwd"   head.LayerNorm.backward       (dx, dweight, dbias)
           "ce_fwd"     head.LinearCE.forward         (loss, lse per token)
           "ce_train"   forward, then backward        (loss, lse, dx, dweight)
           "lowp"       head.LowpLinear               (y)
  norm:    rows, cols, dtype ("bf16", "f32") of the activations, rms
  ce:      tokens, vocab, hidden; BF16 activations and head weight
  lowp:    tokens, rows, cols (the weight is [rows, cols]), form ("mxfp4",
           "fp8"), out ("f32", "bf16"); BF16 activations

Sizes are those of the parameter sets in ``workloads.SHAPES`` (hidden 896, 3584
and 5120 with their vocabularies and MLP widths) or ragged ones in between.

With ``own`` false ``run`` computes the definitions with elementary torch
operations in 32 bits; with ``own`` true it calls the package.
"""
import math

import torch

own = False

EPS = 1e-6
IGNORE = -100
OPS = ("norm_fwd", "norm_bwd", "ce_fwd", "ce_train", "lowp")
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
LARGEST = 4096 * 152064 * 3584  # tokens * vocab * hidden of the largest training case


def listed():
    return [
        # one decoded token's norm: all latency
        {"name": "norm_fwd_1x5120", "op": "norm_fwd", "rows": 1, "cols": 5120, "dtype": "bf16",
         "rms": True},
        # a trainer's packed batch before the head
        {"name": "norm_fwd_16384x3584", "op": "norm_fwd", "rows": 16384, "cols": 3584,
         "dtype": "bf16", "rms": False},
        # its gradient
        {"name": "norm_bwd_16384x3584", "op": "norm_bwd", "rows": 16384, "cols": 3584,
         "dtype": "bf16", "rms": True},
        # a small FP32 run with odd sizes
        {"name": "norm_bwd_f32_1027x897", "op": "norm_bwd", "rows": 1027, "cols": 897,
         "dtype": "f32", "rms": False},
        # log-probabilities of a rollout under the reference weights: no gradient
        {"name": "ce_fwd_2048_0p5b", "op": "ce_fwd", "tokens": 2048, "vocab": 151936,
         "hidden": 896},
        # a trainer's micro-batch at the 7B head: the largest
        {"name": "ce_train_4096_7b", "op": "ce_train", "tokens": 4096, "vocab": 152064,
         "hidden": 3584},
        # one short sequence at the 32B head: few tokens against a weight of 1.6 GB
        {"name": "ce_train_61_32b", "op": "ce_train", "tokens": 61, "vocab": 152064,
         "hidden": 5120},
        # a byte-pair toy model with odd sizes
        {"name": "ce_train_77_odd", "op": "ce_train", "tokens": 77, "vocab": 5003, "hidden": 203},
        # one token through the smallest projection (k_proj of the 0.5B set): all latency
        {"name": "mxfp4_1_kproj_0p5b", "op": "lowp", "tokens": 1, "rows": 128, "cols": 896,
         "form": "mxfp4", "out": "bf16"},
        # one token through the 7B set's down_proj
        {"name": "mxfp4_1_down_7b", "op": "lowp", "tokens": 1, "rows": 3584, "cols": 18944,
         "form": "mxfp4", "out": "bf16"},
        # a served batch's logits at the 32B head
        {"name": "mxfp4_16_head_32b", "op": "lowp", "tokens": 16, "rows": 152064, "cols": 5120,
         "form": "mxfp4", "out": "f32"},
        # a ragged batch through an FP8 receiver's up_proj
        {"name": "fp8_5_up_7b", "op": "lowp", "tokens": 5, "rows": 18944, "cols": 3584,
         "form": "fp8", "out": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, unit):
    """A width between lo and hi: three in four a multiple of `unit`, as models have them."""
    n = _log(rng, lo, hi)
    n = max(lo, n // unit * unit) if rng.random() < 0.75 else n | 1
    return n + unit if n == 3 << 10 else n


def draw(rng):
    op = rng.choice(OPS)
    if op.startswith("norm"):
        return {"op": op, "rows": _log(rng, 1, 16384), "cols": _width(rng, 64, 8192, 64),
                "dtype": rng.choice(("bf16", "bf16", "f32")), "rms": rng.random() < 0.5}
    if op.startswith("ce"):
        hidden, vocab = _width(rng, 64, 5120, 64), _log(rng, 256, 152064)
        return {"op": op, "tokens": min(_log(rng, 1, 8192), LARGEST // (vocab * hidden)),
                "vocab": vocab, "hidden": hidden}
    cols = _width(rng, 64, 27648, 32)
    return {"op": op, "tokens": _log(rng, 1, 64),
            "rows": min(_log(rng, 64, 152064), 152064 * 5120 // cols), "cols": cols,
            "form": rng.choice(("mxfp4", "mxfp4", "fp8")), "out": rng.choice(("f32", "bf16"))}


DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _mxfp4(w):
    """Codes (two a byte, the even value in the low nibble) and E8M0 scale bytes
    of a flat FP32 tensor in blocks of 32, the block's scale from its largest
    magnitude."""
    n = w.numel()
    pad = torch.zeros((n + 31) // 32 * 32, device=w.device)
    pad[:n] = w
    b = pad.view(-1, 32)
    e = (torch.frexp(b.abs().amax(1)).exponent - 3).clamp(-127, 127)
    q = torch.ldexp(b, -e[:, None]).flatten()
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    code = torch.bucketize(q.abs(), edges, out_int32=True).to(torch.uint8)
    code |= (q < 0).to(torch.uint8) << 3
    code = code[:(n + 1) // 2 * 2].view(-1, 2)
    return code[:, 0] | (code[:, 1] << 4), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"op": op}
    if op.startswith("norm"):
        rows, cols, dt = case["rows"], case["cols"], DTYPE[case["dtype"]]
        # residual-stream rows: a common offset, rows of different size
        x = (normal(rows, cols) + 0.25) * (0.5 + 2 * torch.rand(rows, 1, generator=g, device="cuda"))
        s.update(rms=case["rms"], x=x.to(dt), weight=1 + 0.1 * normal(cols),
                 bias=None if case["rms"] else 0.1 * normal(cols))
        if op == "norm_bwd":
            s["dy"] = (0.01 * normal(rows, cols)).to(dt)
            # what the forward pass left
            xf = s["x"].float()
            s["mean"] = None if case["rms"] else xf.mean(1)
            if not case["rms"]:
                xf = xf - s["mean"][:, None]
            s["rstd"] = torch.rsqrt((xf * xf).mean(1) + EPS)
    elif op.startswith("ce"):
        tokens, vocab, hidden = case["tokens"], case["vocab"], case["hidden"]
        # logits of sd 2.8, and targets from hardly to rather likely
        w = torch.empty(vocab, hidden, dtype=torch.bfloat16, device="cuda")
        w.normal_(0.0, 2.5 / math.sqrt(hidden), generator=g)
        y = torch.randint(vocab, (tokens,), generator=g, device="cuda")
        sure = (math.log(vocab) + 5) / 7 * torch.rand(tokens, 1, generator=g, device="cuda")
        s.update(weight=w, x=(normal(tokens, hidden) + sure * w[y].float()).to(torch.bfloat16),
                 # one target in eight belongs to a prompt and has no loss
                 targets=torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.125,
                                     torch.full_like(y, IGNORE), y),
                 # advantage over the number of tokens
                 dloss=normal(tokens) / tokens, scale=1.0 / 0.9)
    else:
        rows, cols, form = case["rows"], case["cols"], case["form"]
        w = normal(rows * cols) * 0.02
        s.update(rows=rows, cols=cols, form=form, out=DTYPE[case["out"]], inv_scale=1.0,
                 scales=None, x=normal(case["tokens"], cols).to(torch.bfloat16))
        if form == "mxfp4":
            s["codes"], s["scales"] = _mxfp4(w)
        else:
            s["inv_scale"] = 448.0 / 0.125
            s["codes"] = (w * s["inv_scale"]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    if own:  # the handle that a program keeps beside its weights
        from paper_2602_03839_amd import head, pulse
        if op.startswith("norm"):
            s["handle"] = head.LayerNorm(s["weight"], s["bias"], eps=EPS, rms=s["rms"])
        elif op.startswith("ce"):
            s["handle"] = head.LinearCE(s["weight"], max_tokens=case["tokens"],
                                        logit_scale=s["scale"])
        else:
            s["handle"] = head.LowpLinear(pulse.MXFP4 if s["form"] == "mxfp4" else pulse.FP8_E4M3,
                                          s["codes"], s["scales"], s["rows"], s["cols"],
                                          inv_scale=s["inv_scale"])
    return s


def _decode(codes, scales, n, inv_scale):
    """The FP32 values of a receiver's codes."""
    if scales is None:
        return codes.view(torch.float8_e4m3fn).float() / inv_scale
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    nib = torch.stack((codes & 15, codes >> 4), 1).flatten()[:n].int()
    step = torch.exp2(scales.float() - 127)
    return table[nib] * step.repeat_interleave(32)[:n]


def _own(s):
    op, h = s["op"], s["handle"]
    if op == "norm_fwd":
        y, mean, rstd = h(s["x"])
        return {"y": y, "rstd": rstd} if mean is None else {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        dx, dw, db = h.backward(s["dy"], s["x"], s["mean"], s["rstd"])
        return {"dx": dx, "dw": dw} if db is None else {"dx": dx, "dw": dw, "db": db}
    if op == "lowp":
        return {"y": h(s["x"], out_dtype=s["out"])}
    loss, lse = h.forward(s["x"], s["targets"])
    if op == "ce_fwd":
        return {"loss": loss, "lse": lse}
    dx, dw = h.backward(s["x"], s["targets"], lse, s["dloss"])
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def run(state):
    s = state
    if own:
        return _own(s)
    op = s["op"]
    if op == "lowp":
        w = _decode(s["codes"], s["scales"], s["rows"] * s["cols"], s["inv_scale"])
        return {"y": (s["x"].float() @ w.view(s["rows"], s["cols"]).t()).to(s["out"])}
    if op == "norm_fwd":
        xf, out = s["x"].float(), {}
        if not s["rms"]:
            out["mean"] = xf.mean(1)
            xf = xf - out["mean"][:, None]
        out["rstd"] = torch.rsqrt((xf * xf).mean(1) + EPS)
        y = xf * out["rstd"][:, None] * s["weight"]
        out["y"] = (y if s["rms"] else y + s["bias"]).to(s["x"].dtype)
        return out
    if op == "norm_bwd":
        dy, r, xf = s["dy"].float(), s["rstd"][:, None], s["x"].float()
        xh = (xf if s["rms"] else xf - s["mean"][:, None]) * r
        a = dy * s["weight"]
        t = a - xh * (a * xh).mean(1, keepdim=True)
        if not s["rms"]:
            t = t - a.mean(1, keepdim=True)
        out = {"dx": (t * r).to(s["x"].dtype), "dw": (dy * xh).sum(0)}
        return out if s["rms"] else {**out, "db": dy.sum(0)}
    x, w, y = s["x"].float(), s["weight"].float(), s["targets"]
    z = (x @ w.t()) * s["scale"]
    top = z.amax(1)
    kept = y >= 0
    at = torch.where(kept, y, 0)[:, None]
    hit = z.gather(1, at)[:, 0]
    z = torch.exp(z - top[:, None])
    total = z.sum(1)
    rest = torch.log(total)
    out = {"loss": torch.where(kept, (top - hit) + rest, 0.0), "lse": top + rest}
    if op == "ce_train":
        by = torch.where(kept, s["dloss"], 0.0) * s["scale"]
        z *= (by / total)[:, None]
        z.scatter_add_(1, at, -by[:, None])
        out["dx"] = (z @ w).to(torch.bfloat16)
        out["dw"] = (z.t() @ x).to(torch.bfloat16)
    return out


def work(case):
    op = case["op"]
    if op.startswith("norm"):
        n, size = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        stats = 4 * case["rows"] * (1 if case["rms"] else 2)
        vec = 4 * case["cols"] * (1 if case["rms"] else 2)
        if op == "norm_fwd":
            return {"bytes": 2 * n * size + vec + stats, "flops": 8 * n}
        return {"bytes": 3 * n * size + 4 * case["cols"] + vec + stats, "flops": 14 * n}
    if op.startswith("ce"):
        t, v, d = case["tokens"], case["vocab"], case["hidden"]
        once = 2 * (t * d + v * d)
        if op == "ce_fwd":
            return {"bytes": once + 16 * t, "flops": 2 * t * v * d}
        return {"bytes": 2 * once + 20 * t, "flops": 6 * t * v * d}
    n, t = case["rows"] * case["cols"], case["tokens"]
    codes = (n + 1) // 2 + (n + 31) // 32 if case["form"] == "mxfp4" else n
    out = (4 if case["out"] == "f32" else 2) * t * case["rows"]
    return {"bytes": codes + 2 * t * case["cols"] + out, "flops": 2 * t * n}


def exact(case, seed):
    s = prepare(case, seed)
    op, x = s["op"], s["x"].double()
    if op == "lowp":
        n = s["rows"] * s["cols"]
        if s["form"] == "fp8":
            c = s["codes"].long()
            bits = torch.arange(256, device="cuda")
            exp, man = (bits >> 3) & 15, (bits & 7).double()
            mag = torch.where(exp == 0, torch.ldexp(man / 8, torch.tensor(-6, device="cuda")),
                              torch.ldexp(1 + man / 8, exp - 7))
            w = torch.where(bits > 127, -mag, mag)[c] / s["inv_scale"]
        else:
            w = torch.empty(n, dtype=torch.float64, device="cuda")
            mags = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
            for half in (0, 1):
                nib = (s["codes"] >> (4 * half)) & 15
                v = mags[(nib & 7).int()]
                part = w[half::2]
                part.copy_(torch.where(nib > 7, -v, v)[:part.numel()])
            for lane in range(32):
                part = w[lane::32]
                part.copy_(torch.ldexp(part, s["scales"][:part.numel()].int() - 127))
        return {"y": x @ w.view(s["rows"], s["cols"]).t()}
    if op.startswith("norm"):
        w = s["weight"].double()
        if op == "norm_fwd":
            mean = torch.zeros_like(x[:, 0]) if s["rms"] else x.sum(1) / x.shape[1]
            c = x - mean[:, None]
            rstd = 1 / torch.sqrt(c.square().sum(1) / x.shape[1] + EPS)
            y = c * rstd[:, None] * w
            if s["rms"]:
                return {"y": y, "rstd": rstd}
            return {"y": y + s["bias"].double(), "mean": mean, "rstd": rstd}
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        xh = x * r if s["rms"] else (x - s["mean"].double()[:, None]) * r
        a, n = dy * w, x.shape[1]
        dx = a - xh * ((a * xh).sum(1) / n)[:, None]
        if not s["rms"]:
            dx -= (a.sum(1) / n)[:, None]
        out = {"dx": dx * r, "dw": (dy * xh).sum(0)}
        if not s["rms"]:
            out["db"] = dy.sum(0)
        return out
    y, piece = s["targets"], 16384
    kept, vocab = y >= 0, case["vocab"]
    z = torch.cat([x @ s["weight"][v:v + piece].double().t() for v in range(0, vocab, piece)], 1)
    z *= s["scale"]
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(len(y), device="cuda")
    hit = z[rows, y.clamp(min=0)]
    out = {"loss": torch.where(kept, lse - hit, torch.zeros_like(lse)), "lse": lse}
    if op == "ce_train":
        g = torch.where(kept, s["dloss"].double(), torch.zeros_like(lse)) * s["scale"]
        z -= lse[:, None]
        z.exp_()
        z[rows, y.clamp(min=0)] -= 1
        z *= g[:, None]
        out["dx"] = torch.zeros_like(x)
        out["dw"] = torch.empty(vocab, x.shape[1], dtype=torch.float64, device="cuda")
        for v in range(0, vocab, piece):
            out["dx"] += z[:, v:v + piece] @ s["weight"][v:v + piece].double()
            out["dw"][v:v + piece] = z[:, v:v + piece].t().contiguous() @ x
    return out
