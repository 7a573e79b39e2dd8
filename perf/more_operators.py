"""What the operators of a learner's step in little memory are measured on.

A learner of a language model runs out of memory on two things: the logits of a large vocabulary with their gradient, and the
activations that the backward pass needs again.  The operators measured here do without the first and keep the second in 8 bits:

  head      cross entropy of hidden states and the output matrix, without keeping the logits, with the gradients of both
  score     log probability and log normaliser of tokens from hidden states and the output matrix
  norm      root-mean-square norm with the residual's addition; outputs in 16 (or 32) bits, and normalised values in 8 bits with scales
  normgrad  its backward pass from the 8 bits
  keep      an activation packed into 8 bits, and read back
  wgrad     the gradient of a weight matrix from a packed activation
  step      norm and linear layer, forward and backward, with nothing but the 8 bits kept between

8 bits: 32 columns of a row share a power of two u = 2^(s - 127); a value is code * u, with code = rint(x / u) cut to +-127 and
u = 2^(floor(log2(max |x|)) - 6), at least 2^-126.  Codes of a row are padded with zeros to a multiple of 32.
"""
import math

import torch

own = False

BLOCK = 32
EPS = 1e-6
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the answers of a small model: few tokens, all latency
        dict(name="head_short", op="head", rows=48, width=256, vocab=32000, masked=0.0, temperature=1.0),
        # odd numbers of rows and entries, a quarter of the rows prompts, a temperature
        dict(name="head_odd", op="head", rows=1000, width=1000, vocab=50257, masked=0.25, temperature=0.7),
        # a learner's batch of 8192 tokens in a large vocabulary, an eighth of them prompt or padding
        dict(name="head_batch", op="head", rows=8192, width=2048, vocab=131072, masked=0.125, temperature=1.0),
        # scoring 512 tokens of a wide model under a reference: the output matrix is read once
        dict(name="score_wide", op="score", rows=512, width=4096, vocab=152000, masked=0.0, temperature=1.0),
        # one token for each of 32 sequences being sampled
        dict(name="norm_token", op="norm", rows=32, width=2048, dtype="bf16", residual=True, out=True),
        # a learner's batch of 16384 tokens: new residual stream, input of the next product, and what the backward pass needs
        dict(name="norm_batch", op="norm", rows=16384, width=4096, dtype="bf16", residual=True, out=True),
        # fp32 activations of an odd width
        dict(name="norm_odd_fp32", op="norm", rows=5003, width=1100, dtype="fp32", residual=False, out=True),
        # backward pass of the same batch
        dict(name="normgrad_batch", op="normgrad", rows=16384, width=4096, dtype="bf16", residual=True),
        # an activation of a wide layer kept and read back
        dict(name="keep_batch", op="keep", rows=8192, width=8192, dtype="bf16"),
        # weight gradient of a small layer from few rows
        dict(name="wgrad_short", op="wgrad", rows=200, outs=768, width=256),
        # weight gradient of a joint projection from a batch of 8192 tokens
        dict(name="wgrad_batch", op="wgrad", rows=8192, outs=8192, width=2048),
        # norm and feed-forward projection of 4096 tokens, forward and backward
        dict(name="step_batch", op="step", rows=4096, outs=8192, width=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """Mostly what models have, multiples of 64; now and then any number."""
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.25 else max(64, w // 64 * 64)


def draw(rng):
    op = rng.choice(["head", "head", "head", "score", "norm", "norm", "normgrad", "keep", "wgrad", "wgrad", "step"])
    if op in ("head", "score"):
        width, vocab = _width(rng, 64, 4096), _log(rng, 500, 160000)
        rows = _log(rng, 1, min(8192, 1.9e12 / (width * vocab), 1e9 / vocab))
        return dict(op=op, rows=rows, width=width, vocab=vocab, masked=rng.choice([0.0, 0.1, 0.5]), temperature=rng.choice([1.0, 0.8]))
    if op in ("norm", "normgrad", "keep"):
        width = _width(rng, 64, 16384)
        case = dict(op=op, rows=_log(rng, 1, min(32768, 6.5e7 / width)), width=width, dtype=rng.choice(["fp32", "bf16", "bf16"]))
        if op != "keep":
            case.update(residual=rng.random() < 0.7)
        if op == "norm":
            case.update(out=rng.random() < 0.8)
        return case
    width, outs = _width(rng, 64, 4096), _width(rng, 64, 8192)
    return dict(op=op, rows=_log(rng, 1, min(8192, 1.3e11 / (width * outs))), outs=outs, width=width)


# ---- inputs -------------------------------------------------------------------------------------------------------

def _activations(rows, width, gen, dtype):
    """Channels of different sizes, as the residual stream of a network has."""
    channels = torch.randn(width, device=gen.device, generator=gen).mul_(0.6).exp_()
    return torch.randn(rows, width, device=gen.device, generator=gen).mul_(channels).to(dtype)


def _randn(shape, scale, gen, dtype):
    return torch.randn(shape, device=gen.device, generator=gen).mul_(scale).to(dtype)


def _gain(width, gen, dtype):
    return torch.randn(width, device=gen.device, generator=gen).mul_(0.1).add_(1.0).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=torch.device("cuda"))
    gen.manual_seed(int(seed) * 2654435761 % (1 << 62))
    op, rows, width, bf16 = case["op"], case["rows"], case["width"], torch.bfloat16
    s = {"op": op, "width": width}
    if op in ("head", "score"):
        s["head"] = _randn((case["vocab"], width), 2.0 / math.sqrt(width), gen, bf16)
        s["tokens"] = torch.randint(0, case["vocab"], (rows,), device=gen.device, generator=gen)
        lift = torch.rand(rows, 1, device=gen.device, generator=gen).mul_(3.0)            # a trained model: the token is mostly likely
        s["hidden"] = torch.randn(rows, width, device=gen.device, generator=gen).add_(lift * s["head"][s["tokens"]].float()).to(bf16)
        s["weights"] = None
        if case["masked"]:
            s["weights"] = torch.ones(rows, device=gen.device)
            s["weights"][torch.randperm(rows, device=gen.device, generator=gen)[:min(rows - 1, round(case["masked"] * rows))]] = 0.0
        s["temperature"] = case["temperature"]
        return s
    dtype = DTYPES[case.get("dtype", "bf16")]
    s["dtype"] = dtype
    if op == "keep":
        s["x"] = _activations(rows, width, gen, dtype)
        return s
    s["gain"] = _gain(width, gen, dtype)
    if op in ("norm", "step"):
        s["x"] = _activations(rows, width, gen, dtype)
        s["residual"] = _activations(rows, width, gen, dtype) if case.get("residual", True) else None
        s["out"] = case.get("out", True)
    else:                                                                                # what the forward pass left: packed values
        x = _activations(rows, width, gen, torch.float32)
        s["rstd"] = torch.rsqrt(x.square().mean(1) + EPS)
        s["codes"], s["scales"] = _pack(x.mul_(s["rstd"][:, None]))
    if op in ("wgrad", "step"):
        s["dout"] = _randn((rows, case["outs"]), 1e-3, gen, bf16)
    if op == "normgrad":
        s["dout"] = _randn((rows, width), 1e-3, gen, dtype)
    if op == "step":
        s["weight"] = _randn((case["outs"], width), 1.0 / math.sqrt(width), gen, bf16)
    if op in ("normgrad", "step"):
        s["dtotal"] = _randn((rows, width), 1e-3, gen, dtype) if case.get("residual", True) else None
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _pack(x):
    """(codes, scales) of fp32 values."""
    rows, width = x.shape
    full = -(-width // BLOCK) * BLOCK
    if full != width:
        x = torch.cat([x, x.new_zeros(rows, full - width)], 1)
    x = x.view(rows, -1, BLOCK)
    e = x.abs().amax(2).view(torch.int32) >> 23
    s = torch.where(e == 255, e, (e - 6).clamp(min=1))
    codes = (x * ((254 - s) << 23).view(torch.float32)[:, :, None]).round().clamp(-127, 127)
    codes = torch.where((s == 255)[:, :, None], torch.zeros_like(codes), codes)
    return codes.to(torch.int8).view(rows, full), s.to(torch.uint8)


def _unpack(codes, scales, width):
    unit = (scales.to(torch.int32) << 23).view(torch.float32)
    return (codes.view(codes.shape[0], -1, BLOCK).float() * unit[:, :, None]).view(codes.shape)[:, :width]


def _plain_head(s):
    h, w, t = s["hidden"].float(), s["head"].float(), s["tokens"][:, None]
    live = None if s["weights"] is None else s["weights"] != 0
    z = h @ w.T
    z /= s["temperature"]
    top = z.amax(1, keepdim=True)
    z_t = z.gather(1, t)
    p = z.sub_(top).exp_()
    total = p.sum(1, keepdim=True)
    lse = top + total.log()
    logp = (z_t - lse)[:, 0]
    lse = lse[:, 0]
    if live is not None:
        logp, lse = torch.where(live, logp, 0.0), torch.where(live, lse, 0.0)
    if s["op"] == "score":
        return {"logp": logp, "lse": lse}
    share = torch.full_like(logp, 1.0 / logp.numel()) if live is None else s["weights"] / s["weights"].sum()
    loss = -(share * logp).sum()
    p /= total
    p.scatter_add_(1, t, torch.full_like(z_t, -1.0))
    p *= (share / s["temperature"])[:, None]
    return {"loss": loss, "logp": logp, "dhidden": (p @ w).to(s["hidden"].dtype), "dhead": (p.T @ h).to(s["head"].dtype)}


def _plain_norm(s):
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["dtype"])
    x = total.float()
    rstd = torch.rsqrt(x.square().mean(1) + EPS)
    n = x * rstd[:, None]
    return total, rstd, n


def _plain_normgrad(dout, n, rstd, gain, dtotal, dtype):
    g = dout * gain.float()
    dx = (g - n * (g * n).mean(1, keepdim=True)) * rstd[:, None]
    if dtotal is not None:
        dx += dtotal.float()
    return {"dx": dx.to(dtype), "dgain": (dout * n).sum(0).to(gain.dtype)}


def _plain(s):
    op = s["op"]
    if op in ("head", "score"):
        return _plain_head(s)
    if op == "keep":
        return {"kept": _unpack(*_pack(s["x"].float()), s["width"]).to(torch.bfloat16)}
    if op == "wgrad":
        return {"dweight": ((s["dout"].float().T @ _unpack(s["codes"], s["scales"], s["width"])) * s["gain"].float()).to(torch.bfloat16)}
    if op == "normgrad":
        return _plain_normgrad(s["dout"].float(), _unpack(s["codes"], s["scales"], s["width"]), s["rstd"], s["gain"], s["dtotal"], s["dtype"])
    total, rstd, n = _plain_norm(s)
    kept = _unpack(*_pack(n), s["width"])
    if op == "norm":
        out = {"kept": kept.to(torch.bfloat16), "rstd": rstd}
        if s["residual"] is not None:
            out["total"] = total
        if s["out"]:
            out["out"] = (n * s["gain"].float()).to(s["dtype"])
        return out
    y = (n * s["gain"].float()).to(s["dtype"]).float()                                    # the product's input is a tensor of 16 bits
    w, dz = s["weight"].float(), s["dout"].float()
    out = {"total": total, "z": (y @ w.T).to(s["dtype"]), "dweight": ((dz.T @ kept) * s["gain"].float()).to(torch.bfloat16)}
    out.update(_plain_normgrad((dz @ w).to(s["dtype"]).float(), kept, rstd, s["gain"], s["dtotal"], s["dtype"]))
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _calls(s):
    import paper_1511_05950_b200 as P
    op = s["op"]
    if op == "head":
        r = P.head_cross_entropy(s["hidden"], s["head"], s["tokens"], weights=s["weights"], temperature=s["temperature"])
        return {"loss": r.stats[0], "logp": r.logp, "dhidden": r.dhidden, "dhead": r.dhead}
    if op == "score":
        r = P.head_logprob(s["hidden"], s["head"], s["tokens"], weights=s["weights"], temperature=s["temperature"])
        return {"logp": r.logp, "lse": r.lse}
    if op == "keep":
        return {"kept": P.unpack8(P.pack8(s["x"]))}
    if op == "wgrad":
        return {"dweight": P.packed_weight_grad(s["dout"], P.Packed8(s["codes"], s["scales"], s["width"]), gain=s["gain"])}
    if op == "normgrad":
        r = P.rms_norm_grad(s["dout"], P.Packed8(s["codes"], s["scales"], s["width"]), s["rstd"], gain=s["gain"], dtotal=s["dtotal"])
        return {"dx": r.dx, "dgain": r.dgain}
    if op == "norm":
        r = P.rms_norm(s["x"], gain=s["gain"], residual=s["residual"], eps=EPS, out=s["out"], pack=True)
        out = {"kept": P.unpack8(r.packed), "rstd": r.rstd}
        if s["residual"] is not None:
            out["total"] = r.total
        if s["out"]:
            out["out"] = r.out
        return out
    x, gain, weight = (s[k].detach().requires_grad_(True) for k in ("x", "gain", "weight"))
    z, total = P.norm_linear(x, gain, weight, residual=s["residual"], eps=EPS)
    torch.autograd.backward([z, total], [s["dout"], s["dtotal"]])
    return {"total": total.detach(), "z": z.detach(), "dweight": weight.grad, "dx": x.grad, "dgain": gain.grad}


def run(state):
    return _calls(state) if own else _plain(state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    op, rows, width = case["op"], case["rows"], case["width"]
    if op in ("head", "score"):
        vocab = case["vocab"]
        live = rows - (min(rows - 1, round(case["masked"] * rows)) if case["masked"] else 0)
        once = 2 * (live * width + vocab * width) + 16 * rows
        return {"bytes": 2 * once if op == "head" else once, "flops": (6 if op == "head" else 2) * live * width * vocab}
    size = 4 if case.get("dtype") == "fp32" else 2
    n, kept = rows * width, rows * width * 33 / 32
    if op == "keep":
        return {"bytes": n * size + 2 * kept + 2 * n, "flops": 4 * n}
    if op == "norm":
        more = (2 if case["residual"] else 0) + (1 if case["out"] else 0)
        return {"bytes": n * size * (1 + more) + 2 * kept + 2 * n, "flops": 8 * n}
    if op == "normgrad":
        return {"bytes": n * size * (3 if case["residual"] else 2) + kept, "flops": 10 * n}
    outs = case["outs"]
    if op == "wgrad":
        return {"bytes": 2 * rows * outs + kept + 2 * outs * width, "flops": 2 * n * outs}
    return {"bytes": 2 * (6 * n + 2 * rows * outs + 3 * outs * width), "flops": 6 * n * outs}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _near(x):
    """The nearest values that 8 bits with a scale stand for, of values in 64 bits."""
    rows, width = x.shape
    blocks = torch.nn.functional.pad(x, (0, -width % BLOCK)).reshape(rows, -1, BLOCK)
    exponent = torch.frexp(blocks.abs().amax(2))[1].double() - 1
    unit = torch.exp2(exponent - 6).clamp(min=2.0 ** -126)[:, :, None]
    return (torch.round(blocks / unit).clamp(-127, 127) * unit).reshape(rows, -1)[:, :width]


def _stands_for(s):
    unit = torch.exp2(s["scales"].double() - 127).repeat_interleave(BLOCK, 1)
    return (s["codes"].double() * unit)[:, :s["width"]]


def _exact_head(s):
    keep = torch.arange(s["tokens"].numel(), device=s["tokens"].device) if s["weights"] is None else s["weights"].nonzero()[:, 0]
    h, w, t = s["hidden"][keep].double(), s["head"].double(), s["tokens"][keep]
    z = (h @ w.T).div_(s["temperature"])
    lse = torch.logsumexp(z, 1)
    logp = z[torch.arange(t.numel(), device=t.device), t] - lse

    def whole(x):
        return x.new_zeros((s["tokens"].numel(),) + x.shape[1:]).index_copy_(0, keep, x)

    if s["op"] == "score":
        return {"logp": whole(logp), "lse": whole(lse)}
    share = torch.ones_like(logp) if s["weights"] is None else s["weights"][keep].double()
    share = share / share.sum()
    dz = z.sub_(lse[:, None]).exp_()
    dz[torch.arange(t.numel(), device=t.device), t] -= 1.0
    dz.mul_((share / s["temperature"])[:, None])
    return {"loss": -(share * logp).sum(), "logp": whole(logp), "dhidden": whole(dz @ w), "dhead": dz.T @ h}


def _exact_normgrad(dout, n, rstd, s):
    gain = s["gain"].double()
    g = dout * gain
    dx = rstd.double()[:, None] * (g - n * (g * n).mean(1, keepdim=True))
    return {"dx": dx if s["dtotal"] is None else dx + s["dtotal"].double(), "dgain": (dout * n).sum(0)}


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("head", "score"):
        return _exact_head(s)
    if op == "keep":
        return {"kept": _near(s["x"].double())}
    if op == "wgrad":
        return {"dweight": s["dout"].double().T @ (_stands_for(s) * s["gain"].double())}
    if op == "normgrad":
        return _exact_normgrad(s["dout"].double(), _stands_for(s), s["rstd"], s)
    total = s["x"].double()
    if s["residual"] is not None:
        total = (total + s["residual"].double()).to(s["dtype"]).double()
    rstd = (total.square().mean(1) + EPS).rsqrt()
    n = total * rstd[:, None]
    kept = _near(n)
    if op == "norm":
        out = {"kept": kept, "rstd": rstd}
        if s["residual"] is not None:
            out["total"] = total
        if s["out"]:
            out["out"] = n * s["gain"].double()
        return out
    y = (n * s["gain"].double()).to(s["dtype"]).double()
    w, dz = s["weight"].double(), s["dout"].double()
    out = {"total": total, "z": y @ w.T, "dweight": dz.T @ (kept * s["gain"].double())}
    out.update(_exact_normgrad((dz @ w).to(s["dtype"]).double(), kept, rstd, s))
    return out
