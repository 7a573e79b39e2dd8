"""What the learner-side and server-side operators are measured on.

The server of this repository applies momentum SGD to gradients that learners compute on stale weights.  The operators
measured here are the ones a language-model learner and its server need next to that:

  norm      the global norm of c staleness-weighted gradients over many tensors, with the clipping factor
  adamw     an AdamW step over many tensors, the gradient being the weighted sum of c pushed ones; moments in 32 or in 8 bits
  logprob   log probability, log normaliser and entropy of chosen tokens from logits
  policy    the clipped policy loss with a KL term and an entropy term, and its gradient with respect to the logits
  pref      the preference loss over pairs of sequences (paired log ratios), and its gradient with respect to the logits

Moments in 8 bits: the tensors' moments lie one behind the other in one array, each tensor starting at a multiple of 256
elements; every 256 elements share a power of two 2^E.  The first moment is a sign, 3 exponent and 4 fraction bits (bias 7), the
second 4 exponent and 4 fraction bits (bias 15), both with subnormals; rounding to a neighbour is random, with the
probability that keeps the expectation, from a hash of the seed, the step and the element's place.
"""
import math
import random

import torch

own = False

BLOCK = 256
MASK32 = 0xFFFFFFFF


# ---- sizes --------------------------------------------------------------------------------------------------------

CNN = [32 * 3 * 25, 32, 32 * 32 * 25, 32, 64 * 32 * 25, 64, 10 * 1024, 10]                      # the small network, 89,578
ALEXNET = [96 * 3 * 121, 96, 256 * 48 * 25, 256, 384 * 256 * 9, 384, 384 * 192 * 9, 384, 256 * 192 * 9, 256,
           4096 * 9216, 4096, 4096 * 4096, 4096, 1000 * 4096, 1000]                              # the large one, 60,965,224


def _lm(layers, width, vocab):
    """A decoder's tensors: embedding, per layer two gains, a joint projection, an output projection, two of a feed-forward."""
    layer = [width, 3 * width * width, width * width, width, 4 * width * width, 4 * width * width]
    return [vocab * width] + layer * layers + [width]


def _split(total, tensors, seed):
    """`tensors` sizes that sum to `total`, most of it in a few (as in a network), odd ones and ones of one element among them."""
    r = random.Random(seed)
    share = [r.random() ** 4 + 1e-6 for _ in range(tensors)]
    sizes = [max(1, int(total * s / sum(share))) for s in share]
    return sizes


def _sizes(case):
    kind = case["tensors"]
    if kind == "cnn":
        return CNN
    if kind == "alexnet":
        return ALEXNET
    if kind == "lm":
        return _lm(case["layers"], case["width"], case["vocab"])
    return _split(case["total"], case["count"], case["split"])


def listed():
    return [
        # one update group of the small configuration: four learners' fp32 gradients in eight tensors; all latency
        dict(name="norm_cnn_c4", op="norm", tensors="cnn", c=4, dtype="fp32"),
        # gradient of a language model of 1.07e9 parameters in 122 tensors, bf16, one learner at a time
        dict(name="norm_lm_bf16", op="norm", tensors="lm", layers=20, width=2048, vocab=32000, c=1, dtype="bf16"),
        # the small network's step, one gradient (pure asynchronous): all latency
        dict(name="adamw_cnn", op="adamw", tensors="cnn", c=1, dtype="fp32", bits=32, mirror=False, clip=False),
        # the large network's step with four gradients a group, clipped, moments in 32 bits
        dict(name="adamw_alexnet_c4", op="adamw", tensors="alexnet", c=4, dtype="fp32", bits=32, mirror=False, clip=True),
        # the language model's step: bf16 gradient, 8-bit moments, bf16 copy of the weights for the learners, clipped
        dict(name="adamw8_lm_bf16", op="adamw", tensors="lm", layers=20, width=2048, vocab=32000, c=1, dtype="bf16", bits=8, mirror=True, clip=True),
        # scoring the tokens that a batch of 32 sequences has just sampled, one each; odd vocabulary, so rows start anywhere
        dict(name="logprob_step", op="logprob", rows=32, vocab=50257, dtype="bf16", masked=0.0, banned=0, temperature=1.0),
        # reference or behaviour log probabilities of 8192 tokens, an eighth of them prompt or padding
        dict(name="logprob_batch", op="logprob", rows=8192, vocab=131072, dtype="bf16", masked=0.125, banned=0, temperature=1.0),
        # a short answer in a small vocabulary
        dict(name="policy_short", op="policy", rows=48, vocab=32000, dtype="bf16", masked=0.0, banned=0, temperature=1.0, kl=0.05, ent=0.0),
        # fp32 logits, odd vocabulary whose last entries are padding (minus infinity), temperature, all terms of the loss
        dict(name="policy_fp32_odd", op="policy", rows=4096, vocab=50257, dtype="fp32", masked=0.25, banned=81, temperature=0.7, kl=0.04, ent=0.01),
        # a learner's batch of 16384 tokens in a large vocabulary
        dict(name="policy_batch", op="policy", rows=16384, vocab=152000, dtype="bf16", masked=0.125, banned=0, temperature=1.0, kl=0.02, ent=0.0),
        # two pairs of short answers
        dict(name="pref_short", op="pref", pairs=2, longest=96, vocab=32000, dtype="bf16", masked=0.0, smooth=0.0),
        # eight pairs of ragged answers of up to 1024 tokens (their prompts' rows masked) in a large vocabulary
        dict(name="pref_batch", op="pref", pairs=8, longest=1024, vocab=131072, dtype="bf16", masked=0.25, smooth=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "adamw", "adamw", "logprob", "policy", "policy", "pref"])
    if op in ("norm", "adamw"):
        c, dtype = rng.choice([1, 1, 2, 4, 7]), rng.choice(["fp32", "bf16"])
        case = dict(op=op, tensors="split", total=_log(rng, 2000, 2e8 / c), count=_log(rng, 1, 400), split=rng.randrange(1 << 30), c=c, dtype=dtype)
        if op == "adamw":
            case.update(bits=rng.choice([8, 32]), mirror=rng.random() < 0.5, clip=rng.random() < 0.5)
        return case
    vocab, dtype = _log(rng, 500, 160000), rng.choice(["fp32", "bf16", "bf16"])
    most = 2e9 if dtype == "bf16" else 1e9
    masked = rng.choice([0.0, 0.1, 0.5])
    if op == "pref":
        pairs = _log(rng, 1, 24)
        longest = _log(rng, 1, max(2, min(2048, most / (2 * pairs * vocab))))
        return dict(op=op, pairs=pairs, longest=longest, vocab=vocab, dtype=dtype, masked=masked, smooth=rng.choice([0.0, 0.1]))
    case = dict(op=op, rows=_log(rng, 1, min(16384, most / vocab)), vocab=vocab, dtype=dtype, masked=masked,
                banned=rng.choice([0, 0, vocab // 100]), temperature=rng.choice([1.0, 0.8]))
    if op == "policy":
        case.update(kl=rng.choice([0.0, 0.05]), ent=rng.choice([0.0, 0.01]))
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
LR, BETAS, EPS, DECAY = 1e-4, (0.9, 0.95), 1e-8, 0.1


def _starts(sizes):
    """Where each tensor's moments begin, and how many elements they take in all."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


def _views(flat, sizes, starts):
    return [flat[o:o + n] for o, n in zip(starts, sizes)]


def _scales(c):
    """1 / (c * sigma) for staleness 1, 2, 3, ...: what the server weights a group's gradients with."""
    return [1.0 / (c * (1 + l % 3)) for l in range(c)]


def _prepare_tensors(case, gen, seed):
    sizes, c, dt = _sizes(case), case["c"], DTYPES[case["dtype"]]
    starts, padded = _starts(sizes)
    dense, n = [], 0
    for count in sizes:
        dense.append(n)
        n += count
    dev = gen.device
    s = {"op": case["op"], "sizes": sizes, "c": c, "scales": _scales(c), "padded": padded}
    mag = torch.randn(n, device=dev, generator=gen).mul_(0.7).exp_().mul_(2e-5)          # every element's gradient has a size of its own
    s["grads"] = []
    for _ in range(c):
        g = torch.randn(n, device=dev, generator=gen).mul_(mag).to(dt)
        s["grads"].append([v.clone() for v in _views(g, sizes, dense)])                  # tensors of their own, as a learner's are
    s["scratch"] = torch.zeros(padded, device=dev)
    s["scratch_views"] = _views(s["scratch"], sizes, starts)
    if case["op"] == "norm":
        s["max_norm"] = 2e-5 * math.sqrt(n)                                             # under the norm, so the factor is below one
        if own:
            import paper_1511_05950_b200 as P
            s["plan"] = P.TensorList(sizes, device=dev)
        return s
    s["w"] = torch.randn(n, device=dev, generator=gen).mul_(0.02)                       # the server's flat vector; the tensors are parts of it
    s["w_views"] = _views(s["w"], sizes, dense)
    s["mirror"] = s["w"].to(torch.bfloat16) if case["mirror"] else None
    s["mirror_views"] = _views(s["mirror"], sizes, dense) if case["mirror"] else None
    s["decay_mult"] = [0.0 if n_i <= 4096 else 1.0 for n_i in sizes]                     # gains and biases do not decay
    s["clip"] = torch.tensor([2.5, 0.4], device=dev) if case["clip"] else None
    s["t"], s["seed"], s["bits"] = 100, seed & 0xFFFF, case["bits"]
    m, v = torch.zeros(padded, device=dev), torch.zeros(padded, device=dev)
    torch._foreach_copy_(_views(m, sizes, starts), _views(torch.randn(n, device=dev, generator=gen).mul_(mag).mul_(0.3), sizes, dense))
    torch._foreach_copy_(_views(v, sizes, starts), _views(mag.mul_(torch.rand(n, device=dev, generator=gen).add_(0.5)).square_(), sizes, dense))
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        half = torch.full((), 1 << 18, dtype=torch.int32, device=dev)
        s["m"], s["m_scale"] = _encode(m, True, half)
        s["v"], s["v_scale"] = _encode(v, False, half)
    if own:                                                                              # the optimiser object that a program keeps
        import paper_1511_05950_b200 as P
        state = (s["m"], s["v"]) if case["bits"] == 32 else (s["m"], s["v"], s["m_scale"], s["v_scale"])
        s["plan"] = P.AdamW(s["w_views"], lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, state_bits=case["bits"],
                            decay_mult=s["decay_mult"], mirrors=s["mirror_views"], state=state, step=s["t"], seed=s["seed"])
    return s


def _logits(rows, vocab, dtype, banned, gen):
    """Logits of a trained model: a spread of values, the chosen token usually among the likely ones."""
    dev = gen.device
    x = torch.randn(rows, vocab, device=dev, generator=gen, dtype=DTYPES[dtype]).mul_(2.0)
    tokens = torch.randint(0, vocab - banned, (rows,), device=dev, generator=gen)
    lift = torch.rand(rows, 1, device=dev, generator=gen).mul_(14.0).to(x.dtype)
    x.scatter_add_(1, tokens[:, None], lift)
    if banned:
        x[:, vocab - banned:] = -math.inf
    return x, tokens


def _kept(rows, masked, gen):
    """1 where a row counts, 0 for prompts and padding: round(masked * rows) of them, at random places."""
    w = torch.ones(rows, device=gen.device)
    w[torch.randperm(rows, device=gen.device, generator=gen)[:int(round(masked * rows))]] = 0.0
    return w


def _lengths(case):
    """Lengths of the 2 * pairs sequences: ragged, the longest as given, one of one token."""
    r = random.Random(case["pairs"] * 7919 + case["longest"])
    n = [r.randint(max(1, case["longest"] // 2), case["longest"]) for _ in range(2 * case["pairs"])]
    n[0] = case["longest"]
    if len(n) > 4:
        n[3] = 1
    return n


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 2654435761 % (1 << 62))
    op = case["op"]
    if op in ("norm", "adamw"):
        return _prepare_tensors(case, gen, int(seed))
    s = {"op": op}
    if op == "pref":
        lengths = _lengths(case)
        rows = sum(lengths)
        s["logits"], s["tokens"] = _logits(rows, case["vocab"], case["dtype"], 0, gen)
        s["weights"] = _kept(rows, case["masked"], gen)
        s["offsets"] = torch.tensor([0] + lengths, device=dev).cumsum(0)
        logp = _token_logprob(s["logits"], s["tokens"], 1.0, s["weights"])[0]
        ref = _per_sequence(logp * s["weights"], s["offsets"])
        s["ref_logp"] = ref + torch.randn(ref.shape, device=dev, generator=gen).mul_(4.0)
        s["beta"], s["smooth"] = 0.1, case["smooth"]
        return s
    rows = case["rows"]
    s["logits"], s["tokens"] = _logits(rows, case["vocab"], case["dtype"], case["banned"], gen)
    s["weights"] = _kept(rows, case["masked"], gen)
    s["temperature"] = case["temperature"]
    if op == "policy":
        logp = _token_logprob(s["logits"], s["tokens"], s["temperature"], s["weights"])[0]
        # most ratios near one, some far off: the weights have moved since these tokens were sampled
        near = torch.randn(rows, device=dev, generator=gen).mul_(0.03)
        far = torch.rand(rows, device=dev, generator=gen).mul_(0.4).add_(0.35) * torch.sign(torch.rand(rows, device=dev, generator=gen) - 0.5)
        s["old_logp"] = logp + torch.where(torch.rand(rows, device=dev, generator=gen) < 0.12, far, near)
        s["ref_logp"] = logp + torch.randn(rows, device=dev, generator=gen).mul_(0.2) if case["kl"] else None
        s["advantages"] = torch.randn(rows, device=dev, generator=gen)
        s["kl"], s["ent"] = case["kl"], case["ent"]
    return s


# ---- plain forms: many tensors ------------------------------------------------------------------------------------

def _gradient(s):
    """The weighted sum of the c gradients in fp32, laid out as the moments are."""
    total = None
    for scale, grads in zip(s["scales"], s["grads"]):
        torch._foreach_copy_(s["scratch_views"], grads)
        part = s["scratch"] * scale
        total = part if total is None else total.add_(part)
    return total


def _norm(s):
    norm = _gradient(s).square_().sum().sqrt()
    return {"norm": torch.stack([norm, torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))])}


def _key(seed, t):
    x = (seed + t * 0x9E3779B97F4A7C15) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & 0xFFFFFFFFFFFFFFFF
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & 0xFFFFFFFFFFFFFFFF
    return (x ^ (x >> 31)) & MASK32


def _hash(n, key, dev):
    x = torch.arange(n, device=dev)
    x = ((x & MASK32) ^ key).add_((x >> 32) * 0x9E3779B9).bitwise_and_(MASK32)
    x ^= x >> 16
    x.mul_(0x7FEB352D).bitwise_and_(MASK32)
    x ^= x >> 15
    x.mul_(0x846CA68B).bitwise_and_(MASK32)
    x ^= x >> 16
    return x


def _decode(codes, scale, signed):
    unit = 2.0 ** 120 if signed else 2.0 ** 112
    x = ((codes & 127 if signed else codes).to(torch.int32) << 19).view(torch.float32).mul_(unit)
    x = x.view(-1, BLOCK).mul_((scale.to(torch.int32) << 23).view(torch.float32)[:, None]).view(-1)
    return torch.where(codes > 127, -x, x) if signed else x


def _encode(x, signed, rnd):
    """8-bit codes of x and the exponents of its blocks.  rnd: 19 random bits for each element."""
    unit, top = (2.0 ** -120, 127) if signed else (2.0 ** -112, 255)
    mag = x.abs()
    e = ((mag.view(-1, BLOCK).amax(1).view(torch.int32) + (1 << 19)) >> 23).clamp_(27, 253)
    bits = mag.view(-1, BLOCK).mul(((254 - e) << 23).view(torch.float32)[:, None]).mul_(unit).view(-1).view(torch.int32)
    code = ((bits + rnd) >> 19).clamp_(max=top)
    if signed:
        code += (x < 0).to(torch.int32) << 7
    else:
        code = torch.maximum(code, (x > 0).to(torch.int32))
    return code.to(torch.uint8), e.to(torch.uint8)


def _adamw(s):
    s["t"] += 1
    t, (b1, b2) = s["t"], BETAS
    g = _gradient(s)
    if s["clip"] is not None:
        g.mul_(s["clip"][1])
    small = s["bits"] == 8
    m = _decode(s["m"], s["m_scale"], True) if small else s["m"]
    v = _decode(s["v"], s["v_scale"], False) if small else s["v"]
    m.mul_(b1).add_(g * (1 - b1))
    v.mul_(b2).add_(g.square_().mul_(1 - b2))
    u = m / (v.sqrt().mul_(1 / math.sqrt(1 - b2 ** t)).add_(EPS))
    u.mul_(LR / (1 - b1 ** t))
    s["scratch"].copy_(u)
    torch._foreach_mul_(s["w_views"], [1 - LR * DECAY * d for d in s["decay_mult"]])
    torch._foreach_sub_(s["w_views"], s["scratch_views"])
    out = {"w": s["w"], "m": m, "v": v}
    if small:
        x = _hash(m.numel(), _key(s["seed"], t), m.device)
        m, m_scale = _encode(m, True, ((x & 0xFFFF) << 3).to(torch.int32))
        v, v_scale = _encode(v, False, ((x >> 16) << 3).to(torch.int32))
        s["m"].copy_(m), s["v"].copy_(v), s["m_scale"].copy_(m_scale), s["v_scale"].copy_(v_scale)
        out["m"], out["v"] = _decode(m, m_scale, True).to(torch.bfloat16), _decode(v, v_scale, False).to(torch.bfloat16)
    if s["mirror"] is not None:
        out["mirror"] = s["mirror"].copy_(s["w"])
    return out


# ---- plain forms: losses from logits ------------------------------------------------------------------------------

def _token_logprob(logits, tokens, temperature, weights):
    """(logp, lse, entropy) of each row's token, zero where the row's weight is zero; also the scaled logits and the softmax."""
    z = logits.float()
    if temperature != 1.0:
        z = z * (1.0 / temperature)
    top = z.amax(1, keepdim=True)
    e = (z - top).exp_()
    total = e.sum(1, keepdim=True)
    lse = (top + total.log()).squeeze(1)
    entropy = lse - torch.where(e > 0, e * z, 0.0).sum(1) / total.squeeze(1)
    logp = z.gather(1, tokens[:, None]).squeeze(1) - lse
    keep = weights != 0
    return torch.where(keep, logp, 0.0), torch.where(keep, lse, 0.0), torch.where(keep, entropy, 0.0), z, e.div_(total)


def _logprob(s):
    logp, lse, entropy, _, _ = _token_logprob(s["logits"], s["tokens"], s["temperature"], s["weights"])
    return {"logp": logp, "lse": lse, "entropy": entropy}


CLIP = 0.2


def _policy(s):
    w = s["weights"]
    logp, lse, entropy, z, p = _token_logprob(s["logits"], s["tokens"], s["temperature"], w)
    keep, share = w != 0, w / w.sum()
    adv = s["advantages"]
    ratio = (logp - s["old_logp"]).exp()
    free, held = ratio * adv, ratio.clamp(1 - CLIP, 1 + CLIP) * adv
    term = -torch.minimum(free, held)
    slope = torch.where(free <= held, -free, 0.0)
    kl = torch.zeros_like(logp)
    if s["ref_logp"] is not None:
        d = s["ref_logp"] - logp
        kl = d.exp() - d - 1
        slope = slope + s["kl"] * (1 - d.exp())
    loss = term + s["kl"] * kl - s["ent"] * entropy
    each = torch.stack([loss, term, kl, entropy, (free > held).float()])
    stats = torch.where(keep, each * share, 0.0).sum(1)
    inv = 1.0 / s["temperature"]
    a = torch.where(keep, slope * share * inv, 0.0)[:, None]
    grad = p * -a
    if s["ent"]:
        b = torch.where(keep, share * (s["ent"] * inv), 0.0)[:, None]
        grad += torch.where(p > 0, p * (z - lse[:, None] + entropy[:, None]), 0.0).mul_(b)
    grad.scatter_add_(1, s["tokens"][:, None], a)
    return {"stats": stats, "logp": logp, "entropy": entropy, "dlogits": grad.to(s["logits"].dtype)}


def _per_sequence(x, offsets):
    """Sums of x over each sequence's rows."""
    at = torch.arange(x.numel(), device=x.device)
    return torch.where((at >= offsets[:-1, None]) & (at < offsets[1:, None]), x, 0.0).sum(1)


def _pref(s):
    w, offsets = s["weights"], s["offsets"]
    logp, _, _, _, p = _token_logprob(s["logits"], s["tokens"], 1.0, w)
    seq = _per_sequence(logp * w, offsets)
    d = seq - s["ref_logp"]
    margin = s["beta"] * (d[0::2] - d[1::2])
    up = (1 + (-margin.abs()).exp()).log()
    loss = (1 - s["smooth"]) * (up + (-margin).clamp(min=0)) + s["smooth"] * (up + margin.clamp(min=0))
    stats = torch.stack([loss.mean(), (margin > 0).float().mean(), margin.mean()])
    slope = (1 / (1 + (-margin).exp()) - (1 - s["smooth"])) * (s["beta"] / margin.numel())
    per_seq = torch.stack([slope, -slope], 1).view(-1)
    row = torch.searchsorted(offsets, torch.arange(w.numel(), device=w.device), right=True) - 1
    a = (per_seq[row] * w)[:, None]
    grad = p.mul_(-a).scatter_add_(1, s["tokens"][:, None], a)
    return {"stats": stats, "seq_logp": seq, "dlogits": grad.to(s["logits"].dtype)}


# ---- one pass -----------------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_1511_05950_b200 as P
    op = s["op"]
    if op == "norm":
        return {"norm": s["plan"].grad_norm(s["grads"], s["scales"], s["max_norm"])}
    if op == "adamw":
        s["plan"].step(s["grads"], s["scales"], clip=s["clip"])
        m, v = s["plan"].moments()
        out = {"w": s["w"], "m": m, "v": v}
        if s["mirror"] is not None:
            out["mirror"] = s["mirror"]
        return out
    if op == "logprob":
        r = P.token_logprob(s["logits"], s["tokens"], weights=s["weights"], temperature=s["temperature"])
        return {"logp": r.logp, "lse": r.lse, "entropy": r.entropy}
    if op == "policy":
        r = P.policy_loss(s["logits"], s["tokens"], s["old_logp"], s["advantages"], weights=s["weights"], ref_logp=s["ref_logp"],
                          clip_low=CLIP, clip_high=CLIP, kl_coef=s["kl"], entropy_coef=s["ent"], temperature=s["temperature"])
        return {"stats": r.stats, "logp": r.logp, "entropy": r.entropy, "dlogits": r.dlogits}
    r = P.preference_loss(s["logits"], s["tokens"], s["offsets"], s["ref_logp"], weights=s["weights"], beta=s["beta"], label_smoothing=s["smooth"])
    return {"stats": r.stats, "seq_logp": r.seq_logp, "dlogits": r.dlogits}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _norm, "adamw": _adamw, "logprob": _logprob, "policy": _policy, "pref": _pref}[state["op"]](state)


def work(case):
    op = case["op"]
    if op in ("norm", "adamw"):
        n, g = sum(_sizes(case)), case["c"] * (4 if case["dtype"] == "fp32" else 2)
        if op == "norm":
            return {"bytes": n * g, "flops": n * (2 * case["c"] + 2)}
        # weights read and written, moments read and written (8 bits: and returned as bf16 values), a bf16 copy written
        moments = 16 if case["bits"] == 32 else 4 + 4 + 4 / BLOCK
        return {"bytes": n * (8 + g + moments + (2 if case["mirror"] else 0)), "flops": n * (2 * case["c"] + 14)}
    rows = sum(_lengths(case)) if op == "pref" else case["rows"]
    used = rows - int(round(case["masked"] * rows))                                       # masked rows need not be read
    b = 4 if case["dtype"] == "fp32" else 2
    write = 0 if op == "logprob" else rows
    return {"bytes": case["vocab"] * b * (used + write) + rows * 28, "flops": case["vocab"] * (5.0 * used + 3.0 * (used if write else 0))}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_moment(codes, exponents, signed):
    """Values of 8-bit codes, from the table of all 256."""
    table = []
    for code in range(256):
        mag = code % 128 if signed else code
        e, f, bias = mag // 16, mag % 16, 7 if signed else 15
        value = (1 + f / 16) * 2.0 ** (e - bias) if e else f / 16 * 2.0 ** (1 - bias)
        table.append(-value if signed and code >= 128 else value)
    x = torch.tensor(table, dtype=torch.float64, device=codes.device)[codes.long()]
    return x * torch.pow(2.0, exponents.double() - 127).repeat_interleave(BLOCK)


def _exact_tensors(case, s):
    sizes, (starts, padded) = s["sizes"], _starts(s["sizes"])
    dev = s["scratch"].device
    g = torch.zeros(padded, dtype=torch.float64, device=dev)
    for scale, grads in zip(s["scales"], s["grads"]):
        for o, x in zip(starts, grads):
            g[o:o + x.numel()] += scale * x.double()
    if case["op"] == "norm":
        norm = float(torch.linalg.vector_norm(g))
        return {"norm": torch.tensor([norm, min(1.0, s["max_norm"] / norm)], dtype=torch.float64)}
    if s["clip"] is not None:
        g *= float(s["clip"][1])
    t, (b1, b2) = s["t"] + 1, BETAS
    if case["bits"] == 8:
        m, v = _exact_moment(s["m"], s["m_scale"], True), _exact_moment(s["v"], s["v_scale"], False)
    else:
        m, v = s["m"].double(), s["v"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    w, at = s["w"].double(), 0
    for o, n, d in zip(starts, sizes, s["decay_mult"]):
        part = w[at:at + n]
        step = (m[o:o + n] / (1 - b1 ** t)) / (torch.sqrt(v[o:o + n] / (1 - b2 ** t)) + EPS)
        w[at:at + n] = part - LR * (step + DECAY * d * part)
        at += n
    out = {"w": w, "m": m, "v": v}                                                         # 8 bits: the moments before they are rounded
    if s["mirror"] is not None:
        out["mirror"] = w
    return out


def _exact_losses(case, s):
    logits, tokens, w = s["logits"], s["tokens"], s["weights"].double()
    rows, vocab = logits.shape
    dev, op = logits.device, case["op"]
    temperature = s.get("temperature", 1.0)
    logp, lse, entropy = (torch.zeros(rows, dtype=torch.float64, device=dev) for _ in range(3))
    step = max(1, int(2e8 // vocab))

    def parts():
        for r in range(0, rows, step):
            x = torch.log_softmax(logits[r:r + step].double() / temperature, 1)
            yield slice(r, r + step), x

    for at, x in parts():
        keep = w[at] != 0
        n = torch.logsumexp(logits[at].double() / temperature, 1)
        h = -torch.nan_to_num(x.exp() * x, nan=0.0).sum(1)
        logp[at] = torch.where(keep, x.gather(1, tokens[at, None])[:, 0], 0.0)
        lse[at], entropy[at] = torch.where(keep, n, 0.0), torch.where(keep, h, 0.0)
    if op == "logprob":
        return {"logp": logp, "lse": lse, "entropy": entropy}
    ent = 0.0
    if op == "policy":
        share, adv, ent = w / w.sum(), s["advantages"].double(), s["ent"]
        ratio = torch.exp(logp - s["old_logp"].double())
        low, high = ratio * adv, torch.clamp(ratio, 1 - CLIP, 1 + CLIP) * adv
        clipped = low > high
        term = torch.where(clipped, -high, -low)
        slope = torch.where(clipped, 0.0, -low)
        kl = torch.zeros_like(logp)
        if s["ref_logp"] is not None:
            d = s["ref_logp"].double() - logp
            kl = torch.expm1(d) - d
            slope = slope - s["kl"] * torch.expm1(d)
        stats = torch.stack([(x * share)[w != 0].sum() for x in (term + s["kl"] * kl - ent * entropy, term, kl, entropy, clipped.double())])
        out = {"stats": stats, "logp": logp, "entropy": entropy}
        a = slope * share
    else:
        ends = s["offsets"].tolist()
        seq = torch.stack([(logp * w)[i:j].sum() for i, j in zip(ends[:-1], ends[1:])])
        d = seq - s["ref_logp"].double()
        margin = s["beta"] * (d[0::2] - d[1::2])
        loss = -(1 - s["smooth"]) * torch.nn.functional.logsigmoid(margin) - s["smooth"] * torch.nn.functional.logsigmoid(-margin)
        out = {"stats": torch.stack([loss.mean(), (margin > 0).double().mean(), margin.mean()]), "seq_logp": seq}
        slope = ((1 - s["smooth"]) * -torch.sigmoid(-margin) + s["smooth"] * torch.sigmoid(margin)) * s["beta"] / len(margin)
        a = torch.zeros(rows, dtype=torch.float64, device=dev)
        for k, (i, j) in enumerate(zip(ends[:-1], ends[1:])):
            a[i:j] = slope[k // 2] * (1 if k % 2 == 0 else -1)
        a, share = a * w, w
    grad = torch.empty(rows, vocab, dtype=torch.float64, device=dev)
    for at, x in parts():
        p = x.exp()
        y = -a[at, None] * p
        if ent:
            y += torch.nan_to_num(p * (x + entropy[at, None]), nan=0.0) * (ent * share[at, None])
        y.scatter_add_(1, tokens[at, None], a[at, None])
        grad[at] = torch.where(w[at, None] != 0, y, 0.0) / temperature
    return {**out, "dlogits": grad}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "adamw"):
        return _exact_tensors(case, s)
    return _exact_losses(case, s)
