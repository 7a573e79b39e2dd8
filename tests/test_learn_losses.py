"""Token log probabilities, policy loss and preference loss (include/softsync_learn.h) against float64 on the CPU.

The reference computes each loss from its formula with torch in float64 and takes the gradient by automatic differentiation,
so the gradient formula in the header is checked by something that does not use it; differences of the operator's own loss
check it once more.
"""
import ctypes as C
import math

import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu
EPS = 2.0 ** -24


def make(rows, vocab, dtype, seed=0, std=3.0, pad=0, shift=0, masked=0.3, banned=0):
    """Logits as rows of a wider buffer (pad extra columns, shift elements off the start), tokens, weights; on the GPU."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(rows * (vocab + pad) + shift + 64, generator=g).mul_(std).to(dtype).cuda()
    x = buf[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    if banned:
        x[:, vocab - banned:] = -math.inf
    tokens = torch.randint(0, vocab - banned, (rows,), generator=g)
    weights = (torch.rand(rows, generator=g) + 0.5) * (torch.rand(rows, generator=g) >= masked)
    return x, tokens.cuda(), weights.cuda()


def reference_stats(x, tokens, weights, temperature):
    """(z leaf, logp, lse, entropy) in float64; zero where the weight is zero."""
    keep = weights.cpu() != 0
    leaf = x.detach().double().cpu().clone()
    leaf[~keep] = 0.0
    leaf.requires_grad_(True)
    z = leaf / temperature
    lse = torch.logsumexp(z, 1)
    logp = z.gather(1, tokens.cpu()[:, None]).squeeze(1) - lse
    p = torch.softmax(z, 1)
    entropy = lse - torch.where(p > 0, p * z.clamp(min=-1e300), 0.0).sum(1)
    zero = torch.zeros((), dtype=torch.float64)
    return leaf, torch.where(keep, logp, zero), torch.where(keep, lse, zero), torch.where(keep, entropy, zero)


def stat_tolerance(x, temperature):
    """The exponent's argument is rounded twice (the difference and its scaling; |d| up to the row's range), exp2 has two units in the
    last place, a thread adds up at most vocab / 32 terms one by one, and the result is a sum of three terms of at most `range + log V`."""
    span = float((x.float().masked_fill(torch.isinf(x.float()), 0.0).abs().max()) * 2 / temperature) + math.log(x.shape[1]) + 1
    return EPS * (8 * span + 4 * span + x.shape[1] / 32 + 32)


SHAPES = [  # rows, vocab, pad, shift
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 0, 1), (4, 33, 3, 0), (2, 255, 0, 0), (7, 1000, 8, 0), (3, 1001, 0, 3), (130, 4099, 0, 0),
    (1, 50257, 0, 0), (9, 50257, 0, 0), (6, 32000, 0, 0), (5, 131072, 0, 0), (2, 152001, 7, 5), (300, 515, 0, 0), (2, 270001, 0, 0), (3, 524288, 0, 0),
]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,pad,shift", SHAPES)
def test_token_logprob(dtype, rows, vocab, pad, shift):
    for temperature, banned in ((1.0, 0), (0.6, vocab // 3)):
        x, tokens, weights = make(rows, vocab, dtype, seed=rows + vocab, pad=pad, shift=shift, banned=banned)
        _, logp, lse, entropy = reference_stats(x, tokens, weights, temperature)
        r = P.token_logprob(x, tokens, weights, temperature)
        tol = stat_tolerance(x, temperature)
        for got, want in ((r.logp, logp), (r.lse, lse), (r.entropy, entropy)):
            assert (got.cpu().double() - want.detach()).abs().max() <= tol
        again = P.token_logprob(x, tokens, weights, temperature)
        assert all(torch.equal(a, b) for a, b in zip(r, again))
        plain = P.token_logprob(x, tokens, None, temperature)
        keep = weights != 0
        assert torch.equal(plain.logp[keep], r.logp[keep])


def policy_reference(x, tokens, weights, old, adv, ref, low, high, kl, ent, temperature):
    leaf, logp, _, entropy = reference_stats(x, tokens, weights, temperature)
    w, old, adv = weights.double().cpu(), old.double().cpu(), adv.double().cpu()
    share = w / w.sum() if float(w.sum()) else w
    ratio = torch.exp(logp - old)
    free, held = ratio * adv, ratio.clamp(1 - low, 1 + high) * adv
    term = -torch.minimum(free, held)
    k3 = torch.zeros_like(logp)
    if ref is not None:
        d = ref.double().cpu() - logp
        k3 = torch.exp(d) - d - 1
    loss = term + (kl if ref is not None else 0.0) * k3 - ent * entropy
    clipped = (free > held).double()
    stats = torch.stack([(share * q).sum() for q in (loss, term, k3, entropy, clipped)])
    grad = torch.autograd.grad(stats[0], leaf)[0]
    p = torch.softmax(leaf.detach() / temperature, 1)
    return stats.detach(), logp.detach(), entropy.detach(), grad, p, share


def policy_inputs(x, tokens, weights, temperature, seed, with_ref=True):
    """Ratios near one and far from it, none within 1 % of the clipping bounds 0.8 and 1.2 (where a rounding decides)."""
    g = torch.Generator().manual_seed(seed)
    rows = x.shape[0]
    logp = reference_stats(x, tokens, weights, temperature)[1].detach().float()
    near = torch.randn(rows, generator=g).mul_(0.05).clamp_(-0.15, 0.15)
    far = (torch.rand(rows, generator=g) + 0.3) * torch.sign(torch.randn(rows, generator=g))
    old = (logp - torch.where(torch.rand(rows, generator=g) < 0.4, far, near)).cuda()
    adv = torch.randn(rows, generator=g).cuda()
    ref = (logp + torch.randn(rows, generator=g) * 0.5).cuda() if with_ref else None
    return old, adv, ref


def gradient_close(got, want, scale, span, dtype):
    """scale: per row, the size of what multiplies p and the one-hot.  Relative error of p: (4 span + 16) eps as in the statistics; the row's
    factor adds that of logp (its exponential) and a dozen roundings.  bf16 output rounds once more."""
    bound = scale[:, None] * EPS * (16 * span + 64) * (want.abs() / scale.clamp(min=1e-300)[:, None] + 2e-2) + scale[:, None] * EPS
    if dtype == torch.bfloat16:
        bound = bound + want.abs() * 2.0 ** -8 + 1e-38
    err = (got.double().cpu() - want).abs()
    assert (err <= bound).all(), float((err / bound.clamp(min=1e-300)).max())


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,pad,shift", SHAPES)
def test_policy_loss(dtype, rows, vocab, pad, shift):
    for temperature, kl, ent, banned, with_ref in ((1.0, 0.1, 0.0, 0, True), (0.7, 0.05, 0.02, vocab // 3, True), (1.0, 0.0, 0.0, 0, False), (1.3, 0.0, 0.03, 0, False)):
        x, tokens, weights = make(rows, vocab, dtype, seed=rows * 3 + vocab, pad=pad, shift=shift, banned=banned)
        old, adv, ref = policy_inputs(x, tokens, weights, temperature, 5, with_ref)
        low, high = 0.2, 0.2
        stats, logp, entropy, grad, p, share = policy_reference(x, tokens, weights, old, adv, ref, low, high, kl, ent, temperature)
        r = P.policy_loss(x, tokens, old, adv, weights, ref, low, high, kl, ent, temperature)
        tol = stat_tolerance(x, temperature)
        assert (r.logp.cpu().double() - logp).abs().max() <= tol and (r.entropy.cpu().double() - entropy).abs().max() <= tol
        # the terms move with logp at most as fast as |rho A| + kl |e^d - 1| <= 20 here
        assert (r.stats.cpu().double() - stats).abs().max() <= 20 * tol + 16 * EPS * float(stats.abs().max())
        span = tol / EPS
        scale = share / temperature * (4 * adv.double().cpu().abs() + kl * 20 + ent * (span + 1))
        gradient_close(r.dlogits, grad, scale, span, dtype)
        assert bool((r.dlogits[weights == 0] == 0).all())
        # other buffers: a strided one, and the logits' own
        wide = torch.full((rows, vocab + 5), 9.0, dtype=dtype, device="cuda")
        P.policy_loss(x, tokens, old, adv, weights, ref, low, high, kl, ent, temperature, grad=wide[:, 2:2 + vocab])
        assert torch.equal(wide[:, 2:2 + vocab], r.dlogits) and bool((wide[:, :2] == 9).all()) and bool((wide[:, 2 + vocab:] == 9).all())
        none = P.policy_loss(x, tokens, old, adv, weights, ref, low, high, kl, ent, temperature, grad=False)
        assert none.dlogits is None and torch.equal(none.stats, r.stats)
        around = x._base.clone() if x._base is not None else None
        same = P.policy_loss(x, tokens, old, adv, weights, ref, low, high, kl, ent, temperature, grad="inplace")
        assert same.dlogits.data_ptr() == x.data_ptr() and torch.equal(x, r.dlogits) and torch.equal(same.stats, r.stats)
        if around is not None and around.dim() == 1 and pad:
            mine = torch.zeros_like(around, dtype=torch.bool)
            mine[shift:shift + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab] = True
            assert torch.equal(around[~mine], x._base[~mine])


@gpu
def test_policy_gradient_against_differences_of_the_loss():
    """Directional derivatives of the operator's own loss: central differences with a step h, error h^2 / 6 |third derivative| plus the
    loss's rounding over h; with h = 1e-2 and a loss of order one both are below 1e-4."""
    x, tokens, weights = make(40, 61, torch.float32, seed=3, std=1.0)
    old, adv, ref = policy_inputs(x, tokens, weights, 1.0, 7)
    args = dict(weights=weights, ref_logp=ref, kl_coef=0.2, entropy_coef=0.1)
    base = P.policy_loss(x, tokens, old, adv, **args)
    g = torch.Generator().manual_seed(1)
    for _ in range(8):
        d = torch.randn(x.shape, generator=g).cuda()
        d /= d.norm()
        h = 1e-2
        up = float(P.policy_loss(x + h * d, tokens, old, adv, grad=False, **args).stats[0])
        down = float(P.policy_loss(x - h * d, tokens, old, adv, grad=False, **args).stats[0])
        assert abs((up - down) / (2 * h) - float((base.dlogits * d).sum())) < 1e-4


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_nothing_may_be_read_from(dtype):
    """NaN, infinities and tokens out of range in rows of weight zero; all rows of weight zero; no rows."""
    for vocab in (37, 4097, 40000):
        x, tokens, weights = make(12, vocab, dtype, seed=2, masked=0.0)
        old, adv, ref = policy_inputs(x, tokens, weights, 1.0, 3)
        weights[3:7] = 0.0
        clean = P.policy_loss(x, tokens, old, adv, weights, ref, kl_coef=0.1, entropy_coef=0.1)
        x[3], x[4, ::2], x[5, 1], x[6] = math.nan, math.inf, -math.inf, -math.inf
        tokens[3], tokens[4], tokens[5] = -100, vocab, 1 << 40
        old[3], adv[4], ref[5] = math.nan, math.inf, math.nan
        dirty = P.policy_loss(x, tokens, old, adv, weights, ref, kl_coef=0.1, entropy_coef=0.1)
        for a, b in zip(clean, dirty):
            assert torch.equal(a, b)
        assert bool((dirty.dlogits[3:7] == 0).all()) and float(dirty.logp[3:7].abs().sum()) == 0.0
        none = P.policy_loss(x, tokens, old, adv, torch.zeros(12, device="cuda"), ref, kl_coef=0.1)
        assert none.stats.tolist() == [0.0] * 5 and not bool(none.dlogits.any())
    empty = P.policy_loss(x[:0], tokens[:0], old[:0], adv[:0])
    assert empty.stats.tolist() == [0.0] * 5 and empty.dlogits.shape == (0, vocab)
    assert P.token_logprob(x[:0], tokens[:0]).logp.numel() == 0


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 5003, 60000, 152000])
def test_extreme_rows(dtype, vocab):
    """A mask of the type's lowest value over everything (uniform), over all but one, over half; large logits; all minus infinity, a NaN, plus
    infinity and a token out of range (NaN, in that row alone)."""
    low = torch.finfo(dtype).min
    x, tokens, weights = make(10, vocab, dtype, seed=9, masked=0.0)
    weights.fill_(1.0)
    x[0] = low
    x[1], x[1, 5], tokens[1] = low, 2.0, 5
    x[2, vocab // 2:] = low
    x[3] *= 1e4
    x[4], x[4, 7], tokens[4] = -math.inf, 3.0, 7
    tokens[2] = 1
    r = P.token_logprob(x, tokens)
    assert abs(float(r.logp[0]) + math.log(vocab)) < 1e-5 * math.log(vocab) and abs(float(r.entropy[0]) - math.log(vocab)) < 1e-5 * math.log(vocab)
    assert float(r.logp[1]) == 0.0 and float(r.logp[4]) == 0.0 and float(r.lse[1]) == 2.0 and float(r.entropy[4]) == 0.0
    z = x[2, :vocab // 2].double()
    assert abs(float(r.lse[2]) - float(torch.logsumexp(z, 0))) < 1e-5
    z = x[3].double()
    assert abs(float(r.lse[3]) - float(torch.logsumexp(z, 0))) <= 4 * EPS * float(z.abs().max())
    old, adv = r.logp.clone(), torch.ones(10, device="cuda")
    g = P.policy_loss(x, tokens, old, adv).dlogits.double()
    for row in (0, 1, 2, 4):
        z = x[row].double()
        p = torch.exp(z - z.max()) / torch.exp(z - z.max()).sum()
        p[int(tokens[row])] -= 1.0
        assert (g[row] - p / 10).abs().max() <= 0.1 * 2.0 ** -8
    fine = P.token_logprob(x, tokens)
    x[5], x[6, 3], x[7, vocab - 1], tokens[8] = -math.inf, math.nan, math.inf, vocab
    r = P.policy_loss(x, tokens, old, adv)
    assert bool(torch.isnan(r.logp[5:9]).all()) and torch.equal(r.logp[:5], fine.logp[:5]) and torch.equal(r.logp[9:], fine.logp[9:])
    assert bool(torch.isnan(r.stats[0])) and bool(torch.isfinite(r.dlogits[:5]).all()) and bool(torch.isfinite(r.dlogits[9:]).all())
    assert bool(torch.isnan(r.dlogits[5:9].float()).any(1).all())


@gpu
def test_a_single_row_and_a_single_entry():
    x = torch.tensor([[1.5]], device="cuda")
    t = torch.zeros(1, dtype=torch.int64, device="cuda")
    r = P.policy_loss(x, t, torch.zeros(1, device="cuda"), torch.ones(1, device="cuda"))
    assert r.stats.tolist()[:2] == [-1.0, -1.0] and r.dlogits.tolist() == [[0.0]] and float(r.entropy) == 0.0


@gpu
def test_row_offsets_beyond_32_bits():
    """Rows that start more than 2^32 elements after the first (8.6 GB of bf16)."""
    vocab, stride = 1000, (1 << 31) + 8
    buf = torch.zeros(stride * 2 + vocab, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, vocab), (stride, 1))
    g = torch.Generator().manual_seed(4)
    small = torch.randn(3, vocab, generator=g).bfloat16().cuda()
    x.copy_(small)
    tokens = torch.tensor([1, 2, 999], device="cuda")
    old, adv = torch.full((3,), -7.0, device="cuda"), torch.ones(3, device="cuda")
    a, b = P.policy_loss(x, tokens, old, adv), P.policy_loss(small, tokens, old, adv)
    assert torch.equal(a.logp, b.logp) and torch.equal(a.dlogits, b.dlogits)
    P.policy_loss(x, tokens, old, adv, grad="inplace")
    assert torch.equal(x, b.dlogits)


# ---- preference loss ----------------------------------------------------------------------------------------------------

def preference_reference(x, tokens, weights, ends, ref, beta, smooth, temperature):
    leaf, logp, _, _ = reference_stats(x, tokens, weights, temperature)
    lw = logp * weights.double().cpu()
    seq = torch.stack([lw[i:j].sum() for i, j in zip(ends[:-1], ends[1:])])
    d = seq - ref.double().cpu()
    margin = beta * (d[0::2] - d[1::2])
    loss = -(1 - smooth) * torch.nn.functional.logsigmoid(margin) - smooth * torch.nn.functional.logsigmoid(-margin)
    stats = torch.stack([loss.mean(), (margin > 0).double().mean(), margin.mean()])
    grad = torch.autograd.grad(stats[0], leaf)[0]
    return stats.detach(), seq.detach(), grad


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths,vocab,pad,shift", [
    ([1, 1], 50, 0, 0), ([5, 0, 3, 7], 1001, 0, 1), ([0, 0], 33, 0, 0), ([20, 31, 1, 64], 4096, 8, 0), ([3, 2], 131072, 0, 0),
    ([40] * 34, 300, 0, 0), ([700, 3, 2, 1100], 129, 0, 0), ([2, 3], 152001, 0, 3),
])
def test_preference_loss(dtype, lengths, vocab, pad, shift):
    before, after = 2, 3                                               # rows that belong to no sequence
    ends = [before]
    for n in lengths:
        ends.append(ends[-1] + n)
    rows = ends[-1] + after
    for temperature, beta, smooth in ((1.0, 0.1, 0.0), (0.8, 0.3, 0.2)):
        x, tokens, weights = make(rows, vocab, dtype, seed=rows + vocab, pad=pad, shift=shift)
        logp = reference_stats(x, tokens, weights, temperature)[1].detach()
        g = torch.Generator().manual_seed(6)
        ref = torch.stack([(logp * weights.double().cpu())[i:j].sum() for i, j in zip(ends[:-1], ends[1:])]) + torch.randn(len(lengths), generator=g) * 5
        ref = ref.float().cuda()
        x[0], x[rows - 1] = math.nan, math.inf                         # outside every sequence
        x64 = x.clone()
        x64[0], x64[rows - 1] = 0.0, 0.0
        stats, seq, grad = preference_reference(x64, tokens, weights, ends, ref, beta, smooth, temperature)
        offs = torch.tensor(ends, device="cuda")
        r = P.preference_loss(x, tokens, offs, ref, weights, beta, smooth, temperature)
        tol = stat_tolerance(x64, temperature)
        longest, heaviest = max(lengths), 1.5
        seq_tol = tol * longest * heaviest + 2 * EPS * float(seq.abs().max())
        assert (r.seq_logp.cpu().double() - seq).abs().max() <= seq_tol
        ref_tol = EPS * float(ref.abs().max())
        slack = 4 * beta * (seq_tol + ref_tol)
        assert abs(float(r.stats[0]) - float(stats[0])) <= slack + 4 * EPS * float(stats[0])
        assert abs(float(r.stats[2]) - float(stats[2])) <= slack + 4 * EPS * abs(float(stats[2]))
        assert float(r.stats[1]) == pytest.approx(float(stats[1]), abs=1e-6)
        scale = weights.double().cpu() * beta / (len(lengths) // 2) / temperature
        want = grad
        err = (r.dlogits.double().cpu() - want).abs()
        bound = scale[:, None] * (slack + EPS * (16 * tol / EPS + 64)) * (want.abs() / scale.clamp(min=1e-300)[:, None] + 2e-2) + scale[:, None] * EPS
        bound = bound + (want.abs() * 2.0 ** -8 + 1e-38 if dtype == torch.bfloat16 else 0.0)
        assert (err <= bound).all()
        assert bool((r.dlogits[weights == 0] == 0).all()) and not bool(r.dlogits[:before].any()) and not bool(r.dlogits[rows - after:].any())
        again = P.preference_loss(x, tokens, offs, ref, weights, beta, smooth, temperature, grad="inplace")
        assert torch.equal(x, r.dlogits) and torch.equal(again.stats, r.stats) and torch.equal(again.seq_logp, r.seq_logp)


@gpu
def test_preference_gradient_against_differences_of_the_loss():
    x, tokens, weights = make(30, 45, torch.float32, seed=8, std=1.0)
    offs = torch.tensor([0, 8, 15, 15, 30], device="cuda")
    ref = torch.tensor([-30.0, -25.0, 0.0, -50.0], device="cuda")
    base = P.preference_loss(x, tokens, offs, ref, weights, 0.2, 0.1)
    g = torch.Generator().manual_seed(1)
    for _ in range(8):
        d = torch.randn(x.shape, generator=g).cuda()
        d /= d.norm()
        h = 1e-2
        up = float(P.preference_loss(x + h * d, tokens, offs, ref, weights, 0.2, 0.1, grad=False).stats[0])
        down = float(P.preference_loss(x - h * d, tokens, offs, ref, weights, 0.2, 0.1, grad=False).stats[0])
        assert abs((up - down) / (2 * h) - float((base.dlogits * d).sum())) < 1e-4


@gpu
def test_large_margins_and_hostile_offsets():
    x, tokens, _ = make(12, 100, torch.float32, seed=1)
    offs = torch.tensor([0, 3, 6, 9, 12], device="cuda")
    for far in (1e4, -1e4, 1e30):
        ref = torch.tensor([-far, 0.0, far, 0.0], device="cuda")
        r = P.preference_loss(x, tokens, offs, ref, beta=1.0)
        assert bool(torch.isfinite(r.stats).all()) and bool(torch.isfinite(r.dlogits).all())
    ref = torch.zeros(4, device="cuda")
    for bad in ([-5, 3, 6, 9, 12], [0, 3, 6, 9, 1 << 40], [9, 3, 6, 2, 12]):           # rows outside the logits are never touched
        r = P.preference_loss(x, tokens, torch.tensor(bad, device="cuda"), ref)
        assert bool(torch.isfinite(r.stats).all())
    none = P.preference_loss(x, tokens, torch.zeros(1, dtype=torch.int64, device="cuda"), ref[:0])
    assert none.stats.tolist() == [0.0] * 3 and not bool(none.dlogits.any())
    empty = P.preference_loss(x[:0], tokens[:0], torch.zeros(3, dtype=torch.int64, device="cuda"), ref[:2])
    assert float(empty.stats[0]) == pytest.approx(math.log(2.0), rel=1e-6) and empty.seq_logp.tolist() == [0.0, 0.0]


# ---- streams, refusals --------------------------------------------------------------------------------------------------

@gpu
def test_losses_run_on_the_current_stream():
    x, tokens, weights = make(64, 8000, torch.bfloat16, seed=4)
    old, adv, ref = policy_inputs(x, tokens, weights, 1.0, 3)
    want = P.policy_loss(x, tokens, old, adv, weights, ref, kl_coef=0.1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [P.policy_loss(x, tokens, old, adv, weights, ref, kl_coef=0.1) for _ in range(5)]
    other = [P.policy_loss(x, tokens, old, adv, weights, ref, kl_coef=0.1) for _ in range(5)]      # at the same time on the default one
    torch.cuda.synchronize()
    for r in got + other:
        assert all(torch.equal(a, b) for a, b in zip(r, want))


@gpu
def test_result_continues_into_autograd():
    h = torch.randn(6, 16, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    w = torch.randn(16, 50, device="cuda", generator=torch.Generator("cuda").manual_seed(2)).requires_grad_(True)
    logits = h @ w
    tokens = torch.arange(6, device="cuda")
    old, adv = torch.full((6,), -4.0, device="cuda"), torch.ones(6, device="cuda")
    r = P.policy_loss(logits, tokens, old, adv)
    logits.backward(r.dlogits)
    assert torch.allclose(w.grad, h.t() @ r.dlogits, rtol=1e-5, atol=1e-6)


def test_refusals_of_the_library_without_a_gpu():
    b = C.c_int64()
    assert P.ps_loss_workspace(10, 2, C.byref(b)) == P.PS_OK and b.value > 0
    assert P.ps_loss_workspace(-1, 0, C.byref(b)) == P.PS_ERR_INVALID_ARG and P.ps_loss_workspace(1, 0, None) == P.PS_ERR_INVALID_ARG

    def lg(**kw):
        k = dict(data_dev=0x1000, dtype=0, rows=4, vocab=8, row_stride=8, tokens_dev=0x2000, weights_dev=None, temperature=1.0)
        k.update(kw)
        return C.byref(P.binding.Logits(*[k[n] for n, _ in P.binding.Logits._fields_]))

    for bad in (dict(dtype=2), dict(rows=-1), dict(vocab=0), dict(row_stride=7), dict(temperature=0.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(temperature=1e-45), dict(data_dev=None), dict(data_dev=0x1002), dict(tokens_dev=None), dict(tokens_dev=0x2004),
                dict(weights_dev=0x3002), dict(rows=1 << 40), dict(row_stride=1 << 62)):
        assert P.ps_token_logprob(lg(**bad), 0x5000, None, None, None) == P.PS_ERR_INVALID_ARG, bad
    assert P.ps_token_logprob(lg(), None, None, None, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_token_logprob(None, 0x5000, None, None, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_token_logprob(lg(rows=0), None, None, None, None) == P.PS_OK

    def policy(grad=None, stride=8, ws=0x9000, ws_bytes=1 << 20, logp=0x5000, stats=0x6000, **kw):
        k = dict(old_logp_dev=0x7000, advantages_dev=0x7100, ref_logp_dev=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0)
        k.update(kw)
        p = P.binding.PolicyInputs(*[k[n] for n, _ in P.binding.PolicyInputs._fields_])
        return P.ps_policy_loss(lg(), C.byref(p), stats, logp, None, grad, stride, ws, ws_bytes, None)

    for bad in (dict(old_logp_dev=None), dict(advantages_dev=None), dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1), dict(clip_high=float("inf")),
                dict(kl_coef=float("nan")), dict(entropy_coef=float("inf")), dict(ws=None), dict(ws_bytes=16), dict(ws=0x9004), dict(logp=None), dict(stats=None),
                dict(grad=0x1010), dict(grad=0x1000, stride=9), dict(grad=0x8000, stride=7), dict(grad=0x8002)):
        assert policy(**bad) == P.PS_ERR_INVALID_ARG, bad

    def pref(**kw):
        k = dict(offsets_dev=0x7000, ref_logp_dev=0x7100, pairs=2, beta=0.1, label_smoothing=0.0)
        k.update(kw)
        p = P.binding.PreferenceInputs(*[k[n] for n, _ in P.binding.PreferenceInputs._fields_])
        return P.ps_preference_loss(lg(), C.byref(p), 0x6000, 0x6100, None, 8, 0x9000, 1 << 20, None)

    for bad in (dict(offsets_dev=None), dict(ref_logp_dev=None), dict(pairs=-1), dict(beta=float("nan")), dict(label_smoothing=1.5), dict(label_smoothing=-0.1),
                dict(offsets_dev=0x7004)):
        assert pref(**bad) == P.PS_ERR_INVALID_ARG, bad


@gpu
def test_refusals_of_the_python_calls():
    x, tokens, weights = make(4, 16, torch.float32)
    old = adv = torch.zeros(4, device="cuda")
    bad = [
        (TypeError, lambda: P.token_logprob(x.half(), tokens)),
        (ValueError, lambda: P.token_logprob(x[0], tokens)),
        (ValueError, lambda: P.token_logprob(x.t(), tokens)),
        (ValueError, lambda: P.token_logprob(x.cpu(), tokens.cpu())),
        (ValueError, lambda: P.token_logprob(x, tokens[:3])),
        (TypeError, lambda: P.token_logprob(x, tokens.int())),
        (ValueError, lambda: P.token_logprob(x, tokens.cpu())),
        (TypeError, lambda: P.token_logprob(x, tokens, weights.double())),
        (ValueError, lambda: P.token_logprob(x, tokens, weights[:2])),
        (P.SoftsyncError, lambda: P.token_logprob(x, tokens, temperature=0.0)),
        (ValueError, lambda: P.policy_loss(x, tokens, old[:3], adv)),
        (ValueError, lambda: P.policy_loss(x, tokens, old, adv, grad="elsewhere")),
        (ValueError, lambda: P.policy_loss(x, tokens, old, adv, grad=torch.zeros(4, 15, device="cuda"))),
        (ValueError, lambda: P.policy_loss(x, tokens, old, adv, grad=torch.zeros(4, 16, device="cuda", dtype=torch.bfloat16))),
        (P.SoftsyncError, lambda: P.policy_loss(x, tokens, old, adv, clip_low=2.0)),
        (ValueError, lambda: P.preference_loss(x, tokens, torch.zeros(4, dtype=torch.int64, device="cuda"), old)),
        (ValueError, lambda: P.preference_loss(x, tokens, torch.zeros(3, dtype=torch.int64, device="cuda"), old)),
        (TypeError, lambda: P.preference_loss(x, tokens, torch.zeros(3, dtype=torch.int32, device="cuda"), old[:2])),
    ]
    for k, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail("case %d was not refused" % k)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,pad,shift", [(1200, 3001, 0, 1), (640, 12001, 7, 0), (310, 50001, 0, 3), (170, 70001, 0, 0), (240, 65536, 8, 0), (160, 150001, 3, 2), (37, 600003, 0, 0)])
def test_policy_loss_of_many_rows(dtype, rows, vocab, pad, shift):
    """Several rows after one another in every block, with runs of rows without a weight between them."""
    x, tokens, weights = make(rows, vocab, dtype, seed=rows + vocab, pad=pad, shift=shift, masked=0.3)
    weights[rows // 3:rows // 2] = 0.0
    weights[-1] = 0.0
    old, adv, ref = policy_inputs(x, tokens, weights, 0.9, 6)
    for kl, ent in ((0.05, 0.0), (0.05, 0.02)):
        stats, logp, entropy, grad, p, share = policy_reference(x, tokens, weights, old, adv, ref, 0.2, 0.2, kl, ent, 0.9)
        r = P.policy_loss(x, tokens, old, adv, weights, ref, 0.2, 0.2, kl, ent, 0.9)
        tol = stat_tolerance(x, 0.9)
        assert (r.logp.cpu().double() - logp).abs().max() <= tol and (r.entropy.cpu().double() - entropy).abs().max() <= tol
        assert (r.stats.cpu().double() - stats).abs().max() <= 20 * tol + 16 * EPS * float(stats.abs().max())
        scale = share / 0.9 * (4 * adv.double().cpu().abs() + kl * 20 + ent * (tol / EPS + 1))
        gradient_close(r.dlogits, grad, scale, tol / EPS, dtype)
        assert bool((r.dlogits[weights == 0] == 0).all())
        del grad, p
    first = r.dlogits.clone()
    again = P.policy_loss(x, tokens, old, adv, weights, ref, 0.2, 0.2, kl, ent, 0.9, grad="inplace")
    assert torch.equal(x, first) and torch.equal(again.stats, r.stats)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab", [(700, 40), (330, 33000), (310, 70000)])
def test_policy_loss_of_mostly_masked_rows(dtype, rows, vocab):
    """More rows than are worked on at a time, of which none, the first, the last or all have a weight.  Masked rows hold NaN: they are not read.
    Weights of one are the same as none given, bit by bit, and what a row contributes does not depend on where it stands."""
    x, tokens, _ = make(rows, vocab, dtype, seed=rows, masked=0.0)
    old = torch.full((rows,), -math.log(vocab), device="cuda")
    adv = torch.linspace(-1, 1, rows, device="cuda")
    every = P.policy_loss(x, tokens, old, adv, torch.ones(rows, device="cuda"), entropy_coef=0.01)
    plain = P.policy_loss(x, tokens, old, adv, entropy_coef=0.01)
    for a, b in zip(every, plain):
        assert torch.equal(a, b)
    for live in ([], [0], [rows - 1], [0, rows // 2, rows - 1]):
        weights = torch.zeros(rows, device="cuda")
        weights[live] = 1.0
        y = torch.full_like(x, math.nan)
        y[live] = x[live]
        r = P.policy_loss(y, tokens, old, adv, weights, entropy_coef=0.01)
        dead = weights == 0
        assert bool((r.dlogits[dead] == 0).all()) and bool((r.logp[dead] == 0).all()) and bool((r.entropy[dead] == 0).all())
        if not live:
            assert r.stats.tolist() == [0.0] * 5
            continue
        few = P.policy_loss(x[live].contiguous(), tokens[live], old[live], adv[live], torch.ones(len(live), device="cuda"), entropy_coef=0.01)
        assert torch.equal(r.logp[live], every.logp[live]) and torch.equal(r.entropy[live], every.entropy[live])
        # the same rows alone may be cut into other parts: sums of fp32 in another order, at most vocab / 32 terms one by one
        tol = EPS * (vocab / 32 + 64) * 16
        assert (r.stats - few.stats).abs().max() <= tol * (1 + few.stats.abs().max())
