"""Losses and the gradient norm where their inputs are far from a well-behaved model's, compared with float64."""
import math

import numpy as np
import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu
EPS = 2.0 ** -24


def large_rows(vocab, dtype):
    """(logits on the GPU, tokens): rows whose softmax is ordinary although their logits are large."""
    g = torch.Generator().manual_seed(vocab)
    r = lambda: torch.randn(vocab, generator=g)
    half = r()
    half[vocab // 2:] = -1e9
    ties = torch.full((vocab,), -1e6)
    ties[::3] = -1e6 - 8192
    rows = [torch.full((vocab,), -1e9), torch.full((vocab,), -1e4), torch.full((vocab,), -65504.0), torch.full((vocab,), 1e7), torch.full((vocab,), -1e15),
            half, ties, r() + 3e4, r() * 1e4, r() * 3, r() + 700.0, torch.full((vocab,), -1e9)]
    x = torch.stack(rows).to(dtype).cuda()
    return x, x.float().argmax(1)                                     # a likely token: its log probability is a number of ordinary size


def softmax64(x, temperature):
    return torch.softmax(x.double() / temperature, 1)


def relative_error_of_p(vocab, dtype):
    """Where p counts (above 2^-40) the exponent is below 40 and comes from a difference, a scaling and a subtraction, rounded once each; a
    thread adds up at most vocab / 32 terms one by one; for bf16 the exponent may be off by 2^-15 as a whole."""
    return EPS * (4 * 40 + 64 + vocab / 32) + (2.0 ** -15 if dtype == torch.bfloat16 else 0.0)


def assert_gradient(got, p, tokens, a, b, dtype, vocab):
    """got against a (1[token] - p) + b p (log p + H), a and b per row."""
    hot = torch.zeros_like(p).scatter_(1, tokens[:, None], 1.0)
    logp = torch.where(p > 0, p, 1.0).log()
    entropy = -(p * logp).sum(1, keepdim=True)
    want = a[:, None] * (hot - p) + b[:, None] * p * (logp + entropy)
    rel = relative_error_of_p(vocab, dtype)
    size = a.abs()[:, None] * (p + 16 * EPS) + b.abs()[:, None] * p * (logp.abs() + entropy + 2)
    bound = rel * size + EPS * (a.abs() + b.abs())[:, None] * 2.0 ** -16 + want.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 16 * EPS)
    err = (got.double() - want).abs()
    worst = (err / bound).amax(1)
    assert (err <= bound).all(), worst.tolist()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 5003, 60000, 152000, 1000003])
@pytest.mark.parametrize("temperature,ent", [(1.0, 0.0), (1.0, 0.02), (0.004, 0.0)])
def test_policy_gradient_of_large_logits(dtype, vocab, temperature, ent):
    x, tokens = large_rows(vocab, dtype)
    rows = x.shape[0]
    p = softmax64(x, temperature)
    old = p.gather(1, tokens[:, None]).squeeze(1).log().float()       # ratio one
    adv = torch.linspace(0.5, 2.0, rows, device="cuda")
    r = P.policy_loss(x, tokens, old, adv, temperature=temperature, entropy_coef=ent)
    a = -adv.double() * (r.logp.double() - old.double()).exp() / rows / temperature      # the ratio that the call's own log probabilities give
    b = torch.full_like(a, ent / rows / temperature)
    assert_gradient(r.dlogits, p, tokens, a, b, dtype, vocab)
    # a buffer whose rows lie elsewhere in a 16-byte vector takes single elements: the same bits
    wide = torch.zeros(rows, vocab + 5, dtype=dtype, device="cuda")
    P.policy_loss(x, tokens, old, adv, temperature=temperature, entropy_coef=ent, grad=wide[:, 1:1 + vocab])
    assert torch.equal(wide[:, 1:1 + vocab], r.dlogits)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [40, 5003, 152000])
def test_preference_gradient_of_large_logits(dtype, vocab):
    x, tokens = large_rows(vocab, dtype)
    rows = x.shape[0]
    p = softmax64(x, 1.0)
    logp = p.gather(1, tokens[:, None]).squeeze(1).log()
    offsets = torch.arange(rows + 1, device="cuda")
    r = P.preference_loss(x, tokens, offsets, logp.float(), beta=0.1)  # margins of zero
    slope = -0.5 * 0.1 / (rows // 2)
    a = torch.where(torch.arange(rows, device="cuda") % 2 == 0, slope, -slope).double()
    # the margin's own error, beta (4 log probabilities of at most ~14 rounded to fp32), moves the slope by a quarter of it
    wide = torch.zeros(rows, vocab + 5, dtype=dtype, device="cuda")
    P.preference_loss(x, tokens, offsets, logp.float(), beta=0.1, grad=wide[:, 1:1 + vocab])
    assert torch.equal(wide[:, 1:1 + vocab], r.dlogits)
    assert_gradient(r.dlogits, p, tokens, a, torch.zeros_like(a), dtype, vocab)


@gpu
@pytest.mark.parametrize("smooth", [0.0, 0.1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_preference_gradient_of_confident_pairs(dtype, smooth):
    """The factor of pair i is beta / pairs (s sigmoid(margin) - (1 - s) sigmoid(-margin)): small for a pair that the model ranks right, and as
    exact as the margin is.  That is rounded to fp32 once, after log probabilities whose errors are below 1e-5 each: relative to a
    sigmoid that falls as e^-margin, at most beta * 4e-5 + 60 * 2^-24 < 5e-5; the products add a dozen roundings."""
    margins = torch.tensor([0.0, 3.0, 9.0, 12.0, 15.0, 17.5, 25.0, 60.0, -3.0, -12.0, -17.5, -60.0], dtype=torch.float64)
    pairs, vocab, beta = len(margins), 97, 0.5
    g = torch.Generator().manual_seed(2)
    x = torch.randn(2 * pairs, vocab, generator=g).to(dtype).cuda()
    tokens = torch.randint(0, vocab, (2 * pairs,), generator=g).cuda()
    p = softmax64(x, 1.0)
    logp = p.gather(1, tokens[:, None]).squeeze(1).log().cpu()
    ref = torch.zeros(2 * pairs, dtype=torch.float64)
    ref[1::2] = margins / beta - (logp[0::2] - logp[1::2])             # margin = beta (logp_0 - logp_1 + ref_1)
    ref = ref.float()
    r = P.preference_loss(x, tokens, torch.arange(2 * pairs + 1, device="cuda"), ref.cuda(), beta=beta, label_smoothing=smooth)
    margin = beta * (logp[0::2] - logp[1::2] + ref[1::2].double())
    slope = (smooth * torch.sigmoid(margin) - (1 - smooth) * torch.sigmoid(-margin)) * beta / pairs
    a = torch.stack([slope, -slope], 1).view(-1).cuda()[:, None]
    want = a * (torch.zeros_like(p).scatter_(1, tokens[:, None], 1.0) - p)
    err = (r.dlogits.double() - want).abs()
    part = (smooth * torch.sigmoid(margin) + (1 - smooth) * torch.sigmoid(-margin)) * beta / pairs      # what rounds before the two are subtracted
    size = torch.stack([part, part], 1).view(-1).cuda()[:, None] * want.abs() / a.abs()
    bound = size * 1e-4 + want.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert (err <= bound).all(), (err / bound).amax(1).tolist()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 40, 5003, 152000])
def test_rows_without_a_result_are_nan_in_every_output(dtype, vocab):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(8, vocab, generator=g).to(dtype).cuda()
    tokens = torch.zeros(8, dtype=torch.int64, device="cuda")
    want = P.token_logprob(x, tokens)
    x[1], x[2, vocab // 2], x[3, vocab - 1] = -math.inf, math.nan, math.inf
    tokens[4], tokens[5], tokens[6] = -1, vocab, 1 << 40
    r = P.token_logprob(x, tokens)
    q = P.policy_loss(x, tokens, torch.zeros(8, device="cuda"), torch.ones(8, device="cuda"), entropy_coef=0.1)
    for got, good in ((r.logp, want.logp), (r.lse, want.lse), (r.entropy, want.entropy), (q.logp, None), (q.entropy, None)):
        assert bool(torch.isnan(got[1:7]).all()) and bool(torch.isfinite(got[[0, 7]]).all())
        assert good is None or torch.equal(got[[0, 7]], good[[0, 7]])
    assert bool(torch.isnan(q.dlogits[1:7].float()).any(1).all()) and bool(torch.isfinite(q.dlogits[[0, 7]].float()).all())


@gpu
@pytest.mark.parametrize("dtype,c,shift", [(torch.bfloat16, 1, 0), (torch.float32, 1, 0), (torch.bfloat16, 2, 0), (torch.float32, 1, 1)])
def test_norm_of_long_gradients(dtype, c, shift):
    """A constant gradient is the worst case of a long sum: every addition rounds the same way.  Sums in fp32 end after at most 8 additions and
    3 joins, so the squares' sum is exact to 12 EPS, the norm to half of that; weighting rounds c products and c - 1 sums, the result once."""
    n = 3 << 27 if dtype == torch.bfloat16 else 3 << 26
    scale = 0.7371
    grads = [[torch.full((n + shift,), 1.171875, dtype=dtype, device="cuda")[shift:]]] * c
    scales = [scale] * c
    got = float(P.TensorList([n]).grad_norm(grads, scales)[0])
    exact = c * float(np.float32(scale)) * 1.171875 * math.sqrt(n)
    assert abs(got - exact) <= (6 + 2 * c + 1) * EPS * exact


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,rows", [(5003, 41), (50257, 41), (152000, 41), (1000003, 5)])
def test_confident_rows(dtype, vocab, rows):
    """Normalised logits (log probabilities) whose token has nearly all the probability and stands late in its row.  The sums are relative to a
    value at most 10 log2(e)-units, 7 natural ones, below the row's maximum.  In units of EPS: the difference to it is rounded to 4, the
    exponent to 6 + 8, 10 of them after the factor ln 2, the exponential to 4, its sum to 4, the logarithm (below 16) to 6 and its product to
    4, the difference of the token's logit to 4: 40 for log probability and normaliser.  The entropy's quotient carries the exponent's error and
    that of a product and a quotient once more: 64."""
    g = torch.Generator("cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, device="cuda", generator=g)
    tokens = torch.randint(vocab // 2, vocab, (rows,), device="cuda", generator=g)
    x.scatter_(1, tokens[:, None], torch.linspace(20 + math.log(vocab / 5e4), 60, rows, device="cuda")[:, None])
    x = torch.log_softmax(x, 1).to(dtype)
    exact = torch.log_softmax(x.double(), 1)
    logp, lse = exact.gather(1, tokens[:, None]).squeeze(1), torch.logsumexp(x.double(), 1)
    entropy = -(exact.exp() * exact).sum(1)
    r = P.token_logprob(x, tokens)
    q = P.policy_loss(x, tokens, torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), grad=False)
    for name, got, want, tol in (("logp", r.logp, logp, 40), ("lse", r.lse, lse, 40), ("entropy", r.entropy, entropy, 64), ("policy logp", q.logp, logp, 40),
                                 ("policy entropy", q.entropy, entropy, 64)):
        err = float((got.double() - want).abs().max())
        assert err <= tol * EPS, (name, err / EPS)
