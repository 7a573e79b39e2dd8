"""The cross entropy and log probabilities from hidden states (include/softsync_learn.h) where they can lose what they promise: weights of any size, products whose
sums are long, confident rows, and the memory that a call asks for.

Tolerances are derived beside each test.  Sums of products in the tensor cores are cut towards zero to 24 bits at each of their additions (16 terms each), and are
taken out and added up to nearest every 1,024 terms: 64 cuts of at most 2^-23 of the sum so far, which in a sum of one sign is half its end on average.
"""
import math

import pytest
import torch

import paper_1511_05950_b200 as P
from tests.test_head_losses import Reference, close, make

gpu = pytest.mark.gpu


def powers(rows, seed=1):
    """Weights of eight bits between a half and three halves: exact at every size used here, subnormal ones included."""
    return (torch.randint(128, 385, (rows,), generator=torch.Generator().manual_seed(seed)) / 256).cuda()


# ---- weights of any size --------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("power", [-140, -126, -100, 40, 64, 100, 126])
def test_the_size_of_the_weights_does_not_matter(power):
    """loss and gradients are divided by the sum of the weights: a power of two in all of them changes no bit, though their sum may be subnormal (exact all the same:
    a multiple of 2^-149) or beyond fp32."""
    rows, width, vocab = 300, 128, 1000
    hidden, head, tokens, _ = make(rows, width, vocab, seed=51)
    weights = powers(rows)
    weights[::7] = 0.0
    want = P.head_cross_entropy(hidden, head, tokens, weights=weights)
    ref = Reference(hidden, head, tokens)
    dhidden, tol_h, dhead, tol_w = ref.gradients(weights.double() / weights.double().sum())
    assert close(want.dhidden, dhidden, tol_h) and close(want.dhead, dhead, tol_w)
    got = P.head_cross_entropy(hidden, head, tokens, weights=(weights.double() * 2.0 ** power).float())
    assert torch.equal(got.logp, want.logp) and torch.equal(got.lse, want.lse) and torch.equal(got.stats[0], want.stats[0])
    assert torch.equal(got.dhidden, want.dhidden) and torch.equal(got.dhead, want.dhead)
    total = (weights.double().sum() * 2.0 ** power).float()
    assert torch.equal(got.stats[1], total)


@gpu
@pytest.mark.parametrize("power", [-112, -60, 60, 100])
def test_the_size_of_dlogp_goes_through(power):
    """Gradients are those of dlogp times the power, but for what bf16 cannot hold (its step below 2^-126 is 2^-133): entries of G of any likelihood are rounded relative
    to the largest dlogp."""
    hidden, head, tokens, _ = make(300, 128, 1000, seed=52)
    dlogp = -powers(300)
    lse = P.head_logprob(hidden, head, tokens).lse
    want = P.head_logprob_grad(hidden, head, tokens, lse, dlogp)
    got = P.head_logprob_grad(hidden, head, tokens, lse, (dlogp.double() * 2.0 ** power).float())
    for a, b in zip(got, want):
        assert bool((((a.double() * 2.0 ** -power) - b.double()).abs() <= 2.0 ** (-134 - power)).all())


@gpu
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_a_dlogp_that_is_no_number_spoils_its_row_alone(bad):
    hidden, head, tokens, _ = make(200, 64, 500, seed=53)
    dlogp = (-powers(200).double() * 2.0 ** -100).float()
    lse = P.head_logprob(hidden, head, tokens).lse
    want = P.head_logprob_grad(hidden, head, tokens, lse, dlogp)
    dlogp[77] = bad
    got = P.head_logprob_grad(hidden, head, tokens, lse, dlogp)
    others = torch.arange(200, device="cuda") != 77
    assert torch.equal(got.dhidden[others], want.dhidden[others]) and not bool(got.dhidden[77].isfinite().any()) and not bool(got.dhead.isfinite().all(1).any())


# ---- memory and refusals (no GPU) -----------------------------------------------------------------------------------------
