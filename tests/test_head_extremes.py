"""The cross entropy and log probabilities from hidden states (include/softsync_learn.h) where they can lose what they promise: weights of any size, products whose
sums are long, confident rows, and the memory that a call asks for.

Tolerances are derived beside each test.  Sums of products in the tensor cores are cut towards zero to 24 bits at each of their additions (16 terms each), and are
taken out and added up to nearest every 1,024 terms: 64 cuts of at most 2^-23 of the sum so far, which in a sum of one sign is half its end on average.
"""
import ctypes as C
import math

import pytest
import torch

import paper_1511_05950_b200 as P
from tests.test_head_losses import BF16, HALF, Reference, close, make, struct

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


# ---- logits that are computed again ---------------------------------------------------------------------------------------

def confident(rows, width, z, seed):
    """Rows whose token 0 has a product of about z, all terms of one sign, and all else products of order one."""
    g = torch.Generator().manual_seed(seed)
    hidden = (0.5 + torch.rand(rows, width, generator=g)).to(BF16).cuda()
    head = (0.2 / math.sqrt(width) * torch.randn(300, width, generator=g))
    head[0] = z / width * (0.5 + torch.rand(width, generator=g))
    return hidden, head.to(BF16).cuda(), torch.zeros(rows, dtype=torch.int64, device="cuda")


@gpu
@pytest.mark.parametrize("width", [1024, 4096, 16384])
def test_wide_confident_rows_from_lse(width):
    """p of the token is 1 but for e^-90, so its G = p - 1 shows how well lse and the logit that is computed again agree: both are the same sum.  What is left is the rounding
    of lse (below 128: 2^-18), and of two products of about 150 in the exponent (2^-17 each, times log 2)."""
    hidden, head, tokens = confident(60, width, 100.0, width)
    score = P.head_logprob(hidden, head, tokens)
    z = hidden.double() @ head.double().T
    assert float(z[:, 0].min()) > 90 and float(z[:, 0].max()) < 128 and float(z[:, 1:].max()) < 10
    dhidden = P.head_logprob_grad(hidden, head, tokens, score.lse, torch.full((60,), -1.0, device="cuda"), grad="hidden").dhidden.double()
    tol = (2.0 ** -18 + 2 * 2.0 ** -17 * math.log(2)) * (1 + 2 * HALF)
    rest = torch.exp(z[:, 1:] - score.lse.double()[:, None]).abs() @ head[1:].double().abs()
    assert bool((dhidden.abs() <= tol * head[0].double().abs() + 2 * rest + 1e-38).all())


@gpu
@pytest.mark.parametrize("temperature", [0.7, 1.0, 0.3])
def test_products_of_hundreds_from_lse(temperature):
    """The difference to lse comes before the exponential's scale: with products over T of up to 512 only lse's own rounding is left (2^-16)."""
    hidden, head, tokens = confident(200, 256, 330.0 * temperature, 61)
    hidden *= torch.linspace(0.8, 1.25, 200, device="cuda")[:, None].to(BF16)
    score = P.head_logprob(hidden, head, tokens, temperature=temperature)
    z = hidden.double() @ head.double().T / temperature
    assert 250 < float(z[:, 0].max()) < 512 and float((z[:, 1:] - z[:, :1]).max()) < -150
    dhidden = P.head_logprob_grad(hidden, head, tokens, score.lse, torch.full((200,), -1.0, device="cuda"), temperature=temperature, grad="hidden").dhidden.double()
    assert bool((dhidden.abs() <= 2.0 ** -16 * (1 + 2 * HALF) * head[0].double().abs() / temperature + 1e-38).all())


@gpu
@pytest.mark.parametrize("width", [1100, 2048])
def test_gradient_from_lse_at_usual_widths(width):
    hidden, head, tokens, weights = make(333, width, 3001, seed=width)
    ref = Reference(hidden, head, tokens, 0.9)
    lse = P.head_logprob(hidden, head, tokens, temperature=0.9).lse
    g = P.head_logprob_grad(hidden, head, tokens, lse, -weights, temperature=0.9)
    dhidden, tol_h, dhead, tol_w = ref.gradients(weights)
    assert close(g.dhidden, dhidden, tol_h) and close(g.dhead, dhead, tol_w)


# ---- memory and refusals (no GPU) -----------------------------------------------------------------------------------------

SLOTS, TILE, STEP, MOST = 74, 256, 64, 3               # CTA pairs, tile, steps of a stage; parts of split tiles that there is room for, in slots
CHOICES = (1, 2, 3, 4, 6, 8, 12, 16, 24, 37, 74)


def up(x, by):
    return -(-x // by)


def parts_of(m, n, k, slots):
    """Parts of split tiles that a product of these extents has, by the rule that the kernels follow."""
    steps, rest = up(k, STEP), up(m, TILE) * up(n, TILE) % slots

    def cost(s):
        if s == 1:
            return 5 * (steps + 6)
        if steps < 16 or s * 4 > steps or rest * s > MOST * slots:
            return 1 << 40
        return 5 * (up(rest * s, slots) * (up(steps, s) + 6) + 8) + rest * s

    best = min(CHOICES, key=cost)
    return rest * best if rest and best > 1 else 0


def head_bytes(rows, width, vocab, grad=1):
    n = C.c_int64()
    h = struct(rows=rows, width=width, vocab=vocab, hidden_stride=width, head_stride=width)
    assert P.ps_head_workspace(C.byref(h), grad, C.byref(n)) == P.PS_OK
    return n.value


def packed_bytes(rows, outs, cols):
    n = C.c_int64()
    a = P.binding.PackedGrad(dout_dev=4096, codes_dev=4096, scales_dev=4096, gain_dtype=P.PS_GRAD_FP32, out_dtype=P.PS_GRAD_BF16, rows=rows, outs=outs, cols=cols, dout_stride=outs,
                             dweight_dev=8192)
    assert P.ps_packed_grad_workspace(C.byref(a), C.byref(n)) == P.PS_OK
    return n.value


def pieces_of(rows, width, vocab):
    """(first column of the kept piece, columns of the others) and the columns of G."""
    most = max(TILE, max(1 << 30, rows * width * 2) // (2 * up(rows, STEP) * STEP) // TILE * TILE)
    first = up(vocab - most, TILE) * TILE if vocab > most else 0
    piece = up(up(first, up(first, most)), TILE) * TILE if first else 0
    return first, piece, up(max(piece, vocab - first), TILE) * TILE


@pytest.mark.parametrize("rows,width,vocab", [(1, 64, 500), (48, 256, 32000), (300, 512, 2000), (1000, 1000, 50257), (700, 4096, 4096), (8192, 2048, 131072), (5000, 64, 200), (2000, 520, 700),
                                              (20001, 64, 60001)])
def test_room_for_every_split(rows, width, vocab):
    """Beside G and the sums over pieces there is room for the parts of both gradients, for any number of rows that take part and any number of pairs of CTAs, and not much more."""
    first, piece, columns = pieces_of(rows, width, vocab)
    others = up(rows, STEP) * STEP * columns * 2 + (rows * up(width, STEP) * STEP * 4 if first else 0)
    room = head_bytes(rows, width, vocab) - head_bytes(rows, width, vocab, 0) - others
    most_h = most_w = 0
    for live in sorted({*range(1, min(rows, 70)), *range(1, rows, max(1, rows // 200)), rows}):
        for slots in (SLOTS, SLOTS - 1, 60, 37, 2):
            for n in {vocab - first, piece or vocab, (first % piece if piece else 0) or vocab - first}:
                most_h, most_w = max(most_h, parts_of(live, width, n, slots)), max(most_w, parts_of(n, width, live, slots))
    part = TILE * TILE * 4
    assert room >= (most_h + most_w) * part
    widest = max(piece, vocab - first)
    ceiling = sum(min(MOST * SLOTS, min(up(m, TILE) * up(width, TILE), SLOTS - 1) * min(74, k // (4 * STEP) + 1)) * part for m, k in ((rows, widest), (widest, rows)) if k > 15 * STEP)
    assert room <= ceiling + 2048


def test_small_calls_ask_for_little():
    assert head_bytes(1, 64, 500) < 1 << 18                                    # it was 116 MB
    assert head_bytes(48, 256, 32000) < 64 * 32256 * 2 + 74 * TILE * TILE * 4 + (1 << 20)
    assert packed_bytes(1, 8, 33) < 1 << 14
    for rows, outs, cols in ((1, 8, 33), (200, 768, 256), (8192, 256, 256), (8192, 8192, 2048), (1023, 64, 64), (1024, 64, 64), (100000, 520, 72)):
        parts = max(parts_of(outs, cols, rows, slots) for slots in (74, 73, 60, 37, 2))
        values = rows * up(cols, 64) * 128
        assert packed_bytes(rows, outs, cols) >= values + parts * TILE * TILE * 4


@pytest.mark.parametrize("bad", [dict(rows=1 << 26, vocab=1 << 28), dict(rows=1 << 26, vocab=1 << 26), dict(temperature=3e-39), dict(temperature=4e-39)], ids=str)
def test_refused_before_anything_is_launched(bad):
    """More tiles than a launch counts, and temperatures whose exponent's scale log2(e) / T is beyond fp32."""
    n = C.c_int64()
    h = struct(**bad)
    assert P.ps_head_workspace(C.byref(h), 1, C.byref(n)) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob(C.byref(h), 256, 256, 256, 256, 1 << 60, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_cross_entropy(C.byref(h), 256, 256, 256, 256, 256, 256, 256, 1 << 60, None) == P.PS_ERR_INVALID_ARG


def test_weight_gradient_of_too_many_tiles_is_refused():
    n = C.c_int64()
    a = P.binding.PackedGrad(dout_dev=4096, codes_dev=4096, scales_dev=4096, gain_dtype=P.PS_GRAD_FP32, out_dtype=P.PS_GRAD_BF16, rows=4, outs=1 << 28, cols=1 << 20, dout_stride=1 << 28,
                             dweight_dev=8192)
    assert P.ps_packed_grad_workspace(C.byref(a), C.byref(n)) == P.PS_ERR_INVALID_ARG
    assert P.ps_packed_weight_grad(C.byref(a), 256, 1 << 60, None) == P.PS_ERR_INVALID_ARG
