"""Losses without logits (include/softsync_learn.h) against float64: log probabilities, cross entropy and gradients from hidden states and the
output matrix.

Tolerances.  Products of bf16 values are exact in fp32.  A sum of K of them is off by at most (K / 16 + 16) 2^-23 of the sum of their magnitudes
(16 at a time, each addition rounded or cut to 24 bits), which is at most |h| |w|: `products`.  The exponent's argument is rounded twice, the exponential
has two units in the last place, the sums of a row are of 32 terms, then of 4 runs, then of its parts.  A gradient's G = a (p - 1[token]) is rounded to bf16 (half a step:
2^-8) and has the error of p, which may come through 16 bits of its own (half a step 2^-11, zero below 2^-62); the sums over vocabulary or rows are products again; the result is rounded to bf16 once.
"""
import ctypes as C
import math

import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu
EPS, HALF = 2.0 ** -24, 2.0 ** -8
BF16 = torch.bfloat16


def matrix(g, rows, cols, scale, pad=0, shift=0):
    """rows x cols of a wider buffer: pad extra columns, shift elements off the start."""
    buf = (torch.randn(rows * (cols + pad) + shift, generator=g) * scale).to(BF16).cuda()
    return buf[shift:].view(rows, cols + pad)[:, :cols]


def make(rows, width, vocab, seed=0, pad=(0, 0), shift=(0, 0), masked=0.3):
    g = torch.Generator().manual_seed(seed)
    head = matrix(g, vocab, width, 2.0 / math.sqrt(width), pad[1], shift[1])
    tokens = torch.randint(0, vocab, (rows,), generator=g).cuda()
    hidden = matrix(g, rows, width, 1.0, pad[0], shift[0])
    hidden.add_((1.5 * torch.rand(rows, 1, generator=g).cuda() * head[tokens].float()).to(BF16))
    weights = (torch.rand(rows, generator=g) + 0.5) * (torch.rand(rows, generator=g) >= masked)
    return hidden, head, tokens, weights.cuda()


def products(a_norm, b_norm, k):
    return (k / 16 + 16) * 2.0 ** -23 * a_norm * b_norm


class Reference:
    """Everything in float64, with the tolerance of each."""

    def __init__(self, hidden, head, tokens, temperature=1.0):
        self.h, self.w, self.t, self.temperature = hidden.double(), head.double(), tokens, temperature
        self.z = self.h @ self.w.T / temperature
        self.lse = torch.logsumexp(self.z, 1)
        self.rows = torch.arange(len(tokens), device="cuda")
        self.logp = self.z[self.rows, tokens] - self.lse
        h_norm, w_norm = float(self.h.norm(dim=1).max()), float(self.w.norm(dim=1).max())
        span = float(self.z.abs().max()) * 2 + math.log(head.shape[0]) + 1
        self.z_tol = products(h_norm, w_norm, hidden.shape[1]) / temperature + EPS * 4 * span
        self.tol = 2 * self.z_tol + EPS * (8 * span + 48 + head.shape[0] / 128)

    def gradients(self, a):
        """(dhidden, its tolerance, dhead, its tolerance) for dloss/dz = a (p - 1[token]), a without the 1 / temperature."""
        p = torch.exp(self.z - self.lse[:, None])
        g = p.clone()
        g[self.rows, self.t] -= 1
        a = a.double()[:, None] / self.temperature
        off = a.abs() * (HALF * g.abs() + (2 * self.tol + 8 * EPS + 2.0 ** -11) * p + 2.0 ** -62)
        g, size = a * g, a.abs() * g.abs()

        def product(m, off, size, other, k):
            value = m @ other
            tol = off @ other.abs() + (k / 16 + 64) * 2.0 ** -23 * (size @ other.abs())
            return value, tol * (1 + HALF) + HALF * value.abs() + 1e-38

        return (*product(g, off, size, self.w, g.shape[1]), *product(g.T, off.T, size.T, self.h, g.shape[0]))


def close(got, want, tol):
    off = (got.double() - want).abs()
    fine = bool((off <= tol).all())
    if not fine:
        print("off by up to %.3g of the tolerance in %d places" % (float((off / tol).max()), int((off > tol).sum())))
    return fine


SHAPES = [  # rows, width, vocab
    (1, 1, 1), (1, 8, 2), (3, 7, 33), (1, 64, 500), (5, 64, 127), (129, 65, 129), (255, 100, 257), (256, 128, 256), (300, 333, 1001), (64, 256, 4099),
    (257, 1024, 300), (1000, 72, 20000), (2, 4096, 513), (48, 256, 32000), (700, 520, 2500),
]


@gpu
@pytest.mark.parametrize("rows,width,vocab", SHAPES)
def test_cross_entropy_and_gradients(rows, width, vocab):
    for temperature, masked in ((1.0, None), (0.7, 0.4)):
        hidden, head, tokens, weights = make(rows, width, vocab, seed=rows + vocab, masked=masked or 0.0)
        if masked is None:
            weights = None
        ref = Reference(hidden, head, tokens, temperature)
        w = torch.ones(rows, device="cuda") if weights is None else weights
        total = float(w.double().sum())
        r = P.head_cross_entropy(hidden, head, tokens, weights=weights, temperature=temperature)
        keep = w != 0
        assert close(r.logp, ref.logp * keep, ref.tol) and close(r.lse, ref.lse * keep, ref.tol)
        assert bool((r.logp[~keep] == 0).all()) and bool((r.lse[~keep] == 0).all()) and bool((r.dhidden[~keep] == 0).all())
        share = w.double() / total if total else w.double()
        want = -float((share * ref.logp).sum())
        assert abs(float(r.stats[0]) - want) <= ref.tol + EPS * 8 * abs(want) and abs(float(r.stats[1]) - total) <= 2 * EPS * total
        dhidden, tol_h, dhead, tol_w = ref.gradients(share)
        assert close(r.dhidden, dhidden, tol_h) and close(r.dhead, dhead, tol_w)
        again = P.head_cross_entropy(hidden, head, tokens, weights=weights, temperature=temperature)
        assert all(torch.equal(x, y) for x, y in zip(r, again))
        score = P.head_logprob(hidden, head, tokens, weights=weights, temperature=temperature)
        assert torch.equal(score.logp, r.logp) and torch.equal(score.lse, r.lse)
        for which in ("hidden", "head"):
            one = P.head_cross_entropy(hidden, head, tokens, weights=weights, temperature=temperature, grad=which)
            got = {"hidden": one.dhidden, "head": one.dhead}
            assert torch.equal(got.pop(which), {"hidden": r.dhidden, "head": r.dhead}[which]) and list(got.values()) == [None]


@gpu
def test_pieces_of_the_vocabulary():
    """More rows and entries than one piece of G holds (1 GiB): the kept one and two that are computed again, of an odd width in all."""
    rows, vocab = 20001, 60001
    hidden, head, tokens, weights = make(rows, 64, vocab, seed=5, masked=0.1)
    r = P.head_cross_entropy(hidden, head, tokens, weights=weights)
    a = weights.double() / weights.double().sum()
    dhead, tol_w = torch.zeros(vocab, 64, dtype=torch.float64, device="cuda"), torch.zeros(vocab, 64, dtype=torch.float64, device="cuda")
    for first in range(0, rows, 5000):                                 # the reference by rows: their gradients of the head add up
        part = slice(first, first + 5000)
        ref = Reference(hidden[part], head, tokens[part])
        keep = weights[part] != 0
        assert close(r.logp[part], ref.logp * keep, ref.tol)
        dhidden, tol_h, more, tol = ref.gradients(a[part])
        assert close(r.dhidden[part], dhidden, tol_h)
        dhead += more
        tol_w += tol
    assert close(r.dhead, dhead, tol_w + (rows / 16) * 2.0 ** -23 * (a[:, None] * hidden.double().abs()).sum(0))
    again = P.head_logprob_grad(hidden, head, tokens, r.lse, -a.float())
    assert float((again.dhidden.double() - r.dhidden.double()).norm()) <= 2 * HALF * float(r.dhidden.double().norm())
    assert float((again.dhead.double() - r.dhead.double()).norm()) <= 2 * HALF * float(r.dhead.double().norm())


@gpu
def test_a_head_of_more_than_two_to_the_31_values():
    rows, width, vocab = 5, 4096, 530001
    hidden, _, _, _ = make(rows, width, 2, seed=6)
    g = torch.Generator("cuda").manual_seed(7)
    head = torch.empty(vocab, width, dtype=BF16, device="cuda").normal_(generator=g).mul_(2.0 / math.sqrt(width))
    tokens = torch.tensor([0, vocab - 1, 5, 524290, vocab - 1], device="cuda")
    r = P.head_cross_entropy(hidden, head, tokens)
    z = torch.cat([hidden.double() @ part.double().T for part in head.split(65536)], 1)
    lse = torch.logsumexp(z, 1)
    logp = z[torch.arange(rows), tokens] - lse
    tol = 2 * products(float(hidden.double().norm(dim=1).max()), float(head[:1000].float().norm(dim=1).max()) * 1.2, width) + EPS * (300 + vocab / 128)
    assert close(r.logp, logp, tol)
    for last in (slice(vocab - 300, vocab), slice(524200, 524400), slice(0, 10)):
        p = torch.exp(z[:, last] - lse[:, None])
        one = (tokens[:, None] == torch.arange(last.start, last.stop, device="cuda")).double()
        want = (p - one).T @ hidden.double() / rows
        size = ((p - one).abs() + p).T @ hidden.double().abs() / rows
        assert close(r.dhead[last], want, (HALF + 2.0 ** -11 + 4 * tol) * size + HALF * want.abs() + 1e-30)


@gpu
@pytest.mark.parametrize("pad,shift", [((8, 16), (0, 8)), ((3, 0), (1, 0)), ((0, 5), (0, 3)), ((1, 1), (1, 1)), ((0, 0), (4, 4))])
def test_strides_and_alignment(pad, shift):
    hidden, head, tokens, weights = make(70, 72, 601, seed=3, pad=pad, shift=shift)
    dense = P.head_cross_entropy(hidden.contiguous(), head.contiguous(), tokens, weights=weights)
    r = P.head_cross_entropy(hidden, head, tokens, weights=weights)
    assert all(torch.equal(x, y) for x, y in zip(r, dense))
    r = P.head_cross_entropy(hidden, head, tokens)
    dense = P.head_cross_entropy(hidden.contiguous(), head.contiguous(), tokens)
    assert all(torch.equal(x, y) for x, y in zip(r, dense))


@gpu
def test_rows_without_a_weight_are_not_read():
    hidden, head, tokens, weights = make(300, 96, 700, seed=9)
    want = P.head_cross_entropy(hidden, head, tokens, weights=weights)
    gone = weights == 0
    spoiled, lost = hidden.clone(), tokens.clone()
    spoiled[gone] = float("nan")
    spoiled[gone.nonzero()[0]] = float("inf")
    lost[gone] = -7
    got = P.head_cross_entropy(spoiled, head, lost, weights=weights)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    dlogp = torch.where(gone, 0.0, -weights)
    lse = torch.where(gone, float("nan"), want.lse)
    a, b = (P.head_logprob_grad(x, head, t, l, dlogp) for x, t, l in ((hidden, tokens, want.lse), (spoiled, lost, lse)))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_no_weight_at_all_and_one_row():
    hidden, head, tokens, _ = make(130, 64, 300, seed=11)
    none = P.head_cross_entropy(hidden, head, tokens, weights=torch.zeros(130, device="cuda"))
    assert all(bool((x == 0).all()) for x in none)
    for at in (0, 127, 129):
        weights = torch.zeros(130, device="cuda")
        weights[at] = 0.25
        r = P.head_cross_entropy(hidden, head, tokens, weights=weights)
        alone = P.head_cross_entropy(hidden[at:at + 1], head, tokens[at:at + 1])
        assert torch.equal(r.logp[at], alone.logp[0]) and abs(float(r.stats[0] - alone.stats[0])) <= 2 * EPS * abs(float(alone.stats[0]))
        assert torch.equal(r.dhidden[at], alone.dhidden[0]) and torch.equal(r.dhead, alone.dhead)
        assert float(r.dhidden.abs().sum()) == float(r.dhidden[at].abs().sum())


@gpu
def test_empty():
    hidden, head, tokens, _ = make(4, 64, 300)
    r = P.head_cross_entropy(hidden[:0], head, tokens[:0])
    assert r.dhidden.shape == (0, 64) and r.logp.numel() == 0 and bool((r.dhead == 0).all()) and r.stats.tolist() == [0, 0]
    g = P.head_logprob_grad(hidden[:0], head, tokens[:0], r.lse, r.logp)
    assert g.dhidden.shape == (0, 64) and bool((g.dhead == 0).all())
    assert P.head_logprob(hidden[:0], head, tokens[:0]).logp.numel() == 0


@gpu
@pytest.mark.parametrize("kind", ["nan", "inf", "token", "negative token"])
def test_a_bad_row_spoils_itself_and_the_sums(kind):
    hidden, head, tokens, _ = make(200, 64, 300, seed=13)
    want = P.head_cross_entropy(hidden, head, tokens)
    hidden, tokens = hidden.clone(), tokens.clone()
    if "token" in kind:
        tokens[77] = -1 if "negative" in kind else 300
    else:
        hidden[77, 5] = float(kind)
    r = P.head_cross_entropy(hidden, head, tokens)
    others = torch.arange(200, device="cuda") != 77
    assert torch.equal(r.logp[others], want.logp[others]) and torch.equal(r.dhidden[others], want.dhidden[others])
    assert bool(r.logp[77].isnan()) and bool(r.lse[77].isnan()) and bool(r.dhidden[77].isnan().all())
    assert bool(r.stats[0].isnan()) and bool(r.dhead.isnan().any())


@gpu
def test_a_bad_token_in_the_gradient():
    hidden, head, tokens, weights = make(70, 64, 300, seed=14, masked=0.0)
    lse = P.head_logprob(hidden, head, tokens).lse
    tokens[3] = 300
    g = P.head_logprob_grad(hidden, head, tokens, lse, -weights)
    assert bool(g.dhidden[3].isnan().all()) and bool(g.dhead.isnan().any()) and int(g.dhidden.isnan().any(1).sum()) == 1
    weights[3] = 0.0                                                   # and now it takes no part
    g = P.head_logprob_grad(hidden, head, tokens, lse, -weights)
    assert bool(g.dhidden.isfinite().all()) and bool(g.dhead.isfinite().all()) and bool((g.dhidden[3] == 0).all())


@gpu
def test_barred_entries():
    """Entries whose product is minus infinity have no probability; a row of nothing else is NaN."""
    hidden, head, tokens, _ = make(40, 64, 300, seed=17)
    hidden[:, 0], head[:, 0] = 1.0, 0.0
    tokens = tokens % 200
    want = P.head_logprob(hidden, head[:200].contiguous(), tokens)
    head[200:, 0] = -math.inf
    got = P.head_logprob(hidden, head, tokens)
    assert close(got.logp, want.logp.double(), 8 * EPS * float(want.logp.abs().max()) + 64 * EPS)
    head[:, 0] = -math.inf
    got = P.head_logprob(hidden, head, tokens)
    assert bool(got.logp.isnan().all()) and bool(got.lse.isnan().all())


@gpu
def test_large_products_and_confident_rows():
    """Products of some thousands: the token's probability is one, or zero, and nothing overflows."""
    hidden, head, tokens, _ = make(64, 128, 1000, seed=19)
    hidden = hidden * 64
    ref = Reference(hidden, head, tokens)
    assert float(ref.z.abs().max()) > 500
    r = P.head_cross_entropy(hidden, head, tokens)
    assert close(r.logp, ref.logp, ref.tol) and bool(r.dhidden.isfinite().all()) and bool(r.dhead.isfinite().all())
    dhidden, tol_h, dhead, tol_w = ref.gradients(torch.full((64,), 1 / 64, device="cuda"))
    assert close(r.dhidden, dhidden, tol_h) and close(r.dhead, dhead, tol_w)


@gpu
def test_same_values_as_from_logits():
    """token_logprob and policy_loss on the logits in fp32, head_logprob and head_logprob_grad without them: the policy loss's factor of each row
    goes back through the head."""
    hidden, head, tokens, weights = make(200, 128, 900, seed=23)
    logits = hidden.float() @ head.float().T
    ref = Reference(hidden, head, tokens)
    a, b = P.token_logprob(logits, tokens, weights), P.head_logprob(hidden, head, tokens, weights=weights)
    assert close(a.logp, b.logp.double(), 2 * ref.tol) and close(a.lse, b.lse.double(), 2 * ref.tol)
    old = a.logp + 0.05
    adv = torch.linspace(-1, 1, 200, device="cuda")
    loss = P.policy_loss(logits, tokens, old, adv, weights=weights)
    ratio = torch.exp(b.logp - old)
    free = ratio * adv <= ratio.clamp(0.8, 1.2) * adv
    dlogp = torch.where(free, -ratio * adv, 0.0) * weights / weights.sum()
    g = P.head_logprob_grad(hidden, head, tokens, b.lse, dlogp)
    dhidden, tol_h, dhead, tol_w = ref.gradients(-dlogp.double())
    assert close(g.dhidden, dhidden, tol_h) and close(g.dhead, dhead, tol_w)
    assert close(g.dhidden, loss.dlogits.double() @ head.double(), tol_h * 1.01 + 1e-6 * dhidden.abs().max())


@gpu
def test_differences_of_the_loss():
    hidden, head, tokens, weights = make(64, 96, 500, seed=29)
    r = P.head_cross_entropy(hidden, head, tokens, weights=weights)
    for name, at, grad in (("hidden", hidden, r.dhidden), ("head", head, r.dhead)):
        step = (torch.randn(at.shape, generator=torch.Generator().manual_seed(1)) * 0.02 * float(at.abs().max())).cuda()
        ends = [(at.float() + s * step).to(BF16) for s in (1, -1)]
        losses = []
        for e in ends:
            call = dict(hidden=hidden, head=head)
            call[name] = e
            losses.append(float(P.head_cross_entropy(call["hidden"], call["head"], tokens, weights=weights, grad=False).stats[0]))
        way = ends[0].double() - ends[1].double()
        # how far a row's products move (to each side); the second end is not quite the mirror of the first, so its curvature counts too
        other = head if name == "hidden" else hidden
        move = float((way @ other.double().T).abs().max()) / 2
        middle = (ends[0].double() + ends[1].double()) / 2 - at.double()
        bent = float((middle @ other.double().T).abs().max())
        predicted = float((grad.double() * way).sum())
        size = float((grad.double().abs() * way.abs()).sum())
        assert abs(losses[0] - losses[1] - predicted) <= 2 * move ** 3 / 3 + 2 * move * bent + 2 * HALF * size + 64 * EPS * abs(losses[0])


@gpu
def test_captured_and_replayed():
    hidden, head, tokens, weights = make(150, 64, 1000, seed=31)
    other = make(150, 64, 1000, seed=32, masked=0.6)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        P.head_cross_entropy(hidden, head, tokens, weights=weights)
        graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            r = P.head_cross_entropy(hidden, head, tokens, weights=weights)
        with torch.cuda.graph(second, stream=stream):
            s = P.head_logprob(hidden, head, tokens)
    torch.cuda.synchronize()
    for x in (None, other):
        if x:
            for a, b in zip((hidden, head, tokens, weights), x):
                a.copy_(b)
        graph.replay()
        second.replay()
        torch.cuda.synchronize()
        want = P.head_cross_entropy(hidden, head, tokens, weights=weights)
        assert all(torch.equal(a, b) for a, b in zip(r, want)) and torch.equal(s.logp, P.head_logprob(hidden, head, tokens).logp)


@gpu
def test_two_streams_at_once():
    calls = [make(300, 128, 5000, seed=k) for k in (41, 42)]
    want = [P.head_cross_entropy(h, w, t, weights=x) for h, w, t, x in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for k, (s, (h, w, t, x)) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                got[k].append(P.head_cross_entropy(h, w, t, weights=x))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for r in got[k] for a, b in zip(r, want[k]))


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------------

def struct(**kw):
    good = dict(hidden_dev=4096, head_dev=8192, rows=4, width=64, vocab=300, hidden_stride=64, head_stride=64, tokens_dev=4096, temperature=1.0)
    return P.binding.Head(**{**good, **kw})


BAD = [dict(rows=-1), dict(rows=1 << 40), dict(width=0), dict(width=1 << 21), dict(vocab=0), dict(vocab=1 << 40), dict(hidden_stride=63), dict(head_stride=10),
       dict(hidden_stride=1 << 39), dict(temperature=0.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-44),
       dict(hidden_dev=None), dict(head_dev=None), dict(tokens_dev=None), dict(hidden_dev=4097), dict(tokens_dev=4100)]


@pytest.mark.parametrize("bad", BAD, ids=[str(b) for b in BAD])
def test_refused_by_the_library(bad):
    n = C.c_int64()
    assert P.ps_head_workspace(C.byref(struct()), 1, C.byref(n)) == P.PS_OK and n.value > 0
    h = struct(**bad)
    assert P.ps_head_workspace(C.byref(h), 1, C.byref(n)) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob(C.byref(h), None, 256, 256, 256, 1 << 40, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob_grad(C.byref(h), 256, 256, 256, 256, 256, 1 << 40, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_cross_entropy(C.byref(h), None, 256, 256, 256, 256, 256, 256, 1 << 40, None) == P.PS_ERR_INVALID_ARG


def test_refused_buffers():
    h, n = struct(), C.c_int64()
    P.ps_head_workspace(C.byref(h), 1, C.byref(n))
    for ws, size in ((None, 1 << 30), (264, 1 << 30), (256, n.value - 1)):
        assert P.ps_head_logprob_grad(C.byref(h), 256, 256, 256, 256, ws, size, None) == P.PS_ERR_INVALID_ARG
        assert P.ps_head_cross_entropy(C.byref(h), 256, 256, 256, 256, 256, 256, ws, min(size, 1000) if ws == 256 else size, None) == P.PS_ERR_INVALID_ARG
        assert P.ps_head_logprob(C.byref(h), 256, 256, 256, ws, 100 if ws == 256 else size, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob(C.byref(h), None, None, 256, 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob(C.byref(h), 257, 256, 256, 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_logprob_grad(C.byref(h), 256, 256, 264, None, 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_cross_entropy(C.byref(h), None, None, 256, 256, None, None, 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_cross_entropy(None, None, 256, 256, 256, None, None, 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_head_workspace(C.byref(h), 1, None) == P.PS_ERR_INVALID_ARG


def test_refused_in_python():
    h, w, t = torch.zeros(4, 64, dtype=BF16), torch.zeros(30, 64, dtype=BF16), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        P.head_logprob(h, w, t)
    with pytest.raises(TypeError, match="bf16"):
        P.head_logprob(h.float(), w.float(), t)
    with pytest.raises(ValueError, match="width"):
        P.head_cross_entropy(h, w[:, :32], t)
    with pytest.raises(ValueError, match="contiguous"):
        P.head_cross_entropy(h.T, w.T, t)
    with pytest.raises(TypeError, match="tensor"):
        P.head_logprob([0], w, t)


@gpu
def test_refused_in_python_on_the_gpu():
    h, w, t, x = make(4, 64, 30)
    lse = torch.zeros(4, device="cuda")
    for call, error in ((lambda: P.head_logprob(h, w, t.int()), TypeError), (lambda: P.head_logprob(h, w, t[:3]), ValueError),
                        (lambda: P.head_logprob(h, w, t.cpu()), ValueError), (lambda: P.head_logprob(h, w, t, weights=x.double()), TypeError),
                        (lambda: P.head_logprob(h, w, t, temperature=0.0), ValueError), (lambda: P.head_logprob(h, w.cpu(), t), ValueError),
                        (lambda: P.head_cross_entropy(h, w, t, grad="logits"), ValueError), (lambda: P.head_cross_entropy(h, w[:0], t), ValueError),
                        (lambda: P.head_logprob_grad(h, w, t, lse, lse[:2]), ValueError), (lambda: P.head_logprob(h, w, [0] * 4), TypeError), (lambda: P.head_logprob_grad(h, w, t, lse, None), TypeError)):
        with pytest.raises(error):
            call()
