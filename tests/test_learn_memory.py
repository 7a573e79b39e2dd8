"""Whose memory the operators use and for how long: streams, versions that autograd watches, workspaces, captured graphs."""
import gc
import threading

import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu


class Busy:
    """Two streams, the second with a fifth of a second of work ahead of what it is given."""

    def __init__(self):
        self.home, self.away = torch.cuda.Stream(), torch.cuda.Stream()

    def start(self):
        gc.collect()                                                   # not while the other stream is at work: it takes a while after many tests
        self.away.wait_stream(self.home)
        with torch.cuda.stream(self.away):
            torch.cuda._sleep(400_000_000)

    def taken(self, places):
        """Whether an allocation of any size of `places` on the first stream gets one of those places now, while the second is still at work."""
        held = []
        with torch.cuda.stream(self.home):
            for place, size in places:
                held += [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
        hit = {t.data_ptr() for t in held} & {place for place, _ in places}
        if self.away.query():
            pytest.skip("the host took too long: the other stream's work has ended, which shows nothing")
        return bool(hit)


def places(tensors):
    return [(t.data_ptr(), t.numel() * t.element_size()) for t in tensors]


SIZES = [3_000_000, 5, 700_001]


@gpu
def test_a_list_dropped_while_another_stream_works_on_it():
    b = Busy()
    with torch.cuda.stream(b.home):
        grads = [torch.ones(n, device="cuda") for n in SIZES]
        plan = P.TensorList(SIZES)
    want = float(plan.grad_norm(grads)[0])
    b.start()
    with torch.cuda.stream(b.away):
        out = plan.grad_norm(grads)
    where = places([plan._workspace])
    del plan
    assert not b.taken(where)
    b.away.synchronize()
    assert float(out[0]) == want


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_an_optimizer_dropped_while_another_stream_works_on_it(bits):
    b = Busy()
    with torch.cuda.stream(b.home):
        grads = [torch.ones(n, device="cuda") for n in SIZES]
        want = [torch.ones(n, device="cuda") for n in SIZES]
        params = [torch.ones(n, device="cuda") for n in SIZES]
        P.AdamW(want, state_bits=bits).step(grads)
        optimizer = P.AdamW(params, state_bits=bits)
    b.home.synchronize()
    b.start()
    with torch.cuda.stream(b.away):
        optimizer.step(grads)
    where = places([optimizer._workspace, *optimizer.state])
    del optimizer
    assert not b.taken(where)
    b.away.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(params, want))


@gpu
def test_pushed_gradients_stay_until_the_update_has_read_them():
    b = Busy()
    with torch.cuda.stream(b.home):
        params = [torch.ones(n, device="cuda") for n in SIZES]
        server = P.AdamWServer(params, 1, 1)
        grads = [torch.ones(n, device="cuda") for n in SIZES]
        server.push(0, grads, server.pull())
    where = places(grads)
    del grads
    b.start()
    with torch.cuda.stream(b.away):
        server.apply_update()
    assert not b.taken(where)
    b.away.synchronize()
    assert all(bool((p < 1).all()) for p in params)


# ---- what autograd sees ---------------------------------------------------------------------------------------------------

def loss_calls(logits):
    """The two losses with their gradient in place of the logits."""
    rows = logits.shape[0]
    tokens = torch.zeros(rows, dtype=torch.int64, device="cuda")
    old, adv = torch.full((rows,), -2.0, device="cuda"), torch.ones(rows, device="cuda")
    return {"policy": lambda grad: P.policy_loss(logits, tokens, old, adv, grad=grad),
            "preference": lambda grad: P.preference_loss(logits, tokens, torch.arange(rows + 1, device="cuda"), old, grad=grad)}


@gpu
@pytest.mark.parametrize("which", ["policy", "preference"])
def test_a_gradient_in_place_of_saved_logits_is_noticed(which):
    x = torch.randn(4, 50, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).requires_grad_(True)
    logits = torch.tanh(x)                                             # saves its output
    before = logits._version
    r = loss_calls(logits)[which]("inplace")
    assert logits._version == before + 1 and r.dlogits.data_ptr() == logits.data_ptr()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logits.backward(r.dlogits)
    w = torch.eye(50, device="cuda").requires_grad_(True)
    logits = torch.tanh(x.detach()) @ w                                # does not
    apart = loss_calls(logits)[which](True).dlogits
    assert logits._version == 0
    logits.backward(loss_calls(logits)[which]("inplace").dlogits)
    assert torch.allclose(w.grad, torch.tanh(x.detach()).t() @ apart, rtol=1e-5, atol=1e-7)


@gpu
@pytest.mark.parametrize("which", ["policy", "preference"])
def test_a_given_buffer_counts_as_written_and_a_refused_call_does_not(which):
    logits = torch.randn(4, 50, device="cuda")
    buffer = torch.zeros(4, 50, device="cuda")
    loss_calls(logits)[which](buffer)
    assert buffer._version == 1 and logits._version == 0
    wide = torch.zeros(5, 50, device="cuda")
    with pytest.raises(P.SoftsyncError):                               # overlaps the logits
        loss_calls(wide[:4])[which](wide[1:])
    assert wide._version == 0
    with torch.inference_mode():
        unwatched = torch.randn(4, 50, device="cuda")
        loss_calls(unwatched)[which]("inplace")


@gpu
def test_a_step_on_saved_parameters_is_noticed():
    w = torch.eye(40, device="cuda")
    mirror = w.bfloat16()
    x = torch.randn(3, 40, device="cuda").requires_grad_(True)
    y, z = x @ w, x.bfloat16() @ mirror                                # both save their second factor
    optimizer = P.AdamW([w], mirrors=[mirror])
    versions = w._version, mirror._version
    optimizer.step([torch.ones_like(w)])
    assert w._version > versions[0] and mirror._version > versions[1]
    for out in (y, z):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()
    with pytest.raises(P.SoftsyncError):
        optimizer.lr = -1.0
        optimizer.step([torch.ones_like(w)])
    assert w._version == versions[0] + 1


# ---- workspaces -------------------------------------------------------------------------------------------------------------

def inputs(rows, vocab, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, vocab, device="cuda", generator=g, dtype=torch.bfloat16).mul_(2)
    tokens = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    weights = (torch.rand(rows, device="cuda", generator=g) > 0.3).float()
    old = torch.randn(rows, device="cuda", generator=g) * 0.1 - 9
    adv = torch.randn(rows, device="cuda", generator=g)
    offsets = torch.linspace(0, rows, 5, device="cuda").long()
    return x, tokens, weights, old, adv, offsets


def both_losses(x, tokens, weights, old, adv, offsets):
    policy = P.policy_loss(x, tokens, old, adv, weights, entropy_coef=0.01)
    preference = P.preference_loss(x, tokens, offsets, old[:4], weights)
    return [policy.stats, policy.logp, policy.entropy, policy.dlogits, preference.stats, preference.seq_logp, preference.dlogits]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


CASES = [(9, 500), (700, 3001), (5, 152000), (2100, 40), (400, 33000)]


@gpu
def test_calls_of_many_threads_share_what_is_kept():
    x = inputs(9, 500, 1)
    want = both_losses(*x)
    results = []

    def work():
        results.append(same(both_losses(*x), want))

    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for _ in range(40):
        t = threading.Thread(target=work)
        t.start()
        t.join()
    torch.cuda.synchronize()
    assert results == [True] * 40 and torch.cuda.memory_allocated() == before


@gpu
def test_losses_of_different_sizes_one_after_the_other():
    """They share a workspace that grows, and the larger ones leave their traces in it."""
    data = [inputs(r, v, k) for k, (r, v) in enumerate(CASES)]
    want = [both_losses(*d) for d in data]
    for order in ([4, 0, 3, 1, 2], [0, 0, 1, 0, 3, 0, 2, 4, 0]):
        for k in order:
            assert same(both_losses(*data[k]), want[k])


@gpu
def test_threads_on_streams_of_their_own_at_the_same_time():
    data = [inputs(r, v, k) for k, (r, v) in enumerate(CASES)]
    want = [both_losses(*d) for d in data]
    torch.cuda.synchronize()
    results = {}

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [both_losses(*data[k]) for _ in range(10)]
            torch.cuda.current_stream().synchronize()
            results[k] = all(same(g, want[k]) for g in got)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(data))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert results == {k: True for k in range(len(data))}


@gpu
@pytest.mark.parametrize("rows,vocab", CASES + [(4, 1000003)])
def test_a_captured_graph_has_a_workspace_of_its_own(rows, vocab):
    """Recorded once, replayed on other inputs, with calls of the same stream in between."""
    x = inputs(rows, vocab, 1)
    both_losses(*x)                                                    # what a kernel asks once of the GPU is asked before
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both_losses(*x)
    for seed in (2, 3):
        y = inputs(rows, vocab, seed)
        for a, b in zip(x, y):
            a.copy_(b)
        graph.replay()
        want = both_losses(*y)
        assert same(out, want)
        graph.replay()
        assert same(out, want)
