"""Whose memory the operators use and for how long: streams, versions that autograd watches, workspaces, captured graphs."""
import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu


class Busy:
    """Two streams, the second with some tens of milliseconds of work ahead of what it is given."""

    def __init__(self):
        self.home, self.away = torch.cuda.Stream(), torch.cuda.Stream()

    def start(self):
        self.away.wait_stream(self.home)
        with torch.cuda.stream(self.away):
            torch.cuda._sleep(100_000_000)

    def taken(self, places):
        """Whether an allocation of any size of `places` on the first stream gets one of those places now, while the second is still at work."""
        held = []
        with torch.cuda.stream(self.home):
            for place, size in places:
                held += [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(3)]
        hit = {t.data_ptr() for t in held} & {place for place, _ in places}
        assert not self.away.query(), "the work ended too early to show anything"
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
