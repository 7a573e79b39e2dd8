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
