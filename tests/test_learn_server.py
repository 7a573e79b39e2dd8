"""AdamWServer: the n-softsync protocol with an AdamW step, against a recount of the staleness and a plain optimizer; and the example."""
import numpy as np
import pytest
import torch

import paper_1511_05950_b200 as P
from oracle import reference as R
from tests.helpers import PULL, staleness_by_recount

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lam,n,bits,max_norm", [(6, 2, 32, None), (5, 5, 32, 0.5), (8, 2, 8, 0.05)])
def test_updates_weigh_gradients_by_their_staleness(lam, n, bits, max_norm):
    """A trace of pulls and pushes; the same gradients go through a plain AdamW with scales 1 / (c max(tau, 1)), tau counted by brute force from
    the trace, in ascending (learner, push index) order.  Both use the same step, so weights and moments are equal bit by bit."""
    sizes, hyper = [700, 33, 2048], dict(lr=1e-2, betas=(0.9, 0.99), weight_decay=0.1, state_bits=bits, seed=5)
    g = torch.Generator("cuda").manual_seed(3)
    start = [torch.randn(k, generator=g, device="cuda") for k in sizes]
    ours, plain = [p.clone() for p in start], [p.clone() for p in start]
    server = P.AdamWServer(ours, lam, n, max_norm=max_norm, **hyper)
    optimizer = P.AdamW(plain, **hyper)
    c = lam // n
    assert server.c == c
    kinds, learners = R.simulate_arrivals("exp", lam, 20 * c, 9)
    taus, _ = staleness_by_recount(kinds, learners, c)
    group, pulled, pushes, updates = [], {}, 0, 0
    counts = [0] * lam
    for kind, l in zip(kinds.tolist(), learners.tolist()):
        if kind == PULL:
            pulled[l] = server.pull()
            assert pulled[l] == updates
            continue
        grad = [torch.randn(k, generator=g, device="cuda") * 0.1 for k in sizes]
        ready = server.push(l, grad, pulled[l])
        group.append((l, counts[l], grad, 1.0 / (c * max(int(taus[pushes]), 1))))
        counts[l] += 1
        pushes += 1
        assert ready == (len(group) == c)
        if ready:
            server.apply_update()
            group.sort(key=lambda e: e[:2])
            scales = [float(np.float32(e[3])) for e in group]
            grads = [e[2] for e in group]
            optimizer.step(grads, scales, clip=None if max_norm is None else optimizer.grad_norm(grads, scales, max_norm))
            group, updates = [], updates + 1
            assert all(torch.equal(a, b) for a, b in zip(ours, plain))
    assert updates == 20 and taus.max() > 1
    assert all(torch.equal(a, b) for a, b in zip(server.optimizer.state, optimizer.state))
    assert server.staleness_histogram().sum() == updates * c
    if max_norm is not None:
        assert float(server.last_norm[0]) > 0 and float(server.last_norm[1]) <= 1.0


def test_a_push_that_the_update_would_refuse_is_refused_and_counts_for_nothing():
    params = [torch.zeros(10, device="cuda"), torch.zeros(3, device="cuda")]
    server = P.AdamWServer(params, 2, 1)
    good = [torch.ones(10, device="cuda"), torch.ones(3, device="cuda")]
    with pytest.raises(ValueError):
        server.push(0, good[:1], 0)
    with pytest.raises(TypeError):
        server.push(0, [x.half() for x in good], 0)
    with pytest.raises(P.SoftsyncError) as e:
        server.push(0, good, 1)                                            # a timestamp ahead of the server's
    assert e.value.status == P.PS_ERR_BAD_TIMESTAMP
    with pytest.raises(P.SoftsyncError) as e:
        server.push(7, good, 0)
    assert e.value.status == P.PS_ERR_BAD_LEARNER
    assert not server.push(0, good, 0) and server.push(1, good, 0)
    assert server.pull() == 1                                              # applies the group first
    assert server.timestamps() == (1, 1) and bool((params[0] < 0).all())


def test_the_example_learns():
    """Chance is 1/32.  Recorded runs reach 0.55 to 0.65 after the first phase and 1.0 after the second."""
    from examples import async_policy
    seen = async_policy.train(policy_turns=3000, preference_turns=800, log=None)
    assert seen["start"] < 0.15 and seen["policy"] > 0.3 and seen["preference"] > 0.9
    assert sum(seen["staleness"][2:]) > 100                                # and on stale gradients
