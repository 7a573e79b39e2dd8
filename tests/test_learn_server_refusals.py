"""AdamWServer: what it refuses leaves its clock, its pending gradients and the weights as they were."""
import ctypes as C
import math

import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu


def test_a_configuration_is_checked_without_a_gpu():
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, seed=0)
    check = lambda **kw: P.ps_adamw_check(C.byref(P.binding.AdamwConfig(**{**good, **kw})))
    assert check() == P.PS_OK and check(lr=0.0, beta1=0.0, beta2=0.0, eps=0.0) == P.PS_OK
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=math.inf), dict(weight_decay=math.nan), dict(step=0)):
        assert check(**bad) == P.PS_ERR_INVALID_ARG, bad
    assert P.ps_adamw_check(None) == P.PS_ERR_INVALID_ARG


def make(**kw):
    params = [torch.ones(10, device="cuda"), torch.ones(300, device="cuda")]
    return params, P.AdamWServer(params, 2, 1, **{**dict(lr=0.1, max_norm=1.0), **kw})


def gradient(dtype=torch.float32):
    return [torch.full((10,), 0.5, dtype=dtype, device="cuda"), torch.full((300,), 0.25, dtype=dtype, device="cuda")]


@gpu
def test_what_no_update_would_take_is_refused_at_once():
    for bad in (dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan)):
        with pytest.raises(ValueError):
            make(**bad)
    for bad in (dict(lr=-0.1), dict(betas=(1.0, 0.9)), dict(eps=math.nan), dict(step=-1)):
        with pytest.raises(P.SoftsyncError) as e:
            make(**bad)
        assert e.value.status == P.PS_ERR_INVALID_ARG


@gpu
@pytest.mark.parametrize("first,other", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_gradients_of_two_types(first, other):
    params, server = make()
    with pytest.raises(P.SoftsyncError):
        server.push(0, gradient(other), 5)                             # refused for its timestamp: its type does not count
    server.push(0, gradient(first), 0)
    with pytest.raises(TypeError):
        server.push(1, gradient(other), 0)
    assert server.timestamps() == (0, 0)
    assert server.push(1, gradient(first), 0)
    assert server.pull() == 1 and bool((params[0] < 1).all())


@gpu
@pytest.mark.parametrize("change", [dict(lr=-1.0), dict(lr=math.nan), dict(betas=(0.9, 1.0)), dict(eps=-1.0), dict(max_norm=0.0), dict(max_norm=math.nan)])
def test_an_update_that_is_refused_can_be_made_later(change):
    want, other = make()
    params, server = make()
    for s in (server, other):
        s.push(0, gradient(), 0)
        s.push(1, gradient(), 0)
    other.apply_update()
    for name, value in change.items():
        owner = server if name == "max_norm" else server.optimizer
        good = getattr(owner, name)
        setattr(owner, name, value)
        for call in (server.apply_update, server.pull):
            with pytest.raises((ValueError, P.SoftsyncError)):
                call()
            assert server.timestamps() == (0, 1) and server.optimizer.steps == 0 and all(bool((p == 1).all()) for p in params)
        setattr(owner, name, good)
    server.apply_update()
    assert server.timestamps() == (1, 1) and server.optimizer.steps == 1
    assert all(torch.equal(a, b) for a, b in zip(params, want)) and torch.equal(server.last_norm, other.last_norm)
    with pytest.raises(P.SoftsyncError) as e:
        server.apply_update()                                          # no group
    assert e.value.status == P.PS_ERR_NOT_READY and server.timestamps() == (1, 1)


@gpu
def test_a_gradient_that_changed_its_shape_after_the_push():
    params, server = make()
    g = gradient()
    server.push(0, g, 0)
    server.push(1, gradient(), 0)
    whole = g[1].data
    g[1].data = whole[:200]
    with pytest.raises(ValueError):
        server.apply_update()
    assert server.timestamps() == (0, 1) and all(bool((p == 1).all()) for p in params)
    g[1].data = whole
    server.apply_update()
    assert server.timestamps() == (1, 1) and bool((params[1] < 1).all())
