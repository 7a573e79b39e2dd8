"""AdamW where its step leaves the short forms of root and quotient, where 8-bit blocks have large scales, and for lists that take a step of
several launches: bit by bit against the same restatement as the ordinary cases."""
import math

import numpy as np
import pytest
import torch

import paper_1511_05950_b200 as P
from tests.test_learn_tensors import Setup, adamw, decode, encode, hashes, key_of, pack, unpack, weighted

gpu = pytest.mark.gpu


def one_step(s, hyper, t, seed=7, scales=None):
    """Makes step t on the GPU and in NumPy and compares everything bit by bit; s holds the state before it."""
    opt = s.optimizer(**hyper, step=t - 1, seed=seed)
    opt.step(s.grads, scales)
    g = weighted(s.grads_np, [1.0] * s.c if scales is None else scales, np.float32)
    with np.errstate(over="ignore", under="ignore"):
        new = [adamw(w, m, v, x, t, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"], 1, 1, np.float32)
               for w, m, v, x in zip(s.w_np, unpack(s.m, s.sizes), unpack(s.v, s.sizes), g)]
    assert np.array_equal(s.flat.cpu().numpy(), np.concatenate([n[0] for n in new]))
    m, v = pack([n[1] for n in new], s.sizes), pack([n[2] for n in new], s.sizes)
    if s.bits == 32:
        for got, want in zip(s.state, (m, v)):
            for a, b in zip(unpack(got.cpu().numpy(), s.sizes), unpack(want, s.sizes)):
                assert np.array_equal(a, b)
        return
    x = hashes(m.size, key_of(seed, t))
    for signed, array, bits16, codes, exps in ((True, m, x & np.uint64(0xFFFF), s.state[0], s.state[2]), (False, v, x >> np.uint64(16), s.state[1], s.state[3])):
        want, we = encode(array, bits16, signed)
        assert np.array_equal(exps.cpu().numpy(), we)
        for a, b in zip(unpack(codes.cpu().numpy(), s.sizes), unpack(want, s.sizes)):
            assert np.array_equal(a, b)
    for got, c, e, signed in zip(opt.moments(), s.state[:2], s.state[2:], (True, False)):
        assert np.array_equal(got.float().cpu().numpy(), decode(c.cpu().numpy(), e.cpu().numpy(), signed).astype(np.float32))


def rescale(s, gradients, moments):
    """Gradients, and moments to match, times powers of two (squared for the second)."""
    for row, row_np in zip(s.grads, s.grads_np):
        for k, g in enumerate(row):
            g.mul_(gradients)
            row_np[k] = g.float().cpu().numpy()
    if s.bits == 32:
        s.m, s.v = s.m * np.float32(moments), s.v * np.float32(moments) * np.float32(moments)
        for t, x in zip(s.state, (s.m, s.v)):
            t.copy_(torch.from_numpy(x))
    else:
        up = int(math.log2(moments))
        s.me, s.ve = (s.me.astype(int) + up).astype(np.uint8), (s.ve.astype(int) + 2 * up).astype(np.uint8)
        s.m, s.v = (decode(c, e, signed).astype(np.float32) for c, e, signed in ((s.mc, s.me, True), (s.vc, s.ve, False)))
        for t, x in zip(s.state[2:], (s.me, s.ve)):
            t.copy_(torch.from_numpy(x))


HYPER = dict(lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = [255, 4096, 1, 10241]


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("change", [dict(eps=1e-13), dict(eps=0.0), dict(lr=1e-14), dict(lr=0.0), dict(eps=1e20), dict(betas=(0.0, 0.0)), dict(betas=(0.9, 0.99999999))])
def test_hyperparameters_outside_the_short_forms(bits, change):
    one_step(Setup(SIZES, 2, torch.float32, bits, seed=31), {**HYPER, **change}, 3, scales=[0.5, 0.25])


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gradients,moments", [(2.0 ** 33, 2.0 ** 33), (2.0 ** 16, 2.0 ** 16), (2.0 ** 50, 2.0 ** 50), (2.0 ** 40, 1.0), (1.0, 2.0 ** 40), (2.0 ** -40, 2.0 ** -20)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_moments_of_all_magnitudes(bits, dtype, gradients, moments):
    """2^50 times 1e-3: first moments of 2^40, second ones of 2^80, beyond the short forms (2^20, 2^30) and beyond where a block's scale and its
    unit fit one factor (2^7, 2^15)."""
    s = Setup(SIZES, 1, dtype, bits, seed=41)
    rescale(s, gradients, moments)
    one_step(s, HYPER, 9)


@gpu
@pytest.mark.parametrize("bits,tensors,c", [(32, 300, 2), (8, 700, 1), (32, 700, 3), (8, 500, 5), (32, 20, 256)])
def test_lists_of_many_pointers(bits, tensors, c):
    """More gradient pointers than the small and the middle parameter block hold, and (700 x 3, 500 x 5, 20 x 256) than one launch carries: the tensors
    after the first launch's have coefficients of their own."""
    r = np.random.default_rng(5)
    sizes = [int(n) for n in r.integers(0, 700, tensors)]
    sizes[3] = 0
    one_step(Setup(sizes, c, torch.bfloat16, bits, seed=51), HYPER, 2, scales=[1.0 / (c + k) for k in range(c)])


@gpu
def test_coefficients_of_every_tensor_over_several_launches():
    tensors, c = 700, 3
    sizes = [1 + k % 5 for k in range(tensors)]
    s = Setup(sizes, c, torch.float32, 32, seed=61)
    lr_mult, decay_mult = [1.0 + k / 64 for k in range(tensors)], [float(k % 7) for k in range(tensors)]
    opt = s.optimizer(**HYPER, lr_mult=lr_mult, decay_mult=decay_mult, step=1)
    opt.step(s.grads)
    new = [adamw(w, m, v, g, 2, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"], lm, dm, np.float32) for w, m, v, g, lm, dm in
           zip(s.w_np, unpack(s.m, sizes), unpack(s.v, sizes), weighted(s.grads_np, [1.0] * c, np.float32), lr_mult, decay_mult)]
    assert np.array_equal(s.flat.cpu().numpy(), np.concatenate([n[0] for n in new]))


@gpu
def test_quotients_below_the_smallest_normal_number():
    """m / (root + eps) below 2^-126 is rounded to a subnormal or kept with all its bits, and only then multiplied with the step size: two results,
    at most one subnormal step (2^-149) apart for a step size of up to one, so only a weight of about zero shows which."""
    n = 1024
    r = np.random.default_rng(3)
    g = (r.standard_normal(n) * 1e-38).astype(np.float32)
    w = torch.zeros(n, device="cuda")
    opt = P.AdamW([w], lr=0.5, betas=(0.0, 0.999), eps=1.0, weight_decay=0.0)
    opt.step([torch.from_numpy(g).cuda()])
    exact = -0.5 * g.astype(np.float64)
    assert np.abs(w.cpu().numpy().astype(np.float64) - exact).max() <= 2.0 ** -149


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_lists_without_elements(bits):
    w = [torch.empty(0, device="cuda"), torch.empty(0, device="cuda")]
    opt = P.AdamW(w, state_bits=bits)
    opt.step(w, clip=opt.grad_norm(w))
    m, v = opt.moments()
    assert m.numel() <= 1 and v.numel() <= 1 and opt.steps == 1
    again = P.AdamW(w, state_bits=bits, state=opt.state, step=opt.steps)
    again.step(w)
    none = [torch.empty(0, dtype=t.dtype, device="cuda") for t in opt.state]
    P.AdamW(w, state_bits=bits, state=none).step(w)
