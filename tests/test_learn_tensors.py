"""Gradient norm and AdamW over a list of tensors (include/softsync_learn.h) against plain NumPy implementations.

The header fixes the order of every rounding, so weights and 32-bit moments are compared bit by bit with a float32 restatement,
and 8-bit moments code by code with a restatement that goes by the formats' value tables and the definition of random
rounding (distance to the lower neighbour) instead of bit shifts.  Both are compared with the formulas in float64 as well.
"""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu
BLOCK = P.PS_STATE_BLOCK
EPS32 = 2.0 ** -24                                  # relative error of one rounding to float32


def offsets(sizes):
    at, out = 0, []
    for n in sizes:
        out.append(at)
        at += -(-n // BLOCK) * BLOCK
    return out, at


def pack(parts, sizes):
    """Per-tensor arrays into a state array (zeros in the gaps)."""
    off, total = offsets(sizes)
    out = np.zeros(total, dtype=parts[0].dtype)
    for o, p in zip(off, parts):
        out[o:o + p.size] = p
    return out


def unpack(array, sizes):
    off, _ = offsets(sizes)
    return [array[o:o + n] for o, n in zip(off, sizes)]


# ---- the 8-bit formats, from their definition ---------------------------------------------------------------------

def values(signed):
    """Values of the codes without a sign, ascending."""
    out = []
    for code in range(128 if signed else 256):
        e, f, bias = code // 16, code % 16, 7 if signed else 15
        out.append((1 + f / 16) * 2.0 ** (e - bias) if e else f / 16 * 2.0 ** (1 - bias))
    return np.array(out)


def decode(codes, exps, signed):
    table = values(signed)
    x = table[codes & 127] * np.where(codes & 128, -1.0, 1.0) if signed else table[codes]
    return x * np.repeat(2.0 ** (exps.astype(np.float64) - 127), BLOCK)


def key_of(seed, step):
    mask = (1 << 64) - 1
    x = (seed + step * 0x9E3779B97F4A7C15) & mask
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & mask
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & mask
    return (x ^ (x >> 31)) & 0xFFFFFFFF


def hashes(n, key):
    m = np.uint64(0xFFFFFFFF)
    x = np.arange(n, dtype=np.uint64)
    x = (((x & m) ^ np.uint64(key)) + (x >> np.uint64(32)) * np.uint64(0x9E3779B9)) & m
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x7FEB352D)) & m
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0x846CA68B)) & m
    return x ^ (x >> np.uint64(16))


def encode(x, rnd16, signed):
    """(codes, exponents) of a float32 state array: the block's power of two, then the lower neighbour in the table or the one above it,
    the latter where the distance to the lower one plus the random part (16 bits) reaches a whole step."""
    table = values(signed)
    mag = np.abs(x.astype(np.float64)).reshape(-1, BLOCK)
    top = mag.max(1)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(top))
        e += top >= 31 / 16 * 2.0 ** np.where(np.isfinite(e), e, 0.0)
    e = np.clip(np.where(top > 0, e, -1000) + 127, 27, 253)
    rel = (mag / 2.0 ** (e - 127)[:, None]).reshape(-1)
    low = np.minimum(np.searchsorted(table, rel, side="right") - 1, len(table) - 1)
    above = np.where(low + 1 < len(table), table[np.minimum(low + 1, len(table) - 1)], 2.0)
    frac = np.floor((rel - table[low]) / (above - table[low]) * (1 << 19))
    code = np.minimum(low + (frac + rnd16.astype(np.float64) * 8 >= (1 << 19)), len(table) - 1).astype(np.int64)
    if signed:
        code |= np.where(x < 0, 128, 0)
    else:
        code = np.maximum(code, x > 0)
    return code.astype(np.uint8), e.astype(np.uint8)


# ---- the step, float32 in the documented order, and float64 ---------------------------------------------------------

def weighted(grads, scales, dtype):
    """Per tensor: the weighted sum of the c gradients."""
    out = []
    for k in range(len(grads[0])):
        acc = None
        for s, g in zip(scales, grads):
            part = dtype(s) * g[k].astype(dtype)
            acc = part if acc is None else acc + part
        out.append(acc)
    return out


def adamw(w, m, v, g, t, lr, betas, eps, wd, lr_mult, decay_mult, dtype):
    """One tensor's new (w, m, v)."""
    b1, b2 = betas
    f = dtype
    m = m * f(b1) + g * f(1 - b1)
    v = v * f(b2) + (g * g) * f(1 - b2)
    den = np.sqrt(v) * f(1 / math.sqrt(1 - b2 ** t)) + f(eps)
    w = w * f(1.0 - lr * wd * (float(np.float32(lr_mult)) * float(np.float32(decay_mult)))) - \
        (m / den) * f(lr / (1 - b1 ** t) * float(np.float32(lr_mult)))
    return w, m, v


class Setup:
    """Random tensors, gradients and moments; the same on the host and the GPU."""

    def __init__(self, sizes, c, dtype, bits, seed=0, shift=0, spread=1.0, mirror=False):
        r = np.random.default_rng(seed)
        self.sizes, self.c, self.bits = sizes, c, bits
        dev = torch.device("cuda")
        total = sum(sizes)
        flat = torch.zeros(total + shift, device=dev)[shift:]          # shift elements off the 16-byte grid
        flat.copy_(torch.from_numpy(r.standard_normal(total).astype(np.float32) * 0.05))
        self.flat = flat
        self.params = list(torch.split(flat, sizes))
        self.mirrors = None
        if mirror:
            self.mirrors = list(torch.split(torch.zeros(total + shift, dtype=torch.bfloat16, device=dev)[shift:], sizes))
        self.grads = []
        for _ in range(c):
            row = []
            for n in sizes:
                x = torch.from_numpy((r.standard_normal(n) * np.exp(spread * r.standard_normal(n)) * 1e-3).astype(np.float32)).to(dtype)
                buf = torch.zeros(n + shift, dtype=dtype, device=dev)[shift:]
                buf.copy_(x)
                row.append(buf)
            self.grads.append(row)
        self.grads_np = [[g.float().cpu().numpy() for g in row] for row in self.grads]
        self.w_np = [p.cpu().numpy() for p in self.params]
        m = [r.standard_normal(n).astype(np.float32) * np.float32(3e-4) for n in sizes]
        v = [(r.standard_normal(n).astype(np.float32) * np.float32(1e-3)) ** 2 for n in sizes]
        self.m, self.v = pack(m, sizes), pack(v, sizes)
        if bits == 8:
            half = np.full(self.m.size, 1 << 15)
            (self.mc, self.me), (self.vc, self.ve) = encode(self.m, half, True), encode(self.v, half, False)
            self.m = decode(self.mc, self.me, True).astype(np.float32)      # exact: five significant bits
            self.v = decode(self.vc, self.ve, False).astype(np.float32)
            state = [self.mc, self.vc, self.me, self.ve]
        else:
            state = [self.m, self.v]
        self.state = [torch.from_numpy(x.copy()).to(dev) for x in state]

    def optimizer(self, **kw):
        return P.AdamW(self.params, state_bits=self.bits, state=self.state, mirrors=self.mirrors, **kw)


LISTS = [[1], [256], [255, 257, 1, 0, 2048, 5], [2049, 4096, 3, 100003], [7] * 40 + [10241], [32 * 3 * 25, 32, 25600, 32, 51200, 64, 10240, 10]]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1, 3, 17])
@pytest.mark.parametrize("shift", [0, 1])
def test_gradient_norm_matches_float64(dtype, c, shift):
    for k, sizes in enumerate(LISTS):
        s = Setup(sizes, c, dtype, 32, seed=k, shift=shift)
        scales = [1.0 / (c * (1 + l % 3)) for l in range(c)]
        exact = math.sqrt(sum(float((g ** 2).sum()) for g in weighted(s.grads_np, scales, np.float64)))
        plan = P.TensorList(sizes)
        # c products and c sums are rounded once each, the squares' sum keeps 24 bits through at most a few hundred additions a thread
        tol = (2 * c + 200) * EPS32
        got = plan.grad_norm(s.grads, scales, max_norm=exact / 4).cpu().numpy()
        assert abs(got[0] - exact) <= tol * exact
        assert abs(got[1] - 0.25) <= 2 * tol
        again = plan.grad_norm(s.grads, scales, max_norm=exact * 4).cpu().numpy()
        assert again[0] == got[0] and again[1] == 1.0                  # the same bits every time; no clipping below the bound


@gpu
def test_gradient_norm_over_several_launches_and_zero():
    sizes = [3] * 700                                                   # 700 tensors x 7 gradients: more pointers than one launch carries
    s = Setup(sizes, 7, torch.bfloat16, 32, seed=5)
    exact = math.sqrt(sum(float((g ** 2).sum()) for g in weighted(s.grads_np, [1.0] * 7, np.float64)))
    plan = P.TensorList(sizes)
    for _ in range(3):
        assert abs(float(plan.grad_norm(s.grads)[0]) - exact) <= 220 * EPS32 * exact
    zero = [[torch.zeros_like(g) for g in s.grads[0]]]
    assert plan.grad_norm(zero, max_norm=1.0).tolist() == [0.0, 1.0]
    empty = P.TensorList([0, 0])
    assert empty.grad_norm([torch.empty(0, device="cuda")] * 2, max_norm=1.0).tolist() == [0.0, 1.0]


@gpu
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_stops_the_step(bad):
    for bits in (32, 8):
        s = Setup([300, 5, 4096], 1, torch.float32, bits, seed=3)
        s.grads[0][2][77] = bad
        opt = s.optimizer(lr=0.1)
        before = [x.clone() for x in [s.flat, *s.state]]
        clip = opt.grad_norm(s.grads, max_norm=1.0)
        assert not math.isfinite(float(clip[0]))
        opt.step(s.grads, clip=clip)
        assert all(torch.equal(a, b) for a, b in zip(before, [s.flat, *s.state]))


@gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c,shift", [(1, 0), (4, 0), (1, 1), (3, 3)])
def test_adamw_steps_match_the_formula(bits, dtype, c, shift):
    for k, sizes in enumerate(LISTS):
        lr_mult = [1.0 if i % 3 else 0.5 for i in range(len(sizes))]
        decay_mult = [float(i % 2) for i in range(len(sizes))]
        s = Setup(sizes, c, dtype, bits, seed=10 + k, shift=shift, mirror=k % 2 == 0)
        hyper = dict(lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
        opt = s.optimizer(**hyper, lr_mult=lr_mult, decay_mult=decay_mult, step=4, seed=99)
        scales = [1.0 / (c * (1 + l % 3)) for l in range(c)]
        clip = torch.tensor([3.0, 0.37], device="cuda") if k % 2 else None
        g32 = weighted(s.grads_np, scales, np.float32)
        if clip is not None:
            g32 = [g * np.float32(0.37) for g in g32]
        g64 = [g * (float(np.float32(0.37)) if clip is not None else 1.0) for g in weighted(s.grads_np, [float(np.float32(x)) for x in scales], np.float64)]
        w, m, v = s.w_np, s.m, s.v
        for t in (5, 6, 7):
            old = (w, m, v)
            opt.step(s.grads, scales, clip=clip)
            args = (t, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"])
            new = [adamw(a, b, d, g, *args, lm, dm, np.float32) for a, b, d, g, lm, dm in
                   zip(w, unpack(m, sizes), unpack(v, sizes), g32, lr_mult, decay_mult)]
            ref = [adamw(a.astype(np.float64), b.astype(np.float64), d.astype(np.float64), g, *args, lm, dm, np.float64) for a, b, d, g, lm, dm in
                   zip(old[0], unpack(old[1], sizes), unpack(old[2], sizes), g64, lr_mult, decay_mult)]
            w = [n[0] for n in new]
            m, v = pack([n[1] for n in new], sizes), pack([n[2] for n in new], sizes)
            got_w = s.flat.cpu().numpy()
            assert np.array_equal(got_w, np.concatenate(w))
            # one step's roundings: about a dozen, on the weight and on an update that is at most a few lr large
            r = np.concatenate([x[0] for x in ref])
            assert np.abs(got_w - r).max(initial=0) <= 16 * EPS32 * (np.abs(r).max(initial=0) + 10 * hyper["lr"])
            if s.mirrors:
                assert all(torch.equal(q, p.to(torch.bfloat16)) for q, p in zip(s.mirrors, s.params))
            if bits == 8:
                x = hashes(m.size, key_of(99, t))
                for signed, array, bits16, codes, exps in ((True, m, x & np.uint64(0xFFFF), s.state[0], s.state[2]),
                                                           (False, v, x >> np.uint64(16), s.state[1], s.state[3])):
                    want, we = encode(array, bits16, signed)
                    assert np.array_equal(exps.cpu().numpy(), we)
                    for a, b in zip(unpack(codes.cpu().numpy(), sizes), unpack(want, sizes)):
                        assert np.array_equal(a, b)
                m = decode(s.state[0].cpu().numpy(), s.state[2].cpu().numpy(), True).astype(np.float32)
                v = decode(s.state[1].cpu().numpy(), s.state[3].cpu().numpy(), False).astype(np.float32)
                mv = [a.cpu().float().numpy() for a in opt.moments()]
                assert np.array_equal(mv[0], m) and np.array_equal(mv[1], v)
            else:
                for a, b in zip(unpack(s.state[0].cpu().numpy(), sizes), unpack(m, sizes)):
                    assert np.array_equal(a, b)
                for a, b in zip(unpack(s.state[1].cpu().numpy(), sizes), unpack(v, sizes)):
                    assert np.array_equal(a, b)


@gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_what_lies_around_the_tensors_stays_untouched(bits):
    """Gaps of the state arrays and the elements between tensors carved out of a larger buffer."""
    sizes = [5, 300, 2049]
    _, total = offsets(sizes)
    dev = torch.device("cuda")
    big = torch.full((3000,), 7.0, device=dev)
    mir = torch.full((3000,), 7.0, dtype=torch.bfloat16, device=dev)
    at = [3, 20, 400]
    params = [big[a:a + n] for a, n in zip(at, sizes)]
    mirrors = [mir[a:a + n] for a, n in zip(at, sizes)]
    grads = [torch.ones(n, device=dev) for n in sizes]
    fill = 3.0 if bits == 32 else 200
    kind = torch.float32 if bits == 32 else torch.uint8
    state = [torch.full((total,), fill, dtype=kind, device=dev) for _ in range(2)]
    off, _ = offsets(sizes)
    for s in state:
        for o, n in zip(off, sizes):
            s[o:o + n] = 0
    if bits == 8:
        state += [torch.full((total // BLOCK,), 120, dtype=torch.uint8, device=dev) for _ in range(2)]
    opt = P.AdamW(params, lr=0.1, state_bits=bits, state=state, mirrors=mirrors)
    opt.step(grads)
    inside = torch.zeros(3000, dtype=torch.bool, device=dev)
    for a, n in zip(at, sizes):
        inside[a:a + n] = True
    assert bool((big[~inside] == 7).all()) and bool((mir[~inside] == 7).all()) and bool((big[inside] != 7).all())
    gap = torch.ones(total, dtype=torch.bool, device=dev)
    for o, n in zip(off, sizes):
        gap[o:o + n] = False
    assert bool((state[0][gap] == fill).all()) and bool((state[1][gap] == fill).all())


@gpu
def test_random_rounding_keeps_the_expectation():
    """The same step under 4000 seeds: the mean of the stored values is the value.  A stored value is one of
    two neighbours a step d apart, so the mean of N has a standard deviation of at most d / (2 sqrt N); six of them are allowed."""
    n, trials = 4 * BLOCK, 4000
    dev = torch.device("cuda")
    r = np.random.default_rng(1)
    g = (np.exp(r.standard_normal(n) * 1.5) * 1e-2).astype(np.float32)
    grad = torch.from_numpy(g).to(dev)
    mean = [np.zeros(n), np.zeros(n)]
    opt = P.AdamW([torch.zeros(n, device=dev)], lr=1e-3, betas=(0.9, 0.999), state_bits=8)
    for seed in range(trials):
        opt.seed, opt.steps = seed, 0
        for t in opt.state:
            t.zero_()
        opt.step([grad])
        for k, x in enumerate(opt.moments()):
            mean[k] += x.double().cpu().numpy()
    for k, exact in enumerate((0.1 * g.astype(np.float64), 0.001 * g.astype(np.float64) ** 2)):
        mean[k] /= trials
        top = np.repeat(exact.reshape(-1, BLOCK).max(1), BLOCK)
        smallest = top * 2.0 ** (-9 if k == 0 else -17)                # the step of the formats' subnormals, relative to the largest, at most
        step = np.maximum(exact / 16, smallest)
        normal = exact > 2 * smallest                                  # below that v is held up to its smallest code by design
        assert (np.abs(mean[k] - exact)[normal] <= (6 * step / (2 * math.sqrt(trials)) + exact * 2.0 ** -15)[normal]).all()


@gpu
def test_a_second_moment_in_8_bits_follows_its_average_down():
    """With no gradient v falls by beta2 a step, a sixtieth of a code step: rounding to the nearest code would hold it still for ever."""
    n, steps, b2 = 64 * BLOCK, 1500, 0.999
    dev = torch.device("cuda")
    opt = P.AdamW([torch.zeros(n, device=dev)], lr=0.0, betas=(0.9, b2), state_bits=8, seed=3)
    opt.step([torch.ones(n, device=dev)])
    start = float(opt.moments()[1].double().mean())
    for _ in range(steps):
        opt.step([torch.zeros(n, device=dev)])
    end = float(opt.moments()[1].double().mean())
    # the mean over 16384 elements: relative spread of one element after 1500 steps below sqrt(1500 * (1/16)^2 / 4) = 1.2, of the mean 1 %
    assert abs(end / start / b2 ** steps - 1) < 0.06


@gpu
def test_infinities_mark_their_block():
    s = Setup([600], 1, torch.float32, 8, seed=8)
    opt = s.optimizer(lr=1e-3)
    s.grads[0][0][300] = float("inf")
    opt.step(s.grads)
    m, v = opt.moments()
    bad = ~torch.isfinite(v.float())
    assert bool(bad[256:512].all()) and not bool(bad[:256].any()) and not bool(bad[512:600].any())
    assert s.state[2].tolist()[1] == 255 and s.state[3].tolist()[1] == 255


@gpu
def test_zero_start_zero_gradients_and_tiny_ones():
    for bits in (32, 8):
        w = torch.linspace(-1, 1, 1000, device="cuda")
        keep = w.clone()
        opt = P.AdamW([w], lr=0.1, weight_decay=0.0, state_bits=bits)
        opt.step([torch.zeros(1000, device="cuda")])
        assert torch.equal(w, keep)                                    # 0 / (0 + eps)
        g = torch.full((1000,), 1e-25, device="cuda")                  # squares below the smallest float
        opt.step([g])
        assert bool(torch.isfinite(w).all())


@gpu
def test_step_runs_on_the_current_stream():
    s = Setup([4096, 100], 1, torch.float32, 32, seed=2)
    opt = s.optimizer(lr=1e-2, step=0)
    want, _, _ = zip(*[adamw(a, b, d, g, 1, 1e-2, (0.9, 0.999), 1e-8, 0.01, 1, 1, np.float32) for a, b, d, g in
                       zip(s.w_np, unpack(s.m, s.sizes), unpack(s.v, s.sizes), weighted(s.grads_np, [1.0], np.float32))])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        clip = opt.grad_norm(s.grads)
        opt.step(s.grads, clip=clip)
    side.synchronize()
    assert np.array_equal(s.flat.cpu().numpy(), np.concatenate(want))


# ---- refusals (no GPU needed below) ---------------------------------------------------------------------------------

def test_sizes_of_a_list():
    e, b = C.c_int64(), C.c_int64()
    sizes = (C.c_int64 * 4)(1, 256, 257, 0)
    assert P.ps_tensors_sizes(4, sizes, C.byref(e), C.byref(b)) == P.PS_OK
    assert e.value == 256 + 256 + 512 and b.value > 0
    assert P.ps_tensors_sizes(0, sizes, C.byref(e), C.byref(b)) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_sizes(4, None, C.byref(e), C.byref(b)) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_sizes(1, (C.c_int64 * 1)(-1), None, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_sizes(1, (C.c_int64 * 1)(1 << 50), None, None) == P.PS_ERR_INVALID_ARG
    h = C.c_void_p()
    assert P.ps_tensors_create(C.byref(h), 4, sizes, None, b.value, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_create(C.byref(h), 4, sizes, 0x1000, b.value - 1, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_create(C.byref(h), 4, sizes, 0x1008, b.value, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_tensors_create(None, 4, sizes, 0x1000, b.value, None) == P.PS_ERR_INVALID_ARG
    fake = C.c_void_p(0x4000)                                          # not a handle this library made
    assert P.ps_tensors_destroy(fake) == P.PS_ERR_INVALID_ARG
    assert P.ps_grad_norm(fake, None, 1, None, 0, 1.0, None, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_adamw_step(fake, None, 1, None, 0, None, None, None) == P.PS_ERR_INVALID_ARG
    assert P.ps_adamw_moments(fake, None, None, None) == P.PS_ERR_INVALID_ARG


@gpu
def test_refusals_leave_everything_alone():
    s = Setup([100, 300], 2, torch.float32, 32, seed=4)
    opt = s.optimizer(lr=1e-2)
    before = [x.clone() for x in [s.flat, *s.state]]
    with pytest.raises(ValueError):
        opt.step([s.grads[0][:1]])                                     # a tensor short
    with pytest.raises(ValueError):
        opt.step(s.grads, scales=[1.0])                                # one scale for two gradients
    with pytest.raises(ValueError):
        opt.step([[s.grads[0][0][:50], s.grads[0][1]]])
    with pytest.raises(ValueError):
        opt.step([[torch.zeros(200, device="cuda")[::2], s.grads[0][1]]])
    with pytest.raises(TypeError):
        opt.step([[s.grads[0][0].half(), s.grads[0][1].half()]])
    with pytest.raises(TypeError):
        opt.step([s.grads[0], [g.bfloat16() for g in s.grads[1]]])
    with pytest.raises(ValueError):
        opt.step([[g.cpu() for g in s.grads[0]]])
    with pytest.raises(ValueError):
        opt.step([])
    for change in (dict(lr=-1.0), dict(lr=float("nan")), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(steps=-1),
                   dict(weight_decay=float("inf"))):
        old = {k: getattr(opt, k) for k in change}
        for k, x in change.items():
            setattr(opt, k, x)
        with pytest.raises(P.SoftsyncError) as e:
            opt.step(s.grads)
        assert e.value.status == P.PS_ERR_INVALID_ARG
        for k, x in old.items():
            setattr(opt, k, x)
    with pytest.raises(P.SoftsyncError):
        opt.step(s.grads, scales=[1.0, float("nan")])
    with pytest.raises(P.SoftsyncError):
        opt.grad_norm(s.grads, max_norm=0.0)
    with pytest.raises(P.SoftsyncError) as e:
        P.AdamW([s.params[0], s.params[0]])                            # overlapping parameters
    assert e.value.status == P.PS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        P.AdamW(s.params, state_bits=16)
    with pytest.raises(ValueError):
        P.AdamW(s.params, state=[torch.zeros(100, device="cuda")] * 2)
    with pytest.raises(TypeError):
        P.AdamW([p.double() for p in s.params])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, [s.flat, *s.state]))
    plan = P.TensorList([4])
    cfg = P.binding.AdamwConfig(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0)
    ptr = (C.c_void_p * 1)(s.grads[0][0].data_ptr())
    assert P.ps_adamw_step(plan._h, ptr, 1, None, 0, C.byref(cfg), None, None) == P.PS_ERR_NO_STATE
    assert P.ps_adamw_moments(opt._h, s.state[0].data_ptr(), s.state[1].data_ptr(), None) == P.PS_ERR_NO_STATE
