"""Norm, activations in 8 bits and the weight gradient from them (include/softsync_learn.h) against plain implementations in float64.

Tolerances.  The squares of a row are added in fp32: eight by eight in a thread (at most 4 times, or in fp64 beyond), then over at most 10 exchanges; the mean,
its root and every product are rounded once: `SUM` roundings.  What is written in bf16 is off by half a step (2^-8) more, fp32 by 2^-24.  Codes
are compared exactly, with the formula applied to the very values that were packed.
"""
import ctypes as C

import pytest
import torch

import paper_1511_05950_b200 as P

gpu = pytest.mark.gpu
EPS = 2.0 ** -24
BF16, FP32 = torch.bfloat16, torch.float32
HALF = {BF16: 2.0 ** -8, FP32: EPS}
SUM = 32


def rows_of(g, rows, cols, dtype, pad=0, shift=0, scale=1.0):
    buf = (torch.randn(rows * (cols + pad) + shift, generator=g) * scale).to(dtype).cuda()
    return buf[shift:].view(rows, cols + pad)[:, :cols]


def plain_pack(x):
    """(codes, scales) of values, from the definition, on the CPU in float64."""
    x = x.detach().cpu().double()
    rows, cols = x.shape
    full = -(-cols // 32) * 32
    blocks = torch.nn.functional.pad(x, (0, full - cols)).view(rows, -1, 32)
    top = blocks.abs().amax(2)
    bad = ~blocks.isfinite().all(2)
    exponent = torch.frexp(torch.where(bad, 1.0, top))[1] - 1
    s = (exponent - 6 + 127).clamp(min=1)
    s[(top == 0) & ~bad] = 1
    codes = torch.round(blocks / torch.exp2(s.double() - 127)[:, :, None]).clamp(-127, 127)
    codes[bad], s[bad] = 0, 255
    return codes.view(rows, full).to(torch.int8), s.to(torch.uint8)


def same_codes(packed, x):
    codes, scales = plain_pack(x)
    return torch.equal(packed.codes.cpu(), codes) and torch.equal(packed.scales.cpu(), scales)


# ---- 8 bits ---------------------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (3, 7, 0, 0), (2, 31, 1, 0), (5, 32, 0, 0), (5, 33, 0, 1), (4, 100, 4, 4), (1, 1000, 0, 0), (37, 1000, 8, 8),
                                                 (37, 1001, 0, 0), (300, 512, 0, 3), (129, 4096, 0, 0), (2, 70001, 0, 0)])
def test_pack_and_unpack(dtype, rows, cols, pad, shift):
    g = torch.Generator().manual_seed(rows * cols)
    x = rows_of(g, rows, cols, dtype, pad, shift)
    x *= torch.exp2(torch.randint(-20, 20, (rows, 1), generator=g).cuda()).to(dtype)
    packed = P.pack8(x)
    assert packed.codes.shape == (rows, -(-cols // 32) * 32) and packed.cols == cols and same_codes(packed, x)
    unit = torch.exp2(packed.scales.double() - 127).repeat_interleave(32, 1)
    values = (packed.codes.double() * unit)[:, :cols]
    for kind in (BF16, FP32):
        back = P.unpack8(packed, kind)
        assert back.dtype == kind and torch.equal(back.double(), values)
    off = (values - x.double()).abs() / unit[:, :cols]
    assert float(off.max()) <= 1.0                                      # half a unit, a whole one where the code is cut to 127
    assert bool((off[(packed.codes[:, :cols].abs() < 127)] <= 0.5).all())


@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_values_at_the_edges(dtype):
    """Zeros, subnormals, the largest values, ties, codes that are cut, infinities and NaN: a block each."""
    info = torch.finfo(dtype)
    x = torch.zeros(12, 32, dtype=dtype)
    x[1] = info.smallest_normal * torch.linspace(0, 1, 32).to(dtype) / 4
    x[2] = info.max * torch.linspace(-1, 1, 32).to(dtype)
    x[3, 0], x[3, 1:] = 1.0, (torch.arange(31) + 0.5).to(dtype) / 64     # ties to even
    x[4], x[4, 3] = 0.25, 1.9921875                                      # 127.5 units
    x[5, 7] = float("inf")
    x[6, 7] = float("nan")
    x[7, 31] = -info.max
    x[8] = -0.0
    x[9] = 2.0 ** -126
    x[10] = 2.0 ** -120 * 1.5
    x[11, 0], x[11, 1] = 1.0, -2.0 ** -40
    for rows in (x, x.reshape(3, 128), x.reshape(1, 384)):
        packed = P.pack8(rows.cuda())
        assert same_codes(packed, rows)
        back = P.unpack8(packed).float().cpu().view(12, 32)
        assert bool(back[5:7].isnan().all()) and bool(back[[k for k in range(12) if k not in (5, 6)]].isfinite().all())


@gpu
def test_nothing_is_written_beside_the_rows():
    x = torch.randn(5, 40, device="cuda")
    packed = P.pack8(x)
    wide = torch.full((5, 48), 7.0, device="cuda", dtype=BF16)
    assert P.ps_unpack8(packed.codes.data_ptr(), packed.scales.data_ptr(), 5, 40, wide.data_ptr(), P.PS_GRAD_BF16, 48, None) == P.PS_OK
    torch.cuda.synchronize()
    assert bool((wide[:, 40:] == 7).all()) and torch.equal(wide[:, :40], P.unpack8(packed))
    assert P.pack8(x[:0]).codes.shape == (0, 64) and P.unpack8(P.pack8(x[:0])).shape == (0, 40)


@gpu
def test_more_than_two_to_the_32_values():
    rows, cols = 70001, 65600
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.empty(rows, cols, dtype=BF16, device="cuda").normal_(generator=g)
    packed = P.pack8(x)
    back = P.unpack8(packed)
    for part in (slice(0, 2), slice(rows // 2, rows // 2 + 2), slice(rows - 2, rows)):
        one = P.Packed8(packed.codes[part], packed.scales[part], cols)
        assert same_codes(one, x[part]) and torch.equal(back[part], P.unpack8(P.pack8(x[part].clone())))
    r = P.rms_norm(x, pack=True)
    want = P.rms_norm(x[-2:].clone(), pack=True)
    assert torch.equal(r.out[-2:], want.out) and torch.equal(r.packed.codes[-2:], want.packed.codes)
    dx = P.rms_norm_grad(x, r.packed, r.rstd).dx
    assert torch.equal(dx[-2:], P.rms_norm_grad(x[-2:].clone(), want.packed, want.rstd).dx)


# ---- norm -----------------------------------------------------------------------------------------------------------------

SHAPES = [  # rows, cols, pad, shift
    (1, 1, 0, 0), (3, 7, 0, 0), (5, 33, 0, 1), (6, 256, 0, 0), (7, 257, 0, 0), (130, 512, 8, 8), (9, 1000, 0, 0), (5, 1024, 0, 0), (4, 1025, 3, 0), (33, 2048, 0, 0), (3, 2056, 0, 0),
    (700, 4096, 0, 0), (2, 4104, 0, 4), (3, 8192, 0, 0), (2, 8200, 0, 0), (3, 16384, 0, 0), (2, 16392, 0, 0), (2, 40001, 0, 0), (1, 200000, 0, 0),
]


def norm_reference(x, residual, gain, eps, dtype):
    total = x if residual is None else (x.float() + residual.float()).to(dtype)
    t = total.double()
    rstd = (t.square().mean(1) + eps).rsqrt()
    n = t * rstd[:, None]
    return total, rstd, n, n if gain is None else n * gain.double()


@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES)
def test_norm(dtype, rows, cols, pad, shift):
    g = torch.Generator().manual_seed(rows + cols)
    x, residual = rows_of(g, rows, cols, dtype, pad, shift), rows_of(g, rows, cols, dtype, 0, shift, scale=3.0)
    for gain, res in ((None, residual), ((torch.randn(cols, generator=g) + 1).cuda(), None), ((torch.randn(cols, generator=g) + 1).to(BF16).cuda(), residual)):
        total, rstd, n, out = norm_reference(x, res, gain, 1e-5, dtype)
        r = P.rms_norm(x, gain, res, eps=1e-5, pack=True)
        assert torch.equal(r.total, total) and (res is not None or r.total is x)
        assert bool(((r.rstd.double() - rstd).abs() <= SUM * EPS * rstd).all())
        assert bool(((r.out.double() - out).abs() <= (SUM + 4) * EPS * out.abs() + HALF[dtype] * out.abs() * (1 + SUM * EPS) + 1e-40).all())
        values = total.float() * r.rstd[:, None]                        # what was packed: one rounding each, as in the kernel
        assert same_codes(r.packed, values)
        only = P.rms_norm(x, gain, res, eps=1e-5, out=False, pack=True)
        assert only.out is None and torch.equal(only.packed.codes, r.packed.codes) and torch.equal(only.rstd, r.rstd)
        bare = P.rms_norm(x, gain, res, eps=1e-5)
        assert bare.packed is None and torch.equal(bare.out, r.out)


@gpu
@pytest.mark.parametrize("cols", [64, 1001, 2048, 20000])
def test_the_total_in_the_residuals_place(cols):
    g = torch.Generator().manual_seed(cols)
    x, residual = rows_of(g, 9, cols, BF16), rows_of(g, 9, cols, BF16, pad=8)
    want = P.rms_norm(x, None, residual, pack=True)
    before = residual._version
    r = P.rms_norm(x, None, residual, pack=True, inplace=True)
    assert r.total.data_ptr() == residual.data_ptr() and residual._version == before + 1 and torch.equal(residual, want.total)
    assert torch.equal(r.out, want.out) and torch.equal(r.packed.codes, want.packed.codes)
    with pytest.raises(ValueError, match="residual"):
        P.rms_norm(x, inplace=True)


@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("cols", [64, 300, 1001, 4096, 20000])
@pytest.mark.parametrize("eps", [1e-12, 1e-5])
def test_codes_of_blocks_of_zeros(dtype, cols, eps):
    """Rows, and blocks within rows, that hold nothing: the least unit, and codes that are 0 whatever the row's factor."""
    g = torch.Generator().manual_seed(cols)
    x = rows_of(g, 4, cols, dtype)
    x[1], x[2, :32], x[3, 32:] = 0.0, 0.0, 0.0
    r = P.rms_norm(x, eps=eps, pack=True)
    assert same_codes(r.packed, x.float() * r.rstd[:, None])
    assert bool((r.packed.codes[1] == 0).all()) and bool((r.packed.scales[1] == 1).all()) and bool((r.out[1] == 0).all())
    assert bool((r.packed.codes[2, :32] == 0).all()) and bool((r.packed.codes[3, 32:] == 0).all())


@gpu
def test_rows_of_zeros_and_bad_rows():
    x = torch.randn(6, 300, device="cuda").to(BF16)
    x[1], x[2, 4], x[3, 5] = 0.0, float("nan"), float("inf")
    r = P.rms_norm(x, eps=1e-6, pack=True)
    clean = P.rms_norm(x[[0, 4, 5]], eps=1e-6, pack=True)
    assert torch.equal(r.out[[0, 4, 5]], clean.out) and torch.equal(r.packed.codes[[0, 4, 5]], clean.packed.codes)
    assert bool((r.out[1] == 0).all()) and bool(r.out[2].isnan().all()) and bool(r.out[3, 5].isnan())
    assert bool(P.unpack8(r.packed)[2].isnan().all())
    assert P.rms_norm(x[:0], pack=True).out.shape == (0, 300)


# ---- its backward pass ----------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols,pad,shift", SHAPES)
def test_norm_backward(dtype, rows, cols, pad, shift):
    g = torch.Generator().manual_seed(rows + cols + 1)
    x, dout = rows_of(g, rows, cols, dtype, 0, shift), rows_of(g, rows, cols, dtype, pad, shift)
    dtotal = rows_of(g, rows, cols, dtype, pad, 0)
    for gain, more in ((None, dtotal), ((torch.randn(cols, generator=g) + 1).cuda(), None), ((torch.randn(cols, generator=g) + 1).to(BF16).cuda(), dtotal)):
        fwd = P.rms_norm(x, gain, pack=True)
        for kept in (fwd.packed, fwd.total):
            rstd = fwd.rstd.double()[:, None]
            n = P.unpack8(kept, FP32).double() if kept is fwd.packed else kept.double() * rstd
            gd = dout.double() if gain is None else dout.double() * gain.double()
            mean = (gd * n).mean(1, keepdim=True)
            dx = rstd * (gd - n * mean) + (0 if more is None else more.double())
            off = (SUM + 8) * EPS * (rstd * (gd.abs() + n.abs() * (gd * n).abs().mean(1, keepdim=True)) + (0 if more is None else more.double().abs()))
            r = P.rms_norm_grad(dout, kept, fwd.rstd, gain, more)
            assert bool(((r.dx.double() - dx).abs() <= off + HALF[dtype] * dx.abs() + 1e-40).all())
            again = P.rms_norm_grad(dout, kept, fwd.rstd, gain, more)
            assert torch.equal(r.dx, again.dx) and (gain is None or torch.equal(r.dgain, again.dgain))
            if gain is None:
                assert r.dgain is None
                continue
            dgain = (dout.double() * n).sum(0)
            off = (rows / 4 + SUM) * EPS * (dout.double() * n).abs().sum(0)
            assert r.dgain.dtype == gain.dtype and bool(((r.dgain.double() - dgain).abs() <= off + HALF[gain.dtype] * dgain.abs() + 1e-40).all())
            assert P.rms_norm_grad(dout, kept, fwd.rstd, gain, more, grad_gain=False).dgain is None


@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols", [(6001, 64), (6001, 1024), (3001, 1100), (5003, 2048), (3001, 4096), (1999, 8192), (1300, 8200)])
def test_many_rows(dtype, rows, cols):
    """More rows than blocks: every block goes round its slots of shared memory several times and adds up the gain's gradient."""
    g = torch.Generator().manual_seed(3)
    x, dout, dtotal = rows_of(g, rows, cols, dtype), rows_of(g, rows, cols, dtype), rows_of(g, rows, cols, dtype, pad=8)
    gain = (torch.randn(cols, generator=g) + 1).cuda()
    fwd = P.rms_norm(x, gain, pack=True)
    n, rstd = P.unpack8(fwd.packed, FP32).double(), fwd.rstd.double()[:, None]
    for more in (None, dtotal):
        r = P.rms_norm_grad(dout, fwd.packed, fwd.rstd, gain, more)
        gd = dout.double() * gain.double()
        dx = rstd * (gd - n * (gd * n).mean(1, keepdim=True)) + (0 if more is None else more.double())
        off = (SUM + 8) * EPS * (rstd * (gd.abs() + n.abs() * (gd * n).abs().mean(1, keepdim=True)) + (0 if more is None else more.double().abs()))
        assert bool(((r.dx.double() - dx).abs() <= off + HALF[dtype] * dx.abs() + 1e-40).all())
        terms = dout.double() * n
        assert bool(((r.dgain.double() - terms.sum(0)).abs() <= (rows / 32 + SUM) * EPS * terms.abs().sum(0)).all())
        assert torch.equal(r.dx, P.rms_norm_grad(dout, fwd.packed, fwd.rstd, gain, more).dx)
    one = P.rms_norm_grad(dout[-1:], P.Packed8(fwd.packed.codes[-1:], fwd.packed.scales[-1:], cols), fwd.rstd[-1:], gain, dtotal[-1:])
    assert torch.equal(one.dx[0], r.dx[-1])


@gpu
def test_norm_gradient_against_differences():
    """The kept total's gradient along random directions, in fp32: the loss is sum(dout out), whose third derivative along a step of
    relative size s is below 16 s^3 of |dout| |out|."""
    g = torch.Generator().manual_seed(5)
    x, dout = rows_of(g, 8, 500, FP32), rows_of(g, 8, 500, FP32)
    gain = (torch.randn(500, generator=g) + 1).cuda()
    fwd = P.rms_norm(x, gain)
    r = P.rms_norm_grad(dout, fwd.total, fwd.rstd, gain)
    s = 1e-2
    way = rows_of(g, 8, 500, FP32) * s
    loss = [(P.rms_norm(x + k * way, gain).out.double() * dout.double()).sum() for k in (1, -1)]
    size = float((dout.norm(dim=1) * fwd.out.norm(dim=1)).sum())
    assert abs(float(loss[0] - loss[1]) / 2 - float((r.dx.double() * way.double()).sum())) <= 16 * s ** 3 * size + 64 * EPS * size
    way = torch.randn(500, generator=g).cuda()
    loss = [(P.rms_norm(x, gain + k * way).out.double() * dout.double()).sum() for k in (1, -1)]
    size = float((dout.double().abs() * (P.rms_norm(x).out.double() * way.double()).abs()).sum() + (dout.double().abs() * fwd.out.double().abs()).sum())
    assert abs(float(loss[0] - loss[1]) / 2 - float((r.dgain.double() * way.double()).sum())) <= (SUM + 16) * EPS * size


# ---- weight gradient from the codes ---------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("rows,outs,cols,pad,shift", [
    (1, 1, 1, 0, 0), (1, 8, 33, 0, 0), (63, 64, 64, 0, 0), (64, 256, 256, 0, 0), (65, 257, 255, 0, 0), (200, 768, 256, 8, 8), (200, 100, 300, 3, 0), (129, 136, 40, 0, 1),
    (3000, 64, 72, 0, 0), (4097, 300, 520, 0, 0), (1000, 1032, 2048, 0, 0), (700, 2500, 1100, 0, 0)])
def test_weight_gradient(rows, outs, cols, pad, shift):
    g = torch.Generator().manual_seed(rows + outs + cols)
    dout = rows_of(g, rows, outs, BF16, pad, shift)
    packed = P.pack8(rows_of(g, rows, cols, FP32) * torch.exp2(torch.randint(-4, 4, (1, cols), generator=g).float()).cuda())
    n = P.unpack8(packed, FP32).double()
    for gain in (None, (torch.randn(cols, generator=g) + 1).cuda(), (torch.randn(cols, generator=g) + 1).to(BF16).cuda()):
        k = 1.0 if gain is None else gain.double()
        want = (dout.double().T @ n) * k
        off = (rows / 16 + 32) * 2.0 ** -23 * (dout.double().abs().T @ n.abs()) * (1.0 if gain is None else gain.double().abs())
        for dtype in (BF16, FP32):
            got = P.packed_weight_grad(dout, packed, gain, dtype)
            assert got.dtype == dtype and got.shape == (outs, cols)
            assert bool(((got.double() - want).abs() <= off + HALF[dtype] * (want.abs() + off) + 1e-38).all())
            assert torch.equal(got, P.packed_weight_grad(dout, packed, gain, dtype))


@gpu
def test_weight_gradient_without_rows_and_of_bad_ones():
    packed = P.pack8(torch.randn(80, 70, device="cuda"))
    none = P.Packed8(packed.codes[:0], packed.scales[:0], 70)
    assert bool((P.packed_weight_grad(torch.zeros(0, 50, device="cuda", dtype=BF16), none) == 0).all())
    x = torch.randn(80, 70, device="cuda")
    x[3, 40] = float("inf")
    dw = P.packed_weight_grad(torch.ones(80, 50, device="cuda", dtype=BF16), P.pack8(x))
    assert bool(dw[:, 32:64].isnan().all()) and bool(dw[:, :32].isfinite().all()) and bool(dw[:, 64:].isfinite().all())


# ---- norm and linear layer for autograd -----------------------------------------------------------------------------------

def kept_gradients(x, residual, gain, weight, dz, dtotal, eps):
    """The gradients that norm_linear promises: of the values that 8 bits stand for."""
    fwd = P.rms_norm(x, gain, residual, eps=eps, pack=True)
    n, rstd = P.unpack8(fwd.packed, FP32).double(), fwd.rstd.double()[:, None]
    dy = (dz @ weight).double()
    gd = dy * gain.double()
    dx = rstd * (gd - n * (gd * n).mean(1, keepdim=True)) + (0 if dtotal is None else dtotal.double())
    return dx, (dy * n).sum(0), (dz.double().T @ n) * gain.double()


@gpu
@pytest.mark.parametrize("lead,width,outs", [((5,), 64, 40), ((2, 3, 7), 100, 33), ((300,), 512, 264)])
def test_norm_linear(lead, width, outs):
    g = torch.Generator().manual_seed(width)
    rand = lambda *s: torch.randn(*s, generator=g).to(BF16).cuda()  # noqa: E731
    x, residual, gain, weight = rand(*lead, width), rand(*lead, width), rand(width) + 1, rand(outs, width) / width ** 0.5
    dz, dtotal = rand(*lead, outs), rand(*lead, width)
    for res in (residual, None):
        leaves = [t.clone().requires_grad_(True) for t in (x, gain, weight)] + ([residual.clone().requires_grad_(True)] if res is not None else [])
        z, total = P.norm_linear(*leaves[:3], residual=leaves[3] if res is not None else None)
        flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        fwd = P.rms_norm(flat(x), gain, None if res is None else flat(res))
        assert torch.equal(flat(z), fwd.out @ weight.T) and torch.equal(flat(total), fwd.total) and z.shape == (*lead, outs)
        torch.autograd.backward([z, total], [dz, dtotal])
        dx, dgain, dweight = kept_gradients(flat(x), None if res is None else flat(res), gain, weight, flat(dz), flat(dtotal), 1e-6)
        direct = P.rms_norm(flat(x), gain, None if res is None else flat(res), pack=True)
        assert torch.equal(leaves[2].grad, P.packed_weight_grad(flat(dz), direct.packed, gain))
        for got, want in ((flat(leaves[0].grad), dx), (leaves[1].grad, dgain), (leaves[2].grad, dweight)):
            size = want.abs().max()
            assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4 * size).all())
        if res is not None:
            assert torch.equal(leaves[3].grad, leaves[0].grad)


@gpu
def test_norm_linear_parts_of_the_gradient():
    g = torch.Generator().manual_seed(8)
    x, gain, weight = (torch.randn(*s, generator=g).to(BF16).cuda() for s in ((20, 64), (64,), (32, 64)))
    a = x.clone().requires_grad_(True)
    z, total = P.norm_linear(a, gain, weight)
    z.sum().backward()                                                 # an expanded gradient, none for the total
    b, w = x.clone().requires_grad_(True), weight.clone().requires_grad_(True)
    z, total = P.norm_linear(b, gain, w, residual=x)
    total.backward(torch.ones_like(total))                             # none for z
    assert bool((b.grad == 1).all()) and (w.grad is None or bool((w.grad == 0).all()))
    w = weight.clone().requires_grad_(True)
    z, _ = P.norm_linear(x, gain, w)
    z.backward(torch.ones_like(z))
    kept = P.rms_norm(x, gain, pack=True).packed
    assert torch.equal(w.grad, P.packed_weight_grad(torch.ones_like(z), kept, gain)) and bool(a.grad.isfinite().all())
    with torch.no_grad():
        assert not P.norm_linear(a, gain, weight)[0].requires_grad
    none, w = x[:0].clone().requires_grad_(True), weight.clone().requires_grad_(True)
    z, total = P.norm_linear(none, gain, w)
    (z.sum() + total.sum()).backward()
    assert z.shape == (0, 32) and none.grad.shape == (0, 64) and bool((w.grad == 0).all())


@gpu
def test_norm_linear_keeps_eight_bits():
    """Between the passes: codes, scales and a number a row, beside what the caller holds."""
    x, gain, weight = (torch.ones(*s, device="cuda", dtype=BF16) for s in ((4096, 2048), (2048,), (64, 2048)))
    x, weight = x.requires_grad_(True), weight.requires_grad_(True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    z, total = P.norm_linear(x, gain, weight)
    kept = torch.cuda.memory_allocated() - before - z.numel() * 2
    assert kept <= 4096 * 2048 * 33 / 32 + 4096 * 4 + 4096


@gpu
def test_a_step_of_all_of_them():
    """Two layers and a loss without logits, forward and backward, and the gradients to a server: near the same model in float32 with autograd and
    full activations.  Each kept value is off by at most 1/64 of its block's largest (2^-7 of it on average less), so the gradients of a whole
    tensor agree to a few parts in a hundred; the loss is not touched by the 8 bits at all."""
    g = torch.Generator().manual_seed(12)
    vocab, width, rows = 1000, 128, 256
    shapes = [(vocab, width), (width,), (width, width), (width,), (width, width), (width,), (vocab, width)]
    masters = [(torch.randn(*s, generator=g) * (s[-1] ** -0.5) if len(s) == 2 else torch.ones(*s)).cuda() for s in shapes]
    tokens = torch.randint(0, vocab, (rows + 1,), generator=g).cuda()
    weights = (torch.rand(rows, generator=g) > 0.3).float().cuda()
    p = [m.to(BF16).requires_grad_(True) for m in masters]
    stream = p[0][tokens[:-1]]
    z, total = P.norm_linear(stream, p[1], p[2])
    z, total = P.norm_linear(torch.relu(z), p[3], p[4], residual=total)
    last = P.rms_norm(z.detach(), p[5].detach(), total.detach(), pack=True)
    r = P.head_cross_entropy(last.out, p[6].detach(), tokens[1:], weights=weights)
    back = P.rms_norm_grad(r.dhidden, last.packed, last.rstd, p[5].detach())
    torch.autograd.backward([z, total], [back.dx, back.dx])
    grads = [t.grad if t.grad is not None else None for t in p]
    grads[5], grads[6] = back.dgain, r.dhead

    q = [t.detach().float().requires_grad_(True) for t in p]
    norm = lambda t, gain: t * torch.rsqrt(t.square().mean(1, keepdim=True) + 1e-6) * gain  # noqa: E731
    s = q[0][tokens[:-1]]
    y = torch.relu(norm(s, q[1]) @ q[2].T)
    s = y + s
    s = norm(s, q[3]) @ q[4].T + s
    logp = torch.log_softmax(norm(s, q[5]) @ q[6].T, 1)[torch.arange(rows), tokens[1:]]
    loss = -(weights * logp).sum() / weights.sum()
    loss.backward()
    assert abs(float(r.stats[0]) - float(loss)) <= 2e-2 * abs(float(loss))
    for got, want in zip(grads, q):
        assert float((got.float() - want.grad).norm()) <= 0.05 * float(want.grad.norm())
    params = [m.clone() for m in masters]
    server = P.AdamWServer(params, 1, 1, max_norm=1.0, lr=1e-3)
    server.push(0, [x.contiguous() for x in grads], server.pull())
    server.apply_update()
    assert all(bool(a.isfinite().all()) and not torch.equal(a, b) for a, b in zip(params, masters))


@gpu
def test_norm_linear_captured():
    """A whole step, forward and backward, replayed with other inputs."""
    g = torch.Generator().manual_seed(23)
    x, residual, dz, dtotal = (rows_of(g, 200, k, BF16) for k in (128, 128, 96, 128))
    gain, weight = (torch.randn(*s, generator=g).to(BF16).cuda() for s in ((128,), (96, 128)))
    leaves = [t.requires_grad_(True) for t in (x, gain, weight)]

    def step():
        for t in leaves:
            t.grad = None
        z, total = P.norm_linear(x, gain, weight, residual=residual)
        torch.autograd.backward([z, total], [dz, dtotal])
        return [z, total] + [t.grad for t in leaves]

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            out = step()
        del out                                                        # no eager graph of these leaves lives on
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = [t.detach() for t in step()]
    with torch.no_grad():
        for t in (x, residual, dz, dtotal):
            t.copy_(rows_of(g, *t.shape, BF16))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in got]
    assert all(torch.equal(a, b) for a, b in zip(got, step()))


@gpu
def test_two_streams_at_once():
    g = torch.Generator().manual_seed(22)
    sets = [(rows_of(g, 500, 1000, BF16), rows_of(g, 500, 300, BF16)) for _ in range(2)]
    gain = torch.ones(1000, device="cuda")

    def run(x, dz):
        fwd = P.rms_norm(x, gain, x, pack=True)
        back = P.rms_norm_grad(x, fwd.packed, fwd.rstd, gain, x)
        return (*fwd.packed[:2], fwd.out, fwd.total, *back, P.packed_weight_grad(dz, fwd.packed, gain))

    want = [run(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(run(*sets[k]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k in range(2) for r in got[k] for a, b in zip(r, want[k]))


@gpu
def test_captured_and_replayed():
    g = torch.Generator().manual_seed(21)
    make = lambda: [rows_of(g, 150, 300, BF16) for _ in range(3)] + [rows_of(g, 150, 200, BF16)]  # noqa: E731
    x, residual, dout, dz = make()
    gain = torch.ones(300, device="cuda")

    def run():
        fwd = P.rms_norm(x, gain, residual, pack=True)
        return (*fwd.packed[:2], fwd.out, *P.rms_norm_grad(dout, fwd.packed, fwd.rstd, gain, dout), P.packed_weight_grad(dz, fwd.packed, gain), P.unpack8(P.pack8(x)))

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = run()
    for fresh in (None, make()):
        if fresh:
            for a, b in zip((x, residual, dout, dz), fresh):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, run()))


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------------

def norm(**kw):
    good = dict(x_dev=4096, dtype=P.PS_GRAD_BF16, gain_dtype=P.PS_GRAD_FP32, rows=4, cols=64, x_stride=64, residual_stride=64, total_stride=64, eps=1e-6, rstd_dev=4096)
    return P.binding.Norm(**{**good, **kw})


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(rows=-1), dict(rows=1 << 33), dict(cols=0), dict(cols=1 << 30), dict(x_dev=None), dict(x_dev=4097), dict(x_stride=63), dict(x_stride=1 << 60), dict(eps=-1.0),
    dict(eps=float("nan")), dict(rstd_dev=None), dict(rstd_dev=4098), dict(gain_dev=4098), dict(gain_dev=4096, gain_dtype=9), dict(residual_dev=4097), dict(residual_dev=64, residual_stride=8),
    dict(total_dev=8192, total_stride=8), dict(total_dev=4096, total_stride=72), dict(out_dev=4096, x_stride=72), dict(out_dev=8192, total_dev=8192), dict(codes_dev=4096), dict(scales_dev=4096),
    dict(codes_dev=4104, scales_dev=4096)], ids=str)
def test_norm_refused(bad):
    assert P.ps_rms_norm(C.byref(norm(**bad)), None) == P.PS_ERR_INVALID_ARG


def grad(**kw):
    good = dict(dout_dev=4096, total_dev=8192, rstd_dev=4096, dtype=P.PS_GRAD_BF16, gain_dtype=P.PS_GRAD_FP32, rows=4, cols=64, dout_stride=64, total_stride=64, dtotal_stride=64, dx_dev=16384)
    return P.binding.NormGrad(**{**good, **kw})


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(rows=-1), dict(cols=0), dict(dout_dev=None), dict(dout_dev=4097), dict(dout_stride=8), dict(total_dev=None), dict(total_stride=3), dict(codes_dev=4096, scales_dev=4096),
    dict(codes_dev=4096, total_dev=None), dict(rstd_dev=None), dict(dx_dev=None), dict(dx_dev=8192), dict(dx_dev=4096, dout_stride=72), dict(dtotal_dev=4097),
    dict(dtotal_dev=4096, dtotal_stride=2), dict(dgain_dev=4098), dict(gain_dev=4096, gain_dtype=3), dict(cols=20000, dout_stride=20000, total_stride=20000, dx_dev=4096, dgain_dev=256)], ids=str)
def test_norm_gradient_refused(bad):
    assert P.ps_rms_norm_grad(C.byref(grad(**bad)), 256, 1 << 30, None) == P.PS_ERR_INVALID_ARG


def test_workspaces_refused():
    n = C.c_int64()
    assert P.ps_norm_grad_workspace(100, 64, C.byref(n)) == P.PS_OK and n.value > 0
    assert P.ps_norm_grad_workspace(100, 0, C.byref(n)) == P.PS_ERR_INVALID_ARG and P.ps_norm_grad_workspace(100, 64, None) == P.PS_ERR_INVALID_ARG
    for ws, size in ((None, 1 << 30), (264, 1 << 30), (256, 100)):
        assert P.ps_rms_norm_grad(C.byref(grad(dgain_dev=4096)), ws, size, None) == P.PS_ERR_INVALID_ARG
    a = packed_grad()
    assert P.ps_packed_grad_workspace(C.byref(a), C.byref(n)) == P.PS_OK and n.value > 0
    for ws, size in ((None, 1 << 30), (264, 1 << 30), (256, n.value - 1)):
        assert P.ps_packed_weight_grad(C.byref(a), ws, size, None) == P.PS_ERR_INVALID_ARG


def packed_grad(**kw):
    good = dict(dout_dev=4096, codes_dev=4096, scales_dev=4096, gain_dtype=P.PS_GRAD_FP32, out_dtype=P.PS_GRAD_BF16, rows=100, outs=64, cols=64, dout_stride=64, dweight_dev=8192)
    return P.binding.PackedGrad(**{**good, **kw})


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 40), dict(outs=0), dict(cols=0), dict(cols=1 << 22), dict(dout_dev=None), dict(dout_dev=4097), dict(dout_stride=8), dict(codes_dev=None),
                                 dict(codes_dev=4104), dict(scales_dev=None), dict(out_dtype=5), dict(gain_dev=4098), dict(gain_dev=4096, gain_dtype=4), dict(dweight_dev=None),
                                 dict(dweight_dev=8200)], ids=str)
def test_weight_gradient_refused(bad):
    assert P.ps_packed_weight_grad(C.byref(packed_grad(**bad)), 256, 1 << 40, None) == P.PS_ERR_INVALID_ARG


def test_packing_refused():
    for args in ((None, 1, 4, 64, 64, 256, 256), (4097, 1, 4, 64, 64, 256, 256), (256, 5, 4, 64, 64, 256, 256), (256, 1, -4, 64, 64, 256, 256), (256, 1, 4, 0, 64, 256, 256),
                 (256, 1, 4, 64, 8, 256, 256), (256, 1, 4, 64, 64, 264, 256), (256, 1, 4, 64, 64, None, 256), (256, 1, 4, 64, 64, 256, None)):
        x, dtype, rows, cols, stride, codes, scales = args
        assert P.ps_pack8(*args, None) == P.PS_ERR_INVALID_ARG
        assert P.ps_unpack8(codes, scales, rows, cols, x, dtype, stride, None) == P.PS_ERR_INVALID_ARG


def test_refused_in_python():
    x = torch.zeros(4, 64)
    codes, scales = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8)
    for call, error in (
            (lambda: P.pack8(x), ValueError), (lambda: P.pack8(x.double()), TypeError), (lambda: P.pack8(x.T), ValueError), (lambda: P.pack8([1]), TypeError),
            (lambda: P.unpack8(P.Packed8(codes, scales, 64)), ValueError), (lambda: P.unpack8(P.Packed8(codes, scales, 65)), ValueError),
            (lambda: P.unpack8(P.Packed8(codes, scales[:, :1], 64)), ValueError), (lambda: P.unpack8(P.Packed8(codes.float(), scales, 64)), TypeError),
            (lambda: P.unpack8(P.Packed8(codes, scales, 64), torch.float16), TypeError), (lambda: P.rms_norm(x), ValueError), (lambda: P.rms_norm(x.half()), TypeError),
            (lambda: P.rms_norm_grad(x, x, x), ValueError), (lambda: P.rms_norm_grad(x, P.Packed8(codes, scales, 63), x), ValueError),
            (lambda: P.packed_weight_grad(x, P.Packed8(codes, scales, 64)), ValueError), (lambda: P.packed_weight_grad(x, P.Packed8(codes, scales, 64), dtype=torch.half), TypeError),
            (lambda: P.norm_linear(x, x[0], x), TypeError), (lambda: P.norm_linear(x.to(BF16), x[0], x[:, :3].to(BF16)), ValueError),
            (lambda: P.norm_linear(x.to(BF16), x[0], x.to(BF16), residual=x[:2].to(BF16)), ValueError)):
        with pytest.raises(error):
            call()


@gpu
def test_refused_in_python_on_the_gpu():
    x = torch.zeros(4, 64, device="cuda")
    kept, r = P.pack8(x), torch.zeros(4, device="cuda")
    for call, error in (
            (lambda: P.rms_norm(x, gain=x[0, :5]), ValueError), (lambda: P.rms_norm(x, gain=x[0].double()), TypeError), (lambda: P.rms_norm(x, residual=x[:3]), ValueError),
            (lambda: P.rms_norm(x, residual=x.to(BF16)), TypeError), (lambda: P.rms_norm(x, eps=-1.0), P.SoftsyncError), (lambda: P.rms_norm(x, gain=x[0].cpu()), ValueError),
            (lambda: P.rms_norm_grad(x, kept, r[:2]), ValueError), (lambda: P.rms_norm_grad(x[:3], kept, r[:3]), ValueError), (lambda: P.rms_norm_grad(x, x.to(BF16), r), TypeError),
            (lambda: P.rms_norm_grad(x, kept, r, dtotal=x[:, :3]), ValueError), (lambda: P.packed_weight_grad(x, kept), TypeError),
            (lambda: P.packed_weight_grad(x[:2].to(BF16), kept), ValueError), (lambda: P.packed_weight_grad(x.to(BF16), kept, gain=x[0, :3]), ValueError)):
        with pytest.raises(error):
            call()
