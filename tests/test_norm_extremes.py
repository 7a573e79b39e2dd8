"""The norm, its backward pass, the weight gradient from 8 bits and norm_linear where they can lose what they promise: values far from one, gains off their alignment, long
sums of one sign, other types of autocast, any strides.  Against float64; the roundings counted are those of test_packed_activations.py."""
import pytest
import torch

import paper_1511_05950_b200 as P
from tests.test_packed_activations import BF16, EPS, FP32, HALF, SUM, norm_reference, rows_of, same_codes

gpu = pytest.mark.gpu


# ---- values far from one --------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 64), (5, 1000), (3, 1001), (400, 2048), (5, 4096), (700, 4096), (3, 16384), (3, 20000), (2, 40001)])
def test_squares_beyond_fp32(dtype, rows, cols):
    """Rows whose squares overflow or vanish in fp32 although their mean's root does not: total and 1 / root are representable, so out and codes are as exact as ever.  A row of
    zeros is there too (NaN without an eps, by the formula), and a usual one."""
    g = torch.Generator().manual_seed(cols)
    x = rows_of(g, rows, cols, dtype)
    x.clamp_(-3.5, 3.5)
    for power in (125, 100, 63, -62, -80, -100, -120):
        big = (x.double() * 2.0 ** power).to(dtype)
        big[-1] = x[-1]
        for eps in (0.0, 1e-6):
            if eps and power < 0:
                continue                                                # eps is all there is: below
            total, rstd, n, out = norm_reference(big, None, None, eps, dtype)
            r = P.rms_norm(big, eps=eps, pack=True)
            assert bool(((r.rstd.double() - rstd).abs() <= SUM * EPS * rstd + 2.0 ** -150).all())
            assert bool(((r.out.double() - out).abs() <= (SUM + 4) * EPS * out.abs() + HALF[dtype] * out.abs() * (1 + SUM * EPS) + 1e-40).all())
            assert same_codes(r.packed, total.float() * r.rstd[:, None])
    small = (x.double() * 2.0 ** -80).to(dtype)
    r = P.rms_norm(small, eps=1e-6)
    assert bool(((r.rstd.double() - 1e3).abs() <= 1e3 * SUM * EPS).all())
    x[0] = 0.0
    assert bool(P.rms_norm(x, eps=0.0).out[0].isnan().all()) and bool((P.rms_norm(x, eps=1e-6).out[0] == 0).all())


@gpu
@pytest.mark.parametrize("cols", [64, 1001, 4096, 20000])
def test_a_large_total_of_residual_and_input(cols):
    g = torch.Generator().manual_seed(cols)
    x, residual = ((rows_of(g, 9, cols, BF16).clamp(-3, 3).double() * 2.0 ** k).to(BF16) for k in (90, 91))
    gain = (torch.randn(cols, generator=g) + 1).cuda()
    total, rstd, n, out = norm_reference(x, residual, gain, 1e-6, BF16)
    r = P.rms_norm(x, gain, residual, inplace=True)
    assert torch.equal(r.total, total) and bool(((r.rstd.double() - rstd).abs() <= SUM * EPS * rstd).all())
    assert bool(((r.out.double() - out).abs() <= (SUM + 4) * EPS * out.abs() + 2.0 ** -8 * out.abs() * (1 + SUM * EPS) + 1e-40).all())


# ---- gains off their alignment --------------------------------------------------------------------------------------------

def gain_at(g, cols, dtype, shift):
    return (torch.randn(cols + shift, generator=g) + 1).to(dtype).cuda()[shift:]


@gpu
@pytest.mark.parametrize("gain_dtype", [FP32, BF16])
@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 64), (40, 1024), (300, 2056), (3, 20000)])
def test_norm_with_a_gain_off_its_alignment(dtype, rows, cols, shift, gain_dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x, residual, dout, dtotal = (rows_of(g, rows, cols, dtype) for _ in range(4))
    gain = gain_at(g, cols, gain_dtype, shift)
    want = P.rms_norm(x, gain.clone(), residual, pack=True)
    got = P.rms_norm(x, gain, residual, pack=True)
    assert gain.data_ptr() % 16 and torch.equal(got.out, want.out) and torch.equal(got.packed.codes, want.packed.codes) and torch.equal(got.total, want.total)
    n, rstd = P.unpack8(want.packed, FP32).double(), want.rstd.double()[:, None]
    r = P.rms_norm_grad(dout, want.packed, want.rstd, gain, dtotal)
    gd = dout.double() * gain.double()
    dx = rstd * (gd - n * (gd * n).mean(1, keepdim=True)) + dtotal.double()
    off = (SUM + 8) * EPS * (rstd * (gd.abs() + n.abs() * (gd * n).abs().mean(1, keepdim=True)) + dtotal.double().abs())
    assert bool(((r.dx.double() - dx).abs() <= off + HALF[dtype] * dx.abs() + 1e-40).all())
    terms = dout.double() * n
    assert bool(((r.dgain.double() - terms.sum(0)).abs() <= (rows / 4 + SUM) * EPS * terms.abs().sum(0) + HALF[gain_dtype] * terms.sum(0).abs()).all())


@gpu
@pytest.mark.parametrize("gain_dtype", [FP32, BF16])
@pytest.mark.parametrize("rows,outs,cols", [(200, 100, 304), (65, 257, 255), (4097, 300, 520), (3000, 64, 72), (3000, 257, 255), (70, 40, 1), (129, 2500, 1104)])
def test_weight_gradient_with_a_gain_off_its_alignment(rows, outs, cols, gain_dtype):
    g = torch.Generator().manual_seed(rows + cols)
    dout, packed = rows_of(g, rows, outs, BF16), P.pack8(rows_of(g, rows, cols, FP32))
    for shift in (1, 3):
        gain = gain_at(g, cols, gain_dtype, shift)
        assert gain.data_ptr() % 16
        for dtype in (BF16, FP32):
            assert torch.equal(P.packed_weight_grad(dout, packed, gain, dtype), P.packed_weight_grad(dout, packed, gain.clone(), dtype))
        want = dout.double().T @ P.unpack8(packed, FP32).double() * gain.double()
        off = (rows / 16 + 32) * 2.0 ** -23 * (dout.double().abs().T @ P.unpack8(packed, FP32).double().abs()) * gain.double().abs()
        got = P.packed_weight_grad(dout, packed, gain, FP32)
        assert bool(((got.double() - want).abs() <= off * (1 + EPS) + EPS * want.abs() + 1e-38).all())


# ---- long sums of one sign ------------------------------------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("rows,outs,cols", [(32768, 74 * 256, 256), (32768, 300, 200), (1000000, 64, 64)])
def test_long_sums_of_one_sign(rows, outs, cols):
    """The tensor cores cut a running sum towards zero at each addition of 16 terms (at most 2^-23 of it), which in a sum of one sign adds up.  They are taken out every
    1,024 terms: 64 cuts of a sum that is half its end on average, 32 x 2^-23; then each turn's sum is added to nearest: rows / 1024 half steps of a sum that is half its end
    on average.  The first case has as many tiles as there are pairs of CTAs, none of which is split."""
    g = torch.Generator("cuda").manual_seed(rows)
    dout = torch.empty(rows, outs, dtype=BF16, device="cuda").uniform_(0.5, 1.5, generator=g)
    packed = P.pack8(torch.empty(rows, cols, device="cuda").uniform_(0.5, 1.5, generator=g))
    got = P.packed_weight_grad(dout, packed, dtype=FP32)
    some = torch.arange(0, outs, max(1, outs // 64), device="cuda")
    want = torch.zeros(len(some), cols, dtype=torch.float64, device="cuda")
    for part in range(0, rows, 65536):
        n = P.unpack8(P.Packed8(packed.codes[part:part + 65536], packed.scales[part:part + 65536], cols), FP32)
        want += dout[part:part + 65536, some].double().T @ n.double()
    assert bool(((got[some].double() / want - 1).abs() <= 32 * 2.0 ** -23 + (rows / 2048 + 2) * EPS).all())


# ---- norm_linear ----------------------------------------------------------------------------------------------------------

def layer(seed, rows=60, width=96, outs=40):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g).to(BF16).cuda()  # noqa: E731
    return rand(rows, width), rand(width) + 1, rand(outs, width) / width ** 0.5, rand(rows, width), rand(rows, outs), rand(rows, width)


@gpu
@pytest.mark.parametrize("kind", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("inside", [True, False])
def test_norm_linear_under_autocast(kind, inside):
    """The layer is bf16 whatever type autocast gives to torch's products, and its backward pass runs with it and without."""
    x, gain, weight, residual, dz, dtotal = layer(3)

    def step():
        leaves = [t.clone().requires_grad_(True) for t in (x, gain, weight, residual)]
        out = P.norm_linear(*leaves[:3], residual=leaves[3])
        if inside:
            torch.autograd.backward(out, [dz, dtotal])
        return leaves, out

    def grads(leaves, out):
        if not inside:
            torch.autograd.backward(out, [dz, dtotal])
        return [t.detach() for t in out] + [t.grad for t in leaves]

    want = grads(*step())
    with torch.autocast("cuda", dtype=kind):
        leaves, out = step()
    got = grads(leaves, out)
    assert all(a.dtype == BF16 for a in got) and all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_norm_linear_takes_any_strides():
    x, gain, weight, residual, dz, dtotal = layer(4)
    forms = {
        "columns apart": lambda t: t.T.contiguous().T,
        "every other": lambda t: torch.stack([t, t], 2).view(len(t), -1)[:, ::2],
        "rows apart": lambda t: torch.cat([t, t], 1)[:, :t.shape[1]],
        "one row for all": lambda t: t[:1].expand(len(t), -1),
        "three dimensions": lambda t: t.view(5, 12, -1).transpose(0, 1),
    }
    for name, form in forms.items():
        results = []
        for dense in (True, False):
            a, b = (form(t.clone()) for t in (x, residual))
            if dense:
                a, b = (t.clone(memory_format=torch.contiguous_format) for t in (a, b))
            leaves = [t.detach().requires_grad_(True) for t in (a, gain.clone(), weight.T.contiguous().T, b)]
            z, total = P.norm_linear(*leaves[:3], residual=leaves[3])
            torch.autograd.backward([z, total], [form(dz).reshape(z.shape), form(dtotal).reshape(total.shape)])
            results.append([z.detach(), total.detach()] + [t.grad for t in leaves])
        assert all(torch.equal(p, q) for p, q in zip(*results)), name
