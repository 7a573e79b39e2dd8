"""The norm, its backward pass, the weight gradient from 8 bits and norm_linear where they can lose what they promise: values far from one, gains off their alignment, long
sums of one sign, other types of autocast, any strides.  Against float64; the roundings counted are those of test_packed_activations.py."""
import pytest
import torch

import paper_1511_05950_b200 as P
from tests.test_packed_activations import BF16, EPS, FP32

gpu = pytest.mark.gpu


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
