"""The norms around a block at the ends of BF16's range: products of a gate and a weight that leave binary32 although the formula's result does
not.  Needs a B200."""
import pytest
import torch

from paper_2608_15531_b200 import binding as fq

import mx_reference as R

pytestmark = pytest.mark.gpu
BF16, FP16, _ = R.TYPES


def _about(rng, shape, exponent):
    """Numbers of either sign near 2^exponent."""
    sign = 1 - 2 * torch.randint(0, 2, shape, generator=rng).double()
    return sign * (1 + torch.rand(shape, generator=rng).double()) * 2.0 ** exponent


# The block's normalised values are near 2^-10 (64 columns) to 2^-4 (4096), apart from one column that carries the row's mean square.
@pytest.mark.parametrize("D", [64, 1000, 4096, 16384])
@pytest.mark.parametrize("gate_exp,weight_exp,alpha,one_gate", [(64, 64, 1.0, False), (64, 64, 1.0, True), (120, 8, 0.5, False), (-80, -80, 2.0 ** 100, False),
                                                                (-80, -80, 2.0 ** 100, True), (-130, -20, 2.0 ** 90, False), (100, -90, 1.0, False)])
def test_norm_block_gate_times_weight_beyond_binary32(D, gate_exp, weight_exp, alpha, one_gate):
    rng = torch.Generator().manual_seed(D + gate_exp)
    rows = 5
    x = torch.zeros(rows, D, dtype=BF16)
    x[1] = _about(rng, (D,), -70).to(BF16)
    block = (_about(rng, (rows, D), -8)).to(BF16)
    block[:, 0] = 64.0
    weight = _about(rng, (D,), weight_exp).to(BF16)
    gate = _about(rng, (1 if one_gate else rows, D), gate_exp).to(BF16)
    gate[:, 0] = 2.0 ** -100                               # the column that is not small
    gate[0, 5], gate[0, 6] = 0.0, -0.0
    weight[7] = 0.0
    if not one_gate:
        gate[3, 8], gate[4, 9] = float("inf"), float("nan")
        gate[3, 7] = 2.0                                   # (weight 0: an infinite gate there would be a NaN as well)
    r, h = R.norm_block(R.f64(x), 1e-6, R.f64(block), R.f64(weight), R.f64(gate), alpha)
    r, h = R.round_to(r, BF16), R.round_to(h, BF16)
    assert bool(r[:3].isfinite().all()) and bool((r[:3, 10:] != 0).all())
    Rd, Hd = torch.empty(rows, D, dtype=BF16, device="cuda"), torch.empty(rows, D, dtype=BF16, device="cuda")
    fq.fq_norm_block(x.cuda(), 1e-6, block=block.cuda(), block_weight=weight.cuda(), gate=gate.cuda(), residual_scale=alpha, R=Rd, H=Hd)
    assert R.same(Rd, r)
    assert R.same(Hd, h)


@pytest.mark.parametrize("D", [96, 2048])
def test_norm_block_gate_times_weight_at_the_ends_of_fp16(D):
    """Two FP16 numbers always have their product in binary32: from the smallest subnormal numbers to the largest."""
    rng = torch.Generator().manual_seed(D)
    block, weight, gate = (torch.randn(s, generator=rng).to(FP16) for s in ((3, D), (D,), (3, D)))
    weight[::2], gate[1], gate[2] = 65504.0, 65504.0, 2.0 ** -24
    weight[1::4] = 2.0 ** -24
    for alpha in (2.0 ** -30, 2.0 ** 30):
        r, h = R.norm_block(torch.zeros(3, D).double().numpy(), 1e-6, R.f64(block), R.f64(weight), R.f64(gate), alpha)
        Rd, Hd = torch.empty(3, D, dtype=FP16, device="cuda"), torch.empty(3, D, dtype=FP16, device="cuda")
        fq.fq_norm_block(torch.zeros(3, D, dtype=FP16, device="cuda"), 1e-6, block=block.cuda(), block_weight=weight.cuda(), gate=gate.cuda(), residual_scale=alpha,
                         R=Rd, H=Hd)
        assert R.same(Rd, R.round_to(r, FP16)) and R.same(Hd, R.round_to(h, FP16))
