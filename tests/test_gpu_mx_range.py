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


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows,D,pad", [(2, 32, 0), (700, 96, 0), (37, 160, 3), (1200, 4096, 0)])
def test_norm_block_on_column_slices_of_one_array(rows, D, pad, dtype):
    """Inputs, R and H lie beside each other in the rows of one array; what is between them stays as it is."""
    rng = torch.Generator().manual_seed(rows + D)
    wide = torch.randn(rows, 5 * D + pad, generator=rng).to(dtype)
    x, block, gate = (wide[:, i * D:(i + 1) * D] for i in (0, 2, 4))
    r, h = R.norm_block(R.f64(x), 1e-5, R.f64(block), None, R.f64(gate), 0.5)
    want = wide.clone()
    want[:, D:2 * D], want[:, 3 * D:4 * D] = R.round_to(r, dtype), R.round_to(h, dtype)
    d = wide.cuda()
    x, Rd, block, Hd, gate = (d[:, i * D:(i + 1) * D] for i in range(5))
    fq.fq_norm_block(x, 1e-5, block=block, gate=gate, residual_scale=0.5, R=Rd, H=Hd)
    assert R.same(d, want)
    with pytest.raises(fq.FqError, match="overlaps"):
        fq.fq_norm_block(x, 1e-5, block=block, R=Rd, H=d[:, 3 * D - 1:4 * D - 1])


def test_read_back_beside_another_matrix():
    """Two matrices of values in one array, read back in turn, each from codes that the call before made of the other."""
    rows, K = 300, 96
    L = fq.fq_mx_get_layout(rows, K, 0)
    wide = torch.randn(rows, 2 * K, generator=torch.Generator().manual_seed(2)).to(BF16)
    want = R.round_to(R.values(*R.quantize(R.f64(wide[:, :K]), 0), 0), BF16)
    d = wide.cuda()
    codes, scales = (torch.zeros(n, dtype=torch.uint8, device="cuda") for n in fq.fq_mx_sizes(L))
    fq.fq_mx_quantize(L, d[:, :K], codes, scales)
    fq.fq_mx_dequantize(L, codes, scales, d[:, K:])
    assert R.same(d[:, K:], want) and torch.equal(d[:, :K].cpu(), wide[:, :K])
