"""Microscaled FP4 operators against the plain 64-bit implementation.  Codes, scales and what is rounded from them have to be equal:
both sides round the same exact numbers.  Needs a B200."""
import numpy as np
import pytest
import torch

from paper_2608_15531_b200 import binding as fq
from paper_2608_15531_b200 import synth

import harness as H
import mx_reference as R

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = R.TYPES


def buffers(L, fill=0xEE):
    return [torch.full((n,), fill, dtype=torch.uint8, device="cuda") for n in fq.fq_mx_sizes(L)]


def scale_tensor(ts):
    return None if ts is None else torch.full((1,), ts, dtype=torch.float32, device="cuda")


def check_stored(L, codes, scales, ref, fill=0xEE):
    """Codes and scales as the reference has them, in the stored order; the bytes of rows beyond the last as they were."""
    code, byte = ref
    want_c, want_s = R.pack(code, byte, fill)
    got_c, got_s = codes.cpu().numpy().reshape(L.rows, -1), scales.cpu().numpy()
    assert np.array_equal(got_s, want_s), np.nonzero(got_s != want_s)[0][:8]
    bad = np.nonzero(got_c != want_c)
    assert bad[0].size == 0, (bad[0][:8], bad[1][:8], got_c[bad][:8], want_c[bad][:8])


def hard_rows(rows, K, dtype, seed):
    """Normal rows of many magnitudes, and in the first ones what quantising can go wrong at."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, K, generator=g) * torch.exp2(torch.randint(-12, 8, (rows, 1), generator=g).float())
    tiny, huge = torch.finfo(dtype).tiny, torch.finfo(dtype).max
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.0])
    special = [ties.repeat(K // 16), ties.repeat(K // 16) * 8, torch.zeros(K), -torch.zeros(K), torch.full((K,), tiny), torch.full((K,), huge),
               torch.randn(K, generator=g) * tiny / 16, torch.linspace(-7.99, 7.99, K), torch.full((K,), -huge)]
    for i, v in enumerate(special):
        if 2 * i + 1 < rows:
            x[2 * i + 1] = v
    if rows > 20:
        x[20, 5], x[20, 40 % K], x[22, 0], x[24, 33 % K] = float("nan"), 3.0, float("inf"), float("-inf")
    return x.to(dtype)


SHAPES = [(1, 32), (1, 4096), (2, 64), (5, 2976), (31, 96), (33, 160), (97, 128), (128, 256), (129, 288), (300, 544)]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("fmt,ts", [(0, None), (1, None), (1, 0.0037), (1, 1.0)])
@pytest.mark.parametrize("rows,K", SHAPES)
def test_quantize(rows, K, fmt, ts, dtype):
    L = fq.fq_mx_get_layout(rows, K, fmt)
    x = hard_rows(rows, K, dtype, rows + K)
    codes, scales = buffers(L)
    fq.fq_mx_quantize(L, x.cuda(), codes, scales, tensor_scale=scale_tensor(ts))
    ref = R.quantize(R.f64(x), fmt, 1.0 if ts is None else ts)
    check_stored(L, codes, scales, ref)
    for out in R.TYPES:
        y = torch.full((rows, K), 7.0, dtype=out, device="cuda")
        fq.fq_mx_dequantize(L, codes, scales, y, tensor_scale=scale_tensor(ts))
        assert R.same(y, R.round_to(R.values(*ref, fmt, 1.0 if ts is None else ts), out))


@pytest.mark.parametrize("ts", [0.0, -1.0, float("nan"), float("inf"), 2.0 ** -60.5, 2.0 ** 60.5])
def test_a_tensor_scale_out_of_range_gives_nan(ts):
    L = fq.fq_mx_get_layout(3, 64, 1)
    codes, scales = buffers(L)
    y = torch.zeros(3, 64, dtype=FP32, device="cuda")
    fq.fq_mx_quantize(L, torch.ones(3, 64, dtype=BF16, device="cuda"), codes, scales, tensor_scale=scale_tensor(ts))
    check_stored(L, codes, scales, (np.zeros((3, 64), np.uint8), np.full((3, 4), 0x7F, np.uint8)))
    fq.fq_mx_dequantize(L, codes, scales, y, tensor_scale=scale_tensor(ts))
    assert bool(y.isnan().all())


@pytest.mark.parametrize("ts", [2.0 ** -60, 2.0 ** 60, 1.5 * 2.0 ** -41])
def test_tensor_scales_at_the_ends_of_their_range(ts):
    L = fq.fq_mx_get_layout(9, 96, 1)
    x = (torch.randn(9, 96, generator=torch.Generator().manual_seed(1)).double() * ts * 100).float()
    codes, scales = buffers(L)
    fq.fq_mx_quantize(L, x.cuda(), codes, scales, tensor_scale=scale_tensor(ts))
    check_stored(L, codes, scales, R.quantize(R.f64(x), 1, ts))


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("dtype", R.TYPES)
def test_quantize_rows_of_any_stride_on_any_boundary(fmt, dtype):
    rows, K = 37, 160
    L = fq.fq_mx_get_layout(rows, K, fmt)
    x = hard_rows(rows, K, dtype, 3)
    ref = R.quantize(R.f64(x), fmt)
    for ld, at in ((K + 8, 0), (K + 1, 0), (K, 1), (K + 3, 5), (2 * K, K)):
        wide = torch.full((rows * ld + at,), 9.0, dtype=dtype, device="cuda")
        view = torch.as_strided(wide, (rows, K), (ld, 1), at)
        view.copy_(x)
        codes, scales = buffers(L)
        fq.fq_mx_quantize(L, view, codes, scales)
        check_stored(L, codes, scales, ref)
        out = torch.full_like(wide, 9.0)
        fq.fq_mx_dequantize(L, codes, scales, torch.as_strided(out, (rows, K), (ld, 1), at))
        assert R.same(torch.as_strided(out, (rows, K), (ld, 1), at), R.round_to(R.values(*ref, fmt), dtype))
        rest = torch.ones_like(out, dtype=torch.bool)
        torch.as_strided(rest, (rows, K), (ld, 1), at).fill_(False)
        assert bool((out[rest] == 9.0).all())


def test_dequantize_every_code_under_every_scale():
    for fmt in (0, 1):
        L = fq.fq_mx_get_layout(256, 32 * 8, fmt)
        rng = np.random.default_rng(fmt)
        code = rng.integers(0, 16, (256, 256)).astype(np.uint8)
        byte = np.broadcast_to(np.arange(256, dtype=np.uint8)[:, None], (256, 256 // R.BLOCK[fmt]))
        c, s = R.pack(code, byte)
        for dtype in R.TYPES:
            y = torch.zeros(256, 256, dtype=dtype, device="cuda")
            fq.fq_mx_dequantize(L, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), y)
            assert R.same(y, R.round_to(R.values(code, byte, fmt), dtype))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("fmt,ts", [(0, None), (1, 0.011)])
@pytest.mark.parametrize("rows,K", [(1, 32), (1, 14336), (8, 992), (130, 160), (300, 1024)])
def test_quantize_swiglu(rows, K, fmt, ts, dtype):
    g = torch.Generator().manual_seed(rows * K)
    gu = (torch.randn(rows, 2 * K, generator=g) * 2).to(dtype)
    if rows > 7:
        gu[1, :K] = torch.linspace(-120, 120, K).to(dtype)
        gu[2, :K], gu[3, K:], gu[4] = 0.0, 0.0, -0.0
        gu[5] *= 2.0 ** -10
        gu[6, 3], gu[6, 40 % K], gu[7, K + 1] = float("nan"), float("-inf"), float("inf")
    L = fq.fq_mx_get_layout(rows, K, fmt)
    h = R.round_to(R.swiglu(R.f64(gu[:, :K]), R.f64(gu[:, K:])), dtype)
    ref = R.quantize(R.f64(h), fmt, 1.0 if ts is None else ts)
    for at, ld in ((0, 2 * K), (3, 2 * K + 5)):
        wide = torch.zeros(rows * ld + at, dtype=dtype, device="cuda")
        d = torch.as_strided(wide, (rows, 2 * K), (ld, 1), at)
        d.copy_(gu)
        codes, scales = buffers(L)
        fq.fq_mx_quantize_swiglu(L, d[:, :K], d[:, K:], codes, scales, tensor_scale=scale_tensor(ts))
        check_stored(L, codes, scales, ref)


NORM_D = [1, 7, 32, 96, 512, 520, 1024, 2048, 2976, 4096, 4100, 8192, 16384]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("post,gate", [(None, None), (False, None), (True, None), (True, "row"), (False, "full"), (True, "full")])
@pytest.mark.parametrize("D", NORM_D)
def test_norm_block(D, post, gate, dtype):
    rows = 5 if D < 4096 else 3
    g = torch.Generator().manual_seed(D + 7)
    x = (torch.randn(rows, D, generator=g) * 3).to(dtype)
    weight = (1 + 0.1 * torch.randn(D, generator=g)).to(dtype)
    kw, ref = {}, {}
    if post is not None:
        kw["block"] = torch.randn(rows, D, generator=g).to(dtype)
        if post:
            kw["block_weight"] = (1 + 0.1 * torch.randn(D, generator=g)).to(dtype)
        if gate:
            kw["gate"] = torch.randn(1 if gate == "row" else rows, D, generator=g).to(dtype)
        ref = {k: R.f64(v) for k, v in kw.items()}
    alpha = 0.37 if post else 1.0
    r, h = R.norm_block(R.f64(x), 1e-5, ref.get("block"), ref.get("block_weight"), ref.get("gate"), alpha, R.f64(weight))
    r, h = R.round_to(r, dtype), R.round_to(h, dtype)
    kw = {k: v.cuda() for k, v in kw.items()}
    xd, w = x.cuda(), weight.cuda()
    Rd, Hd = torch.empty_like(xd), torch.empty_like(xd)
    fq.fq_norm_block(xd, 1e-5, R=Rd, H=Hd, weight=w, residual_scale=alpha, **kw)
    assert R.same(Rd, r) and R.same(Hd, h) and R.same(xd, x)
    for fmt, ts in ((0, None), (1, 0.002)) if D % 32 == 0 else ():
        L = fq.fq_mx_get_layout(rows, D, fmt)
        codes, scales = buffers(L)
        fq.fq_norm_block(xd, 1e-5, weight=w, residual_scale=alpha, layout=L, codes=codes, scales=scales, tensor_scale=scale_tensor(ts), **kw)
        check_stored(L, codes, scales, R.quantize(R.f64(h), fmt, 1.0 if ts is None else ts))
    # the sum in place, without a weight; the next norm over the block's own output
    _, h1 = R.norm_block(R.f64(x), 1e-5, ref.get("block"), ref.get("block_weight"), ref.get("gate"), alpha)
    over = kw["block"] if "block" in kw else Hd
    fq.fq_norm_block(xd, 1e-5, R=xd, H=over, residual_scale=alpha, **kw)
    assert R.same(xd, r) and R.same(over, R.round_to(h1, dtype))


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("rows,D", [(1, 4096), (129, 256), (200, 160), (260, 1056), (150, 2976), (151, 4096), (149, 8192), (160, 32)])
def test_norm_block_many_rows_and_strides(rows, D, dtype):
    g = torch.Generator().manual_seed(rows)
    x, o = torch.randn(rows, D, generator=g).to(dtype), torch.randn(rows, D, generator=g).to(dtype)
    gate = torch.randn(1, D, generator=g).to(dtype)
    r, h = R.norm_block(R.f64(x), 1e-6, R.f64(o), None, R.f64(gate), 1.0)
    r, h = R.round_to(r, dtype), R.round_to(h, dtype)
    L = fq.fq_mx_get_layout(rows, D, 1)
    for ld, at in ((D, 0), (D + 8, 8), (D + 1, 3)):
        def place(t):
            v = torch.as_strided(torch.zeros(rows * ld + at, dtype=dtype, device="cuda"), (rows, D), (ld, 1), at)
            return v.copy_(t)
        xd, od, Rd, Hd = place(x), place(o), place(x), place(x)
        codes, scales = buffers(L)
        fq.fq_norm_block(xd, 1e-6, block=od, gate=gate.cuda().expand(rows, D) if at else gate.cuda(), R=Rd, H=Hd, layout=L, codes=codes, scales=scales)
        assert R.same(Rd, r) and R.same(Hd, h)
        check_stored(L, codes, scales, R.quantize(R.f64(h), 1))


def test_norm_block_nan_infinity_and_zero_rows():
    x = torch.randn(6, 64, generator=torch.Generator().manual_seed(5)).to(BF16)
    x[1], x[2, 3], x[3, 4], x[4] = 0.0, float("nan"), float("inf"), -0.0
    r, h = R.norm_block(R.f64(x), 1e-5)
    L = fq.fq_mx_get_layout(6, 64, 0)
    codes, scales = buffers(L)
    Hd = torch.empty_like(x, device="cuda")
    fq.fq_norm_block(x.cuda(), 1e-5, H=Hd, layout=L, codes=codes, scales=scales)
    assert R.same(Hd, R.round_to(h, BF16))
    check_stored(L, codes, scales, R.quantize(R.f64(R.round_to(h, BF16)), 0))


# ------------------------------------------------------------------------------------------------------- the product

def operand(rng, rows, K, fmt, exact):
    """Random codes under random scales (`exact`: few scales near 1, so that every partial sum is a number of FP32), stored and as float64."""
    code = rng.integers(0, 16, (rows, K)).astype(np.uint8)
    nb = K // R.BLOCK[fmt]
    if fmt == 0:
        byte = rng.integers(126, 129, (rows, nb)) if exact else rng.integers(118, 134, (rows, nb))
    else:
        byte = rng.choice([0x30, 0x38, 0x40], (rows, nb)) if exact else rng.integers(8, 0x70, (rows, nb))
    byte = byte.astype(np.uint8)
    c, s = R.pack(code, byte, 0xFF)                        # NaN scales in the rows that are not there
    return torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), R.values(code, byte, fmt)


def product(LX, x, LW, w, dtype, ws, **kw):
    Y = torch.full((LX.rows, LW.rows), 7.0, dtype=dtype, device="cuda")
    fq.fq_mx_gemm(LX, x[0], x[1], LW, w[0], w[1], Y, ws, **kw)
    fq.fq_check_status(ws)
    return Y


@pytest.fixture
def ws():
    return torch.zeros(fq.FQ_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(1, 1, 32), (1, 128, 64), (1, 129, 96), (2, 100, 160), (16, 256, 256), (17, 130, 288), (32, 127, 512), (33, 384, 544),
                                   (64, 200, 1024), (65, 129, 992), (100, 64, 2048), (128, 300, 320), (129, 257, 736), (300, 333, 1056), (520, 700, 416),
                                   (1, 4096, 1024), (3, 513, 2048), (777, 130, 96), (1, 20000, 128), (1000, 2000, 64), (1011, 9400, 160), (1040, 9472, 544), (1160, 9300, 96), (129, 19200, 96), (150, 19300, 320), (260, 9500, 288), (384, 9500, 64)])
def test_gemm_exact_sums(M, N, K, fmt, ws):
    """Products are multiples of 2^-4 of magnitude up to 144, and K of them below 2^18: each sum has at most 24 bits,
    in whatever order, so that the result is the exact one rounded once."""
    rng = np.random.default_rng(M + N + K)
    LX, LW = fq.fq_mx_get_layout(M, K, fmt), fq.fq_mx_get_layout(N, K, fmt)
    x, w = operand(rng, M, K, fmt, True), operand(rng, N, K, fmt, True)
    want = x[2] @ w[2].T
    for dtype in R.TYPES:
        Y = product(LX, x, LW, w, dtype, ws)
        got = R.f64(Y)
        bad = np.nonzero(got != R.f64(R.round_to(want, dtype)))
        assert bad[0].size == 0, (bad[0][:8], bad[1][:8], got[bad][:8], want[bad][:8], bad[0].size)


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (16, 4096, 14336), (77, 1133, 2976), (260, 1000, 4096), (1100, 9500, 1056)])
def test_gemm_general_scales(M, N, K, fmt, ws):
    """Sums that FP32 cannot hold.  Each of the K additions may be off by 2^-23 of the magnitudes summed (a truncated addition), the
    tensor scales' product and its multiplication by 2^-23 of the result, and the final rounding by half a step."""
    rng = np.random.default_rng(K)
    LX, LW = fq.fq_mx_get_layout(M, K, fmt), fq.fq_mx_get_layout(N, K, fmt)
    x, w = operand(rng, M, K, fmt, False), operand(rng, N, K, fmt, False)
    kw = {} if fmt == 0 else dict(x_tensor_scale=scale_tensor(0.3), w_tensor_scale=scale_tensor(0.0007))
    alpha = 1.0 if fmt == 0 else float(np.float32(0.3)) * float(np.float32(0.0007))
    want, mag = alpha * (x[2] @ w[2].T), alpha * (np.abs(x[2]) @ np.abs(w[2]).T)
    for dtype in (BF16, FP32):
        got = R.f64(product(LX, x, LW, w, dtype, ws, **kw))
        err = np.abs(got - want)
        assert np.all(err <= K * 2.0 ** -23 * mag + (torch.finfo(dtype).eps / 2 + 2.0 ** -22) * np.abs(want) * 1.01)
        # and all together: errors of either sign add up as their squares do
        assert np.linalg.norm(err) <= (torch.finfo(dtype).eps / 2 + 2.0 ** -18) * np.linalg.norm(want)


@pytest.mark.parametrize("fmt", [0, 1])
def test_gemm_nan_scales_reach_their_rows_only(fmt, ws):
    rng = np.random.default_rng(1)
    M, N, K = 20, 140, 256
    LX, LW = fq.fq_mx_get_layout(M, K, fmt), fq.fq_mx_get_layout(N, K, fmt)
    x, w = operand(rng, M, K, fmt, True), operand(rng, N, K, fmt, True)
    want = x[2] @ w[2].T
    nan = 0xFF if fmt == 0 else 0x7F
    x[1][3 * 16 + 1] = nan                                 # row 3, block 1
    w[1][(LW.K // R.BLOCK[fmt] + 3) // 4 * 512 + 5 * 16] = nan          # row 133, block 0
    want[3], want[:, 133] = np.nan, np.nan
    assert R.same(product(LX, x, LW, w, FP32, ws), torch.from_numpy(want))


@pytest.mark.parametrize("M,N", [(3, 140), (1030, 9472)])
@pytest.mark.parametrize("fmt,xb,wb", [(0, [0, 1, 2], [252, 253, 254]), (0, [254, 253], [0, 1]), (1, list(range(8)), list(range(8))), (1, [0x7e, 1], [0x7e, 0x38])])
def test_gemm_scales_at_the_ends_of_their_range(M, N, fmt, xb, wb, ws):
    """Powers of two at both ends, one of which FP32 holds only as a subnormal number; subnormal E4M3 numbers, zeros, and the largest.  One
    scale to a row, so that a sum is 64 products of codes, exact, times two scales."""
    rng = np.random.default_rng(4)
    K = 64
    nb = K // R.BLOCK[fmt]
    sides = []
    for rows, choice in ((M, xb), (N, wb)):
        code = rng.integers(0, 16, (rows, K)).astype(np.uint8)
        byte = np.broadcast_to(rng.choice(choice, (rows, 1)), (rows, nb)).astype(np.uint8)
        c, s = R.pack(code, byte, 0xFF)
        sides.append((torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda(), R.values(code, byte, fmt)))
    Y = product(fq.fq_mx_get_layout(M, K, fmt), sides[0], fq.fq_mx_get_layout(N, K, fmt), sides[1], FP32, ws)
    assert R.same(Y, torch.from_numpy((sides[0][2] @ sides[1][2].T).astype(np.float32)))


def test_gemm_rows_of_y_with_a_stride(ws):
    rng = np.random.default_rng(2)
    for M, N, K in ((5, 130, 128), (140, 260, 512), (1030, 9401, 64)):
        LX, LW = fq.fq_mx_get_layout(M, K, 0), fq.fq_mx_get_layout(N, K, 0)
        x, w = operand(rng, M, K, 0, True), operand(rng, N, K, 0, True)
        want = R.round_to(x[2] @ w[2].T, BF16)
        for ld, at in ((N + 1, 3), (2 * N, N), (N + 8, 0)):
            wide = torch.full((M * ld + at,), 9.0, dtype=BF16, device="cuda")
            Y = torch.as_strided(wide, (M, N), (ld, 1), at)
            fq.fq_mx_gemm(LX, x[0], x[1], LW, w[0], w[1], Y, ws)
            assert R.same(Y, want)
            Y.fill_(9.0)
            assert bool((wide == 9.0).all())


@pytest.mark.parametrize("M,N,K", [(8, 512, 8192), (1030, 9600, 288)])
def test_gemm_is_reproducible_and_shares_its_workspace(M, N, K, ws):
    rng = np.random.default_rng(3)
    LX, LW = fq.fq_mx_get_layout(M, K, 1), fq.fq_mx_get_layout(N, K, 1)
    x, w = operand(rng, M, K, 1, False), operand(rng, N, K, 1, False)
    first = product(LX, x, LW, w, FP32, ws)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for s in streams:
            Y = torch.empty_like(first)
            fq.fq_mx_gemm(LX, x[0], x[1], LW, w[0], w[1], Y, ws, stream=s)
            outs.append(Y)
    torch.cuda.synchronize()
    fq.fq_check_status(ws)
    assert all(torch.equal(Y, first) for Y in outs)


def test_gemm_reads_what_the_call_before_it_wrote(ws):
    """Weights and activations quantised by the calls directly before, into buffers that the product before still reads."""
    M, N, K = 24, 1024, 2048
    LX, LW = fq.fq_mx_get_layout(M, K, 0), fq.fq_mx_get_layout(N, K, 0)
    g = torch.Generator(device="cuda").manual_seed(0)
    xs = [torch.randn(M, K, generator=g, device="cuda").to(BF16) for _ in range(6)]
    wts = [torch.randn(N, K, generator=g, device="cuda").to(BF16) for _ in range(6)]
    xb, wb = buffers(LX), buffers(LW)
    want, got = [], []
    for sync in (True, False):
        out = want if sync else got
        for x, w in zip(xs, wts):
            Y = torch.empty(M, N, dtype=FP32, device="cuda")
            fq.fq_mx_quantize(LX, x, *xb)
            fq.fq_mx_quantize(LW, w, *wb)
            if sync:
                torch.cuda.synchronize()
            fq.fq_mx_gemm(LX, *xb, LW, *wb, Y, ws)
            if sync:
                torch.cuda.synchronize()
            out.append(Y)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and not torch.equal(want[0], want[1])


@pytest.mark.parametrize("fmt", [0, 1])
def test_offsets_beyond_32_bits(fmt, ws):
    """Rows that lie 2^31 values apart: the third begins beyond 2^32 values, 8 GB from the first."""
    rows, K, ld = 3, 96, 1 << 31
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    L = fq.fq_mx_get_layout(rows, K, fmt)
    x = hard_rows(rows, K, BF16, 9)
    ref = R.quantize(R.f64(x), fmt)
    wide = torch.empty(2 * ld + K + 64, dtype=BF16, device="cuda")
    view = torch.as_strided(wide, (rows, K), (ld, 1))
    view.copy_(x)
    codes, scales = buffers(L)
    fq.fq_mx_quantize(L, view, codes, scales)
    check_stored(L, codes, scales, ref)
    view.zero_()
    fq.fq_mx_dequantize(L, codes, scales, view)
    assert R.same(view, R.round_to(R.values(*ref, fmt), BF16))
    fq.fq_mx_quantize_swiglu(L, view, torch.as_strided(wide, (rows, K), (ld, 1)), *buffers(L))
    r, h = R.norm_block(R.f64(view), 1e-5)
    fq.fq_norm_block(view, 1e-5, R=view, H=(out := torch.empty(rows, K, dtype=BF16, device="cuda")))
    assert R.same(view, R.round_to(r, BF16)) and R.same(out, R.round_to(h, BF16))
    rng = np.random.default_rng(0)
    X, W = operand(rng, rows, K, fmt, True), operand(rng, 96, K, fmt, True)
    fq.fq_mx_gemm(L, X[0], X[1], fq.fq_mx_get_layout(96, K, fmt), W[0], W[1], view, ws)
    assert R.same(view, R.round_to(X[2] @ W[2].T, BF16))


def test_gemm_tensor_scales_whose_product_is_small(ws):
    """Scales of 2^-60 and 2^-59: their product is a normal number of FP32, and so are the results."""
    rng = np.random.default_rng(8)
    LX, LW = fq.fq_mx_get_layout(4, 64, 1), fq.fq_mx_get_layout(140, 64, 1)
    x, w = operand(rng, 4, 64, 1, True), operand(rng, 140, 64, 1, True)
    a, b = 2.0 ** -60, 2.0 ** -59
    Y = product(LX, x, LW, w, FP32, ws, x_tensor_scale=scale_tensor(a), w_tensor_scale=scale_tensor(b))
    assert R.same(Y, torch.from_numpy((x[2] @ w[2].T) * (a * b)))


_CAPTURED_FIRST = """
import torch
from paper_2608_15531_b200 import binding as fq
x = torch.randn(300, 512, device="cuda").bfloat16()
L, W = fq.fq_mx_get_layout(300, 512, 0), fq.fq_mx_get_layout(300, 512, 0)
c, s = (torch.zeros(n, dtype=torch.uint8, device="cuda") for n in fq.fq_mx_sizes(L))
Y, H, ws = torch.empty(300, 300, device="cuda"), torch.empty_like(x), torch.zeros(fq.FQ_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
def run():
    fq.fq_norm_block(x, 1e-5, H=H, layout=L, codes=c, scales=s)
    fq.fq_mx_gemm(L, c, s, W, c, s, Y, ws)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run()
g.replay()
torch.cuda.synchronize()
first = Y.clone()
run()
fq.fq_check_status(ws)
assert torch.equal(first, Y) and bool(Y.any())
"""


def test_the_first_calls_of_a_process_are_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", _CAPTURED_FIRST], cwd=root, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-800:]


# --------------------------------------------------------------------------------------- a decoder's block, and captured

def mlp_reference(x, o, w, wgu, wd, fmt):
    """Residual sum and norm, gate_up, gated product, down, and the residual sum and norm behind it; each result rounded to BF16."""
    r, h = R.norm_block(R.f64(x), 1e-5, R.f64(o), None, None, 1.0, R.f64(w))
    h = R.round_to(h, BF16)
    q = lambda t: R.values(*R.quantize(R.f64(t), fmt), fmt)  # noqa: E731
    gu = R.round_to(q(h) @ q(wgu).T, BF16)
    F = gu.shape[1] // 2
    a = R.round_to(R.swiglu(R.f64(gu[:, :F]), R.f64(gu[:, F:])), BF16)
    return R.round_to(r, BF16), gu, a, q


def test_a_block_of_them_together_and_the_int4_path_behind(ws):
    """norm + quantise -> gate_up -> SwiGLU + quantise -> down -> residual sum and norm -> the fused INT4 call on its result.  Each
    step is checked on the bits that the step before it gave, by that step's own bound."""
    M, D, F, fmt = 6, 512, 768, 1
    g = torch.Generator().manual_seed(11)
    x, o, w = (torch.randn(*s, generator=g).to(BF16) for s in ((M, D), (M, D), (D,)))
    wgu, wd = (0.05 * torch.randn(2 * F, D, generator=g)).to(BF16), (0.05 * torch.randn(D, F, generator=g)).to(BF16)
    lay = {k: fq.fq_mx_get_layout(r, c, fmt) for k, (r, c) in dict(h=(M, D), a=(M, F), gu=(2 * F, D), d=(D, F)).items()}
    b = {k: buffers(v) for k, v in lay.items()}
    for k, t in (("gu", wgu), ("d", wd)):
        fq.fq_mx_quantize(lay[k], t.cuda(), *b[k])
    xd, od, wdv = x.cuda(), o.cuda(), w.cuda()
    GU, DN = torch.empty(M, 2 * F, dtype=BF16, device="cuda"), torch.empty(M, D, dtype=BF16, device="cuda")
    r1, r2, h2 = (torch.empty(M, D, dtype=BF16, device="cuda") for _ in range(3))
    P = H.pack_layer(synth.layer(synth.tensor_seed(3, 3), D, 512, density=0.01, layout="mixed"), 128)

    def block():
        fq.fq_norm_block(xd, 1e-5, block=od, weight=wdv, R=r1, layout=lay["h"], codes=b["h"][0], scales=b["h"][1])
        fq.fq_mx_gemm(lay["h"], *b["h"], lay["gu"], *b["gu"], GU, ws)
        fq.fq_mx_quantize_swiglu(lay["a"], GU[:, :F], GU[:, F:], *b["a"])
        fq.fq_mx_gemm(lay["a"], *b["a"], lay["d"], *b["d"], DN, ws)
        fq.fq_norm_block(r1, 1e-5, block=DN, weight=wdv, R=r2, H=h2)
        fq.fq_fused_w4a16_outlier_gemm(P.L, h2, M, P.d["wq"], P.d["scale"], P.d["zero"], P.d["indptr"], P.d["info"], P.d["packed"], Y4, P.ws)

    Y4 = torch.empty(M, 512, dtype=torch.int16, device="cuda")
    block()
    fq.fq_check_status(ws)
    r, gu, _, q = mlp_reference(x, o, w, wgu, wd, fmt)
    assert R.same(r1, r)
    # sums of at most 768 products: off by 768 * 2^-23 of the magnitudes, which are at most 100 times the result's scale, and half a step
    near = lambda t, ref: np.linalg.norm(R.f64(t) - ref) <= (2.0 ** -8 + 768 * 2.0 ** -23 * 100) * np.linalg.norm(ref)  # noqa: E731
    assert near(GU, R.f64(gu))
    a = R.round_to(R.swiglu(R.f64(GU[:, :F]), R.f64(GU[:, F:])), BF16)
    check_stored(lay["a"], *b["a"], R.quantize(R.f64(a), fmt))
    assert near(DN, q(a) @ q(wd).T)
    rr, hh = R.norm_block(R.f64(r1), 1e-5, R.f64(DN), None, None, 1.0, R.f64(w))
    assert R.same(r2, R.round_to(rr, BF16)) and R.same(h2, R.round_to(hh, BF16))
    bits = h2.cpu().view(torch.int16).numpy().view(np.uint16)
    assert np.array_equal(H.bf16_bits(Y4), H.run_fused(P, bits))

    # captured and replayed on new inputs, twice in a row
    eager = [t.clone() for t in (r2, h2, Y4)]
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        block()
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        block()
    for t in (r1, r2, h2, Y4, GU, DN):
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(eager, (r2, h2, Y4)))
    xd.copy_(-x)
    od.copy_(-o)
    graph.replay()
    graph.replay()
    assert torch.equal(r1, -r.cuda())
    xd.copy_(x)
    od.copy_(o)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(eager, (r2, h2, Y4)))


# ------------------------------------------------------------------------------------------------ what the binding refuses

def test_the_binding_refuses_what_does_not_fit(ws):
    L = fq.fq_mx_get_layout(4, 64, 0)
    x, (c, s) = torch.zeros(4, 64, dtype=BF16, device="cuda"), buffers(L)
    bad = [torch.zeros(4, 65, dtype=BF16, device="cuda")[:, :63], torch.zeros(3, 64, dtype=BF16, device="cuda"), x.cpu(), x.double(), x.to_sparse(),
           torch.zeros(64, 4, dtype=BF16, device="cuda").t(), torch.zeros(4, 128, dtype=BF16, device="cuda")[:, ::2], x.view(2, 2, 64), None]
    for t in bad:
        with pytest.raises((ValueError, RuntimeError)):
            fq.fq_mx_quantize(L, t, c, s)
        with pytest.raises((ValueError, RuntimeError)):
            fq.fq_mx_dequantize(L, c, s, t)
        with pytest.raises((ValueError, RuntimeError)):
            fq.fq_mx_quantize_swiglu(L, x, t, c, s)
    with pytest.raises(ValueError, match="bytes"):
        fq.fq_mx_quantize(L, x, c[:-1], s)
    with pytest.raises(ValueError, match="bytes"):
        fq.fq_mx_quantize(L, x, c, s[:-1])
    with pytest.raises(ValueError, match="type"):
        fq.fq_mx_quantize_swiglu(L, x, x.to(FP16), c, s)
    with pytest.raises(ValueError, match="float32"):
        fq.fq_mx_quantize(L, x, c, s, tensor_scale=torch.ones(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(fq.FqError):
        fq.fq_mx_quantize(L, x, c, s, tensor_scale=torch.ones(1, device="cuda"))
    with pytest.raises(fq.FqError) as e:
        fq.fq_mx_gemm(L, c, s, L, c, s, torch.empty(4, 4, dtype=BF16, device="cuda"), ws[:-16])
    assert e.value.code == fq.FQ_ERR_BUFFER_TOO_SMALL
    with pytest.raises(fq.FqError):
        fq.fq_norm_block(x, 1e-5, R=x, H=x)
    with pytest.raises(ValueError, match="layout"):
        fq.fq_norm_block(x, 1e-5, codes=c, scales=s)
    with pytest.raises(ValueError):
        fq.fq_norm_block(x, 1e-5, H=torch.empty_like(x), weight=torch.ones(63, dtype=BF16, device="cuda"))
    with pytest.raises(TypeError):
        fq.fq_mx_quantize(fq.fq_get_layout(128, 128, 128), x, c, s)
    torch.cuda.synchronize()
    assert bool((c == 0xEE).all()) and bool((s == 0xEE).all())
