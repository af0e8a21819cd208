"""Microscaled FP4: the kernels that only large or particular calls are routed to.  Rows taken four to a warp, CTAs that go through several tiles, splits of
K on every width of tile, norms whose CTAs go through several rows.  Needs a B200; sizes follow from its number of SMs."""
import numpy as np
import pytest
import torch

from paper_2608_15531_b200 import binding as fq

import mx_reference as R

pytestmark = pytest.mark.gpu
BF16, FP16, FP32 = R.TYPES
FILL = 0xEE


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def buffers(L):
    return [torch.full((n,), FILL, dtype=torch.uint8, device="cuda") for n in fq.fq_mx_sizes(L)]


def scale_tensor(ts):
    return None if ts is None else torch.full((1,), ts, dtype=torch.float32, device="cuda")


def place(rows, blocks, total):
    """Where the scale of each row and block is stored."""
    atoms = -(-total // 4)
    r, b = torch.as_tensor(rows, device="cuda").view(-1, 1), torch.as_tensor(blocks, device="cuda").view(1, -1)
    return (r // 128 * atoms + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4


def stored_scales(byte, fill):
    """Scale bytes (rows x blocks) in the stored order; absent blocks 0, absent rows `fill`."""
    rows, nb = byte.shape
    out = torch.full((-(-rows // 128) * -(-nb // 4) * 512,), fill, dtype=torch.uint8, device="cuda")
    out[place(torch.arange(rows), torch.arange(-(-nb // 4) * 4), nb)] = torch.nn.functional.pad(byte, (0, -nb % 4))
    return out


def check_rows(which, x, L, codes, scales, ts):
    """Rows `which` against the 64-bit reference on their values x."""
    nb = L.K // R.BLOCK[L.format]
    code, byte = R.quantize(R.f64(x), L.format, 1.0 if ts is None else ts)
    got = codes.view(L.rows, -1)[which].cpu().numpy()
    assert np.array_equal(got, code[:, 0::2] | code[:, 1::2] << 4)
    got = scales[place(which, torch.arange(-(-nb // 4) * 4), nb)].cpu().numpy()
    assert np.array_equal(got, np.pad(byte, ((0, 0), (0, -nb % 4))))
    return code, byte


def values(rows, K, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, K, generator=g, device="cuda") * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g, device="cuda").float())
    ties = torch.tensor([0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5.0, 6.0], device="cuda").repeat(K // 8)
    x[3], x[-1], x[-2], x[rows // 2] = ties, -ties, 0.0, ties * 4
    x[rows // 3, 5], x[rows // 5, K - 1] = float("nan"), float("inf")
    return x.to(dtype)


def sample(rows):
    """The first and the last rows, those around the last multiple of 128, and some between."""
    rng = np.random.default_rng(rows)
    last = rows // 128 * 128
    pick = [0, 1, 31, 32, 96, 127, 128, rows // 2, rows // 3, rows // 5, rows - 1, rows - 2, 3] + list(range(max(last - 40, 0), rows, 7)) + list(rng.integers(0, rows, 40))
    return torch.tensor(sorted(set(int(r) for r in pick)))


# ---------------------------------------------------------------------- many rows: four to a warp, or one in CTAs of eight warps

# K, rows beyond the last whole 128, ld - K, offset of the first value
MANY = [(32, 1, 0, 0), (96, 31, 0, 0), (160, 33, 16, 8), (480, 97, 3, 1), (544, 127, 8, 8), (1056, 96, 0, 0), (2976, 65, 1, 3), (4096, 0, 0, 0), (20000, 33, 0, 0)]


@pytest.mark.parametrize("dtype", R.TYPES)
@pytest.mark.parametrize("fmt,ts", [(0, None), (1, 0.0037)])
@pytest.mark.parametrize("K,tail,pad,at", MANY)
def test_quantize_and_read_back_many_rows(K, tail, pad, at, fmt, ts, dtype):
    """More than 256 tasks of 512 values to an SM: a warp takes four rows that are 32 apart.  Every byte is that of calls on pieces of 128 to some hundred
    rows, each row its own warp's, and rows at either end and between are compared with the reference."""
    chunks = -(-K // 512)
    rows = (256 * sms() // chunks // 128 + 1) * 128 + tail
    assert rows * chunks > 256 * sms()
    L = fq.fq_mx_get_layout(rows, K, fmt)
    x = values(rows, K, dtype, K + tail)
    flat = torch.zeros(rows * (K + pad) + at, dtype=dtype, device="cuda")
    view = torch.as_strided(flat, (rows, K), (K + pad, 1), at)
    view.copy_(x)
    codes, scales = buffers(L)
    fq.fq_mx_quantize(L, view, codes, scales, tensor_scale=scale_tensor(ts))
    which = sample(rows)
    code, byte = check_rows(which, x[which], L, codes, scales, ts)
    # all the rest: the same calls on pieces
    step = max(128, 200 * sms() // chunks // 128 * 128)
    atoms = -(-(K // R.BLOCK[fmt]) // 4)
    y = torch.full_like(flat, 9.0)
    fq.fq_mx_dequantize(L, codes, scales, torch.as_strided(y, (rows, K), (K + pad, 1), at), tensor_scale=scale_tensor(ts))
    back = torch.as_strided(y, (rows, K), (K + pad, 1), at)
    assert R.same(back[which], R.round_to(R.values(code, byte, fmt, 1.0 if ts is None else ts), dtype))
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        P = fq.fq_mx_get_layout(n, K, fmt)
        assert n * chunks <= 256 * sms()
        c, s = buffers(P)
        fq.fq_mx_quantize(P, x[r0:r0 + n], c, s, tensor_scale=scale_tensor(ts))
        assert torch.equal(codes[r0 * K // 2:(r0 + n) * K // 2], c) and torch.equal(scales[r0 // 128 * atoms * 512:][:s.numel()], s)
        out = torch.empty(n, K, dtype=dtype, device="cuda")
        fq.fq_mx_dequantize(P, c, s, out, tensor_scale=scale_tensor(ts))
        assert torch.equal(back[r0:r0 + n].nan_to_num(1e4), out.nan_to_num(1e4))
    # bytes of absent rows, and the values between the rows
    absent = torch.arange(rows, -(-rows // 128) * 128)
    if absent.numel():
        assert bool((scales[place(absent, torch.arange(atoms * 4), atoms * 4)] == FILL).all())
    rest = torch.ones_like(y, dtype=torch.bool)
    torch.as_strided(rest, (rows, K), (K + pad, 1), at).fill_(False)
    assert bool((y[rest] == 9.0).all())


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("fmt,ts", [(0, None), (1, 0.011)])
@pytest.mark.parametrize("rows,K,pad,at", [(2500, 992, 0, 0), (1237, 2976, 8, 8), (40001, 160, 5, 3), (500, 14336, 0, 0)])
def test_quantize_swiglu_many_rows(rows, K, pad, at, fmt, ts, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows)
    gu = (torch.randn(rows, 2 * K, generator=g, device="cuda") * 2).to(dtype)
    gu[7, :K], gu[8, 3] = torch.linspace(-120, 120, K, device="cuda").to(dtype), float("nan")
    L = fq.fq_mx_get_layout(rows, K, fmt)
    d = torch.as_strided(torch.zeros(rows * (2 * K + pad) + at, dtype=dtype, device="cuda"), (rows, 2 * K), (2 * K + pad, 1), at)
    d.copy_(gu)
    codes, scales = buffers(L)
    fq.fq_mx_quantize_swiglu(L, d[:, :K], d[:, K:], codes, scales, tensor_scale=scale_tensor(ts))
    which = torch.cat([sample(rows), torch.tensor([7, 8])])
    some = gu[which]
    check_rows(which, R.round_to(R.swiglu(R.f64(some[:, :K]), R.f64(some[:, K:])), dtype), L, codes, scales, ts)
    # all rows: the product taken in 64 bits on the device, quantised by the call of its own
    gd, ud = gu[:, :K].double(), gu[:, K:].double()
    h = (gd / (1 + torch.exp(-gd)) * ud).float().to(dtype)
    c, s = buffers(L)
    fq.fq_mx_quantize(L, h, c, s, tensor_scale=scale_tensor(ts))
    assert torch.equal(codes, c) and torch.equal(scales, s)


@pytest.mark.parametrize("fmt", [0, 1])
def test_gated_products_of_rows_beyond_32_bits(fmt):
    """Gate and up in rows 2^31 values apart, the third beyond 2^32."""
    rows, K, ld = 3, 96, 1 << 31
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    gu = torch.randn(rows, 2 * K, generator=torch.Generator().manual_seed(4)).to(BF16)
    d = torch.as_strided(torch.empty(2 * ld + 2 * K, dtype=BF16, device="cuda"), (rows, 2 * K), (ld, 1))
    d.copy_(gu)
    L = fq.fq_mx_get_layout(rows, K, fmt)
    codes, scales = buffers(L)
    fq.fq_mx_quantize_swiglu(L, d[:, :K], d[:, K:], codes, scales)
    check_rows(torch.arange(rows), R.round_to(R.swiglu(R.f64(gu[:, :K]), R.f64(gu[:, K:])), BF16), L, codes, scales, None)


# -------------------------------------------------------------------------------- norms: several rows to a CTA, one after the other

def norm_reference(x, eps, block, block_weight, gate, alpha, weight):
    x, block, weight, eps, alpha = x.double(), block.double(), weight.double(), float(np.float32(eps)), float(np.float32(alpha))
    y = block
    if block_weight is not None:
        y = y / torch.sqrt((y * y).mean(1, keepdim=True) + eps) * block_weight.double()
    if gate is not None:
        y = y * gate.double()
    r = x + alpha * y
    return r, r / torch.sqrt((r * r).mean(1, keepdim=True) + eps) * weight


# (more than three rows for each of the CTAs that fit: 8 to an SM of four rows each up to 512 columns, 8 up to 2048, 4 up to 4096, 2 beyond)
LOOPS = [(96, 96), (256, 96), (520, 26), (1024, 26), (2976, 13), (4096, 13), (5120, 7), (8192, 7), (12288, 7), (16384, 7)]


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("post,gate", [(True, "full"), (False, "full"), (True, "row"), (True, None)])
@pytest.mark.parametrize("D,per_sm", LOOPS)
def test_norm_block_rows_one_after_the_other(D, per_sm, post, gate, dtype):
    rows, alpha = per_sm * sms() + 3, 0.75
    g = torch.Generator(device="cuda").manual_seed(D)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    scale = torch.exp2(torch.randint(-6, 6, (rows, 1), generator=g, device="cuda").float())       # (a neighbour's sum would be far off)
    x, block = (rand(rows, D) * scale).to(dtype), (rand(rows, D) * scale).to(dtype)
    weight, block_weight = (1 + 0.1 * rand(D)).to(dtype), (1 + 0.1 * rand(D)).to(dtype) if post else None
    gate = None if gate is None else rand(1 if gate == "row" else rows, D).to(dtype)
    r, h = (t.float().to(dtype) for t in norm_reference(x, 1e-5, block, block_weight, gate, alpha, weight))
    same = lambda a, b: torch.equal(a, b)  # noqa: E731
    for pad, at in ((0, 0), (1, 3)):                       # rows on 16-byte boundaries, which are fetched ahead, and on others
        def put(t):
            v = torch.as_strided(torch.zeros(t.shape[0] * (D + pad) + at, dtype=dtype, device="cuda"), t.shape, (D + pad, 1), at)
            return v.copy_(t)
        xd, bd, gd = put(x), put(block), None if gate is None else put(gate)
        kw = dict(block_weight=block_weight, gate=gd, residual_scale=alpha, weight=weight)
        Rd, Hd = put(x), put(x)
        fq.fq_norm_block(xd, 1e-5, block=bd, R=Rd, H=Hd, **kw)
        assert same(Rd, r) and same(Hd, h)
        fq.fq_norm_block(xd, 1e-5, block=bd, R=(alone := put(x)), **kw)                   # (one sum to a row, or none)
        assert same(alone, r)
        for fmt, ts in ((0, None), (1, 0.01)) if D % 32 == 0 else ():
            L = fq.fq_mx_get_layout(rows, D, fmt)
            (codes, scales), (c, s) = buffers(L), buffers(L)
            fq.fq_norm_block(xd, 1e-5, block=bd, layout=L, codes=codes, scales=scales, tensor_scale=scale_tensor(ts), **kw)
            fq.fq_mx_quantize(L, h, c, s, tensor_scale=scale_tensor(ts))
            assert same(codes, c) and same(scales, s)
            which = sample(rows)
            check_rows(which, h[which], L, codes, scales, ts)
        fq.fq_norm_block(xd, 1e-5, block=bd, R=xd, H=bd, **kw)                            # in place
        assert same(xd, r) and same(bd, h)


# ---------------------------------------------------------------------------------------------------------- the product

GRID = torch.tensor(R.VALUES)


def operand(rng, rows, K, fmt):
    """Random codes under a few scales near 1, stored and as float64; absent rows have NaN scales."""
    g = torch.Generator(device="cuda").manual_seed(rng)
    code = torch.randint(0, 16, (rows, K), generator=g, device="cuda", dtype=torch.uint8)
    choice = torch.tensor([126, 127, 128] if fmt == 0 else [0x30, 0x38, 0x40], dtype=torch.uint8, device="cuda")
    byte = choice[torch.randint(0, 3, (rows, K // R.BLOCK[fmt]), generator=g, device="cuda")]
    d = torch.tensor([0.5, 1.0, 2.0], dtype=torch.float64, device="cuda")[(byte - choice[0]).int() // (1 if fmt == 0 else 8)]
    v = GRID.cuda()[code.int()] * d.repeat_interleave(R.BLOCK[fmt], 1)
    return code[:, 0::2] | code[:, 1::2] << 4, stored_scales(byte, 0xFF), v


def test_the_operands_are_what_they_are_said_to_be():
    for fmt in (0, 1):
        codes, scales, v = operand(1, 131, 96, fmt)
        L = fq.fq_mx_get_layout(131, 96, fmt)
        y = torch.empty(131, 96, dtype=FP32, device="cuda")
        fq.fq_mx_dequantize(L, codes.view(-1), scales, y)
        assert torch.equal(y.double(), v)


def check_product(M, N, K, fmt, strides):
    x, w = operand(M + K, M, K, fmt), operand(N + 1, N, K, fmt)
    LX, LW = fq.fq_mx_get_layout(M, K, fmt), fq.fq_mx_get_layout(N, K, fmt)
    # products are multiples of 2^-4, and any sum of them is below 2^20: FP32 holds each, in whatever order they are added
    assert float((x[2].abs() @ w[2].abs().t()).max()) < 2.0 ** 20
    want = x[2] @ w[2].t()
    ws = torch.zeros(fq.FQ_MX_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    for dtype in R.TYPES:
        for pad, at in strides:
            flat = torch.full((M * (N + pad) + at,), 9.0, dtype=dtype, device="cuda")
            Y = torch.as_strided(flat, (M, N), (N + pad, 1), at)
            fq.fq_mx_gemm(LX, x[0].view(-1), x[1], LW, w[0].view(-1), w[1], Y, ws)
            fq.fq_check_status(ws)
            off = (Y != want.float().to(dtype)).nonzero()
            assert off.numel() == 0, (dtype, pad, at, off[:6].tolist(), off.shape[0])
            Y.fill_(9.0)
            assert bool((flat == 9.0).all())


# The comments say how many CTAs share a tile of how many tokens on 148 SMs; the results are the same on any number.
SPLITS = [(8, 8901, 4096),       # 2, of 16
          (1, 8900, 4128),       # 2, of 16: 17 steps
          (16, 4099, 4352),      # 4, of 16: 17 steps
          (3, 515, 8224),        # 8, of 16: 33 steps
          (24, 8449, 4096),      # 2, of 32
          (32, 4100, 4096),      # 4, of 32
          (17, 300, 8224),       # 8, of 32
          (64, 4227, 8192),      # 2, of 64
          (40, 1001, 8192),      # 4, of 64
          (33, 515, 16640),      # 8, of 64: 65 steps
          (65, 4700, 8192),      # 2, of 128
          (100, 515, 14336),     # 4, of 128
          (128, 260, 16416),     # 8, of 128
          (200, 300, 8192),      # 4, of 128, two tiles of tokens
          (300, 130, 16640)]     # 8, of 128, three


@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,N,K", SPLITS)
def test_gemm_split_along_k(M, N, K, fmt):
    """Rows of Y on boundaries that allow four features to a store, and on others; features that are no multiple of four."""
    check_product(M, N, K, fmt, [(0, 0), (-N % 4, 0), (-N % 4 + 4, 2), (1, 3)])


# Tiles of 128 features: with more than two to an SM a CTA goes on to a second one, with more than four to a third
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("M,per_sm,K", [(5, 2.2, 544), (1, 4.3, 96), (20, 4.3, 320), (40, 4.3, 96), (64, 2.2, 1056), (128, 2.2, 1056), (97, 4.3, 160), (65, 6.4, 64)])
def test_gemm_several_tiles_to_a_cta(M, per_sm, K, fmt):
    check_product(M, int(per_sm * sms()) * 128 + 65, K, fmt, [(0, 0), (7, 1)])
