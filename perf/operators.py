"""What is timed of the microscaled FP4 operators: quantising rows of values (and reading them back), quantising the gated product of
a decoder's MLP, the norms and the residual sum around a block with the quantisation that follows, and the product of two
quantised matrices, from one token to a prefill.

Formats.  "mx": blocks of 32 values along K, a power of two as scale (E8M0 byte).  "nv": blocks of 16, an E4M3 scale, and
one FP32 scale for the tensor.  Codes are e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte, the lower nibble first.
Scales are stored in atoms of 128 rows by 4 blocks: byte (row % 32) * 16 + row % 128 // 32 * 4 + block % 4 of the atom, a row
tile's atoms one after the other.

Kinds of case:
  quantize  rows x K values to codes and scales, and back
  swiglu    silu(gate) * up to codes and scales, and back
  norm      residual sum, norm, and quantisation of its result (read back)
  gemm      (rows x K) times (N x K) transposed
"""
from __future__ import annotations

import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = {"mx": 32, "nv": 16}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MOST_VALUES = 28672 * 4096            # of the largest listed matrix to quantise
MOST_PRODUCTS = 4096 * 28672 * 4096   # of the largest listed product


def _case(name, kind, M, K, N=0, fmt="mx", type="bf16", post=False, gate="none"):
    return dict(name=name, kind=kind, M=M, K=K, N=N, fmt=fmt, type=type, post=post, gate=gate)


def listed():
    return [
        # one token's activations before a projection of the 8B decoder: two launches, latency only
        _case("quantize m1", "quantize", 1, 4096),
        # odd rows, a width that is no multiple of 64, FP32 from an accumulator
        _case("quantize ragged", "quantize", 333, 2976, fmt="nv", type="fp32"),
        # a weight matrix as it is loaded (8B gate_up): the largest matrix
        _case("quantize weights", "quantize", 28672, 4096, fmt="nv"),
        # a decode batch between gate_up and down
        _case("swiglu m8", "swiglu", 8, 14336),
        # a prefill between gate_up and down
        _case("swiglu m4096", "swiglu", 4096, 14336, fmt="nv", type="fp16"),
        # one token between attention output and gate_up: residual sum, norm, quantisation
        _case("norm m1", "norm", 1, 4096),
        # a prefill through a block with norms on both sides and a gate per token and channel
        _case("norm m4096", "norm", 4096, 4096, post=True, gate="full"),
        # one token through the smallest projection
        _case("gemm m1", "gemm", 1, 4096, 4096),
        # a decode batch through the down projection: long K, few columns
        _case("gemm m16", "gemm", 16, 14336, 4096, fmt="nv"),
        # ragged in every direction
        _case("gemm ragged m77", "gemm", 77, 2976, 11133, fmt="nv", type="fp16"),
        # the largest matrix (70B gate_up) for a full batch of this repository's decode path
        _case("gemm m128 70b", "gemm", 128, 8192, 57344),
        # a prefill through the 8B gate_up: the tensor cores' rate
        _case("gemm m4096", "gemm", 4096, 4096, 28672),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    kind = rng.choice(["quantize", "swiglu", "norm", "gemm", "gemm"])
    fmt = rng.choice(["mx", "nv"])
    type = rng.choice(["bf16", "fp16", "fp32"] if kind in ("quantize", "gemm") else ["bf16", "bf16", "fp16"])
    post, gate = (rng.random() < 0.5, rng.choice(["none", "row", "full"])) if kind == "norm" else (False, "none")
    while True:
        M, K = round(_log_uniform(rng, 1, 8192)), 32 * round(_log_uniform(rng, 4, 512))
        N = round(_log_uniform(rng, 64, 57344)) if kind == "gemm" else 0
        if M * K * N <= MOST_PRODUCTS and max(M, N) * K <= MOST_VALUES // (1 if kind == "quantize" else 2):
            return dict(kind=kind, M=M, K=K, N=N, fmt=fmt, type=type, post=post, gate=gate)


# ------------------------------------------------------------------------------------------------- plain forms

def _pow2(e):
    """2^e exactly, in 64 bits (the library's powers may be off in the last place, which moves ties)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(v):
    """Nearest E4M3 value, ties to even, of v >= 0 (64 bits), at most 448."""
    _, e = torch.frexp(v.clamp_min(2.0 ** -6))
    step = _pow2(e - 4)
    return ((v / step).round() * step).clamp_max(448.0)


def _quantize(x, fmt, ts):
    """Codes (rows x K, one to a byte) and scale bytes (rows x blocks) of x."""
    rows, K = x.shape
    v = x.view(rows, -1, BLOCK[fmt])
    amax = v.abs().amax(2).double()
    bad = ~torch.isfinite(amax)
    if fmt == "mx":
        _, e = torch.frexp(amax)                                       # amax = m 2^e, 0.5 <= m < 1
        e = torch.where(amax > 0, e - 3, -127).clamp(-127, 127)
        d, byte = _pow2(e), torch.where(bad, 255, e + 127).to(torch.uint8)
    else:
        s = torch.where(amax > 0, _e4m3(amax / (6.0 * ts.double())).clamp_min(2.0 ** -9), 0.0)
        d = (s.float() * ts).double()
        byte = torch.where(bad, 0x7F, s.float().to(torch.float8_e4m3fn).view(torch.uint8)).to(torch.uint8)
    q = (v.abs().double() / d.unsqueeze(2)).nan_to_num_(0.0).clamp_max_(6.0)
    # the grid's steps: 0.5 up to 2, 1 up to 4, 2 up to 6; codes count the steps
    low, mid = q < 2, q < 4
    code = torch.where(low, (q * 2).round(), torch.where(mid, q.round() + 2, (q / 2).round() + 4)).to(torch.uint8)
    code += v.signbit().to(torch.uint8) * 8
    return torch.where((bad | (d == 0)).unsqueeze(2), 0, code).to(torch.uint8).view(rows, K), byte


def _values(code, byte, fmt, ts, dtype):
    """What codes and scale bytes stand for, in 32 bits, rounded to dtype."""
    rows, K = code.shape
    q = torch.tensor(GRID + tuple(-g for g in GRID), device=code.device)[code.int()]
    if fmt == "mx":
        d = torch.where(byte == 255, math.nan, _pow2(byte.int() - 127)).float()
    else:
        d = byte.view(torch.float8_e4m3fn).float() * ts
    return (q.view(rows, -1, BLOCK[fmt]) * d.unsqueeze(2)).view(rows, K).to(dtype)


def _pack(code, byte):
    """The stored form: two codes to a byte, scales in atoms of 128 rows by 4 blocks."""
    rows, nb = byte.shape
    tiles, atoms = -(-rows // 128), -(-nb // 4)
    full = torch.zeros(tiles * 128, atoms * 4, dtype=torch.uint8, device=byte.device)
    full[:rows, :nb] = byte
    return code[:, 0::2] | (code[:, 1::2] << 4), full.view(tiles, 4, 32, atoms, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _unpack(codes, scales, rows, nb):
    tiles, atoms = -(-rows // 128), -(-nb // 4)
    code = torch.stack((codes & 15, codes >> 4), 2).view(rows, -1)
    return code, scales.view(tiles, atoms, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(tiles * 128, atoms * 4)[:rows, :nb].contiguous()


def _norm_block(s):
    """Residual sum and norm in 64 bits: what the four bits become depends on which side of a border a value falls."""
    y = s["O"].double()
    if s["w_post"] is not None:
        y = y * torch.rsqrt(y.square().mean(1, keepdim=True) + s["eps"]) * s["w_post"].double()
    if s["gate"] is not None:
        y = y * s["gate"].double()
    r = s["X"].double() + s["alpha"] * y
    return r, r * torch.rsqrt(r.square().mean(1, keepdim=True) + s["eps"]) * s["w"].double()


# -------------------------------------------------------------------------------------------------------- inputs

def _activations(gen, rows, K):
    """Normal values with a few channels that are an order of magnitude larger, as a decoder's activations have them."""
    x = torch.randn(rows, K, generator=gen, device="cuda")
    x[:, torch.randperm(K, generator=gen, device="cuda")[: max(1, K // 200)]] *= 12
    return x


def _tensor_scale(x):
    """The FP32 scale of a tensor whose largest block scale is then 448."""
    return (x.abs().amax().float() / (6 * 448)).view(1)


def _operand(gen, x, fmt):
    ts = _tensor_scale(x) if fmt == "nv" else None
    return (*_pack(*_quantize(x, fmt, ts)), ts)


def _buffers(rows, K, fmt):
    nb = K // BLOCK[fmt]
    return (torch.zeros(rows, K // 2, dtype=torch.uint8, device="cuda"),
            torch.zeros(-(-rows // 128) * -(-nb // 4) * 512, dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    M, K, fmt, dtype, kind = case["M"], case["K"], case["fmt"], TYPES[case["type"]], case["kind"]
    s = dict(case=case, ts=None)
    if kind == "gemm":
        s["x"] = _operand(gen, _activations(gen, M, K), fmt)
        s["w"] = _operand(gen, 0.02 * torch.randn(case["N"], K, generator=gen, device="cuda"), fmt)
        s["Y"] = torch.empty(M, case["N"], dtype=dtype, device="cuda")
        s["workspace"] = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
        return s
    s["codes"], s["scales"] = _buffers(M, K, fmt)
    s["Y"] = torch.empty(M, K, dtype=dtype, device="cuda")
    if kind == "quantize":
        x = 0.02 * torch.randn(M, K, generator=gen, device="cuda") if M > 8192 else _activations(gen, M, K)
        s["X"] = x.to(dtype)
        ts = _tensor_scale(x)
    elif kind == "swiglu":
        gu = torch.randn(M, 2 * K, generator=gen, device="cuda")
        s["GU"] = gu.to(dtype)
        ts = torch.full((1,), 30.0 / (6 * 448), device="cuda")            # as a calibration gives it
    else:
        s["X"], s["O"] = _activations(gen, M, K).to(dtype), torch.randn(M, K, generator=gen, device="cuda").to(dtype)
        weight = lambda: (1 + 0.1 * torch.randn(K, generator=gen, device="cuda")).to(dtype)  # noqa: E731
        s["w"], s["w_post"] = weight(), weight() if case["post"] else None
        rows = {"none": 0, "row": 1, "full": M}[case["gate"]]
        s["gate"] = torch.randn(rows, K, generator=gen, device="cuda").to(dtype) if rows else None
        s["alpha"], s["eps"] = (0.5 if case["post"] else 1.0), 1e-5
        s["R"], s["H"] = torch.empty_like(s["X"]), torch.empty_like(s["X"])
        ts = torch.full((1,), 30.0 / (6 * 448), device="cuda")
    s["ts"] = ts if fmt == "nv" else None
    return s


# --------------------------------------------------------------------------------------------------------- a pass

def _run_own(s):
    from paper_2608_15531_b200 import binding as fq
    case = s["case"]
    M, K, kind = case["M"], case["K"], case["kind"]
    if "L" not in s:                                       # the layouts, which a program keeps beside its buffers
        fmt = fq.FQ_MXFP4 if case["fmt"] == "mx" else fq.FQ_NVFP4
        s["L"] = fq.fq_mx_get_layout(M, K, fmt)
        s["LW"] = fq.fq_mx_get_layout(case["N"], K, fmt) if kind == "gemm" else None
    L = s["L"]
    if kind == "gemm":
        (xc, xs, xt), (wc, ws, wt) = s["x"], s["w"]
        fq.fq_mx_gemm(L, xc, xs, s["LW"], wc, ws, s["Y"], s["workspace"], x_tensor_scale=xt, w_tensor_scale=wt)
        return s["Y"]
    if kind == "quantize":
        fq.fq_mx_quantize(L, s["X"], s["codes"], s["scales"], tensor_scale=s["ts"])
    elif kind == "swiglu":
        fq.fq_mx_quantize_swiglu(L, s["GU"][:, :K], s["GU"][:, K:], s["codes"], s["scales"], tensor_scale=s["ts"])
    else:
        fq.fq_norm_block(s["X"], s["eps"], block=s["O"], block_weight=s["w_post"], gate=s["gate"], residual_scale=s["alpha"], R=s["R"],
                         weight=s["w"], H=s["H"], layout=L, codes=s["codes"], scales=s["scales"], tensor_scale=s["ts"])
    fq.fq_mx_dequantize(L, s["codes"], s["scales"], s["Y"], tensor_scale=s["ts"])
    return [s["R"], s["H"], s["Y"]] if kind == "norm" else s["Y"]


def run(state):
    if own:
        return _run_own(state)
    s = state
    case = s["case"]
    M, K, fmt, dtype, kind = case["M"], case["K"], case["fmt"], TYPES[case["type"]], case["kind"]
    if kind == "gemm":
        nb = K // BLOCK[fmt]
        (xc, xs, xt), (wc, ws, wt) = s["x"], s["w"]
        x = _values(*_unpack(xc, xs, M, nb), fmt, xt, torch.float32)
        w = _values(*_unpack(wc, ws, case["N"], nb), fmt, wt, torch.float32)
        return (x @ w.t()).to(dtype)
    if kind == "quantize":
        return _values(*_quantize(s["X"], fmt, s["ts"]), fmt, s["ts"], dtype)
    if kind == "swiglu":
        g, u = s["GU"][:, :K].double(), s["GU"][:, K:].double()        # 64 bits, as for the norm
        h = (g / (1 + torch.exp(-g)) * u).to(dtype)
        return _values(*_quantize(h, fmt, s["ts"]), fmt, s["ts"], dtype)
    r, h = (t.to(dtype) for t in _norm_block(s))
    return [r, h, _values(*_quantize(h, fmt, s["ts"]), fmt, s["ts"], dtype)]


def work(case):
    M, K, N, kind = case["M"], case["K"], case["N"], case["kind"]
    size = 4 if case["type"] == "fp32" else 2
    stored = 0.5 + 1 / BLOCK[case["fmt"]]
    if kind == "gemm":
        return {"bytes": stored * (M + N) * K + size * M * N, "flops": 2 * M * N * K}
    read = {"quantize": 1, "swiglu": 2, "norm": 2 + (case["gate"] == "full")}[kind]
    written = 1 + 2 * (kind == "norm")                     # the values read back; r and h
    flops = {"quantize": 4, "swiglu": 10, "norm": 12}[kind]
    # codes and scales are written by one call and read by the next
    return {"bytes": (size * (read + written) + 2 * stored) * M * K, "flops": flops * M * K}


# ------------------------------------------------------------------------------------------------- in 64 bits

def _exact_values(h, fmt, ts):
    """Quantised and read back, from the definition: the nearest grid value by comparison with the borders between grid values, an exact tie
    going to the value whose code is even."""
    rows, K = h.shape
    v = h.double().view(rows, -1, BLOCK[fmt])
    top = v.abs().amax(2, keepdim=True)
    if fmt == "mx":
        powers = torch.tensor([2.0 ** i for i in range(-127, 126)], dtype=torch.float64, device=h.device)
        d = powers[(torch.bucketize(top, 4 * powers, right=True) - 1).clamp_min(0)]   # the largest with 4 d <= top
    else:
        e4m3 = torch.arange(127, dtype=torch.uint8, device=h.device).view(torch.float8_e4m3fn).double()
        ask = top / (6 * ts.double())
        at = torch.bucketize(ask, (e4m3[1:] + e4m3[:-1]) / 2, right=False)            # a tie stays below
        lower = at.clamp_max(125)
        up = (ask == (e4m3[lower] + e4m3[lower + 1]) / 2) & (lower % 2 == 1)
        s = e4m3[torch.where(up, lower + 1, at)].clamp_min(2.0 ** -9)
        d = torch.where(top > 0, (s.float() * ts).double(), 1.0)
    grid = torch.tensor(GRID, dtype=torch.float64, device=h.device)
    borders = (grid[1:] + grid[:-1]) / 2
    q = v.abs() / d
    at = torch.bucketize(q, borders, right=False)
    tie = (at < 7) & (q == borders[at.clamp_max(6)]) & (at % 2 == 1)
    return (torch.copysign(grid[at + tie.long()], v) * d).view(rows, K)


def exact(case, seed):
    s = prepare(case, seed)
    K, fmt, dtype, kind = case["K"], case["fmt"], TYPES[case["type"]], case["kind"]
    if kind == "gemm":
        def operand(codes, scales, ts, rows):
            grid = torch.tensor([(-1.0) ** (c >> 3) * GRID[c & 7] for c in range(16)], dtype=torch.float64, device="cuda")
            v = torch.empty(rows, K, dtype=torch.float64, device="cuda")
            v[:, 0::2], v[:, 1::2] = grid[(codes % 16).long()], grid[(codes // 16).long()]
            r, b = torch.arange(rows, device="cuda")[:, None], torch.arange(K // BLOCK[fmt], device="cuda")[None]
            byte = scales[(r // 128 * -(-(K // BLOCK[fmt]) // 4) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4]
            d = torch.tensor([2.0 ** (i - 127) for i in range(256)], dtype=torch.float64, device="cuda")[byte.long()] if fmt == "mx" else byte.view(torch.float8_e4m3fn).double() * ts.double()
            return v.mul_(d.repeat_interleave(BLOCK[fmt], 1))
        return operand(*s["x"], case["M"]) @ operand(*s["w"], case["N"]).t()
    if kind == "quantize":
        return _exact_values(s["X"], fmt, s["ts"])
    if kind == "swiglu":
        g, u = s["GU"].double().split(K, 1)
        return _exact_values((torch.sigmoid(g) * g * u).to(dtype), fmt, s["ts"])
    o, x = s["O"].double(), s["X"].double()
    if case["post"]:
        o = o / torch.sqrt((o * o).sum(1, keepdim=True) / K + s["eps"]) * s["w_post"].double()
    r = torch.addcmul(x, o if s["gate"] is None else o * s["gate"].double(), torch.full((), s["alpha"], dtype=torch.float64, device="cuda"))
    h = r / torch.sqrt((r * r).sum(1, keepdim=True) / K + s["eps"]) * s["w"].double()
    return [r, h, _exact_values(h.to(dtype), fmt, s["ts"])]
