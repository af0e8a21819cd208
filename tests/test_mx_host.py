"""Microscaled FP4: layouts, sizes, and what the calls refuse before anything is launched.  CPU only: the addresses are made up."""
import ctypes

import numpy as np
import pytest

from paper_2608_15531_b200 import binding as fq

import mx_reference as R

BF16, FP16, FP32 = 0, 1, 2
A = 1 << 32            # addresses far apart, 2^32 bytes each


class NormArgs(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint32), ("D", ctypes.c_uint32), ("type", ctypes.c_uint32), ("eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
                ("X", ctypes.c_void_p), ("ld_x", ctypes.c_uint64), ("block", ctypes.c_void_p), ("ld_block", ctypes.c_uint64),
                ("block_weight", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("ld_gate", ctypes.c_uint64), ("weight", ctypes.c_void_p),
                ("R", ctypes.c_void_p), ("ld_r", ctypes.c_uint64), ("H", ctypes.c_void_p), ("ld_h", ctypes.c_uint64),
                ("layout", ctypes.c_void_p), ("tensor_scale", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p)]


def _p(v):
    return ctypes.c_void_p(v)


def _u64(v):
    return ctypes.c_uint64(v)


def quantize(L, x=A, type=BF16, ldx=None, ts=0, codes=2 * A, scales=3 * A):
    return fq.lib().fq_mx_quantize(ctypes.byref(L), _p(x), type, _u64(L.K if ldx is None else ldx), _p(ts), _p(codes), _p(scales), _p(0))


def dequantize(L, y=A, type=BF16, ldy=None, ts=0, codes=2 * A, scales=3 * A):
    return fq.lib().fq_mx_dequantize(ctypes.byref(L), _p(codes), _p(scales), _p(ts), _p(y), type, _u64(L.K if ldy is None else ldy), _p(0))


def swiglu(L, g=A, u=4 * A, type=BF16, ldg=None, ldu=None, ts=0, codes=2 * A, scales=3 * A):
    return fq.lib().fq_mx_quantize_swiglu(ctypes.byref(L), _p(g), _u64(L.K if ldg is None else ldg), _p(u), _u64(L.K if ldu is None else ldu), type, _p(ts),
                                          _p(codes), _p(scales), _p(0))


def gemm(LX, LW, y=A, type=BF16, ldy=None, xt=0, wt=0, xc=2 * A, xs=3 * A, wc=4 * A, ws=5 * A, work=6 * A, bytes=None):
    return fq.lib().fq_mx_gemm(ctypes.byref(LX), _p(xc), _p(xs), _p(xt), ctypes.byref(LW), _p(wc), _p(ws), _p(wt), _p(y), type,
                               _u64(LW.rows if ldy is None else ldy), _p(work), ctypes.c_size_t(fq.FQ_MX_WORKSPACE_BYTES if bytes is None else bytes), _p(0))


def norm(**kw):
    rows, D = kw.get("rows", 4), kw.get("D", 256)
    d = dict(rows=rows, D=D, type=BF16, eps=1e-5, residual_scale=1.0, X=A, ld_x=D, ld_block=D, ld_gate=D, ld_r=D, H=2 * A, ld_h=D)
    d.update(kw)
    layout = d.pop("layout", None)
    a = NormArgs(**d)
    a.layout = ctypes.addressof(layout) if layout is not None else None
    return fq.lib().fq_norm_block(ctypes.byref(a), _p(0))


@pytest.mark.parametrize("rows,K,fmt,code,scale", [(1, 32, 0, 16, 512), (1, 32, 1, 16, 512), (128, 128, 0, 8192, 512), (129, 160, 0, 129 * 80, 2 * 2 * 512),
                                                   (129, 160, 1, 129 * 80, 2 * 3 * 512), (28672, 4096, 1, 28672 * 2048, 224 * 64 * 512)])
def test_sizes(rows, K, fmt, code, scale):
    L = fq.fq_mx_get_layout(rows, K, fmt)
    assert (L.rows, L.K, L.format) == (rows, K, fmt)
    assert fq.fq_mx_sizes(L) == (code, scale)


@pytest.mark.parametrize("rows,K,fmt,code", [(0, 32, 0, -1), (1, 0, 0, -2), (1, 48, 0, -2), (1, 16, 1, -2), (1, 32, 2, -1), (1, (1 << 20) + 32, 0, -2),
                                             (2 ** 31, 32, 0, -2), (-1, 32, 0, -1), (1, 2 ** 32 + 32, 0, -1)])
def test_layouts_that_are_refused(rows, K, fmt, code):
    with pytest.raises(fq.FqError) as e:
        fq.fq_mx_get_layout(rows, K, fmt)
    assert e.value.code == code


def _refused(status, word=""):
    assert status == fq.FQ_ERR_INVALID_ARG and word in fq.fq_last_error(), (status, fq.fq_last_error())


def test_a_made_up_layout_is_refused():
    for field, value in (("abi", 7), ("rows", 0), ("rows", 2 ** 31), ("K", 33), ("K", 0), ("K", 1 << 21), ("format", 2)):
        L = fq.fq_mx_get_layout(4, 64, 0)
        setattr(L, field, value)
        with pytest.raises(fq.FqError):
            fq.fq_mx_sizes(L)
        G = fq.fq_mx_get_layout(4, 64, 0)
        for status in (quantize(L), dequantize(L), swiglu(L), gemm(L, G), gemm(G, L), norm(D=64, codes=4 * A, scales=5 * A, layout=L)):
            _refused(status, "layout")


def test_null_misaligned_and_unknown():
    L = fq.fq_mx_get_layout(4, 64, 0)
    for status in (quantize(L, x=0), quantize(L, codes=0), quantize(L, scales=0), dequantize(L, y=0), dequantize(L, codes=0), swiglu(L, g=0), swiglu(L, u=0),
                   gemm(L, L, y=0), gemm(L, L, xc=0), gemm(L, L, ws=0), gemm(L, L, work=0), norm(X=0)):
        _refused(status, "null")
    for status in (quantize(L, codes=2 * A + 8), quantize(L, scales=3 * A + 4), quantize(L, x=A + 1), quantize(L, x=A + 2, type=FP32), dequantize(L, y=A + 1),
                   swiglu(L, g=A + 1), swiglu(L, u=A + 1), gemm(L, L, y=A + 1), gemm(L, L, xc=2 * A + 8), gemm(L, L, work=6 * A + 8), norm(weight=3 * A + 1),
                   norm(X=A + 1), norm(H=2 * A + 1)):
        _refused(status, "misaligned")
    for status in (quantize(L, type=3), dequantize(L, type=3), swiglu(L, type=FP32), gemm(L, L, type=3), norm(type=FP32)):
        _refused(status, "type")
    for status in (quantize(L, ldx=63), dequantize(L, ldy=63), swiglu(L, ldg=63), swiglu(L, ldu=0), gemm(L, L, ldy=3), norm(ld_x=255), norm(ld_h=0),
                   norm(block=4 * A, ld_block=1), norm(block=4 * A, gate=5 * A, ld_gate=1), quantize(L, ldx=2 ** 63)):
        _refused(status, "row stride")
    assert gemm(L, L, bytes=fq.FQ_MX_WORKSPACE_BYTES - 1) == fq.FQ_ERR_BUFFER_TOO_SMALL


def test_tensor_scales_belong_to_nvfp4():
    L = fq.fq_mx_get_layout(4, 64, 0)
    for status in (quantize(L, ts=7 * A), dequantize(L, ts=7 * A), swiglu(L, ts=7 * A), gemm(L, L, xt=7 * A), gemm(L, L, wt=7 * A),
                   norm(D=64, codes=4 * A, scales=5 * A, tensor_scale=7 * A, layout=L)):
        _refused(status, "tensor scale")
    _refused(quantize(fq.fq_mx_get_layout(4, 64, 1), ts=7 * A + 2), "misaligned")


def test_a_product_of_different_formats_or_lengths_is_refused():
    L = fq.fq_mx_get_layout
    _refused(gemm(L(4, 64, 0), L(4, 64, 1)), "differ")
    _refused(gemm(L(4, 64, 0), L(4, 96, 0)), "differ")


def test_outputs_that_overlap_are_refused():
    L = fq.fq_mx_get_layout(4, 64, 0)          # codes 128 bytes, scales 512
    N = fq.fq_mx_get_layout(4, 64, 1)
    for status in (quantize(L, codes=A + 496), quantize(L, scales=A - 496), quantize(L, codes=3 * A + 496), quantize(N, ts=3 * A + 4),
                   dequantize(L, y=2 * A + 112), swiglu(L, codes=4 * A), gemm(L, L, y=3 * A), gemm(L, L, y=6 * A + 32768), gemm(L, L, work=5 * A + 496),
                   norm(H=A + 2), norm(H=A, ld_h=512), norm(R=2 * A), norm(block=4 * A, H=4 * A - 2), norm(block=4 * A, gate=5 * A, H=5 * A), norm(weight=2 * A + 16),
                   norm(R=A, H=A), norm(D=64, codes=2 * A + 16, scales=5 * A, layout=L)):
        _refused(status, "overlaps")


def test_norm_arguments_that_do_not_go_together():
    L = fq.fq_mx_get_layout(4, 256, 0)
    _refused(norm(rows=0))
    assert norm(D=0) == fq.FQ_ERR_UNSUPPORTED_SHAPE and norm(D=16385) == fq.FQ_ERR_UNSUPPORTED_SHAPE
    _refused(norm(eps=-1.0), "eps")
    _refused(norm(eps=float("nan")), "eps")
    _refused(norm(H=0), "no output")
    _refused(norm(gate=5 * A), "without a block")
    _refused(norm(block_weight=5 * A), "without a block")
    _refused(norm(rows=5, codes=4 * A, scales=5 * A, layout=L), "layout is 4 x 256")
    _refused(norm(codes=4 * A, layout=L), "null")
    _refused(norm(codes=4 * A, scales=5 * A), "layout")


def test_the_reference_quantises_by_the_formula():
    """The oracle itself, value by value in the naive way."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 64)) * np.exp2(rng.integers(-8, 8, (3, 1)))
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 4.0]
    for fmt, ts in ((0, 1.0), (1, 1.0), (1, 0.037)):
        code, byte = R.quantize(x, fmt, ts)
        B = R.BLOCK[fmt]
        for r in range(3):
            for b in range(64 // B):
                blk = x[r, b * B:(b + 1) * B]
                amax = np.abs(blk).max()
                if fmt == 0:
                    d = 2.0 ** (np.floor(np.log2(amax)) - 2)
                else:
                    ask = amax / (6 * float(np.float32(ts)))
                    s = min(range(127), key=lambda i: (abs(R.E4M3[i] - ask), i % 2))
                    assert byte[r, b] == max(s, 1)
                    d = float(np.float32(R.E4M3[max(s, 1)]) * np.float32(ts))
                for i, v in enumerate(blk):
                    c = min(range(8), key=lambda j: (abs(R.GRID[j] * d - abs(v)), j % 2))
                    assert code[r, b * B + i] == c + 8 * (v < 0), (fmt, r, b, i, v, d)
