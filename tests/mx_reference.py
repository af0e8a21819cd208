"""Plain implementation in 64 bits of the microscaled FP4 formats, the gated product and the norms around a block (numpy, one formula
after the other), and helpers of the tests."""
from __future__ import annotations

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([GRID, -GRID])
E4M3 = np.array([(b & 7) * 2.0 ** -9 if b < 8 else (1 + (b & 7) / 8) * 2.0 ** ((b >> 3) - 7) for b in range(127)])     # byte -> value
BLOCK = {0: 32, 1: 16}
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def nearest(q, table):
    """Index of the nearest entry of an ascending table, ties to the even index, beyond the last the last."""
    borders = (table[1:] + table[:-1]) / 2
    at = np.searchsorted(borders, q, side="left")
    tie = (at < len(borders)) & (q == borders[np.minimum(at, len(borders) - 1)]) & (at % 2 == 1)
    return at + tie


def quantize(x, fmt, ts=1.0):
    """x: rows x K float64 -> codes (rows x K), scale bytes (rows x blocks)."""
    rows, K = x.shape
    v = x.reshape(rows, -1, BLOCK[fmt])
    with np.errstate(all="ignore"):
        amax = np.max(np.where(np.isnan(v), np.inf, np.abs(v)), axis=2)
        bad = ~np.isfinite(amax)
        amax = np.where(bad, 1.0, amax)
        if fmt == 0:
            _, e = np.frexp(amax)
            byte = np.where(amax > 0, np.maximum(e - 1 - 2, -127), -127) + 127
            d = np.ldexp(1.0, byte - 127)
            byte = np.where(bad, 255, byte)
        else:
            ts32 = np.float32(ts)
            if not (np.float32(2.0 ** -60) <= ts32 <= np.float32(2.0 ** 60)):
                bad = np.ones_like(bad)
                ts32 = np.float32(1.0)
            byte = nearest(amax / (6.0 * np.float64(ts32)), E4M3)
            byte = np.where(amax > 0, np.maximum(byte, 1), 0)
            d = (E4M3[byte].astype(np.float32) * ts32).astype(np.float64)
            byte = np.where(bad, 0x7F, byte)
        q = np.where(d[:, :, None] > 0, np.abs(v) / np.where(d > 0, d, 1.0)[:, :, None], 0.0)
        code = nearest(np.where(np.isnan(q), 0.0, q), GRID) + 8 * np.signbit(v)
        code = np.where((bad | (d == 0))[:, :, None], 0, code)
    return code.reshape(rows, K).astype(np.uint8), byte.astype(np.uint8)


def steps(byte, fmt, ts=1.0):
    """Scale bytes -> d as float64 (binary32 values)."""
    if fmt == 0:
        return np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(int) - 127))
    table = np.concatenate([E4M3, [np.nan]])
    table = np.concatenate([table, -table])
    with np.errstate(all="ignore"):
        return (table[byte].astype(np.float32) * np.float32(ts)).astype(np.float64)


def values(code, byte, fmt, ts=1.0):
    return VALUES[code] * np.repeat(steps(byte, fmt, ts), BLOCK[fmt], axis=1)


def pack(code, byte, fill=0):
    """Stored codes (rows x K/2) and scales (flat); bytes of rows beyond the last hold `fill`."""
    rows, nb = byte.shape
    tiles, atoms = -(-rows // 128), -(-nb // 4)
    out = np.full((tiles * atoms, 512), fill, dtype=np.uint8)
    for r in range(rows):
        for b in range(atoms * 4):
            out[r // 128 * atoms + b // 4, r % 32 * 16 + r % 128 // 32 * 4 + b % 4] = byte[r, b] if b < nb else 0
    return code[:, 0::2] | code[:, 1::2] << 4, out.reshape(-1)


def round_to(x, dtype):
    """float64 -> the type, through binary32 as a tensor library rounds (a second rounding matters once in 2^29 values)."""
    with np.errstate(all="ignore"):
        return torch.from_numpy(np.ascontiguousarray(x.astype(np.float32))).to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def swiglu(g, u):
    with np.errstate(all="ignore"):
        return g / (1 + np.exp(-g)) * u


def norm_block(x, eps, block=None, block_weight=None, gate=None, alpha=1.0, weight=None):
    with np.errstate(all="ignore"):
        r = x
        if block is not None:
            y = block
            if block_weight is not None:
                y = y / np.sqrt(np.mean(y * y, axis=1, keepdims=True) + np.float64(np.float32(eps))) * block_weight
            if gate is not None:
                y = y * gate
            r = x + np.float64(np.float32(alpha)) * y
        h = r / np.sqrt(np.mean(r * r, axis=1, keepdims=True) + np.float64(np.float32(eps)))
        return r, h if weight is None else h * weight


def same(a, b):
    """Equal values; NaN equals NaN."""
    a, b = f64(a), f64(b)
    return np.array_equal(a, b, equal_nan=True)
