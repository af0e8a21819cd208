"""Which arrays of a call share memory: the rule against a byte map, and what the FP4 calls then refuse or take.  CPU only; the addresses are made up."""
import os
import subprocess

import pytest
import torch

from paper_2608_15531_b200 import binding as fq

from test_mx_host import A, FP32, dequantize, gemm, norm, quantize, swiglu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "fq_overlap.h"
using namespace fq;
static const uintptr_t B = 1ull << 40;
struct M { uint64_t at, rows, cols, ld; size_t size; };
static std::vector<char> map(const M& m) {
    std::vector<char> v(1024, 0);
    for (uint64_t r = 0; r < m.rows; ++r)
        for (uint64_t b = 0; b < m.cols * m.size; ++b) v[m.at + r * m.ld * m.size + b] = 1;
    return v;
}
static Piece piece(const M& m) { return matrix((const void*)(B + m.at), m.rows, m.cols, m.ld, m.size); }
int main() {
    std::mt19937 rng(7);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
    long hits = 0, exact = 0;
    for (long t = 0; t < 400000; ++t) {
        M a, b;
        for (M* m : {&a, &b}) {
            m->size = upto(2) ? 2 : 4, m->rows = 1 + upto(5), m->cols = 1 + upto(9), m->ld = m->cols + (upto(3) ? upto(12) : 0), m->at = upto(150) * 2;
            if (m->rows == 1 && upto(2)) m->ld = 0;
        }
        if (upto(2)) b.ld = a.ld, b.size = a.size;
        for (M* m : {&a, &b})
            if (m->rows > 1) m->ld = std::max(m->ld, m->cols);        // (what a call lets through)
        const auto x = map(a), y = map(b);
        bool want = false;
        for (size_t i = 0; i < x.size(); ++i) want |= x[i] && y[i];
        const Piece p = piece(a), q = piece(b);
        const bool got = p.overlaps(q), back = q.overlaps(p);
        const bool sure = p.rows == 1 || q.rows == 1 || p.stride == q.stride;
        if (got != back || (sure ? got != want : (want && !got))) {
            std::printf("%llu: %llu x %llu, %llu of %zu; %llu: %llu x %llu, %llu of %zu: %d %d, is %d\n", (unsigned long long)a.at, (unsigned long long)a.rows,
                        (unsigned long long)a.cols, (unsigned long long)a.ld, a.size, (unsigned long long)b.at, (unsigned long long)b.rows, (unsigned long long)b.cols,
                        (unsigned long long)b.ld, b.size, got, back, want);
            return 1;
        }
        hits += want, exact += sure;
    }
    // the largest that a call lets through: a row stride of 2^40 values of four bytes, 2^16 rows
    const Piece big = matrix((const void*)B, 1 << 16, 1 << 20, 1ull << 40, 4);
    for (uint64_t r : {0ull, 1ull, 65535ull}) {
        if (!big.overlaps(matrix((const void*)(B + (r << 42) + 1000), 3, 8, 100, 4))) return 2;                          // (strides differ, ranges overlap)
        if (big.overlaps(Piece{(const void*)(B + (r << 42) + (4ull << 20)), 4096})) return 3;                            // behind row r
        if (!big.overlaps(Piece{(const void*)(B + (r << 42) + (4ull << 20) - 1), 4096})) return 4;
    }
    if (big.overlaps(matrix((const void*)(B + (4ull << 20)), 1 << 16, 1 << 20, 1ull << 40, 4))) return 5;                // the columns beside
    if (!big.overlaps(matrix((const void*)(B + (4ull << 20) - 4), 1 << 16, 1 << 20, 1ull << 40, 4))) return 6;
    if (Piece{nullptr, 10}.overlaps(Piece{nullptr, 10}) || Piece{(const void*)B, 0}.overlaps(Piece{(const void*)B, 4})) return 7;
    std::printf("%ld overlap, %ld decided exactly\n", hits, exact);
    return hits > 1000 ? 0 : 8;
}
"""


def test_the_rule_against_a_map_of_bytes(tmp_path):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(_PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "paper_2608_15531_b200", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, (p.returncode, p.stdout, p.stderr[-500:])


def outcome(call, *args, **kw):
    status = call(*args, **kw)
    return status, fq.fq_last_error()


D = 64                                                     # of one array of four times D columns, D a slice
WIDE = dict(D=D, X=A, ld_x=4 * D, ld_r=4 * D, ld_h=4 * D, ld_block=4 * D, ld_gate=4 * D)
LAYOUT = fq.fq_mx_get_layout(4, 64, 0)                     # codes 128 bytes, scales 512
S = 2 * D                                                  # bytes of a slice


def wide(**kw):
    return norm, (), {**WIDE, **kw}


def over(call, *layouts, **kw):
    return call, layouts or (LAYOUT,), kw


APART = [wide(R=A + S, H=A + 2 * S), wide(block=A + S, gate=A + 3 * S, H=A + 2 * S, R=A), wide(X=A + 3 * S, R=A, H=A + S), wide(H=A + 16 * S),
         wide(H=A + S, codes=A + 16 * S, scales=5 * A, layout=LAYOUT),
         over(quantize, ldx=4096, codes=A + 128), over(quantize, ldx=4096, codes=A + 256, scales=A + 1024), over(quantize, ldx=4096, codes=A + 8192 - 128),
         over(dequantize, y=2 * A + 128, ldy=128), over(swiglu, ldg=4096, ldu=4096, u=A + 128, codes=A + 256),
         over(gemm, LAYOUT, LAYOUT, y=A, ldy=1 << 17, work=A + 16), over(gemm, LAYOUT, LAYOUT, y=2 * A + 128, ldy=256)]
SHARED = [wide(R=A + S - 2, H=A + 2 * S), wide(R=A + S, H=A + 2 * S - 2), wide(H=A + 4 * S - 2), wide(H=A - 4 * S + 2), wide(H=A - 3 * 4 * S - S + 2),
          wide(H=A + S, ld_h=4 * D + 8), wide(R=A + S, H=A + S), wide(H=A + S, weight=A + 2 * S - 2), wide(H=A + S, codes=A + S - 16, scales=5 * A, layout=LAYOUT),
          over(quantize, ldx=4096, codes=A + 112), over(quantize, ldx=4096, codes=A + 8192 - 112), over(quantize, ldx=128, codes=A + 4096, scales=A + 1024 - 272),
          over(dequantize, y=2 * A + 126, ldy=128), over(swiglu, ldg=4096, ldu=4096, u=A + 128, codes=A + 240),
          over(gemm, LAYOUT, LAYOUT, y=A, ldy=1 << 17, work=A + (1 << 18) - 16), over(quantize, type=FP32, ldx=128, codes=A + 240), over(quantize, codes=A + 400)]


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: the call has to end at the missing device")
@pytest.mark.parametrize("case", range(len(APART)))
def test_column_slices_of_one_array_are_taken(case):
    call, args, kw = APART[case]
    status, text = outcome(call, *args, **kw)
    assert status == fq.FQ_ERR_CUDA, (status, text)


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_slices_that_share_a_byte_are_refused(case):
    call, args, kw = SHARED[case]
    status, text = outcome(call, *args, **kw)
    assert status == fq.FQ_ERR_INVALID_ARG and "overlaps" in text, (status, text)
