// Whether two arrays of a call share a byte, from their addresses, row lengths and row strides.
#pragma once
#include <cstddef>
#include <cstdint>

namespace fq {

// `rows` stretches of `bytes` bytes, `stride` bytes from one to the next (bytes <= stride); null or empty: not there.
struct Piece {
    const void* p;
    size_t bytes;
    uint64_t rows = 1, stride = 0;
    uintptr_t begin() const { return (uintptr_t)p; }
    uintptr_t end() const { return begin() + (rows - 1) * stride + bytes; }
    // Exact if one of the two is contiguous, or both have the same stride.  Otherwise a number-theoretic question that no caller has
    // asked yet: taken to overlap where the address ranges do.
    bool overlaps(const Piece& o) const {
        if (!p || !o.p || !bytes || !o.bytes || begin() >= o.end() || o.begin() >= end()) return false;
        if (rows == 1) return o.rows == 1 || o.has_row_in(begin(), end());
        if (o.rows == 1) return has_row_in(o.begin(), o.end());
        if (stride != o.stride) return true;
        // o's row j lies (j - i) strides and this much from row i: whole strides and a remainder
        const int64_t s = (int64_t)stride, d = (int64_t)(o.begin() - begin()), q = d >= 0 ? d / s : -((s - 1 - d) / s), rest = d - q * s;
        auto pair = [&](int64_t k) { return k > -(int64_t)rows && k < (int64_t)o.rows; };      // is there one with j - i = k?
        return (pair(-q) && rest < (int64_t)bytes) || (pair(-q - 1) && s - rest < (int64_t)o.bytes);
    }

  private:
    // (the ranges overlap)
    bool has_row_in(uintptr_t lo, uintptr_t hi) const {
        const uint64_t first = lo < begin() + bytes ? 0 : (lo - begin() - bytes) / stride + 1;     // that ends behind lo
        return first < rows && begin() + first * stride < hi;
    }
};
// rows x cols values of `size` bytes with a row stride of ld values
inline Piece matrix(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, size_t size) {
    if (rows == 1 || ld <= cols) return Piece{p, (size_t)(((rows - 1) * ld + cols) * size)};
    return Piece{p, (size_t)(cols * size), rows, ld * size};
}
// No output on another output or on an input.
inline bool disjoint(const Piece* out, int nout, const Piece* in, int nin) {
    for (int i = 0; i < nout; ++i) {
        for (int j = i + 1; j < nout; ++j)
            if (out[i].overlaps(out[j])) return false;
        for (int j = 0; j < nin; ++j)
            if (out[i].overlaps(in[j])) return false;
    }
    return true;
}

}  // namespace fq
