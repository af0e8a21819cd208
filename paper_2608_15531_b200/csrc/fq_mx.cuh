// Microscaled FP4: quantising consecutive values of a row that a lane holds, its block being spread over the lanes beside it.
// Included by fq_mx_kernels.cu.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fq_ptx.cuh"

namespace fq {

// PER: values that a lane holds (8 or 16)
template <bool NV, int PER>
struct Mx {
    static constexpr int BLOCK = NV ? 16 : 32;
    static constexpr int LANES = BLOCK / PER;         // lanes that hold a block
    static constexpr int ATOM = 4 * BLOCK;            // values of K that an atom of scales covers
    static constexpr int ATOM_LANES = ATOM / PER;
};

// ------------------------------------------------------------------------------------------------ values of a type

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return make_float2(bf16lo(w), bf16hi(w)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_float(float v) { return v; }

// Loads that a grid before this one may have written the data of: coherent, past the wait (memory clobber), not kept in L1.
__device__ __forceinline__ uint4 ld16(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
struct alignas(32) Words8 {
    uint32_t w[8];
    __device__ __forceinline__ uint4 half(int i) const { return make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]); }
};
// 32 bytes.  How rows lie: kOdd on any boundary of their type, kVec16 or kVec32 on one of 16 or 32 bytes.
enum RowsLie : int { kOdd = 0, kVec16 = 1, kVec32 = 2 };
__device__ __forceinline__ Words8 ld32(const void* p) {
    Words8 v;
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]), "=r"(v.w[7]) : "l"(p) : "memory");
    return v;
}
template <class T>                                         // 32 bytes of values of T
__device__ __forceinline__ Words8 load32(const T* p, int lie) {
    if (lie == kVec32) return ld32(p);
    Words8 v;
    if (lie == kVec16) {
        const uint4 a = ld16(p), b = ld16(reinterpret_cast<const uint4*>(p) + 1);
        v.w[0] = a.x, v.w[1] = a.y, v.w[2] = a.z, v.w[3] = a.w, v.w[4] = b.x, v.w[5] = b.y, v.w[6] = b.z, v.w[7] = b.w;
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.w[i] = reinterpret_cast<const volatile uint32_t*>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v.w[i] = (uint32_t)reinterpret_cast<const volatile uint16_t*>(p)[2 * i] | (uint32_t)reinterpret_cast<const volatile uint16_t*>(p)[2 * i + 1] << 16;
    }
    return v;
}
template <class T>
__device__ __forceinline__ void store32(T* p, int lie, const Words8& v) {
    if (lie == kVec32) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]),
                     "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7]) : "memory");
    } else if (lie == kVec16) {
        reinterpret_cast<uint4*>(p)[0] = v.half(0), reinterpret_cast<uint4*>(p)[1] = v.half(1);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) reinterpret_cast<uint32_t*>(p)[i] = v.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            reinterpret_cast<uint16_t*>(p)[2 * i] = (uint16_t)v.w[i], reinterpret_cast<uint16_t*>(p)[2 * i + 1] = (uint16_t)(v.w[i] >> 16);
    }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Eight values of a 16-bit type, as they lie in memory.
template <class T>
__device__ __forceinline__ void unpack8(const uint4& q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(w[i], T());
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}
template <class T>
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    return make_uint4(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()), pack2(v[4], v[5], T()), pack2(v[6], v[7], T()));
}
// p[0..7] on any boundary, of which only the first `n` exist (the others are 0).
template <class T>
__device__ __forceinline__ uint4 load_raw(const T* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i / 2] |= (uint32_t)reinterpret_cast<const volatile uint16_t*>(p)[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The same way back; `vec`: all exist, on a 16-byte boundary.
template <class T>
__device__ __forceinline__ void store_raw(T* p, int n, bool vec, const uint4& q) {
    if (vec) {
        *reinterpret_cast<uint4*>(p) = q;
        return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <class T> struct IsBf16 { static constexpr bool value = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };

// --------------------------------------------------------------------------------------------------- quantising

// Eight e2m1 codes, v[0] in the lowest nibble: nearest, ties to even, at most 6.
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8]) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Two E4M3 numbers, `lo` in the lower byte: nearest, ties to even, at most 448.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Value of an E4M3 byte with sign 0.
__device__ __forceinline__ float e4m3_value(uint32_t b) {
    return b >= 8 ? __uint_as_float((b << 20) + (120u << 23)) : (float)b * 0x1p-9f;      // (b << 20: exponent and fraction in place)
}
__device__ __forceinline__ float e2m1_value(uint32_t c) {                                  // of the three lower bits
    return c & 6 ? __uint_as_float(((c & 7) << 22) + (126u << 23)) : 0.5f * (float)(c & 1);
}
constexpr float kMinTensorScale = 0x1p-60f, kMaxTensorScale = 0x1p60f;       // (the product of two is a normal number)

// The tensor's part of an FQ_NVFP4 quantisation.
struct TensorScale {
    float ts, inv6;       // the scale, and about 1 / (6 ts)
    bool bad;
    __device__ __forceinline__ void read(const float* p) {
        ts = 1.0f;
        if (p) asm volatile("ld.global.f32 %0, [%1];" : "=f"(ts) : "l"(p) : "memory");
        bad = !(ts >= kMinTensorScale && ts <= kMaxTensorScale);
        inv6 = 1.0f / (6.0f * ts);
    }
};

// E4M3 scale of a block: nearest to amax / (6 ts).  The quotient in binary32 is off by less than 2^-21 of it, so if the numbers
// 2^-20 above and below round alike that is the result; else the quotient is taken in binary64, and brought to binary32 by
// rounding to odd, so that rounding it again to E4M3 is a single rounding.
__device__ __forceinline__ uint32_t nv_scale(float amax, const TensorScale& t) {
    const float q = amax * t.inv6;
    const uint32_t two = e4m3x2(q * (1.0f - 0x1p-20f), q * (1.0f + 0x1p-20f));
    uint32_t s = two & 0xffu;
    if (s != two >> 8) {
        const double e = (double)amax / (6.0 * (double)t.ts);
        float f = __double2float_rz(e);
        if ((double)f != e) f = __uint_as_float(__float_as_uint(f) | 1u);
        s = e4m3x2(f, f) & 0xffu;
    }
    return amax > 0.0f ? max(s, 1u) : 0u;
}

// One of two neighbouring codes for the exact |v| / d: the sign of |v| - border * d, which one fused multiply-add gives exactly.
__device__ __noinline__ uint32_t settle_codes(uint32_t lo, uint32_t hi, float d, float v0, float v1, float v2, float v3, float v4, float v5,
                                              float v6, float v7) {
    const float v[8] = {v0, v1, v2, v3, v4, v5, v6, v7};
    uint32_t out = lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = (lo >> (4 * i)) & 7u, b = (hi >> (4 * i)) & 7u;
        if (a == b) continue;
        const float border = 0.5f * (e2m1_value(a) + e2m1_value(b)), r = fmaf(-border, d, fabsf(v[i]));
        const uint32_t c = r > 0.0f ? b : (r < 0.0f ? a : (a & 1 ? b : a));
        out = (out & ~(7u << (4 * i))) | c << (4 * i);
    }
    return out;
}

// The scale of a block and what its values are multiplied by.
template <bool NV>
struct BlockScale {
    uint32_t byte;
    float d, inv;                // FQ_MXFP4: inv = 1 / d; FQ_NVFP4: about that
    bool bad;                    // NaN: codes 0
    // amax: bits of the largest magnitude (which compare as magnitudes do; NaN is above infinity)
    __device__ __forceinline__ BlockScale(uint32_t amax, const TensorScale& t) {
        bad = amax >= 0x7f800000u;
        if constexpr (!NV) {
            // 2^floor(log2 amax) is amax's exponent field; two less, and not below 0, is the byte, also for subnormal amax
            byte = (uint32_t)max((int)(amax >> 23) - 2, 0);
            inv = __uint_as_float((254u - byte) << 23);
            d = 0.0f;
        } else {
            bad = bad || t.bad;
            byte = nv_scale(__uint_as_float(amax), t);
            d = e4m3_value(byte) * t.ts;
            asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(d));
            if (byte == 0) inv = 0.0f;                     // a block of zeros
        }
        if (bad) byte = NV ? 0x7fu : 0xffu;
    }
    // codes of eight values
    __device__ __forceinline__ uint32_t codes(const float (&v)[8]) const {
        float y[8];
        uint32_t c;
        if constexpr (!NV) {
            // the quotient is a product with a power of two, exact wherever the result does not round to 0
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i] * inv;
            c = e2m1x8(y);
        } else {
            // a quotient that is off by less than 2^-21: if the numbers 2^-20 below and above round alike that is the result
            const float below = inv * (1.0f - 0x1p-20f), above = inv * (1.0f + 0x1p-20f);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i] * below;
            c = e2m1x8(y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = v[i] * above;
            const uint32_t hi = e2m1x8(y);
            if (c != hi) c = settle_codes(c, hi, d, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
            if (byte == 0) c = 0;
        }
        return bad ? 0 : c;
    }
};
template <int LANES>
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}
// Eight values of a 16-bit type, two to a word: their magnitudes are compared two at a time.
__device__ __forceinline__ uint32_t max_magnitude(const uint4& q) {
    return max_u16x2(max_u16x2(q.x & 0x7fff7fffu, q.y & 0x7fff7fffu), max_u16x2(q.z & 0x7fff7fffu, q.w & 0x7fff7fffu));
}
template <bool NV, class T>
__device__ __forceinline__ void quantize8(const uint4& q, const TensorScale& t, uint32_t& codes, uint32_t& scale) {
    uint32_t m = max_magnitude(q);
    m = block_max<Mx<NV, 8>::LANES>(max(m & 0xffffu, m >> 16));
    const BlockScale<NV> s(__float_as_uint(unpack2(m, T()).x), t);
    float v[8];
    unpack8<T>(q, v);
    codes = s.codes(v);
    scale = s.byte;
}
template <bool NV, class T>
__device__ __forceinline__ void quantize16(const Words8& q, const TensorScale& t, uint2& codes, uint32_t& scale) {
    uint32_t m = max_u16x2(max_magnitude(q.half(0)), max_magnitude(q.half(1)));
    m = block_max<Mx<NV, 16>::LANES>(max(m & 0xffffu, m >> 16));
    const BlockScale<NV> s(__float_as_uint(unpack2(m, T()).x), t);
    float v[8];
    unpack8<T>(q.half(0), v);
    codes.x = s.codes(v);
    unpack8<T>(q.half(1), v);
    codes.y = s.codes(v);
    scale = s.byte;
}
template <bool NV>
__device__ __forceinline__ void quantize16(const Words8& a, const Words8& b, const TensorScale& t, uint2& codes, uint32_t& scale) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, max(a.w[i] & 0x7fffffffu, b.w[i] & 0x7fffffffu));
    const BlockScale<NV> s(block_max<Mx<NV, 16>::LANES>(m), t);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(a.w[i]);
    codes.x = s.codes(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(b.w[i]);
    codes.y = s.codes(v);
    scale = s.byte;
}

// Values of eight codes.
__device__ __forceinline__ void e2m1_values8(uint32_t codes, float (&v)[8]) {
    uint32_t h[4];
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(h[i], __half());
        v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
}

// The four scale bytes of an atom's row, from the lanes that hold its blocks, in all of them.
template <bool NV, int PER>
__device__ __forceinline__ uint32_t gather_scales(uint32_t scale) {
    constexpr int LANES = Mx<NV, PER>::LANES;
    uint32_t w = scale << (8 * ((threadIdx.x & 31) / LANES % 4));
    w |= __shfl_xor_sync(0xffffffffu, w, LANES);
    w |= __shfl_xor_sync(0xffffffffu, w, 2 * LANES);
    return w;
}
// Place of row r's four bytes in atom `atom` (of `atoms` along K).
__device__ __forceinline__ size_t scale_word(uint32_t r, uint32_t atoms, uint32_t atom) {
    return ((size_t)(r >> 7) * atoms + atom) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4;
}

}  // namespace fq
