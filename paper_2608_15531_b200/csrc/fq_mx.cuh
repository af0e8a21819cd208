// Microscaled FP4: quantising eight consecutive values of a row that a lane holds, its block being spread over the lanes
// beside it.  Included by fq_mx_kernels.cu.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fq_ptx.cuh"

namespace fq {

template <bool NV>
struct Mx {
    static constexpr int BLOCK = NV ? 16 : 32;
    static constexpr int LANES = BLOCK / 8;           // lanes that hold a block
    static constexpr int ATOM = 4 * BLOCK;            // values of K that an atom of scales covers
    static constexpr int ATOM_LANES = ATOM / 8;
};

// ------------------------------------------------------------------------------------------------ values of a type

__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) { return make_float2(bf16lo(w), bf16hi(w)); }
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(float v) { return v; }
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
// Eight values from p[0..7], of which only the first `n` exist (the others are 0).  VEC: all eight do, on a 16-byte boundary.
template <class T, bool VEC>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
    if constexpr (VEC && sizeof(T) == 2) {
        const uint4 q = ld16(p);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(w[i], T());
            v[2 * i] = f.x, v[2 * i + 1] = f.y;
        }
    } else if constexpr (VEC) {
        const uint4 a = ld16(p), b = ld16(p + 4);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const T a = from_float<T>(lo), b = from_float<T>(hi);
    return (uint32_t)*reinterpret_cast<const uint16_t*>(&a) | (uint32_t)*reinterpret_cast<const uint16_t*>(&b) << 16;
}
template <class T, bool VEC>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
    if constexpr (VEC && sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    } else if constexpr (VEC) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = from_float<T>(v[i]);
    }
}

// Whether rounding `h` to T may come out differently from rounding the exact value, of which h is a binary32 result that is off
// by a few units in its last place: h lies within 4 units of a border (the middle between two values of T), or below
// T's normal range, where borders lie elsewhere.  True of 1 in 8192 values for BF16, 1 in 1024 for FP16.
__device__ __forceinline__ bool near_border(float h, __nv_bfloat16) {
    const uint32_t b = __float_as_uint(h);
    return ((b - 0x7ffcu) & 0xffffu) <= 8u || (b & 0x7fffffffu) < 0x00800000u;
}
__device__ __forceinline__ bool near_border(float h, __half) {
    const uint32_t b = __float_as_uint(h);
    return ((b - 0x0ffcu) & 0x1fffu) <= 8u || (b & 0x7fffffffu) < 0x38800000u;
}

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
constexpr float kMinTensorScale = 0x1p-100f, kMaxTensorScale = 0x1p100f;

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

// Codes of this lane's eight values and the scale byte of their block.  All lanes of the block take part.
template <bool NV>
__device__ __forceinline__ void quantize8(const float (&v)[8], const TensorScale& t, uint32_t& codes, uint32_t& scale) {
    uint32_t amax = 0;                                     // magnitudes compare as their bits do; NaN is above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < Mx<NV>::LANES; o *= 2) amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const bool bad = amax >= 0x7f800000u || (NV && t.bad);
    float y[8];
    if constexpr (!NV) {
        // 2^floor(log2 amax) is amax's exponent field; two less, and not below 0, is the byte, also for subnormal amax.  The
        // quotient is a product with a power of two, exact wherever the result does not round to 0.
        const uint32_t b = (uint32_t)max((int)(amax >> 23) - 2, 0);
        const float inv = __uint_as_float((254u - b) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[i] * inv;
        codes = e2m1x8(y);
        scale = b;
    } else {
        scale = nv_scale(__uint_as_float(amax), t);
        const float d = e4m3_value(scale) * t.ts, inv = scale ? 1.0f / d : 0.0f;
        const float below = inv * (1.0f - 0x1p-20f), above = inv * (1.0f + 0x1p-20f);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[i] * below;
        codes = e2m1x8(y);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[i] * above;
        const uint32_t hi = e2m1x8(y);
        if (codes != hi) codes = settle_codes(codes, hi, d, v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]);
        if (!scale) codes = 0;
    }
    if (bad) codes = 0, scale = NV ? 0x7fu : 0xffu;
}

// The four scale bytes of an atom's row, from the lanes that hold its blocks, in all of them.
template <bool NV>
__device__ __forceinline__ uint32_t gather_scales(uint32_t scale) {
    uint32_t w = scale << (8 * ((threadIdx.x & 31) / Mx<NV>::LANES % 4));
    w |= __shfl_xor_sync(0xffffffffu, w, Mx<NV>::LANES);
    w |= __shfl_xor_sync(0xffffffffu, w, 2 * Mx<NV>::LANES);
    return w;
}
// Place of row r's four bytes in atom `atom` (of `atoms` along K).
__device__ __forceinline__ size_t scale_word(uint32_t r, uint32_t atoms, uint32_t atom) {
    return ((size_t)(r >> 7) * atoms + atom) * 512 + (r & 31) * 16 + (r >> 5 & 3) * 4;
}

}  // namespace fq
