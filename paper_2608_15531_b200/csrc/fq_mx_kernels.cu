// Microscaled FP4 (sm_100a): quantising rows, also of a gated product or of the norm between two blocks, reading them back, and
// the launchers of these kernels and of the product (fq_mx_gemm_kernel.cuh).  The formats stand in fq.h.
//
// Every kernel is launched so that it may become resident while the grid before it drains (programmatic dependent
// launch), and executes griddepcontrol.wait before it reads or writes global memory: any array may come from that grid.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>

#include "fq_internal.h"
#include "fq_launch.h"
#include "fq_mx.cuh"
#include "fq_mx_gemm_kernel.cuh"
#include "fq_overlap.h"
#include "fq_ptx.cuh"
#include "fq_shares.h"

namespace fq {

static_assert(FQ_MX_WORKSPACE_BYTES == kWsHeaderBytes + kWsCounterBytes, "fq_check_status clears that much");

__device__ __forceinline__ void grid_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------------------------ quantising and reading back

// A warp takes 512 consecutive values, 16 to a lane (32 bytes of a 16-bit type: one load), of G rows that are 32 apart.  With
// G = 4 their scales share the 16-byte lines of an atom, and four loads are in flight; with G = 1 a small matrix is spread over
// more warps, and gated products, which are bound by instructions, keep to 64 registers (those of BF16 spill 8 and 20 bytes for it).  16 values are a
// block of FQ_NVFP4, whose scale (a quotient and its rounding) is then computed by one lane.
// Measured (28672 x 4096 of BF16): MXFP4 45.5 us (6.5 TB/s, the rate of a copy), reading back 46.2; NVFP4 55.9 (5.3 TB/s: 11.7 instructions a
// value, each rounded twice to see whether the quotient is near a border, 69 % of the issue slots).  That is with a tensor scale that no ratio of
// short numbers is.  With other ones quotients lie on borders all the time, as values of eight bits over scales of four do, and nearly every warp settles some one by
// one: with 1 BF16 takes 129 us and FP16 75.  FP32: 76.4 and 85.3.  Gated products, 4096 x 14336: 64.3 us (MXFP4, BF16;
// 28 instructions a value, 72 % of the issue slots, and two of them on the quarter-rate pipe) and 82 to 87 (NVFP4, FP16; about 40; with a tensor scale
// of 1 95, BF16 111).
struct MxParams {
    const void* a;               // X, or the gate
    const void* b;               // up
    uint64_t ld_a, ld_b;         // in values
    const float* ts;
    uint32_t* codes;
    uint8_t* scales;
    void* y;                     // (reading back)
    uint32_t rows, K, atoms, chunks;      // chunks of 512 values
    Divisor by_chunks;
    uint64_t tasks;
    int lie;                     // RowsLie
    uint32_t sms;
};
template <int G>
struct MxTask {
    uint32_t row0, k;            // the first of the rows, this lane's first value
    bool any;
    __device__ __forceinline__ explicit MxTask(const MxParams& p) {
        const uint64_t w = (uint64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
        uint64_t line;
        if ((p.tasks >> 32) == 0) line = p.by_chunks((uint32_t)w);
        else line = w / p.chunks;
        any = w < p.tasks;
        row0 = G == 1 ? (uint32_t)line : (uint32_t)(line >> 5) * (32 * G) + (uint32_t)(line & 31);
        k = (uint32_t)(w - line * p.chunks) * 512 + (threadIdx.x & 31) * 16;
    }
};
constexpr int kMxThreads = 256;

// gate / (1 + exp(-gate)) * up in binary32, off by at most 5.5 * 2^-23 of the result as long as the gate is not below -60 (far below that 1 +
// exp(-g) leaves binary32): 2^-22 (ex2), 2^-23 (rcp), four roundings and, BF16, half a unit.  exp(-g) is 2^t (1 + c) with
//   FP16   t = -g log2(e) as rounded, c = -g - t ln(2), what the rounding left (below 2^-17)
//   BF16   t = -g H, exact: H is log2(e) cut to 16 bits, and c = -g (log2(e) - H) ln(2), whose square (below 2^-23.3) is left out
template <class T>
__device__ __forceinline__ float gated(float g, float u) {
    float t, c;
    if constexpr (IsBf16<T>::value) {
        t = -1.44268798828125f * g;
        c = -4.88849543e-6f * g;
    } else {
        constexpr float L = 1.44269504f, N = 0.693147181f, N2 = -1.90465421e-9f;  // log2(e); ln(2) and what binary32 leaves of it
        t = -L * g;
        c = fmaf(-N2, t, fmaf(-N, t, -g));
    }
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    e = fmaf(e, c, e) + 1.0f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(e));
    return g * s * u;
}
__device__ __noinline__ float gated_exact(float g, float u) { return (float)((double)g / (1.0 + exp(-(double)g)) * (double)u); }

// A lane's 16 gated products, rounded to T and quantised.  The exact product lies between the computed one a little less and a little
// more; where both round alike that is the result.  Where some do not (1 in 4000 values of BF16, 1 in 500 of FP16), but
// give the same codes and scales, no matter (h itself is not put out); else (one in some thousand warps) the warp takes what
// is in question in binary64.  `again`: loads gate and up once more.
template <class T, bool NV, class F>
__device__ __forceinline__ void quantize_gated16(const Words8& gate, const Words8& up, F&& again, const TensorScale& ts, uint2& codes, uint32_t& scale) {
    constexpr float E = 0x1.8p-21f;                        // 6 * 2^-23: the bound, and half a unit for the step's rounding
    Words8 hi;                                             // the larger magnitude; the smaller one is hi, or the number below it where
    uint32_t below = 0;                                    // below has a bit: i and 16 + i for the two of word i
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 g = unpack2(gate.w[i], T()), u = unpack2(up.w[i], T());
        const float a = gated<T>(g.x, u.x), b = gated<T>(g.y, u.y);
        hi.w[i] = pack2(a * (1.0f + E), b * (1.0f + E), T());
        below += (hi.w[i] - pack2(a * (1.0f - E), b * (1.0f - E), T())) << i;
    }
    // the gate's bits as an unsigned number are above those of -60 where it is below -60 (or a NaN with a sign)
    constexpr bool BF = IsBf16<T>::value;
    constexpr uint32_t deep = BF ? 0xc270u : 0xd380u;
    const uint4 g0 = gate.half(0), g1 = gate.half(1);
    const uint32_t gm = max_u16x2(max_u16x2(max_u16x2(g0.x, g0.y), max_u16x2(g0.z, g0.w)), max_u16x2(max_u16x2(g1.x, g1.y), max_u16x2(g1.z, g1.w)));
    // products so small that binary32 may have lost bits on the way: only where a whole block is
    const uint32_t m = max_u16x2(max_magnitude(hi.half(0)), max_magnitude(hi.half(1)));
    const bool all = max(gm & 0xffffu, gm >> 16) > deep || (BF && max(m & 0xffffu, m >> 16) < 0x1780u && m);
    quantize16<NV, T>(hi, ts, codes, scale);
    if (__any_sync(0xffffffffu, below != 0 || all)) {
        Words8 lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) lo.w[i] = hi.w[i] - (below >> i & 0x10001u);
        uint2 other;
        uint32_t other_scale;
        quantize16<NV, T>(lo, ts, other, other_scale);
        if (__any_sync(0xffffffffu, all || other.x != codes.x || other.y != codes.y || other_scale != scale)) {
            Words8 g, u;
            again(g, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t ask = all ? 0x10001u : below >> i & 0x10001u;
                const float2 gi = unpack2(g.w[i], T()), ui = unpack2(u.w[i], T());
                if (ask & 0xffffu) hi.w[i] = (hi.w[i] & 0xffff0000u) | pack2(gated_exact(gi.x, ui.x), 0.0f, T());
                if (ask >> 16) hi.w[i] = (hi.w[i] & 0xffffu) | pack2(0.0f, gated_exact(gi.y, ui.y), T());
            }
            quantize16<NV, T>(hi, ts, codes, scale);
        }
    }
}

template <class T, bool NV, bool GATED, int G>
__global__ void __launch_bounds__(kMxThreads, sizeof(T) == 2 ? (GATED || NV ? 4 : 5) : 1) fq_mx_quantize_kernel(const MxParams p) {
    const MxTask<G> task(p);
    grid_start();
    if (!task.any) return;
    TensorScale ts;
    if constexpr (NV) ts.read(p.ts);
    const uint32_t k = task.k;
    constexpr bool F32 = sizeof(T) == 4, TWO = F32 || GATED;
    Words8 in[G], in2[TWO ? G : 1];                        // the second: values 8 to 15 of FP32, or up
    const bool inside = k < p.K;
    auto load = [&](int g, Words8& one, Words8& two) {
        const uint32_t r = task.row0 + 32 * g;
        if (inside && r < p.rows) {
            const T* a = (const T*)p.a + (uint64_t)r * p.ld_a + k;
            one = load32(a, p.lie);
            if constexpr (F32) two = load32(a + 8, p.lie);
            if constexpr (GATED) two = load32((const T*)p.b + (uint64_t)r * p.ld_b + k, p.lie);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) one.w[i] = two.w[i] = 0;
        }
    };
#pragma unroll
    for (int g = 0; g < G; ++g) load(g, in[g], in2[TWO ? g : 0]);
    uint32_t words[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const uint32_t r = task.row0 + 32 * g;
        uint2 codes;
        uint32_t scale;
        if constexpr (F32) quantize16<NV>(in[g], in2[g], ts, codes, scale);
        else if constexpr (GATED) quantize_gated16<T, NV>(in[g], in2[g], [&](Words8& a, Words8& b) { load(g, a, b); }, ts, codes, scale);
        else quantize16<NV, T>(in[g], ts, codes, scale);
        if (!inside) scale = 0;                                            // blocks beyond K
        words[g] = gather_scales<NV, 16>(scale);
        if (inside && r < p.rows) *reinterpret_cast<uint2*>(p.codes + (((uint64_t)r * p.K + k) >> 3)) = codes;
    }
    const uint32_t atom = k / Mx<NV, 16>::ATOM;
    if ((threadIdx.x & 31) % Mx<NV, 16>::ATOM_LANES == 0 && atom < p.atoms) {
        uint8_t* to = p.scales + scale_word(task.row0, p.atoms, atom);
        if (G == 4 && task.row0 + 96 < p.rows) {
            *reinterpret_cast<uint4*>(to) = make_uint4(words[0], words[1 % G], words[2 % G], words[3 % G]);
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (task.row0 + 32 * g < p.rows) reinterpret_cast<uint32_t*>(to)[g] = words[g];
        }
    }
}

template <class T, bool NV, int G>
__global__ void __launch_bounds__(kMxThreads) fq_mx_dequantize_kernel(const MxParams p) {
    const MxTask<G> task(p);
    grid_start();
    const uint32_t k = task.k;
    if (!task.any || k >= p.K) return;
    float ts = 1.0f;
    if (NV && p.ts) asm volatile("ld.global.f32 %0, [%1];" : "=f"(ts) : "l"(p.ts) : "memory");
    const uint32_t block = k / Mx<NV, 16>::BLOCK;
    const uint8_t* line = p.scales + scale_word(task.row0, p.atoms, block >> 2) + (block & 3);
    uint32_t codes[G][2], scale[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const uint32_t r = task.row0 + 32 * g;
        codes[g][0] = codes[g][1] = 0, scale[g] = 0;
        if (r < p.rows) {
            asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(codes[g][0]), "=r"(codes[g][1])
                         : "l"(p.codes + (((uint64_t)r * p.K + k) >> 3)) : "memory");
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(scale[g]) : "l"(line + 4 * g) : "memory");
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const uint32_t r = task.row0 + 32 * g, s = scale[g];
        if (r >= p.rows) return;
        float d;
        if constexpr (NV) d = (s & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : copysignf(e4m3_value(s & 0x7f), s & 0x80 ? -1.0f : 1.0f) * ts;
        else d = s == 255 ? __uint_as_float(0x7fc00000u) : (s ? __uint_as_float(s << 23) : 0x1p-127f);
        T* y = (T*)p.y + (uint64_t)r * p.ld_a + k;
        Words8 out;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
            e2m1_values8(codes[g][h], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= d;
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < 8; ++i) out.w[i] = __float_as_uint(v[i]);
                store32(y + 8 * h, p.lie, out);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) out.w[4 * h + i] = pack2(v[2 * i], v[2 * i + 1], T());
            }
        }
        if constexpr (sizeof(T) == 2) store32(y, p.lie, out);
    }
}

// -------------------------------------------------------------------------------------- the norms around a block

struct NormParams {
    const void *x, *block, *block_weight, *gate, *weight;
    void *r, *h;
    uint64_t ld_x, ld_block, ld_gate, ld_r, ld_h;
    const float* ts;
    uint32_t* codes;
    uint8_t* scales;
    uint32_t rows, D, atoms;
    float eps, alpha;
    bool vec;
};

// Sum over the TPR threads of a row, in all of them, in a fixed order.  `part`: one cell for each warp of the CTA.
template <int TPR>
__device__ __forceinline__ double row_sum(double s, double* part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = s;
        __syncthreads();
        s = part[threadIdx.x % W];                         // (a warp's lanes hold each cell 32 / W times)
#pragma unroll
        for (int o = W / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    }
    return s;
}

// A thread's 16 bytes to its own place in shared memory, asynchronously.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// CTAs to an SM that the registers have to allow: 768 threads (80 registers; 4096 rows of 4096 with 512 threads 55 us, 768 49, 1024 52 with
// spills), one CTA where each is alone on its SM.
constexpr int norm_ctas(int tpr, int v) { return v == 1 || tpr >= 768 ? 1 : 768 / (tpr < 128 ? 128 : tpr); }

// TPR threads to a row, V vectors of eight values to a thread, which stay in registers from the sum to the last store: one
// pass over the data.  A CTA goes through rows; the next row's values are on their way to shared memory meanwhile, to the other of two places (each
// thread copies and reads its own, so that no barrier is needed; values are read when they are wanted: with all of a row in registers 50 us).  Rows of up to 512 values share a CTA (TPR = 32, a warp to a row).
// Sums and results run in binary64.  In binary32 a value of H would cross a border of its type in 1 of 10^4 cases, and a code of every tenth
// million be a step off.  Only a gate and a weight are multiplied in binary32, exactly (8 + 8 or 11 + 11 bits), as long as the product is a normal number
// of it.  FP16 products always are; of BF16 a thread looks at its eight, and takes gate and weight one after the other where one is not (or is 0).
// Norm and gate, 4096 rows of 4096: BF16 49.2 us, FP16 47.7; one after the other throughout 50.8.  What bounds it: 62 instructions
// a value, half of them the sums over a row and what else a thread does once a row, on 61 % of the issue slots at three rows to an SM (80
// registers); six conversions a value from and to binary64 keep their pipe 50 % busy.  4096 rows of 4096, with a norm behind the block, a gate
// and everything put out 49 us (3.6 TB/s), without norm and gate 37; R and H alone 44 and 32.  Rows of more than 4096 columns have an SM to themselves,
// and above 8192 columns 64 registers are too few (52 to 200 bytes spilled): 4096 rows of 5120 104 and 74 us, of 8192 113 and 81; 2048 of 16384 118 and 83.
template <class T, int TPR, int V, int FORMAT>                             // FORMAT: FQ_MXFP4, FQ_NVFP4, or 2 for none
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, norm_ctas(TPR, V)) fq_norm_kernel(const NormParams p) {
    extern __shared__ uint4 ahead[];                       // [2][V][3][threads]: this and the next row's X, block and gate
    __shared__ double part[4][32];
    constexpr bool NV = FORMAT == (int)FQ_NVFP4;
    constexpr int RPC = TPR < 128 ? 128 / TPR : 1, THREADS = TPR * RPC;
    const uint32_t t = RPC > 1 ? threadIdx.x % TPR : threadIdx.x, stride = gridDim.x * RPC;
    uint32_t row = blockIdx.x * RPC + (RPC > 1 ? threadIdx.x / TPR : 0);
    const bool post = p.block_weight, gated = p.gate;
    const double inv_d = 1.0 / p.D;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto column = [&](int j) { return (j * TPR + t) * 8; };
    auto start = [&](uint32_t r, uint32_t half) {          // p.vec only: whole vectors
        if (r >= p.rows) return;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = column(j), to = smem_u32(ahead + (half * V + j) * 3 * THREADS + threadIdx.x);
            if (c >= p.D) continue;
            copy16(to, (const T*)p.x + r * p.ld_x + c);
            if (p.block) copy16(to + THREADS * 16, (const T*)p.block + r * p.ld_block + c);
            if (gated) copy16(to + 2 * THREADS * 16, (const T*)p.gate + r * p.ld_gate + c);
        }
    };
    uint32_t odd = 0;
    auto fetch = [&](const void* base, uint64_t at, int j, int slot) {
        const uint32_t c = column(j);
        if (!base || c >= p.D) return zero;
        if (p.vec) return ahead[((odd * V + j) * 3 + slot) * THREADS + threadIdx.x];
        return load_raw((const T*)base + at + c, (int)p.D - (int)c);
    };
    auto weight = [&](const void* base, int j, float (&v)[8]) {            // (from the L1 after the first row)
        const uint32_t c = column(j);
        uint4 q = zero;
        if (c < p.D) q = p.vec ? *reinterpret_cast<const uint4*>((const T*)base + c) : load_raw((const T*)base + c, (int)p.D - (int)c);
        unpack8<T>(q, v);
    };
    grid_start();
    if (p.vec) start(row, 0);
    TensorScale ts;
    if constexpr (NV) ts.read(p.ts);
    for (; row < p.rows; row += stride, odd ^= 1) {        // (whole warps; all warps of a CTA of one row)
        if (p.vec) asm volatile("cp.async.wait_all;" ::: "memory");
        if (p.vec) start(row + stride, odd ^ 1);
        double r[V][8];
        double c1 = p.alpha;
        if (post) {
            double s[2] = {0.0, 0.0};
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v[8];
                unpack8<T>(fetch(p.block, row * p.ld_block, j, 1), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    r[j][i] = (double)v[i];
                    s[i & 1] = fma(r[j][i], r[j][i], s[i & 1]);
                }
            }
            c1 *= rsqrt(fma(row_sum<TPR>(s[0] + s[1], part[odd]), inv_d, (double)p.eps));
        }
        double s[2] = {0.0, 0.0};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float v[8], b[8];
            if (p.block) {
                if (!post) {
                    unpack8<T>(fetch(p.block, row * p.ld_block, j, 1), v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[j][i] = (double)v[i];
                }
                if (post || gated) {
                    if (gated) unpack8<T>(fetch(p.gate, row * p.ld_gate, j, 2), b);
                    if (post) {
                        weight(p.block_weight, j, v);
                        bool together = true;
                        if (gated && IsBf16<T>::value) {
                            float most = 0.0f, least = 0x1p-126f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(b[i] * v[i])), least = fminf(least, fabsf(b[i] * v[i]));
                            together = most <= 0x1.fffffep127f && least >= 0x1p-126f;
                        }
                        if (!together) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) r[j][i] *= (double)v[i];
                        } else {
#pragma unroll
                            for (int i = 0; i < 8; ++i) b[i] = gated ? b[i] * v[i] : v[i];
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) r[j][i] *= (double)b[i];
                }
            }
            unpack8<T>(fetch(p.x, row * p.ld_x, j, 0), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                r[j][i] = p.block ? fma(r[j][i], c1, (double)v[i]) : (double)v[i];
                s[i & 1] = fma(r[j][i], r[j][i], s[i & 1]);
            }
        }
        if (p.r) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint32_t c = column(j);
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (float)r[j][i];
                if (c < p.D) store_raw((T*)p.r + row * p.ld_r + c, (int)p.D - (int)c, p.vec, pack8<T>(v));
            }
        }
        if (!p.h && FORMAT == 2) continue;
        const double rstd = rsqrt(fma(row_sum<TPR>(s[0] + s[1], part[2 + odd]), inv_d, (double)p.eps));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = column(j);
            const int n = (int)p.D - (int)c;
            float f[8], b[8];
            if (p.weight) {
                weight(p.weight, j, b);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = 1.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = (float)(r[j][i] * rstd * (double)b[i]);
            const uint4 h = pack8<T>(f);
            if (p.h && n > 0) store_raw((T*)p.h + row * p.ld_h + c, n, p.vec, h);
            if constexpr (FORMAT != 2) {
                uint32_t codes, scale;
                quantize8<NV, T>(n > 0 ? h : zero, ts, codes, scale);
                if (n <= 0) scale = 0;
                const uint32_t word = gather_scales<NV, 8>(scale), atom = c / Mx<NV, 8>::ATOM;
                if (n > 0) p.codes[((uint64_t)row * p.D + c) >> 3] = codes;
                if (t % Mx<NV, 8>::ATOM_LANES == 0 && atom < p.atoms) *reinterpret_cast<uint32_t*>(p.scales + scale_word(row, p.atoms, atom)) = word;
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------ launches

template <class... P, class... A>
static fq_status_t launch(void (*fn)(P...), dim3 grid, uint32_t threads, uint32_t smem, uint32_t cluster, void* stream, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute at[2];
    std::memset(at, 0, sizeof(at));
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, std::forward<A>(args)...);
    return e == cudaSuccess ? FQ_OK : fail(FQ_ERR_CUDA, "kernel launch: %s", cudaGetErrorString(e));
}

static inline uint32_t mx_block(uint32_t format) { return format == FQ_NVFP4 ? 16 : 32; }
static inline uint32_t mx_atoms(const fq_mx_layout_t* L) { return (L->K / mx_block(L->format) + 3) / 4; }
static inline size_t mx_code_bytes(const fq_mx_layout_t* L) { return (size_t)L->rows * L->K / 2; }
static inline size_t mx_scale_bytes(const fq_mx_layout_t* L) { return ((size_t)L->rows + 127) / 128 * mx_atoms(L) * 512; }
static inline size_t type_bytes(uint32_t type) { return type == FQ_TYPE_FP32 ? 4 : 2; }

static bool mx_layout_ok(const fq_mx_layout_t* L) {
    return L && L->abi == FQ_ABI_VERSION && L->format <= FQ_NVFP4 && L->rows && L->rows <= FQ_MX_MAX_ROWS && L->K && L->K % 32 == 0 && L->K <= FQ_MX_MAX_K;
}

static fq_status_t check_stride(const char* what, const void* p, uint64_t rows, uint64_t cols, uint64_t ld, size_t size) {
    if (!aligned(p, size)) return fail(FQ_ERR_INVALID_ARG, "%s is misaligned", what);
    if ((rows > 1 && ld < cols) || ld > (1ull << 40) || (rows - 1) > (1ull << 56) / (ld + 1)) return fail(FQ_ERR_INVALID_ARG, "%s: row stride %llu for %llu columns", what, (unsigned long long)ld, (unsigned long long)cols);
    return FQ_OK;
}
static fq_status_t check_mx(const fq_mx_layout_t* L, const void* codes, const void* scales, const float* ts) {
    if (!mx_layout_ok(L)) return fail(FQ_ERR_INVALID_ARG, "bad layout");
    if (!codes || !scales) return fail(FQ_ERR_INVALID_ARG, "null codes or scales");
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(ts, 4)) return fail(FQ_ERR_INVALID_ARG, "misaligned codes, scales or tensor scale");
    if (ts && L->format != FQ_NVFP4) return fail(FQ_ERR_INVALID_ARG, "FQ_MXFP4 has no tensor scale");
    return FQ_OK;
}
static bool rows_aligned(const void* p, uint64_t ld, size_t size, uint64_t rows, size_t to = 16) { return aligned(p, to) && (rows <= 1 || ld * size % to == 0); }
static int rows_lie(const void* p, uint64_t ld, size_t size, uint64_t rows) {
    return rows_aligned(p, ld, size, rows, 32) ? kVec32 : rows_aligned(p, ld, size, rows) ? kVec16 : kOdd;
}

static MxParams mx_params(const fq_mx_layout_t* L, const float* ts) {
    MxParams p;
    std::memset(&p, 0, sizeof(p));
    p.ts = ts;
    p.rows = L->rows, p.K = L->K, p.atoms = mx_atoms(L);
    p.chunks = (L->K + 511) / 512;
    p.by_chunks = Divisor::of(p.chunks);
    p.sms = (uint32_t)std::max(sm_count_cached(), 1);      // (without a device the launch reports it)
    return p;
}
typedef void (*MxFn)(const MxParams);
// Rows that a warp takes: four for large matrices (28672 x 4096 of BF16, MXFP4, us, one / four 51.0 / 45.3, NVFP4 74.2 / 55.9, read back 48.6 /
// 46.1; 8192 x 4096 15.9 / 15.8, 22.6 / 19.3, 14.9 / 13.4), one for others, whose time is that of a warp (4096 x 4096 8.9 / 9.7, 12.4 / 12.0, 8.2 / 7.7;
// 1024 x 4096 2.9 / 3.4, 3.9 / 4.9, 3.1 / 3.2).
static bool one_row_tasks(const MxParams& p) { return (uint64_t)p.rows * p.chunks <= 256ull * p.sms; }
template <class T, bool GATED>
static MxFn pick_quantize(bool nv, bool one) {
    constexpr int G = GATED ? 1 : 4;
    if (nv) return one ? (MxFn)fq_mx_quantize_kernel<T, true, GATED, 1> : (MxFn)fq_mx_quantize_kernel<T, true, GATED, G>;
    return one ? (MxFn)fq_mx_quantize_kernel<T, false, GATED, 1> : (MxFn)fq_mx_quantize_kernel<T, false, GATED, G>;
}
template <class T>
static MxFn pick_dequantize(bool nv, bool one) {
    if (nv) return one ? (MxFn)fq_mx_dequantize_kernel<T, true, 1> : (MxFn)fq_mx_dequantize_kernel<T, true, 4>;
    return one ? (MxFn)fq_mx_dequantize_kernel<T, false, 1> : (MxFn)fq_mx_dequantize_kernel<T, false, 4>;
}
// G: rows that a task takes
static fq_status_t launch_mx(MxFn fn, MxParams& p, uint32_t G, void* stream) {
    // lines of tasks: the first 32 rows of each 32 G (rows 32 further on go with them)
    p.tasks = ((uint64_t)(p.rows / (32 * G)) * 32 + std::min<uint32_t>(p.rows % (32 * G), 32)) * p.chunks;
    // few warps in CTAs of two, so that they are spread over the SMs (MXFP4, us, two / eight warps: 256 x 4096 1.7 / 1.8, 512 x 4096 2.7 / 2.3)
    const uint32_t threads = p.tasks <= 16ull * p.sms ? 64 : kMxThreads;
    const uint64_t warps = threads / 32, ctas = (p.tasks + warps - 1) / warps;
    if (ctas > 0x7fffffffull) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "matrix too large for one launch");
    return launch(fn, dim3((uint32_t)ctas), threads, 0, 1, stream, p);
}

typedef void (*NormFn)(const NormParams);
// `tpr`: threads to a row, `v`: vectors of eight to a thread.  Two, which halves what a thread spends on the sums over the row (4096 rows
// of 4096 49 us, with one 66); but one where every row has an SM to itself and only latency counts.
template <class T, int FORMAT>
static NormFn pick_norm(uint32_t D, bool few, uint32_t& tpr, uint32_t& v) {
    const uint32_t vectors = (D + 7) / 8;
    if (few) {
        v = 1;
        if (vectors <= 128) return tpr = 128, (NormFn)fq_norm_kernel<T, 128, 1, FORMAT>;
        if (vectors <= 256) return tpr = 256, (NormFn)fq_norm_kernel<T, 256, 1, FORMAT>;
        if (vectors <= 512) return tpr = 512, (NormFn)fq_norm_kernel<T, 512, 1, FORMAT>;
        if (vectors <= 1024) return tpr = 1024, (NormFn)fq_norm_kernel<T, 1024, 1, FORMAT>;
    }
    v = 2;
    if (vectors <= 64) return tpr = 32, (NormFn)fq_norm_kernel<T, 32, 2, FORMAT>;
    if (vectors <= 256) return tpr = 128, (NormFn)fq_norm_kernel<T, 128, 2, FORMAT>;
    if (vectors <= 512) return tpr = 256, (NormFn)fq_norm_kernel<T, 256, 2, FORMAT>;
    if (vectors <= 1024) return tpr = 512, (NormFn)fq_norm_kernel<T, 512, 2, FORMAT>;
    return tpr = 1024, (NormFn)fq_norm_kernel<T, 1024, 2, FORMAT>;
}
template <class T>
static NormFn pick_norm(int format, uint32_t D, bool few, uint32_t& tpr, uint32_t& v) {
    if (format == (int)FQ_MXFP4) return pick_norm<T, (int)FQ_MXFP4>(D, few, tpr, v);
    if (format == (int)FQ_NVFP4) return pick_norm<T, (int)FQ_NVFP4>(D, few, tpr, v);
    return pick_norm<T, 2>(D, few, tpr, v);
}
// CTAs of a persistent kernel that fit on an SM, asked once per kernel (all devices are alike: sm_100a).
static int ctas_per_sm(const void* fn, int threads, size_t smem) {
    struct Seen { const void* fn; int n; };
    static Seen seen[64];
    static int count = 0;
    static std::mutex mu;
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < count; ++i)
        if (seen[i].fn == fn) return seen[i].n;
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, fn, threads, smem) != cudaSuccess || n < 1) {
        cudaGetLastError();
        return 1;
    }
    if (count < 64) seen[count++] = Seen{fn, n};
    return n;
}

// ---- the product

// Codes of a matrix: rows of K/2 bytes; a copy takes 128 bytes (256 codes) of `rows` rows, swizzled.
static fq_status_t encode_codes(EncodeFn fn, const fq_mx_layout_t* L, const void* codes, uint32_t rows, CUtensorMap* map) {
    const cuuint64_t dims[2] = {L->K / 2, L->rows}, strides[1] = {L->K / 2};
    const cuuint32_t box[2] = {128, rows}, ones[2] = {1, 1};
    const CUresult e = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, (void*)codes, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return e == CUDA_SUCCESS ? FQ_OK : fail(FQ_ERR_CUDA, "cuTensorMapEncodeTiled: %d", (int)e);
}
// Its scales: atoms of 128 words, in a row tile's order along K; a copy takes `atoms` of `tiles` row tiles (beyond K: zeros).
static fq_status_t encode_scales(EncodeFn fn, const fq_mx_layout_t* L, const void* scales, uint32_t atoms, uint32_t tiles, CUtensorMap* map) {
    const cuuint64_t dims[3] = {128, mx_atoms(L), (L->rows + 127) / 128}, strides[2] = {512, (cuuint64_t)mx_atoms(L) * 512};
    const cuuint32_t box[3] = {128, atoms, tiles}, ones[3] = {1, 1, 1};
    const CUresult e = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, (void*)scales, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return e == CUDA_SUCCESS ? FQ_OK : fail(FQ_ERR_CUDA, "cuTensorMapEncodeTiled: %d", (int)e);
}

template <class T, int NT, bool NV>
static fq_status_t launch_mx_gemm(const fq_mx_layout_t* LX, const void* xc, const void* xs, const fq_mx_layout_t* LW, const void* wc, const void* ws,
                                  MxGemmParams& p, uint32_t sms, void* stream) {
    using G = MxGemm<NT, NV>;
    const EncodeFn enc = tensor_map_encoder();
    if (!enc) return fail(FQ_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
    CUtensorMap mw, mx, mws, mxs;
    fq_status_t st;
    if ((st = encode_codes(enc, LW, wc, 128, &mw)) != FQ_OK || (st = encode_codes(enc, LX, xc, NT, &mx)) != FQ_OK ||
        (st = encode_scales(enc, LW, ws, G::ATOMS, 1, &mws)) != FQ_OK || (st = encode_scales(enc, LX, xs, G::ATOMS, 1, &mxs)) != FQ_OK)
        return st;
    p.tiles_m = (LX->rows + NT - 1) / NT;
    const uint64_t tiles = (uint64_t)p.tiles_m * ((LW->rows + 127) / 128);
    if (tiles > 0x7fffffffull) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "too many tiles");
    p.tiles = (uint32_t)tiles;
    p.steps = (p.K + kMxStageK - 1) / kMxStageK;
    // The steps of a tile over up to eight CTAs.  The first halving costs an exchange of about a microsecond (more tokens: two), each
    // halving saves 0.18 us for each step of a CTA that it takes away, and CTAs that share an SM, or wait for one, lose it again.
    // So: from 16 steps (more than 32 tokens: 32) while a CTA has 8 (16), on as many CTAs as there are SMs, or twice that where the tile is
    // already split.  us for 1, 2, 4, 8 CTAs: 8 steps, 64 tiles, one token 3.7, 4.4, 4.5, 9.0; 16 steps, 32 tiles 5.2, 4.8, 4.5, 4.9, 64 tokens
    // 5.2, 5.9, 6.8, 7.8; 56 steps, 32 tiles 12.0, 9.7, 9.0, 8.5, 64 tokens 12.8, 10.7, 10.2, 11.5; 12 steps, 87 tiles 6.6, 7.7, 11, 15.
    // Clusters of four and eight do not fill every group of SMs: an eighth is left out of the count (16 steps, 34 tiles of eight CTAs, two to
    // an SM, 8.1 us, of four 4.5).
    constexpr uint32_t least = NT <= 32 ? 8 : 16;
    const uint32_t most = sms - sms / 8;
    p.split = 1;
    while (p.split < 8 && p.steps >= 2 * least && p.steps >= least * p.split &&
           p.tiles * p.split * 2 <= (p.split == 1 ? sms : (NT <= 32 ? 2 : 1) * most))
        p.split *= 2;
    const uint32_t grid = p.split > 1 ? p.tiles * p.split : std::min(p.tiles, 2 * sms);
    // a CTA that has its SM to itself, and more steps than the shorter ring holds, gets all of the shared memory (4096 x 4096, 128 tokens:
    // three stages 7.8 us, six 5.8; 11133 x 2976, 77 tokens, 12.0 and 9.9), but not where its cluster would then wait for SMs (36 tiles of four CTAs,
    // 32 steps, one token: 11.6 us, with the shorter ring 7.0)
    const uint32_t alone = p.split == 8 ? sms - sms / 4 : p.split == 4 ? most : sms;
    p.stages = grid <= alone && (p.steps + p.split - 1) / p.split > G::STAGES ? G::STAGES_ALONE : G::STAGES;
    const auto fn = fq_mx_gemm_kernel<T, NT, NV>;
    const uint32_t smem = p.stages * G::STAGE + 1024;
    const cudaError_t e = ensure_smem_attr((const void*)fn, (int)(G::STAGES_ALONE * G::STAGE + 1024));
    if (e != cudaSuccess) return fail(FQ_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    return launch(fn, dim3(grid), G::THREADS, smem, p.split, stream, mw, mx, mws, mxs, p);
}
template <class T, bool NV>
static fq_status_t launch_mx_pair(const fq_mx_layout_t* LX, const void* xc, const void* xs, const fq_mx_layout_t* LW, const void* wc, const void* ws,
                                  const MxGemmParams& g, uint32_t tokens, uint32_t sms, void* stream) {
    using G = MxPair<NV>;
    const EncodeFn enc = tensor_map_encoder();
    if (!enc) return fail(FQ_ERR_CUDA, "cuTensorMapEncodeTiled is not available");
    CUtensorMap mw, mx, mws, mxs;
    fq_status_t st;
    if ((st = encode_codes(enc, LW, wc, 128, &mw)) != FQ_OK || (st = encode_codes(enc, LX, xc, tokens / 2, &mx)) != FQ_OK ||
        (st = encode_scales(enc, LW, ws, G::ATOMS, 1, &mws)) != FQ_OK || (st = encode_scales(enc, LX, xs, G::ATOMS, tokens / 128, &mxs)) != FQ_OK)
        return st;
    MxPairParams p;
    std::memset(&p, 0, sizeof(p));
    p.Y = g.Y, p.ldy = g.ldy, p.ts_x = g.ts_x, p.ts_w = g.ts_w, p.status = g.status, p.M = g.M, p.N = g.N, p.K = g.K;
    p.tokens = tokens;
    p.tiles_m = (p.M + tokens - 1) / tokens;
    const uint64_t tiles = (uint64_t)p.tiles_m * ((p.N + 255) / 256);
    if (tiles > 0x7fffffffull) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "too many tiles");
    p.tiles = (uint32_t)tiles;
    p.steps = (p.K + kMxStageK - 1) / kMxStageK;
    p.stages = G::STAGES;
    const auto fn = fq_mx_pair_kernel<T, NV>;
    const uint32_t smem = p.stages * G::STAGE + 1024;
    const cudaError_t e = ensure_smem_attr((const void*)fn, (int)smem);
    if (e != cudaSuccess) return fail(FQ_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    return launch(fn, dim3(2 * std::min(p.tiles, sms / 2)), 32 * kPairWarps, smem, 1, stream, mw, mx, mws, mxs, p);
}
// Tokens of a tile of the pair kernel, 128 or 256: what leaves the busiest pair the fewest bytes to copy, which is what its time goes by (a step's
// codes and scales of 256 features, and of the tokens that a tile has).  us, tiles of 128 / 256, tokens x K x features: 129 x 4096 x 19200 15.0 / 14.1,
// 200 x 4096 x 28672 19.9 / 16.4, 2048 x 4096 x 4096 17.9 / 15.4, 640 x 4096 x 28672 37.4 / 32.9; 1024 x 4096 x 6144, the other way, 14.4 / 14.7.
static uint32_t pair_tokens(uint32_t M, uint32_t N, uint32_t sms) {
    auto work = [&](uint32_t t) {
        const uint64_t tiles_m = (M + t - 1) / t, tiles = tiles_m * ((N + 255) / 256), pairs = sms / 2;
        return (tiles + pairs - 1) / pairs * (19 + M / tiles_m / 16);
    };
    return work(128) < work(256) ? 128 : 256;
}
template <class T, bool NV>
static fq_status_t launch_mx_gemm(const fq_mx_layout_t* LX, const void* xc, const void* xs, const fq_mx_layout_t* LW, const void* wc, const void* ws,
                                  MxGemmParams& p, uint32_t sms, void* stream) {
    if (p.M <= 16) return launch_mx_gemm<T, 16, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
    if (p.M <= 32) return launch_mx_gemm<T, 32, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
    if (p.M <= 64) return launch_mx_gemm<T, 64, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
    // More than 128 tokens: single CTAs while each of their tiles has an SM (K 4096, 4096 features, 512 tokens, 128 tiles, 6.8 us, pairs 7.7; K 14336, 4096
    // features, 256 tokens, 13.2 and 15.3), pairs beyond (K 4096, 4096 features, 2048 tokens, 17.7 and 15.4; K 14336 51 and 41).
    if (p.M > 128 && (uint64_t)((p.M + 127) / 128) * ((p.N + 127) / 128) > sms && sms >= 2)
        return launch_mx_pair<T, NV>(LX, xc, xs, LW, wc, ws, p, pair_tokens(p.M, p.N, sms), sms, stream);
    return launch_mx_gemm<T, 128, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
}

}  // namespace fq

using namespace fq;

extern "C" {

fq_status_t fq_mx_get_layout(uint32_t rows, uint32_t K, uint32_t format, fq_mx_layout_t* out) {
    if (!out) return fail(FQ_ERR_INVALID_ARG, "null output");
    if (format > FQ_NVFP4) return fail(FQ_ERR_INVALID_ARG, "format = %u", format);
    if (rows == 0) return fail(FQ_ERR_INVALID_ARG, "no rows");
    if (K == 0 || K % 32 || K > FQ_MX_MAX_K) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "K = %u is not a multiple of 32 in [32, %u]", K, FQ_MX_MAX_K);
    if (rows > FQ_MX_MAX_ROWS) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "%u rows, at most %u", rows, FQ_MX_MAX_ROWS);
    std::memset(out, 0, sizeof(*out));
    out->abi = FQ_ABI_VERSION, out->rows = rows, out->K = K, out->format = format;
    return FQ_OK;
}

fq_status_t fq_mx_sizes(const fq_mx_layout_t* L, size_t* code_bytes, size_t* scale_bytes) {
    if (!mx_layout_ok(L) || !code_bytes || !scale_bytes) return fail(FQ_ERR_INVALID_ARG, "bad layout or null output");
    *code_bytes = mx_code_bytes(L), *scale_bytes = mx_scale_bytes(L);
    return FQ_OK;
}

fq_status_t fq_mx_quantize(const fq_mx_layout_t* L, const void* X, uint32_t type, uint64_t ldx, const float* tensor_scale,
                           void* codes, void* scales, void* cuda_stream) {
    fq_status_t st = check_mx(L, codes, scales, tensor_scale);
    if (st != FQ_OK) return st;
    if (!X) return fail(FQ_ERR_INVALID_ARG, "null X");
    if (type > FQ_TYPE_FP32) return fail(FQ_ERR_INVALID_ARG, "type = %u", type);
    const size_t size = type_bytes(type);
    if ((st = check_stride("X", X, L->rows, L->K, ldx, size)) != FQ_OK) return st;
    const Piece out[2] = {{codes, mx_code_bytes(L)}, {scales, mx_scale_bytes(L)}}, in[2] = {matrix(X, L->rows, L->K, ldx, size), {tensor_scale, 4}};
    if (!disjoint(out, 2, in, 2)) return fail(FQ_ERR_INVALID_ARG, "an output overlaps another array of the call");
    MxParams p = mx_params(L, tensor_scale);
    p.a = X, p.ld_a = ldx, p.codes = (uint32_t*)codes, p.scales = (uint8_t*)scales;
    p.lie = rows_lie(X, ldx, size, L->rows);
    const bool nv = L->format == FQ_NVFP4, one = one_row_tasks(p);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_quantize<__nv_bfloat16, false>(nv, one) : type == FQ_TYPE_FP16 ? pick_quantize<__half, false>(nv, one)
                                                                                                               : pick_quantize<float, false>(nv, one), p, one ? 1 : 4, cuda_stream);
}

fq_status_t fq_mx_quantize_swiglu(const fq_mx_layout_t* L, const void* gate, uint64_t ld_gate, const void* up, uint64_t ld_up,
                                  uint32_t type, const float* tensor_scale, void* codes, void* scales, void* cuda_stream) {
    fq_status_t st = check_mx(L, codes, scales, tensor_scale);
    if (st != FQ_OK) return st;
    if (!gate || !up) return fail(FQ_ERR_INVALID_ARG, "null gate or up");
    if (type > FQ_TYPE_FP16) return fail(FQ_ERR_INVALID_ARG, "type = %u", type);
    if ((st = check_stride("gate", gate, L->rows, L->K, ld_gate, 2)) != FQ_OK || (st = check_stride("up", up, L->rows, L->K, ld_up, 2)) != FQ_OK) return st;
    const Piece out[2] = {{codes, mx_code_bytes(L)}, {scales, mx_scale_bytes(L)}};
    const Piece in[3] = {matrix(gate, L->rows, L->K, ld_gate, 2), matrix(up, L->rows, L->K, ld_up, 2), {tensor_scale, 4}};
    if (!disjoint(out, 2, in, 3)) return fail(FQ_ERR_INVALID_ARG, "an output overlaps another array of the call");
    MxParams p = mx_params(L, tensor_scale);
    p.a = gate, p.ld_a = ld_gate, p.b = up, p.ld_b = ld_up, p.codes = (uint32_t*)codes, p.scales = (uint8_t*)scales;
    p.lie = std::min(rows_lie(gate, ld_gate, 2, L->rows), rows_lie(up, ld_up, 2, L->rows));
    const bool nv = L->format == FQ_NVFP4, one = one_row_tasks(p);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_quantize<__nv_bfloat16, true>(nv, one) : pick_quantize<__half, true>(nv, one), p, 1, cuda_stream);
}

fq_status_t fq_mx_dequantize(const fq_mx_layout_t* L, const void* codes, const void* scales, const float* tensor_scale, void* Y,
                             uint32_t type, uint64_t ldy, void* cuda_stream) {
    fq_status_t st = check_mx(L, codes, scales, tensor_scale);
    if (st != FQ_OK) return st;
    if (!Y) return fail(FQ_ERR_INVALID_ARG, "null Y");
    if (type > FQ_TYPE_FP32) return fail(FQ_ERR_INVALID_ARG, "type = %u", type);
    const size_t size = type_bytes(type);
    if ((st = check_stride("Y", Y, L->rows, L->K, ldy, size)) != FQ_OK) return st;
    const Piece out[1] = {matrix(Y, L->rows, L->K, ldy, size)}, in[3] = {{codes, mx_code_bytes(L)}, {scales, mx_scale_bytes(L)}, {tensor_scale, 4}};
    if (!disjoint(out, 1, in, 3)) return fail(FQ_ERR_INVALID_ARG, "Y overlaps another array of the call");
    MxParams p = mx_params(L, tensor_scale);
    p.y = Y, p.ld_a = ldy, p.codes = (uint32_t*)codes, p.scales = (uint8_t*)scales;      // (read)
    p.lie = rows_lie(Y, ldy, size, L->rows);
    const bool nv = L->format == FQ_NVFP4, one = one_row_tasks(p);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_dequantize<__nv_bfloat16>(nv, one) : type == FQ_TYPE_FP16 ? pick_dequantize<__half>(nv, one)
                                                                                                          : pick_dequantize<float>(nv, one), p, one ? 1 : 4, cuda_stream);
}

fq_status_t fq_norm_block(const fq_norm_args_t* a, void* cuda_stream) {
    if (!a) return fail(FQ_ERR_INVALID_ARG, "null arguments");
    if (!a->rows || a->rows > FQ_MX_MAX_ROWS) return fail(FQ_ERR_INVALID_ARG, "%u rows", a->rows);
    if (!a->D || a->D > FQ_NORM_MAX_D) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "D = %u outside [1, %u]", a->D, FQ_NORM_MAX_D);
    if (a->type > FQ_TYPE_FP16) return fail(FQ_ERR_INVALID_ARG, "type = %u", a->type);
    if (!a->X) return fail(FQ_ERR_INVALID_ARG, "null X");
    if (!(a->eps >= 0.0f)) return fail(FQ_ERR_INVALID_ARG, "eps = %g", (double)a->eps);
    if (!a->R && !a->H && !a->codes) return fail(FQ_ERR_INVALID_ARG, "no output");
    if (!a->block && (a->block_weight || a->gate)) return fail(FQ_ERR_INVALID_ARG, "a weight or gate without a block");
    fq_status_t st;
    const bool quantised = a->codes || a->scales || a->layout || a->tensor_scale;
    if (quantised) {
        if ((st = check_mx(a->layout, a->codes, a->scales, a->tensor_scale)) != FQ_OK) return st;
        if (a->layout->rows != a->rows || a->layout->K != a->D) return fail(FQ_ERR_INVALID_ARG, "the layout is %u x %u", a->layout->rows, a->layout->K);
    }
    const uint64_t rows = a->rows, D = a->D;
    const bool one_gate = a->gate && a->ld_gate == 0;
    struct Matrix { const char* name; const void* p; uint64_t ld; bool single; };
    const Matrix all[5] = {{"X", a->X, a->ld_x, false}, {"block", a->block, a->ld_block, false}, {"gate", a->gate, a->ld_gate, one_gate}, {"R", a->R, a->ld_r, false}, {"H", a->H, a->ld_h, false}};
    bool vec = a->D % 8 == 0 && aligned(a->block_weight, 16) && aligned(a->weight, 16);
    for (const Matrix& m : all) {
        if (!m.p) continue;
        if ((st = check_stride(m.name, m.p, m.single ? 1 : rows, D, m.ld, 2)) != FQ_OK) return st;
        vec = vec && rows_aligned(m.p, m.ld, 2, m.single ? 1 : rows);
    }
    if (!aligned(a->block_weight, 2) || !aligned(a->weight, 2)) return fail(FQ_ERR_INVALID_ARG, "a weight is misaligned");
    const Piece out[4] = {matrix(a->R, rows, D, a->ld_r, 2), matrix(a->H, rows, D, a->ld_h, 2),
                          {a->codes, quantised ? mx_code_bytes(a->layout) : 0}, {a->scales, quantised ? mx_scale_bytes(a->layout) : 0}};
    const Piece in[6] = {matrix(a->X, rows, D, a->ld_x, 2), matrix(a->block, rows, D, a->ld_block, 2), matrix(a->gate, one_gate ? 1 : rows, D, a->ld_gate, 2),
                         {a->block_weight, (size_t)D * 2}, {a->weight, (size_t)D * 2}, {a->tensor_scale, 4}};
    // in place: a thread has read its values of X and block before it writes R or H there
    const uint64_t ld_out[2] = {a->ld_r, a->ld_h}, ld_in[2] = {a->ld_x, a->ld_block};
    bool ok = true;
    for (int i = 0; i < 4 && ok; ++i) {
        for (int j = i + 1; j < 4; ++j) ok = ok && !out[i].overlaps(out[j]);
        for (int j = 0; j < 6; ++j) {
            const bool in_place = i < 2 && j < 2 && out[i].p == in[j].p && (rows == 1 || ld_out[i] == ld_in[j]);
            ok = ok && (in_place || !out[i].overlaps(in[j]));
        }
    }
    if (!ok) return fail(FQ_ERR_INVALID_ARG, "an output overlaps another array of the call");
    NormParams p;
    std::memset(&p, 0, sizeof(p));
    p.x = a->X, p.block = a->block, p.block_weight = a->block_weight, p.gate = a->gate, p.weight = a->weight, p.r = a->R, p.h = a->H;
    p.ld_x = a->ld_x, p.ld_block = a->ld_block, p.ld_gate = a->ld_gate, p.ld_r = a->ld_r, p.ld_h = a->ld_h;
    p.ts = a->tensor_scale, p.codes = (uint32_t*)a->codes, p.scales = (uint8_t*)a->scales;
    p.rows = a->rows, p.D = a->D, p.atoms = quantised ? mx_atoms(a->layout) : 0, p.eps = a->eps, p.alpha = a->residual_scale;
    const int format = quantised ? (int)a->layout->format : 2;
    p.vec = vec;
    const int sms = sm_count_cached();
    if (sms <= 0) return fail(FQ_ERR_CUDA, "no CUDA device: %s", cudaGetErrorString(cudaGetLastError()));
    uint32_t tpr = 0, v = 0;
    const bool few = a->rows <= (uint32_t)sms;
    const NormFn fn = a->type == FQ_TYPE_BF16 ? pick_norm<__nv_bfloat16>(format, a->D, few, tpr, v) : pick_norm<__half>(format, a->D, few, tpr, v);
    const uint32_t threads = std::max<uint32_t>(tpr, 128), per = threads / tpr, smem = 96 * v * threads;
    const cudaError_t e = ensure_smem_attr((const void*)fn, (int)smem);
    if (e != cudaSuccess) return fail(FQ_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    const uint32_t grid = std::min<uint32_t>((a->rows + per - 1) / per, (uint32_t)(sms * ctas_per_sm((const void*)fn, (int)threads, smem)));
    return launch(fn, dim3(grid), threads, smem, 1, cuda_stream, p);
}

fq_status_t fq_mx_gemm(const fq_mx_layout_t* LX, const void* x_codes, const void* x_scales, const float* x_tensor_scale,
                       const fq_mx_layout_t* LW, const void* w_codes, const void* w_scales, const float* w_tensor_scale, void* Y,
                       uint32_t type, uint64_t ldy, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    fq_status_t st = check_mx(LX, x_codes, x_scales, x_tensor_scale);
    if (st != FQ_OK || (st = check_mx(LW, w_codes, w_scales, w_tensor_scale)) != FQ_OK) return st;
    if (LX->K != LW->K || LX->format != LW->format) return fail(FQ_ERR_INVALID_ARG, "the layouts differ in K or format");
    if (!Y || !workspace) return fail(FQ_ERR_INVALID_ARG, "null Y or workspace");
    if (type > FQ_TYPE_FP32) return fail(FQ_ERR_INVALID_ARG, "type = %u", type);
    if (!aligned(workspace, 16)) return fail(FQ_ERR_INVALID_ARG, "misaligned workspace");
    if (workspace_bytes < FQ_MX_WORKSPACE_BYTES) return fail(FQ_ERR_BUFFER_TOO_SMALL, "workspace holds %zu bytes, %u needed", workspace_bytes, FQ_MX_WORKSPACE_BYTES);
    const size_t size = type_bytes(type);
    if ((st = check_stride("Y", Y, LX->rows, LW->rows, ldy, size)) != FQ_OK) return st;
    const Piece out[2] = {matrix(Y, LX->rows, LW->rows, ldy, size), {workspace, FQ_MX_WORKSPACE_BYTES}};
    const Piece in[6] = {{x_codes, mx_code_bytes(LX)}, {x_scales, mx_scale_bytes(LX)}, {x_tensor_scale, 4},
                         {w_codes, mx_code_bytes(LW)}, {w_scales, mx_scale_bytes(LW)}, {w_tensor_scale, 4}};
    if (!disjoint(out, 2, in, 6)) return fail(FQ_ERR_INVALID_ARG, "an output overlaps another array of the call");
    const int sms = sm_count_cached();
    if (sms <= 0) return fail(FQ_ERR_CUDA, "no CUDA device: %s", cudaGetErrorString(cudaGetLastError()));
    MxGemmParams p;
    std::memset(&p, 0, sizeof(p));
    p.Y = Y, p.ldy = ldy, p.ts_x = x_tensor_scale, p.ts_w = w_tensor_scale, p.status = (uint32_t*)workspace;
    p.M = LX->rows, p.N = LW->rows, p.K = LX->K;
    const bool nv = LX->format == FQ_NVFP4;
#define FQ_GEMM(T) (nv ? launch_mx_gemm<T, true>(LX, x_codes, x_scales, LW, w_codes, w_scales, p, (uint32_t)sms, cuda_stream) \
                       : launch_mx_gemm<T, false>(LX, x_codes, x_scales, LW, w_codes, w_scales, p, (uint32_t)sms, cuda_stream))
    return type == FQ_TYPE_BF16 ? FQ_GEMM(__nv_bfloat16) : type == FQ_TYPE_FP16 ? FQ_GEMM(__half) : FQ_GEMM(float);
#undef FQ_GEMM
}

}  // extern "C"
