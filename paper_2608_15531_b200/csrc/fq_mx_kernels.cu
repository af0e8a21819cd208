// Microscaled FP4 (sm_100a): quantising rows, also of a gated product or of the norm between two blocks, reading them back, and
// the launchers of these kernels and of the product (fq_mx_gemm_kernel.cuh).
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
#include "fq_ptx.cuh"

namespace fq {

__device__ __forceinline__ void grid_start() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------------------------ quantising and reading back

// A warp takes 256 consecutive values of four rows that are 32 apart, whose scales share the 16-byte lines of an atom:
// eight values of each row to a lane, four loads in flight.
struct MxParams {
    const void* a;               // X, or the gate
    const void* b;               // up
    uint64_t ld_a, ld_b;         // in values
    const float* ts;
    uint32_t* codes;
    uint8_t* scales;
    void* y;                     // (reading back)
    uint32_t rows, K, atoms, chunks;      // chunks of 256 values
    uint64_t tasks;
};
struct MxTask {
    uint32_t row0, k;            // the first of the four rows, this lane's first value
    bool any;
    __device__ __forceinline__ explicit MxTask(const MxParams& p) {
        const uint64_t w = (uint64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
        const uint64_t line = w / p.chunks;                               // row inside a tile, and the tile
        any = w < p.tasks;
        row0 = (uint32_t)(line >> 5) * 128 + (uint32_t)(line & 31);
        k = (uint32_t)(w - line * p.chunks) * 256 + (threadIdx.x & 31) * 8;
    }
};
constexpr int kMxThreads = 256;

template <class T, bool VEC>
__device__ __forceinline__ void gated8(const T* gate, const T* up, float (&h)[8]) {
    float g[8], u[8];
    load8<T, VEC>(gate, 8, g);
    load8<T, VEC>(up, 8, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f = (g[i] / (1.0f + expf(-g[i]))) * u[i];
        // 1 + exp(-g) beyond -60 loses what the product may still hold
        if ((near_border(f, T()) && g[i] != 0.0f && u[i] != 0.0f) || g[i] < -60.0f) f = (float)((double)g[i] / (1.0 + exp(-(double)g[i])) * (double)u[i]);
        h[i] = to_float(from_float<T>(f));
    }
}

template <class T, bool NV, bool GATED, bool VEC>
__global__ void __launch_bounds__(kMxThreads) fq_mx_quantize_kernel(const MxParams p) {
    const MxTask task(p);
    grid_start();
    if (!task.any) return;
    TensorScale ts;
    if constexpr (NV) ts.read(p.ts);
    const uint32_t lane = threadIdx.x & 31, k = task.k;
    constexpr int AL = Mx<NV>::ATOM_LANES;
    float v[4][8];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t r = task.row0 + 32 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[g][i] = 0.0f;
        if (r < p.rows && k < p.K) {
            const T* a = (const T*)p.a + (uint64_t)r * p.ld_a + k;
            if constexpr (GATED) gated8<T, VEC>(a, (const T*)p.b + (uint64_t)r * p.ld_b + k, v[g]);
            else load8<T, VEC>(a, 8, v[g]);
        }
    }
    uint32_t words[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t r = task.row0 + 32 * g;
        uint32_t codes, scale;
        quantize8<NV>(v[g], ts, codes, scale);
        if (k >= p.K) scale = 0;                                           // blocks beyond K
        words[g] = gather_scales<NV>(scale);
        if (r < p.rows && k < p.K) p.codes[((uint64_t)r * p.K + k) >> 3] = codes;
    }
    const uint32_t atom = k / Mx<NV>::ATOM;
    if (lane % AL == 0 && atom < p.atoms) {
        uint8_t* to = p.scales + scale_word(task.row0, p.atoms, atom);
        if (task.row0 + 96 < p.rows) {
            *reinterpret_cast<uint4*>(to) = make_uint4(words[0], words[1], words[2], words[3]);
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (task.row0 + 32 * g < p.rows) reinterpret_cast<uint32_t*>(to)[g] = words[g];
        }
    }
}

template <class T, bool NV, bool VEC>
__global__ void __launch_bounds__(kMxThreads) fq_mx_dequantize_kernel(const MxParams p) {
    const MxTask task(p);
    grid_start();
    const uint32_t k = task.k;
    if (!task.any || k >= p.K) return;
    float ts = 1.0f;
    if (NV && p.ts) asm volatile("ld.global.f32 %0, [%1];" : "=f"(ts) : "l"(p.ts) : "memory");
    const uint32_t block = k / Mx<NV>::BLOCK;
    const uint8_t* line = p.scales + scale_word(task.row0, p.atoms, block >> 2) + (block & 3);
    uint32_t codes[4], scale[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t r = task.row0 + 32 * g;
        codes[g] = 0, scale[g] = 0;
        if (r < p.rows) {
            asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(codes[g]) : "l"(p.codes + (((uint64_t)r * p.K + k) >> 3)) : "memory");
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(scale[g]) : "l"(line + 4 * g) : "memory");
        }
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const uint32_t r = task.row0 + 32 * g, s = scale[g];
        if (r >= p.rows) return;
        float d;
        if constexpr (NV) d = (s & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : copysignf(e4m3_value(s & 0x7f), s & 0x80 ? -1.0f : 1.0f) * ts;
        else d = s == 255 ? __uint_as_float(0x7fc00000u) : (s ? __uint_as_float(s << 23) : 0x1p-127f);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t c = codes[g] >> (4 * i);
            v[i] = copysignf(e2m1_value(c), c & 8 ? -1.0f : 1.0f) * d;
        }
        store8<T, VEC>((T*)p.y + (uint64_t)r * p.ld_a + k, 8, v);
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
};

// Sum over the TPR threads of a row, in all of them, in a fixed order.  `part`: one cell for each warp of the CTA.
template <int TPR>
__device__ __forceinline__ double row_sum(double s, double* part) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const uint32_t warp = threadIdx.x / 32;
        if (threadIdx.x % 32 == 0) part[warp] = s;
        __syncthreads();
        s = 0.0;
#pragma unroll
        for (int i = 0; i < W; ++i) s += part[i];
    }
    return s;
}

// TPR threads to a row, V vectors of eight values to a thread, which stay in registers from the first load to the last
// store: one pass over the data.  Rows of up to 512 values share a CTA (TPR = 32, a warp to a row).
// Binary64 where it decides: the sums, the residual sum, and a result too near a border.  That costs conversions (two per
// input value, at a quarter of the FP32 rate), not time: the loads and stores of a value take longer.
template <class T, int TPR, int V, bool VEC, int FORMAT>                   // FORMAT: FQ_MXFP4, FQ_NVFP4, or 2 for none
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) fq_norm_kernel(const NormParams p) {
    __shared__ double part[2][32];
    constexpr bool NV = FORMAT == (int)FQ_NVFP4;
    constexpr int RPC = TPR < 128 ? 128 / TPR : 1;
    const uint32_t row = blockIdx.x * RPC + (RPC > 1 ? threadIdx.x / TPR : 0), t = RPC > 1 ? threadIdx.x % TPR : threadIdx.x;
    grid_start();
    if (row >= p.rows) return;                             // (whole warps; CTAs of one row have it)
    const T* x = (const T*)p.x + row * p.ld_x;
    const T* block = (const T*)p.block + row * p.ld_block;
    const T* gate = (const T*)p.gate + row * p.ld_gate;
    float y[V][8], lo[V][8], in[V][8];
    double rstd = 1.0;
    if (p.block) {
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = (j * TPR + t) * 8;
            const int n = (int)p.D - (int)c;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[j][i] = 0.0f, in[j][i] = 0.0f;
            if (n > 0) load8<T, VEC>(block + c, n, y[j]), load8<T, VEC>(x + c, n, in[j]);
        }
        if (p.block_weight) {
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fma((double)y[j][i], (double)y[j][i], s);
            rstd = 1.0 / sqrt(row_sum<TPR>(s, part[0]) / p.D + (double)p.eps);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = (j * TPR + t) * 8;
            const int n = (int)p.D - (int)c;
#pragma unroll
            for (int i = 0; i < 8; ++i) in[j][i] = 0.0f;
            if (n > 0) load8<T, VEC>(x + c, n, in[j]);
        }
    }
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint32_t c = (j * TPR + t) * 8;
        const int n = (int)p.D - (int)c;
        float w[8], g[8];
        if (p.block && p.block_weight && n > 0) load8<T, VEC>((const T*)p.block_weight + c, n, w);
        if (p.block && p.gate && n > 0) load8<T, VEC>(gate + c, n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            double r = in[j][i];
            if (p.block && n > 0) {
                double f = y[j][i];
                if (p.block_weight) f = f * rstd * (double)w[i];
                if (p.gate) f *= (double)g[i];
                r = fma((double)p.alpha, f, r);
            }
            s = fma(r, r, s);
            in[j][i] = (float)r;                           // the sum as two binary32 numbers
            lo[j][i] = (float)(r - (double)in[j][i]);
        }
    }
    if (p.r) {
        T* to = (T*)p.r + row * p.ld_r;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = (j * TPR + t) * 8;
            if (c < p.D) store8<T, VEC>(to + c, (int)p.D - (int)c, in[j]);
        }
    }
    if (!p.h && FORMAT == 2) return;
    rstd = 1.0 / sqrt(row_sum<TPR>(s, part[1]) / p.D + (double)p.eps);
    const float rs = (float)rstd;
    TensorScale ts;
    if constexpr (NV) ts.read(p.ts);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const uint32_t c = (j * TPR + t) * 8;
        const int n = (int)p.D - (int)c;
        float w[8], h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.0f, h[i] = 0.0f;
        if (p.weight && n > 0) load8<T, VEC>((const T*)p.weight + c, n, w);
        if (n > 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float f = in[j][i] * rs * w[i];
                if (near_border(f, T()) && in[j][i] != 0.0f) f = (float)(((double)in[j][i] + (double)lo[j][i]) * rstd * (double)w[i]);
                h[i] = to_float(from_float<T>(f));
            }
            if (p.h) store8<T, VEC>((T*)p.h + row * p.ld_h + c, n, h);
        }
        if constexpr (FORMAT != 2) {
            uint32_t codes, scale;
            quantize8<NV>(h, ts, codes, scale);
            if (n <= 0) scale = 0;
            const uint32_t word = gather_scales<NV>(scale), atom = c / Mx<NV>::ATOM;
            if (n > 0) p.codes[((uint64_t)row * p.D + c) >> 3] = codes;
            if (t % Mx<NV>::ATOM_LANES == 0 && atom < p.atoms) *reinterpret_cast<uint32_t*>(p.scales + scale_word(row, p.atoms, atom)) = word;
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

// A piece of memory that a call reads or writes.
struct Piece {
    const void* p;
    size_t bytes;
    bool overlaps(const Piece& o) const {
        const uintptr_t a = (uintptr_t)p, b = (uintptr_t)o.p;
        return p && o.p && bytes && o.bytes && a < b + o.bytes && b < a + bytes;
    }
};
// rows x cols values of `size` bytes with a row stride of ld values
static Piece matrix(const void* p, uint64_t rows, uint64_t cols, uint64_t ld, size_t size) { return Piece{p, (size_t)(((rows - 1) * ld + cols) * size)}; }
// No output on another output or on an input.
static bool disjoint(const Piece* out, int nout, const Piece* in, int nin) {
    for (int i = 0; i < nout; ++i) {
        for (int j = i + 1; j < nout; ++j)
            if (out[i].overlaps(out[j])) return false;
        for (int j = 0; j < nin; ++j)
            if (out[i].overlaps(in[j])) return false;
    }
    return true;
}
static fq_status_t check_stride(const char* what, const void* p, uint64_t rows, uint64_t cols, uint64_t ld, size_t size) {
    if (!aligned(p, size)) return fail(FQ_ERR_INVALID_ARG, "%s is misaligned", what);
    if ((rows > 1 && ld < cols) || ld > (1ull << 40)) return fail(FQ_ERR_INVALID_ARG, "%s: row stride %llu for %llu columns", what, (unsigned long long)ld, (unsigned long long)cols);
    return FQ_OK;
}
static fq_status_t check_mx(const fq_mx_layout_t* L, const void* codes, const void* scales, const float* ts) {
    if (!mx_layout_ok(L)) return fail(FQ_ERR_INVALID_ARG, "bad layout");
    if (!codes || !scales) return fail(FQ_ERR_INVALID_ARG, "null codes or scales");
    if (!aligned(codes, 16) || !aligned(scales, 16) || !aligned(ts, 4)) return fail(FQ_ERR_INVALID_ARG, "misaligned codes, scales or tensor scale");
    if (ts && L->format != FQ_NVFP4) return fail(FQ_ERR_INVALID_ARG, "FQ_MXFP4 has no tensor scale");
    return FQ_OK;
}
// Rows on 16-byte boundaries.
static bool rows_aligned(const void* p, uint64_t ld, size_t size, uint64_t rows) { return aligned(p, 16) && (rows <= 1 || ld * size % 16 == 0); }

static MxParams mx_params(const fq_mx_layout_t* L, const float* ts) {
    MxParams p;
    std::memset(&p, 0, sizeof(p));
    p.ts = ts;
    p.rows = L->rows, p.K = L->K, p.atoms = mx_atoms(L);
    p.chunks = (L->K + 255) / 256;
    p.tasks = ((uint64_t)(L->rows / 128) * 32 + std::min<uint32_t>(L->rows % 128, 32)) * p.chunks;   // (a last tile of fewer than 32 rows has fewer lines)
    return p;
}
typedef void (*MxFn)(const MxParams);
template <class T, bool GATED>
static MxFn pick_quantize(bool nv, bool vec) {
    if (nv) return vec ? (MxFn)fq_mx_quantize_kernel<T, true, GATED, true> : (MxFn)fq_mx_quantize_kernel<T, true, GATED, false>;
    return vec ? (MxFn)fq_mx_quantize_kernel<T, false, GATED, true> : (MxFn)fq_mx_quantize_kernel<T, false, GATED, false>;
}
template <class T>
static MxFn pick_dequantize(bool nv, bool vec) {
    if (nv) return vec ? (MxFn)fq_mx_dequantize_kernel<T, true, true> : (MxFn)fq_mx_dequantize_kernel<T, true, false>;
    return vec ? (MxFn)fq_mx_dequantize_kernel<T, false, true> : (MxFn)fq_mx_dequantize_kernel<T, false, false>;
}
static fq_status_t launch_mx(MxFn fn, const MxParams& p, void* stream) {
    const uint64_t warps = kMxThreads / 32, ctas = (p.tasks + warps - 1) / warps;
    if (ctas > 0x7fffffffull) return fail(FQ_ERR_UNSUPPORTED_SHAPE, "matrix too large for one launch");
    return launch(fn, dim3((uint32_t)ctas), kMxThreads, 0, 1, stream, p);
}

typedef void (*NormFn)(const NormParams);
template <class T, int FORMAT, bool VEC>
static NormFn pick_norm(uint32_t D, uint32_t& tpr) {
    const uint32_t vectors = (D + 7) / 8;
    if (vectors <= 64) return tpr = 32, (NormFn)fq_norm_kernel<T, 32, 2, VEC, FORMAT>;
    if (vectors <= 128) return tpr = 128, (NormFn)fq_norm_kernel<T, 128, 1, VEC, FORMAT>;
    if (vectors <= 256) return tpr = 256, (NormFn)fq_norm_kernel<T, 256, 1, VEC, FORMAT>;
    if (vectors <= 512) return tpr = 512, (NormFn)fq_norm_kernel<T, 512, 1, VEC, FORMAT>;
    if (vectors <= 1024) return tpr = 512, (NormFn)fq_norm_kernel<T, 512, 2, VEC, FORMAT>;
    return tpr = 1024, (NormFn)fq_norm_kernel<T, 1024, 2, VEC, FORMAT>;
}
template <class T, bool VEC>
static NormFn pick_norm(int format, uint32_t D, uint32_t& tpr) {
    if (format == (int)FQ_MXFP4) return pick_norm<T, (int)FQ_MXFP4, VEC>(D, tpr);
    if (format == (int)FQ_NVFP4) return pick_norm<T, (int)FQ_NVFP4, VEC>(D, tpr);
    return pick_norm<T, 2, VEC>(D, tpr);
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
    p.stages = G::STAGES < 16 ? G::STAGES : 16;
    p.split = 1;
    while (p.split < 8 && p.tiles * p.split * 2 <= sms && p.steps >= 4 * p.split) p.split *= 2;
    const uint32_t grid = p.split > 1 ? p.tiles * p.split : std::min(p.tiles, sms);
    const auto fn = fq_mx_gemm_kernel<T, NT, NV>;
    const uint32_t smem = p.stages * G::STAGE + 1024;
    const cudaError_t e = ensure_smem_attr((const void*)fn, (int)smem);
    if (e != cudaSuccess) return fail(FQ_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    return launch(fn, dim3(grid), 256, smem, p.split, stream, mw, mx, mws, mxs, p);
}
template <class T, bool NV>
static fq_status_t launch_mx_gemm(const fq_mx_layout_t* LX, const void* xc, const void* xs, const fq_mx_layout_t* LW, const void* wc, const void* ws,
                                  MxGemmParams& p, uint32_t sms, void* stream) {
    if (p.M <= 16) return launch_mx_gemm<T, 16, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
    if (p.M <= 32) return launch_mx_gemm<T, 32, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
    if (p.M <= 64) return launch_mx_gemm<T, 64, NV>(LX, xc, xs, LW, wc, ws, p, sms, stream);
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
    const bool nv = L->format == FQ_NVFP4, vec = rows_aligned(X, ldx, size, L->rows);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_quantize<__nv_bfloat16, false>(nv, vec) : type == FQ_TYPE_FP16 ? pick_quantize<__half, false>(nv, vec)
                                                                                                               : pick_quantize<float, false>(nv, vec), p, cuda_stream);
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
    const bool nv = L->format == FQ_NVFP4, vec = rows_aligned(gate, ld_gate, 2, L->rows) && rows_aligned(up, ld_up, 2, L->rows);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_quantize<__nv_bfloat16, true>(nv, vec) : pick_quantize<__half, true>(nv, vec), p, cuda_stream);
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
    const bool nv = L->format == FQ_NVFP4, vec = rows_aligned(Y, ldy, size, L->rows);
    return launch_mx(type == FQ_TYPE_BF16 ? pick_dequantize<__nv_bfloat16>(nv, vec) : type == FQ_TYPE_FP16 ? pick_dequantize<__half>(nv, vec)
                                                                                                          : pick_dequantize<float>(nv, vec), p, cuda_stream);
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
    uint32_t tpr = 0;
    NormFn fn;
    if (a->type == FQ_TYPE_BF16) fn = vec ? pick_norm<__nv_bfloat16, true>(format, a->D, tpr) : pick_norm<__nv_bfloat16, false>(format, a->D, tpr);
    else fn = vec ? pick_norm<__half, true>(format, a->D, tpr) : pick_norm<__half, false>(format, a->D, tpr);
    const uint32_t threads = std::max<uint32_t>(tpr, 128), per = threads / tpr;
    return launch(fn, dim3((a->rows + per - 1) / per), threads, 0, 1, cuda_stream, p);
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
