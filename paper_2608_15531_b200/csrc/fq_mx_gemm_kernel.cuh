// Product of two microscaled FP4 matrices on the block-scaled tensor path (tcgen05.mma kind::mxf4nvf4, FP32 accumulation).
// Included by fq_mx_kernels.cu.
//
// The weights are on the M side (a lane of tensor memory = an output feature), the tokens on the N side, so that one
// layout serves one token (16 columns) and a prefill.  Codes go to shared memory by tiled tensor copies (a row's 256
// codes are 128 bytes, 128-byte swizzle: the K-major operand), the scales as whole atoms, which tcgen05.cp spreads over tensor
// memory: lane = row % 32, one column of four scales for each 32 rows.
//
//   warp 0      producer: per stage of 256 k the codes of 128 features and NT tokens and their scales, one barrier
//   warp 1      tensor: copies the stage's scales to tensor memory, four MMAs of K = 64, one commit
//   warp 2      allocates the tensor memory
//   warps 4-    drain: tcgen05.ld, tensor scales, Y (a warp stores 32 features of a token: whole sectors)
//
// Few tokens are bound by reading the weights once, and by latency on small layers: the k-steps of a tile are then split
// over a cluster of CTAs, whose sums meet in shared memory and are added in rank order by all of them, each its tokens.
// Tensor memory is given back before a CTA waits for its cluster, so that no CTA holds it while it waits for another one.
// Measured (us, calls back to back in a graph, weights from DRAM): one token 4096 x 4096 4.5, 4096 x 28672 12.0 (5.2 TB/s), 14336 x 4096 NVFP4 8.5
// (3.9); 128 tokens 5.9, 13.8, 12.0; 128 tokens 8192 x 57344 46 (5.7 TB/s, tensor pipe 35 % busy).  What bounds the small ones is the chain launch,
// first copy, seven or fewer steps, tensor memory to registers, exchange, store: 3.7 us for 8 steps of 64 tiles.
#pragma once
#include <cooperative_groups.h>

#include "fq_mx.cuh"
#include "fq_ptx.cuh"

namespace fq {

constexpr uint32_t kMxStageK = 256, kMxStages = 12;       // k of a stage; stages of the longest ring

struct MxGemmParams {
    void* Y;
    uint64_t ldy;
    const float *ts_x, *ts_w;
    uint32_t* status;
    uint32_t M, N, K;
    uint32_t steps;                // stages of 256 k
    uint32_t tiles_m, tiles;       // token tiles; all tiles
    uint32_t split;                // CTAs of a cluster, which share the steps of a tile
    uint32_t stages;
};

// NT: tokens of a tile.
template <int NT, bool NV>
struct MxGemm {
    static constexpr uint32_t ATOMS = NV ? 4 : 2;                          // atoms of scales to a stage, of 64 or 128 k
    static constexpr uint32_t W_BYTES = 128 * 128, X_BYTES = NT * 128, S_BYTES = ATOMS * 512;
    static constexpr uint32_t STAGE = W_BYTES + X_BYTES + 2 * S_BYTES;
    static constexpr uint32_t OFF_X = W_BYTES, OFF_WS = OFF_X + X_BYTES, OFF_XS = OFF_WS + S_BYTES;
    // tensor memory: accumulators, then the scales of a stage
    static constexpr uint32_t COL_WS = NT, COL_XS = COL_WS + ATOMS * 4, USED = COL_XS + ATOMS * 4;
    static constexpr uint32_t COLS = USED <= 64 ? 64 : (USED <= 128 ? 128 : (USED <= 256 ? 256 : 512));
    static_assert(STAGE % 1024 == 0 && COLS <= 256, "stage, tensor memory of two CTAs");
    // Two CTAs to an SM: the one drains while the other multiplies, and the next launch's start beside this one's.
    static constexpr uint32_t STAGES = (113 * 1024 - 2048) / STAGE, STAGES_ALONE = (kSmemBudget - 2048) / STAGE;
    static constexpr uint32_t DRAIN = NT >= 64 ? 8 : 4, THREADS = 128 + 32 * DRAIN;        // drain warps: one or two for each 32 features
    static_assert(STAGES >= 3 && STAGES_ALONE <= kMxStages && STAGES * STAGE >= NT * 128 * 4, "stages, exchange of a split tile");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// A tile on its way to the L2 only: harmless to what another kernel is still writing there.
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* map, uint32_t x, uint32_t y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// A stage's work: its scales to tensor memory (one copy for each atom: 32 rows of 16 bytes, to the same lanes of each of the four
// subpartitions), then D (+)= A B for each 64 of its 256 k.  tcgen05.cp and tcgen05.mma of one thread run in the order of their issue.
// Whole warp, converged, with warp-uniform operands; one elected lane issues.  One asm block, so that the address arithmetic
// is not in a divergent branch, where each operand has to be moved into a uniform register: 440 clocks a stage of the pair kernel
// went to its issue, now 245, and the loop around it took 270, now 100 (4096 x 4096 x 28672 238 us, now 197).
//   cw, cx     tensor-memory columns of the two matrices' scales, multiples of four: an MMA whose scales begin in another
//              column ends in an address error
//   ws, xs     lower words of the descriptors of their atoms in shared memory, s_hi the upper word
//   a, b, hi   the same of the codes
//   mmas       how many of the four 64s of k there are
struct StageWork {
    uint32_t d, cw, cx, ws, xs, s_hi, a, b, hi, idesc, acc, mmas, tiles_x;
};
// CP: tensor-memory column BASE + COL, descriptor DESC + OFF (in 16 bytes), predicate
#define FQ_CP(GROUP, BASE, COL, DESC, OFF, PRED)                                                            \
    " add.u32 t, " BASE ", " COL ";\n add.u32 q, " DESC ", " OFF ";\n mov.b64 y, {q, %5};\n"                 \
    " @" PRED " tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [t], y;\n"
// MMA of k 64 j to 64 j + 63: OFF = 2 j, columns of the scales, scale bytes ID (added to idesc), predicate
#define FQ_MMA(GROUP, VEC, OFF, CW, CX, ID, PRED)                                                           \
    " add.u32 q, %6, " OFF ";\n mov.b64 x, {q, %8};\n add.u32 q, %7, " OFF ";\n mov.b64 y, {q, %8};\n"       \
    " add.u32 t, %1, " CW ";\n add.u32 u, %2, " CX ";\n add.u32 i, %9, " ID ";\n"                            \
    " @" PRED " tcgen05.mma.cta_group::" GROUP ".kind::mxf4nvf4.block_scale.scale_vec::" VEC " [%0], x, y, i, [t], [u], f;\n" \
    " setp.eq.b32 f, %10, %10;\n"
#define FQ_STAGE_BEGIN                                                                                      \
    "{\n .reg .pred e, f, m1, m2, m3, t1;\n .reg .b32 t, u, q, i;\n .reg .b64 x, y;\n"                       \
    " elect.sync _|e, 0xffffffff;\n setp.ne.b32 f, %10, 0;\n"                                               \
    " setp.gt.and.u32 m1, %11, 1, e;\n setp.gt.and.u32 m2, %11, 2, e;\n setp.gt.and.u32 m3, %11, 3, e;\n"     \
    " setp.gt.and.u32 t1, %12, 1, e;\n"
#define FQ_STAGE_END(w)                                                                                     \
    "}" ::"r"(w.d), "r"(w.cw), "r"(w.cx), "r"(w.ws), "r"(w.xs), "r"(w.s_hi), "r"(w.a), "r"(w.b), "r"(w.hi), "r"(w.idesc), "r"(w.acc), "r"(w.mmas), \
        "r"(w.tiles_x) : "memory"
// (scale bytes 2 and 3 of an atom's column: 2 << 29 and 2 << 4 in idesc)
template <bool NV>
__device__ __forceinline__ void stage_one(const StageWork& w) {            // a CTA of its own, one row tile of tokens
    if constexpr (NV)
        asm volatile(FQ_STAGE_BEGIN
            FQ_CP("1", "%1", "0", "%3", "0", "e") FQ_CP("1", "%2", "0", "%4", "0", "e") FQ_CP("1", "%1", "4", "%3", "32", "e") FQ_CP("1", "%2", "4", "%4", "32", "e")
            FQ_CP("1", "%1", "8", "%3", "64", "e") FQ_CP("1", "%2", "8", "%4", "64", "e") FQ_CP("1", "%1", "12", "%3", "96", "e") FQ_CP("1", "%2", "12", "%4", "96", "e")
            FQ_MMA("1", "4X", "0", "0", "0", "0", "e") FQ_MMA("1", "4X", "2", "4", "4", "0", "m1") FQ_MMA("1", "4X", "4", "8", "8", "0", "m2")
            FQ_MMA("1", "4X", "6", "12", "12", "0", "m3") FQ_STAGE_END(w));
    else
        asm volatile(FQ_STAGE_BEGIN
            FQ_CP("1", "%1", "0", "%3", "0", "e") FQ_CP("1", "%2", "0", "%4", "0", "e") FQ_CP("1", "%1", "4", "%3", "32", "e") FQ_CP("1", "%2", "4", "%4", "32", "e")
            FQ_MMA("1", "2X", "0", "0", "0", "0", "e") FQ_MMA("1", "2X", "2", "0", "0", "0x40000020", "m1") FQ_MMA("1", "2X", "4", "4", "4", "0", "m2")
            FQ_MMA("1", "2X", "6", "4", "4", "0x40000020", "m3") FQ_STAGE_END(w));
}
template <bool NV>
__device__ __forceinline__ void stage_pair(const StageWork& w) {           // a pair of CTAs, one or two row tiles of tokens
    if constexpr (NV)
        asm volatile(FQ_STAGE_BEGIN
            FQ_CP("2", "%1", "0", "%3", "0", "e") FQ_CP("2", "%1", "4", "%3", "32", "e") FQ_CP("2", "%1", "8", "%3", "64", "e") FQ_CP("2", "%1", "12", "%3", "96", "e")
            FQ_CP("2", "%2", "0", "%4", "0", "e") FQ_CP("2", "%2", "8", "%4", "32", "e") FQ_CP("2", "%2", "16", "%4", "64", "e") FQ_CP("2", "%2", "24", "%4", "96", "e")
            FQ_CP("2", "%2", "4", "%4", "128", "t1") FQ_CP("2", "%2", "12", "%4", "160", "t1") FQ_CP("2", "%2", "20", "%4", "192", "t1") FQ_CP("2", "%2", "28", "%4", "224", "t1")
            FQ_MMA("2", "4X", "0", "0", "0", "0", "e") FQ_MMA("2", "4X", "2", "4", "8", "0", "m1") FQ_MMA("2", "4X", "4", "8", "16", "0", "m2")
            FQ_MMA("2", "4X", "6", "12", "24", "0", "m3") FQ_STAGE_END(w));
    else
        asm volatile(FQ_STAGE_BEGIN
            FQ_CP("2", "%1", "0", "%3", "0", "e") FQ_CP("2", "%1", "4", "%3", "32", "e") FQ_CP("2", "%2", "0", "%4", "0", "e") FQ_CP("2", "%2", "8", "%4", "32", "e")
            FQ_CP("2", "%2", "4", "%4", "64", "t1") FQ_CP("2", "%2", "12", "%4", "96", "t1")
            FQ_MMA("2", "2X", "0", "0", "0", "0", "e") FQ_MMA("2", "2X", "2", "0", "0", "0x40000020", "m1") FQ_MMA("2", "2X", "4", "4", "8", "0", "m2")
            FQ_MMA("2", "2X", "6", "4", "8", "0x40000020", "m3") FQ_STAGE_END(w));
}
#undef FQ_CP
#undef FQ_MMA
#undef FQ_STAGE_BEGIN
#undef FQ_STAGE_END
__device__ __forceinline__ void commit_elected(uint32_t bar) {             // converged warp
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void pair_commit_elected(uint32_t bar) {        // to that barrier of both CTAs
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n"
                 " @e tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

// C tokens of this lane's feature, one row of Y after the other.  Whole tiles without a comparison for each: a drain warp works alone
// on its scheduler, and what it executes is what a tile's end takes (23 instructions a token bound the rate at 4096 tokens).
template <class T, int C>
__device__ __forceinline__ void store_tokens(T* y, uint64_t ldy, const float (&v)[C], float alpha, uint32_t rows) {
    if (rows >= (uint32_t)C) {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            *y = from_float<T>(v[i] * alpha);
            y += ldy;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) {
            if ((uint32_t)i < rows) *y = from_float<T>(v[i] * alpha);
            y += ldy;
        }
    }
}

template <class T, int NT, bool NV>
__global__ void __launch_bounds__(MxGemm<NT, NV>::THREADS, 2)
fq_mx_gemm_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_ws,
                  const __grid_constant__ CUtensorMap map_xs, const MxGemmParams p) {
    using G = MxGemm<NT, NV>;
    extern __shared__ uint8_t mx_smem[];
    __shared__ uint64_t bars[2 * kMxStages + 3];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t abort_word;
    namespace cg = cooperative_groups;
    // (the shuffle tells the compiler that a warp's lanes agree: the tensor warp's operands then stay in uniform registers)
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31, S = p.stages;
    const uint32_t smem = (smem_u32(mx_smem) + 1023) & ~1023u;
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * kMxStages, bar_acc = bar_empty + 8 * kMxStages, bar_free = bar_acc + 8, bar_final = bar_free + 8;
    volatile uint32_t* abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < S; ++s) mbar_init(bar_full + 8 * s, 1), mbar_init(bar_empty + 8 * s, 1);
        mbar_init(bar_acc, 1), mbar_init(bar_free, G::DRAIN), mbar_init(bar_final, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 96) prefetch_map(&map_w), prefetch_map(&map_x), prefetch_map(&map_ws), prefetch_map(&map_xs);
    if (warp == 2) {
        tmem_alloc(smem_u32(&tmem_slot), G::COLS);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // Only here: a CTA of the next grid may take tensor memory, and waits for this grid while it holds it.
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const uint32_t rank = blockIdx.x % p.split, first = blockIdx.x / p.split, stride = gridDim.x / p.split;
    const uint32_t k0 = p.steps * rank / p.split, k1 = p.steps * (rank + 1) / p.split;      // (at most 4096 steps, 8 ranks)

    if (warp == 0) {
        uint32_t issued = 0;
        const bool leader = elect_one();
        if (leader) {
            const uint32_t n0 = first / p.tiles_m * 128;
            for (uint32_t k = k0; k < k1 && k < k0 + S; ++k) tma_prefetch_2d(&map_w, k * 128, n0);
        }
        asm volatile("griddepcontrol.wait;" ::: "memory");
        uint32_t s = 0, ph = 0;
        bool ok = true;
        for (uint32_t tile = first; ok && tile < p.tiles; tile += stride) {
            const uint32_t tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m;
            for (uint32_t k = k0; k < k1; ++k) {
                if (!(ok = warp_wait(bar_empty + 8 * s, ph ^ 1, abort_flag, p.status))) break;
                if (leader) {
                    const uint32_t at = smem + s * G::STAGE, bar = bar_full + 8 * s;
                    mbar_arrive_expect_tx(bar, G::STAGE);
                    tma_load_2d(at, &map_w, k * 128, tn * 128, bar);
                    tma_load_2d(at + G::OFF_X, &map_x, k * 128, tm * NT, bar);
                    tma_load_3d(at + G::OFF_WS, &map_ws, 0, k * G::ATOMS, tn, bar);
                    tma_load_3d(at + G::OFF_XS, &map_xs, 0, k * G::ATOMS, tm, bar);
                }
                ++issued;
                if (++s == S) s = 0, ph ^= 1;
            }
        }
        let_copies_land(bar_full, issued, S);             // (at once, unless another warp gives up)
    } else if (warp == 1) {
        asm volatile("griddepcontrol.wait;" ::: "memory");     // (its waits are limited in time, the grid before is not)
        // e2m1 times e2m1, scales E8M0 (bit 23) or E4M3, N = NT, M = 128
        StageWork w;
        w.idesc = (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | (NV ? 0u : 1u << 23) | (8u << 24);
        w.cw = tmem + G::COL_WS, w.cx = tmem + G::COL_XS, w.tiles_x = 1;
        w.s_hi = (uint32_t)(desc_plain(0, 128) >> 32), w.hi = (uint32_t)(desc_sw128(0) >> 32);
        const uint32_t codes0 = (uint32_t)desc_sw128(smem), scales0 = (uint32_t)desc_plain(smem, 128);
        w.d = tmem;
        uint32_t s = 0, ph = 0, aph = 0;
        for (uint32_t tile = first; tile < p.tiles; tile += stride) {
            if (!warp_wait(bar_free, aph ^ 1, abort_flag, p.status)) break;
            tc_fence_after();
            bool ok = true;
            for (uint32_t k = k0; k < k1; ++k) {
                if (!(ok = warp_wait(bar_full + 8 * s, ph, abort_flag, p.status))) break;
                tc_fence_after();
                const uint32_t at = s * (G::STAGE >> 4);
                w.a = codes0 + at, w.b = codes0 + at + (G::OFF_X >> 4), w.ws = scales0 + at + (G::OFF_WS >> 4), w.xs = scales0 + at + (G::OFF_XS >> 4);
                w.acc = k > k0;
                w.mmas = (min(p.K - k * kMxStageK, kMxStageK) + 63) / 64;  // (beyond K the scales are not there)
                stage_one<NV>(w);
                commit_elected(bar_empty + 8 * s);
                if (k + 1 == k1) commit_elected(bar_acc);
                if (++s == S) s = 0, ph ^= 1;
            }
            if (!ok) break;
            aph ^= 1;
        }
        // No MMA is in flight when the tensor memory is given back and the CTA leaves, whoever gave up.
        commit_elected(bar_final);
        mbar_wait_leaving(bar_final, 0);
        __syncwarp();
    } else if (warp >= 4) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        float alpha = 1.0f;
        if (NV) {
            float a = 1.0f, b = 1.0f;
            if (p.ts_x) asm volatile("ld.global.f32 %0, [%1];" : "=f"(a) : "l"(p.ts_x) : "memory");
            if (p.ts_w) asm volatile("ld.global.f32 %0, [%1];" : "=f"(b) : "l"(p.ts_w) : "memory");
            alpha = a * b;
        }
        const uint32_t quarter = warp & 3, half = (warp - 4) / 4, f = quarter * 32 + lane;             // (two warps take 32 tokens in turn)
        uint32_t aph = 0;
        constexpr int C = NT < 32 ? NT : 32;
        for (uint32_t tile = first; tile < p.tiles; tile += stride, aph ^= 1) {
            if (!warp_wait(bar_acc, aph, abort_flag, p.status)) break;
            tc_fence_after();
            const uint32_t tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m, n = tn * 128 + f, m0 = tm * NT;
            const uint32_t rows = min((uint32_t)NT, p.M - m0);
            T* y = (T*)p.Y + (uint64_t)m0 * p.ldy + n;
            for (uint32_t c = C * half; c < rows; c += C * (G::DRAIN / 4)) {
                float v[C];
                tmem_ld<C>(tmem + (quarter << 21) + c, v);
                tmem_wait_ld();
                if (p.split > 1) {
                    float* part = reinterpret_cast<float*>(mx_smem + (smem - smem_u32(mx_smem))) + c * 128 + f;
#pragma unroll
                    for (int i = 0; i < C; ++i) part[i * 128] = v[i];
                } else if (n < p.N) {
                    store_tokens<T, C>(y + (uint64_t)c * p.ldy, p.ldy, v, alpha, rows - c);
                }
            }
            tc_fence_before();
            if (lane == 0) mbar_arrive(bar_free);
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, G::COLS);
    }
    if (p.split > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const uint32_t tn = first / p.tiles_m, tm = first - tn * p.tiles_m, m0 = tm * NT, rows = min((uint32_t)NT, p.M - m0);
        float alpha = 1.0f;
        asm volatile("griddepcontrol.wait;" ::: "memory");     // (over long ago, but not every warp has asked)
        if (NV) alpha = (p.ts_x ? *(const volatile float*)p.ts_x : 1.0f) * (p.ts_w ? *(const volatile float*)p.ts_w : 1.0f);
        // A warp takes a token, a lane four of its features.  Eight loads in flight, of as many tokens as it takes (the
        // split is a power of two): number q is of the batch's token q / split, from rank q % split.
        float* mine = reinterpret_cast<float*>(mx_smem + (smem - smem_u32(mx_smem)));
        const uint32_t n = tn * 128 + 4 * lane, last = p.split - 1, shift = 31 - __clz(p.split);
        const bool wide = p.ldy % 4 == 0 && (reinterpret_cast<uintptr_t>(p.Y) & (4 * sizeof(T) - 1)) == 0;
        constexpr uint32_t WARPS = G::THREADS / 32;
        for (uint32_t m = rank + p.split * warp; m < rows; m += 8 * WARPS) {
            float4 v[8], sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) {
                const uint32_t at = m + (q >> shift) * WARPS * p.split;
                if (at < rows) v[q] = reinterpret_cast<const float4*>(cluster.map_shared_rank(mine, q & last))[at * 32 + lane];
            }
#pragma unroll
            for (uint32_t q = 0; q < 8; ++q) {
                const uint32_t at = m + (q >> shift) * WARPS * p.split;
                if (at >= rows || *abort_flag) continue;
                if ((q & last) == 0) sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                sum.x += v[q].x, sum.y += v[q].y, sum.z += v[q].z, sum.w += v[q].w;
                if ((q & last) != last) continue;
                T* y = (T*)p.Y + (uint64_t)(m0 + at) * p.ldy + n;
                const T out[4] = {from_float<T>(sum.x * alpha), from_float<T>(sum.y * alpha), from_float<T>(sum.z * alpha), from_float<T>(sum.w * alpha)};
                if (wide && n + 3 < p.N) {
                    struct alignas(4 * sizeof(T)) Four { T v[4]; };
                    *reinterpret_cast<Four*>(y) = Four{{out[0], out[1], out[2], out[3]}};
                } else {
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        if (n + j < p.N) y[j] = out[j];
                }
            }
        }
        cluster.sync();
    }
}

// ---- many tokens: a pair of CTAs (cta_group::2) on 256 features by up to 256 tokens
//
// Each CTA of the pair holds 128 of the features and half of the tokens; the tensor cores of both read both halves, so that
// a byte from the L2 serves twice the operations of the kernel above, which many tokens are bound by.  The accumulators
// take 256 columns of tensor memory, and there is no room for two beside the scales: the eight drain warps take a tile's
// sums into registers, all at once, give the columns back, and convert and store while the next tile is multiplied.
// Tiles begin on multiples of 128 tokens, as the atoms of scales do; the last tile of a column multiplies only the tokens that it has,
// rounded up to 32.
// What bounds it: of the 12500 clocks of a tile of 4096 k the MMAs need 8200 (tensor pipe 68 % busy, 83 at the first launch on a cool device); 1700 pass between a tile's last
// MMA and the next one's first (commit, tensor memory to registers, arrival from the other CTA), the rest waits for copies: six
// stages of 35 KB are all the shared memory, and the L2 delivers 13 TB/s.  4096 x 4096 x 28672 165 us for the first milliseconds (5.8 PFLOP/s; NVFP4 173),
// 197 to 220 once the power cap has lowered the clock to 1.6 GHz; 1024 x 4096 x 18944 30 (5.3 PFLOP/s; NVFP4 31).  Copies of the next tile's weights to the L2 ahead of time changed nothing.
constexpr uint32_t kPairWarps = 12;        // copies, MMAs, allocation, one idle; eight drain warps: two for each 32 features

struct MxPairParams {
    void* Y;
    uint64_t ldy;
    const float *ts_x, *ts_w;
    uint32_t* status;
    uint32_t M, N, K;
    uint32_t steps, tiles_m, tiles, stages;
    uint32_t tokens;               // of a tile: 128 or 256
};

template <bool NV>
struct MxPair {
    static constexpr uint32_t ATOMS = NV ? 4 : 2, W_BYTES = 128 * 128, X_BYTES = 128 * 128, S_BYTES = ATOMS * 512;
    static constexpr uint32_t OFF_X = W_BYTES, OFF_WS = OFF_X + X_BYTES, OFF_XS = OFF_WS + S_BYTES, STAGE = OFF_XS + 2 * S_BYTES;
    static constexpr uint32_t COL_WS = 256, COL_XS = COL_WS + ATOMS * 4, USED = COL_XS + ATOMS * 8;
    static_assert(USED <= 512 && STAGE % 1024 == 0, "tensor memory, swizzle");
    static constexpr uint32_t STAGES = (kSmemBudget - 2048) / STAGE;
    static_assert(STAGES <= 8, "barriers");
};
// Tokens that a tile multiplies; each CTA holds half of them.
__device__ __forceinline__ uint32_t pair_tile_tokens(const MxPairParams& p, uint32_t m0) { return min(p.tokens, (p.M - m0 + 31) / 32 * 32); }

__device__ __forceinline__ uint32_t in_leader(uint32_t saddr) {            // the pair's first CTA's copy of a shared-memory address
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(saddr));
    return r;
}
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// What it tells of is a read of tensor memory that has been waited for; nothing in memory goes with it, so that it need not wait for the
// thread's stores to Y (as a release it took 1900 clocks, a tenth of a tile of 4096 k).
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
template <class T, bool NV>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(32 * kPairWarps, 1)
fq_mx_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_ws,
                  const __grid_constant__ CUtensorMap map_xs, const MxPairParams p) {
    using G = MxPair<NV>;
    extern __shared__ uint8_t mx_smem[];
    __shared__ uint64_t bars[2 * 8 + 3];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t abort_word;
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    // (the shuffle tells the compiler that a warp's lanes agree: the tensor warp's operands then stay in uniform registers)
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x & 31, S = p.stages, rank = blockIdx.x & 1;
    const uint32_t smem = (smem_u32(mx_smem) + 1023) & ~1023u;
    // full: the leader's, for the copies of both CTAs; empty, acc, final: each CTA's own, by commits to both; free: the leader's
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 64, bar_acc = bar_empty + 64, bar_free = bar_acc + 8, bar_final = bar_free + 8;
    volatile uint32_t* abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < S; ++s) mbar_init(bar_full + 8 * s, 1), mbar_init(bar_empty + 8 * s, 1);
        mbar_init(bar_acc, 1);
        mbar_init(bar_free, 16);
        mbar_init(bar_final, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 96) prefetch_map(&map_w), prefetch_map(&map_x), prefetch_map(&map_ws), prefetch_map(&map_xs);
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster.sync();                                        // both CTAs' barriers and tensor memory are there
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);
    const uint32_t first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (warp == 0) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        const bool leader = elect_one();
        const uint32_t bytes = G::W_BYTES + p.tokens / 2 * 128 + G::S_BYTES * (1 + p.tokens / 128), to = in_leader(bar_full);
        uint32_t s = 0, ph = 0, issued = 0;
        bool ok = true;
        for (uint32_t tile = first; ok && tile < p.tiles; tile += stride) {
            const uint32_t tn = tile / p.tiles_m, m0 = (tile - tn * p.tiles_m) * p.tokens, half = pair_tile_tokens(p, m0) / 2;
            for (uint32_t k = 0; k < p.steps; ++k) {
                if (!(ok = warp_wait(bar_empty + 8 * s, ph ^ 1, abort_flag, p.status))) break;
                if (leader) {
                    const uint32_t at = smem + s * G::STAGE, bar = to + 8 * s;
                    if (rank == 0) mbar_arrive_expect_tx(bar_full + 8 * s, 2 * bytes);
                    pair_load_2d(at, &map_w, k * 128, tn * 256 + rank * 128, bar);
                    pair_load_2d(at + G::OFF_X, &map_x, k * 128, m0 + rank * half, bar);
                    pair_load_3d(at + G::OFF_WS, &map_ws, 0, k * G::ATOMS, tn * 2 + rank, bar);
                    pair_load_3d(at + G::OFF_XS, &map_xs, 0, k * G::ATOMS, m0 / 128, bar);
                }
                ++issued;
                if (++s == S) s = 0, ph ^= 1;
            }
        }
        if (rank == 0) let_copies_land(bar_full, issued, S);               // the other CTA's too
        // the commits to this CTA's barriers arrive before it leaves
        for (uint32_t j = (issued > S ? issued - S : 0); j < issued; ++j) mbar_wait_leaving(bar_empty + 8 * (j % S), (j / S) & 1);
    } else if (warp == 1) {
        if (rank == 0) {
            asm volatile("griddepcontrol.wait;" ::: "memory");     // (its waits are limited in time, the grid before is not)
            // e2m1 times e2m1, scales E8M0 (bit 23) or E4M3, M = 256
            const uint32_t idesc = (1u << 7) | (1u << 10) | (NV ? 0u : 1u << 23) | (16u << 24);
            StageWork w;
            w.d = tmem, w.cw = tmem + G::COL_WS, w.cx = tmem + G::COL_XS;
            w.s_hi = (uint32_t)(desc_plain(0, 128) >> 32), w.hi = (uint32_t)(desc_sw128(0) >> 32);
            const uint32_t codes0 = (uint32_t)desc_sw128(smem), scales0 = (uint32_t)desc_plain(smem, 128);
            uint32_t s = 0, ph = 0, aph = 0;
            for (uint32_t tile = first; tile < p.tiles; tile += stride) {
                if (!warp_wait(bar_free, aph ^ 1, abort_flag, p.status)) break;
                tc_fence_after();
                const uint32_t tokens = pair_tile_tokens(p, tile % p.tiles_m * p.tokens);
                w.idesc = idesc | (tokens >> 3) << 17, w.tiles_x = tokens > 128 ? 2 : 1;
                bool ok = true;
                for (uint32_t k = 0; k < p.steps; ++k) {
                    if (!(ok = warp_wait(bar_full + 8 * s, ph, abort_flag, p.status))) break;
                    tc_fence_after();
                    const uint32_t at = s * (G::STAGE >> 4);
                    w.a = codes0 + at, w.b = codes0 + at + (G::OFF_X >> 4), w.ws = scales0 + at + (G::OFF_WS >> 4), w.xs = scales0 + at + (G::OFF_XS >> 4);
                    w.acc = k > 0;
                    w.mmas = (min(p.K - k * kMxStageK, kMxStageK) + 63) / 64;
                    stage_pair<NV>(w);
                    pair_commit_elected(bar_empty + 8 * s);
                    if (k + 1 == p.steps) pair_commit_elected(bar_acc);
                    if (++s == S) s = 0, ph ^= 1;
                }
                if (!ok) break;
                aph ^= 1;
            }
            // what is under way to this CTA arrives, and no MMA runs, before it leaves (the other CTA waits for this one below)
            if (first < p.tiles) mbar_wait_leaving(bar_free, aph ^ 1);
            pair_commit_elected(bar_final);
            mbar_wait_leaving(bar_final, 0);
            __syncwarp();
        }
    } else if (warp >= 4) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        float alpha = 1.0f;
        if (NV) {
            float a = 1.0f, b = 1.0f;
            if (p.ts_x) asm volatile("ld.global.f32 %0, [%1];" : "=f"(a) : "l"(p.ts_x) : "memory");
            if (p.ts_w) asm volatile("ld.global.f32 %0, [%1];" : "=f"(b) : "l"(p.ts_w) : "memory");
            alpha = a * b;
        }
        const uint32_t quarter = warp & 3, half = (warp - 4) / 4, free_bar = in_leader(bar_free);      // takes 128 of the tokens
        uint32_t aph = 0;
        for (uint32_t tile = first; tile < p.tiles; tile += stride, aph ^= 1) {
            if (!warp_wait(bar_acc, aph, abort_flag, p.status)) break;
            tc_fence_after();
            const uint32_t tn = tile / p.tiles_m, m0 = (tile - tn * p.tiles_m) * p.tokens, n = tn * 256 + rank * 128 + quarter * 32 + lane;
            const uint32_t there = min(p.tokens, p.M - m0), rows = there > 128 * half ? min(there - 128 * half, 128u) : 0;
            float v[4][32];
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q)
                if (32 * q < rows) tmem_ld<32>(tmem + (quarter << 21) + 128 * half + 32 * q, v[q]);
            tmem_wait_ld();
            tc_fence_before();
            if (lane == 0) arrive_remote(free_bar);
            if (n < p.N) {
                T* y = (T*)p.Y + (uint64_t)(m0 + 128 * half) * p.ldy + n;
#pragma unroll
                for (uint32_t q = 0; q < 4; ++q)
                    if (32 * q < rows) store_tokens<T, 32>(y + (uint64_t)(32 * q) * p.ldy, p.ldy, v[q], alpha, rows - 32 * q);
            }
        }
    }
    if (*abort_flag) {                                     // copies of a pair that gave up: a millisecond is ample
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 1000000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    cluster.sync();                                        // neither CTA leaves while the other's MMAs may read its memory
    if (warp == 2) {
        mbar_wait_leaving(bar_final, 0);                   // (the commit to the second CTA may come after the one to the first)
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

}  // namespace fq
