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
//   warps 4-7   drain: tcgen05.ld, tensor scales, Y (a warp stores 32 features of a token: whole sectors)
//
// Few tokens are bound by reading the weights once, and by latency on small layers: the k-steps of a tile are then split
// over a cluster of CTAs, whose sums meet in shared memory and are added in rank order by all of them, each its tokens.
// Tensor memory is given back before a CTA waits for its cluster, so that no CTA holds it while it waits for another one.
#pragma once
#include <cooperative_groups.h>

#include "fq_mx.cuh"
#include "fq_ptx.cuh"

namespace fq {

constexpr uint32_t kMxStageK = 256;

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
    static constexpr uint32_t ACCS = 2, D_COLS = ACCS * NT, COL_WS = D_COLS, COL_XS = COL_WS + ATOMS * 4, USED = COL_XS + ATOMS * 4;
    static constexpr uint32_t COLS = USED <= 64 ? 64 : (USED <= 128 ? 128 : (USED <= 256 ? 256 : 512));
    static_assert(STAGE % 1024 == 0 && USED <= 512, "stage, tensor memory");
    // Two CTAs to an SM (the next launch's beside this one's) with up to 64 tokens.
    static constexpr uint32_t SMEM = NT <= 64 ? 113 * 1024 : 227 * 1024;
    static constexpr uint32_t STAGES = (SMEM - 2048) / STAGE;
    static_assert(STAGES >= 3 && STAGES * STAGE >= NT * 128 * 4, "stages, exchange of a split tile");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t x, uint32_t y, uint32_t z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// A tile on its way to the L2 only: harmless to what another kernel is still writing there.
__device__ __forceinline__ void tma_prefetch_2d(const CUtensorMap* map, uint32_t x, uint32_t y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global.tile [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}
// One atom of scales: 32 rows of 16 bytes to the same lanes of each of the four subpartitions.
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint32_t saddr) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc_plain(saddr, 128)) : "memory");
}
template <bool NV>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    if constexpr (NV)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc) : "memory");
}

template <class T, int NT, bool NV>
__global__ void __launch_bounds__(256, 1)
fq_mx_gemm_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_ws,
                  const __grid_constant__ CUtensorMap map_xs, const MxGemmParams p) {
    using G = MxGemm<NT, NV>;
    extern __shared__ uint8_t mx_smem[];
    __shared__ uint64_t bars[2 * 16 + 2 * G::ACCS + 1];
    __shared__ uint32_t tmem_slot;
    __shared__ uint32_t abort_word;
    namespace cg = cooperative_groups;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x & 31, S = p.stages;
    const uint32_t smem = (smem_u32(mx_smem) + 1023) & ~1023u;
    const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * 16, bar_acc = bar_empty + 8 * 16, bar_free = bar_acc + 8 * G::ACCS, bar_final = bar_free + 8 * G::ACCS;
    volatile uint32_t* abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < S; ++s) mbar_init(bar_full + 8 * s, 1), mbar_init(bar_empty + 8 * s, 1);
        for (uint32_t i = 0; i < G::ACCS; ++i) mbar_init(bar_acc + 8 * i, 1), mbar_init(bar_free + 8 * i, 4);
        mbar_init(bar_final, 1);
        abort_word = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
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
        // e2m1 times e2m1, scales E8M0 (bit 23) or E4M3, N = NT, M = 128
        const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | (NV ? 0u : 1u << 23) | (8u << 24);
        uint32_t s = 0, ph = 0, acc = 0, aph = 0;
        const bool leader = elect_one();
        for (uint32_t tile = first; tile < p.tiles; tile += stride) {
            if (!warp_wait(bar_free + 8 * acc, aph ^ 1, abort_flag, p.status)) break;
            tc_fence_after();
            const uint32_t d = tmem + acc * NT;
            bool ok = true;
            for (uint32_t k = k0; k < k1; ++k) {
                if (!(ok = warp_wait(bar_full + 8 * s, ph, abort_flag, p.status))) break;
                tc_fence_after();
                if (leader) {
                    const uint32_t at = smem + s * G::STAGE;
                    const uint32_t left = p.K - k * kMxStageK, mmas = left >= kMxStageK ? 4 : (left + 63) / 64;   // (beyond K the scales are not there)
#pragma unroll
                    for (uint32_t a = 0; a < G::ATOMS; ++a) {
                        scales_to_tmem(tmem + G::COL_WS + 4 * a, at + G::OFF_WS + 512 * a);
                        scales_to_tmem(tmem + G::COL_XS + 4 * a, at + G::OFF_XS + 512 * a);
                    }
                    const uint64_t a = desc_sw128(at), b = desc_sw128(at + G::OFF_X);
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        if (j < mmas) {
                            const uint32_t atom = NV ? j : j / 2, id = NV ? 0 : 2 * (j & 1);           // which of the atom's scales
                            umma_fp4<NV>(d, a + 2 * j, b + 2 * j, idesc | id << 29 | id << 4, tmem + G::COL_WS + 4 * atom, tmem + G::COL_XS + 4 * atom,
                                         k > k0 || j > 0);
                        }
                    umma_commit(bar_empty + 8 * s);
                    if (k + 1 == k1) umma_commit(bar_acc + 8 * acc);
                }
                __syncwarp();
                if (++s == S) s = 0, ph ^= 1;
            }
            if (!ok) break;
            if (++acc == G::ACCS) acc = 0, aph ^= 1;
        }
        // No MMA is in flight when the tensor memory is given back and the CTA leaves, whoever gave up.
        if (leader) umma_commit(bar_final);
        __syncwarp();
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
        const uint32_t quarter = warp - 4, f = quarter * 32 + lane;
        uint32_t acc = 0, aph = 0;
        constexpr int C = NT < 32 ? NT : 32;
        for (uint32_t tile = first; tile < p.tiles; tile += stride) {
            if (!warp_wait(bar_acc + 8 * acc, aph, abort_flag, p.status)) break;
            tc_fence_after();
            const uint32_t tn = tile / p.tiles_m, tm = tile - tn * p.tiles_m, n = tn * 128 + f, m0 = tm * NT;
            const uint32_t rows = min((uint32_t)NT, p.M - m0);
            T* y = (T*)p.Y + (uint64_t)m0 * p.ldy + n;
            for (uint32_t c = 0; c < rows; c += C) {
                float v[C];
                tmem_ld<C>(tmem + (quarter << 21) + acc * NT + c, v);
                tmem_wait_ld();
                if (p.split > 1) {
                    float* part = reinterpret_cast<float*>(mx_smem + (smem - smem_u32(mx_smem))) + c * 128 + f;
#pragma unroll
                    for (int i = 0; i < C; ++i) part[i * 128] = v[i];
                } else if (n < p.N) {
#pragma unroll
                    for (int i = 0; i < C; ++i)
                        if (c + i < rows) y[(uint64_t)(c + i) * p.ldy] = from_float<T>(v[i] * alpha);
                }
            }
            tc_fence_before();
            if (lane == 0) mbar_arrive(bar_free + 8 * acc);
            if (++acc == G::ACCS) acc = 0, aph ^= 1;
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
        if (NV) alpha = (p.ts_x ? *(const volatile float*)p.ts_x : 1.0f) * (p.ts_w ? *(const volatile float*)p.ts_w : 1.0f);
        float* mine = reinterpret_cast<float*>(mx_smem + (smem - smem_u32(mx_smem)));
        const uint32_t f = threadIdx.x & 127, n = tn * 128 + f;
        for (uint32_t m = rank + p.split * (threadIdx.x >> 7); m < rows; m += 2 * p.split) {
            float v[8];
#pragma unroll
            for (uint32_t r = 0; r < 8; ++r)
                if (r < p.split) v[r] = cluster.map_shared_rank(mine, r)[m * 128 + f];
            float sum = 0.0f;
#pragma unroll
            for (uint32_t r = 0; r < 8; ++r)
                if (r < p.split) sum += v[r];
            if (n < p.N && !*abort_flag) ((T*)p.Y)[(uint64_t)(m0 + m) * p.ldy + n] = from_float<T>(sum * alpha);
        }
        cluster.sync();
    }
}

}  // namespace fq
