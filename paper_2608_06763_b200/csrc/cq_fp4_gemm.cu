// y[M][N] = x[M][K] W[N][K]^T, both sides 4-bit floating point with block scales (cq_fp4.cuh): tcgen05.mma takes the codes from
// shared memory and the scales from tensor memory and applies them, so nothing is decoded on the way.
#include "cq_fp4.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"

#include <type_traits>

namespace cq {
namespace fp4 {

struct GemmArgs {
    const uint8_t *w, *x;
    const float *w_scale, *x_scale;
    const int32_t *offset;   // routed: first rows of the groups
    uint16_t *y;
    int *status;
    int E, NB, KT, steps;    // matrices; row blocks of W; k tiles; 64-wide steps of the tensor core that K has
    int token_tiles, band;   // dense: tiles along the rows of x; how many of them are swept together
    int M;                   // rows of x
    int64_t N;
    bool f16;
};

// D[tmem] (+)= A B, codes by shared-memory descriptors, scales in tensor memory
template <int FMT>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    if (FMT == MX)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// 512 bytes of scales (32 rows of 16 bytes) to four columns of tensor memory, in all four groups of 32 lanes
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// descriptor of such a piece: eight-row groups of 128 contiguous bytes, no swizzle
__device__ __forceinline__ uint64_t smem_desc_plain(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)8 << 16) | ((uint64_t)8 << 32) | ((uint64_t)1 << 46);
}
// Instruction descriptor: e2m1 both, scale type (bit 23: e8m0), M = 128, N by the tile.  sf: which scales of a 32-bit column an
// MXFP4 step takes (0: the first two, 2: the last two).
template <int FMT>
__device__ __forceinline__ uint32_t idesc_fp4(uint32_t n, uint32_t sf) {
    return (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (FMT == MX ? 1u << 23 : 0u) | (1u << 27) | (sf << 4) | (sf << 29);
}

template <int FMT, int BN>
struct Shape {
    static constexpr int SB = scale_bytes(FMT), HALVES = BN / 128;
    static constexpr int STAGE = CODE_BYTES + SB + HALVES * (CODE_BYTES + SB);
    static constexpr int STAGES = BN == 256 ? 4 : 6;
    static constexpr int ACCS = BN == 256 ? 1 : 2;             // accumulators: while one is read the next tile fills the other
    static constexpr int ATOMS = SB / 512;                     // scale pieces of a row block and stage
    static constexpr int SF_COLS = ATOMS * 4 * (1 + HALVES);   // scale columns of a stage; each stage has its own
    static constexpr int SF0 = ACCS * BN;
    static_assert(SF0 + STAGES * SF_COLS <= 512, "tensor memory");
    static constexpr size_t smem(int E, bool routed) { return 1024 + (size_t)STAGES * STAGE + 256 + (routed ? 3 * (size_t)(E + 1) * 4 : 0); }
};

struct Item { int e, nb, row0, rows, xblk; int64_t yrow; };   // matrix, row block, first row inside the group, rows, row block of x, row of y

// The idx-th output tile.  Token tiles run fastest within a band of them, so that the CTAs that work at the same time share the
// weights of few row blocks and the activations of one band; both then come from L2.
template <int BN>
__device__ __forceinline__ Item item_of(const GemmArgs &p, int idx, const int *s_off, const int *s_blk, const int *s_item) {
    Item t;
    int rows = p.M, tiles = p.token_tiles, first_blk = 0;
    int64_t first_row = 0;
    t.e = 0;
    if (p.offset) {
        t.e = find_group(s_item, p.E, idx);
        idx -= s_item[t.e];
        first_row = s_off[t.e];
        rows = s_off[t.e + 1] - s_off[t.e];
        first_blk = s_blk[t.e];
        tiles = (rows + BN - 1) / BN;
    }
    const int per_band = p.NB * p.band, g = idx / per_band, rem = idx - g * per_band;
    const int wide = min(p.band, tiles - g * p.band);
    t.nb = rem / wide;
    const int tt = g * p.band + rem - t.nb * wide;
    t.row0 = tt * BN;
    t.rows = min(BN, rows - t.row0);
    t.xblk = first_blk + tt * (BN / 128);
    t.yrow = first_row + t.row0;
    return t;
}

// Warp 0 brings tiles (bulk copies), warp 1 issues the MMAs, warps 2 to 5 write y.
// SPLIT: the CTAs of a cluster share one output tile, each a run of its k tiles; the partial sums meet in the shared memory of the
// cluster, where rank r adds the channels 128 / S r .. in the order of the ranks.  One tile a CTA then; else CTAs take tiles in turn.
template <int FMT, int BN, bool SPLIT>
__global__ void __launch_bounds__(192, 1) fp4_gemm_kernel(const GemmArgs p, int S, int64_t n_items) {
    using SH = Shape<FMT, BN>;
    constexpr int ST = SH::STAGES, SB = SH::SB, ACCS = SH::ACCS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *full = reinterpret_cast<uint64_t *>(ring + ST * SH::STAGE), *empty = full + ST, *acc_full = empty + ST, *acc_empty = acc_full + ACCS;
    uint64_t *drained = acc_empty + ACCS;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(drained + 1);
    volatile int *dead = reinterpret_cast<volatile int *>(s_tmem + 1);
    int *s_off = reinterpret_cast<int *>(ring + ST * SH::STAGE + 256), *s_blk = s_off + p.E + 1, *s_item = s_blk + p.E + 1;
    static_assert((2 * ST + 2 * ACCS + 1) * 8 + 8 <= 256, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = SPLIT ? (int)tc::cluster_rank() : 0;

    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) { tc::mbar_init(&full[i], 1); tc::mbar_init(&empty[i], 1); }
        for (int i = 0; i < ACCS; ++i) { tc::mbar_init(&acc_full[i], 1); tc::mbar_init(&acc_empty[i], 4); }
        tc::mbar_init(drained, 1);
        *dead = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        tc::tmem_alloc(s_tmem, 512);
        tc::tmem_relinquish();
    }
    tc::wait_for_previous_kernel();
    if (p.offset && warp == 2) {
        scan_groups(p.offset, p.E, p.M, s_off, s_blk);
        __syncwarp();
        int sum = 0;   // tiles in front of each group
        for (int e0 = 0; e0 <= p.E; e0 += 32) {
            const int e = e0 + lane;
            int v = e > 0 && e <= p.E ? p.NB * ((s_off[e] - s_off[e - 1] + BN - 1) / BN) : 0;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int u = __shfl_up_sync(~0u, v, d);
                if (lane >= d) v += u;
            }
            v += sum;
            if (e <= p.E) s_item[e] = v;
            sum = __shfl_sync(~0u, v, 31);
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *s_tmem;
    const int items = p.offset ? s_item[p.E] : (int)n_items;
    const int first = SPLIT ? (int)(blockIdx.x / S) : (int)blockIdx.x, stride = SPLIT ? items : (int)gridDim.x;   // split: one tile
    // this CTA's k tiles
    const int k0 = SPLIT ? (int)((int64_t)p.KT * rank / S) : 0, k1 = SPLIT ? (int)((int64_t)p.KT * (rank + 1) / S) : p.KT;

    int it = 0;   // stages filled (warp 0) or used (warp 1) so far
    if (warp == 0) {
        if (lane == 0) {
            for (int idx = first; idx < items && !*dead; idx += stride) {
                const Item t = item_of<BN>(p, idx, s_off, s_blk, s_item);
                const int n = (t.rows + 15) & ~15;
                const uint8_t *wt = p.w + ((int64_t)(t.e * (int64_t)p.NB + t.nb) * p.KT + k0) * tile_bytes(FMT);
                const uint8_t *xt = p.x + ((int64_t)t.xblk * p.KT + k0) * tile_bytes(FMT);
                const int64_t next_block = (int64_t)p.KT * tile_bytes(FMT);
                const int n0 = n < 128 ? n : 128, n1 = n - n0;
                const uint32_t bytes = tile_bytes(FMT) + (uint32_t)n * 128 + SB + (n1 ? SB : 0);
                for (int kt = k0; kt < k1; ++kt, ++it, wt += tile_bytes(FMT), xt += tile_bytes(FMT)) {
                    const int s = it % ST;
                    if (it >= ST && !tc::mbar_wait(&empty[s], (it / ST - 1) & 1, p.status, 51, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead)) { *dead = 1; break; }
                    uint8_t *a = ring + s * SH::STAGE, *b = a + CODE_BYTES + SB, *bs = b + SH::HALVES * CODE_BYTES;
                    tc::mbar_arrive_expect_tx(&full[s], bytes);
                    tc::bulk_load(a, wt, tile_bytes(FMT), &full[s]);
                    tc::bulk_load(b, xt, (uint32_t)n0 * 128, &full[s]);
                    tc::bulk_load(bs, xt + CODE_BYTES, SB, &full[s]);
                    if (n1) {
                        tc::bulk_load(b + CODE_BYTES, xt + next_block, (uint32_t)n1 * 128, &full[s]);
                        tc::bulk_load(bs + SB, xt + next_block + CODE_BYTES, SB, &full[s]);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        int local = 0;
        bool ok = true;
        for (int idx = first; idx < items && ok; idx += stride, ++local) {
            const Item t = item_of<BN>(p, idx, s_off, s_blk, s_item);
            const int n = (t.rows + 15) & ~15, acc = local % ACCS;
            const uint32_t d = tmem + acc * BN;
            if (local >= ACCS) ok = tc::mbar_wait(&acc_empty[acc], (local / ACCS - 1) & 1, p.status, 53, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead);
            tc::tc_fence_after();
            for (int kt = k0; kt < k1 && ok; ++kt, ++it) {
                const int s = it % ST;
                ok = tc::mbar_wait(&full[s], (it / ST) & 1, p.status, 54, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead);
                if (!ok) break;
                tc::tc_fence_after();
                const uint32_t a = tc::smem_u32(ring + s * SH::STAGE), b = a + CODE_BYTES + SB, bs = b + SH::HALVES * CODE_BYTES;
                const uint32_t sfa = tmem + SH::SF0 + s * SH::SF_COLS, sfb = sfa + SH::ATOMS * 4;
                const int steps = min(4, p.steps - 4 * kt);
                if (tc::elect_one()) {
                    const uint64_t da = tc::smem_desc_sw128(a), db = tc::smem_desc_sw128(b);
                    const uint64_t dsa = smem_desc_plain(a + CODE_BYTES), dsb = smem_desc_plain(bs);
#pragma unroll
                    for (int j = 0; j < SH::ATOMS; ++j) {
                        copy_scales(sfa + j * 4, dsa + j * 32);
#pragma unroll
                        for (int h = 0; h < SH::HALVES; ++h) copy_scales(sfb + (j * SH::HALVES + h) * 4, dsb + j * 32 + h * (SB / 16));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (j >= steps) break;
                        const int atom = FMT == MX ? j / 2 : j;
                        umma_fp4<FMT>(d, da + 2 * j, db + 2 * j, idesc_fp4<FMT>(n, FMT == MX ? (j & 1) * 2 : 0), sfa + atom * 4, sfb + atom * 4 * SH::HALVES, kt > k0 || j > 0);
                    }
                    tc::umma_commit(&empty[s]);
                    if (kt == k1 - 1) tc::umma_commit(&acc_full[acc]);
                }
                __syncwarp();
            }
        }
        if (!ok) {   // what was issued completes before tensor memory is given back
            if (lane == 0) *dead = 1;
            if (tc::elect_one()) tc::umma_commit(drained);
            __syncwarp();
            tc::mbar_wait(drained, 0, p.status, 55);
        }
    } else {
        const int quad = warp & 3;   // the 32 lanes of tensor memory that a warp may read
        int local = 0;
        for (int idx = first; idx < items; idx += stride, ++local) {
            const Item t = item_of<BN>(p, idx, s_off, s_blk, s_item);
            const int acc = local % ACCS;
            const bool ok = tc::mbar_wait(&acc_full[acc], (local / ACCS) & 1, p.status, 56, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead);
            if (!__all_sync(~0u, ok)) { *dead = 1; break; }
            tc::tc_fence_after();
            if constexpr (!SPLIT) {
                const float alpha = (p.w_scale ? p.w_scale[t.e] : 1.0f) * (p.x_scale ? *p.x_scale : 1.0f);
                const int64_t ch = (int64_t)t.nb * 128 + quad * 32 + lane;
                uint16_t *out = p.y + t.yrow * p.N + ch;
                for (int c0 = 0; c0 < t.rows; c0 += 32) {
                    uint32_t v[32];
                    tc::tmem_ld32(tmem + acc * BN + c0 + ((uint32_t)(quad * 32) << 16), v);
                    tc::tmem_ld_wait();
                    if (ch < p.N) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (c0 + i >= t.rows) break;
                            const float f = __uint_as_float(v[i]) * alpha;
                            out[(int64_t)(c0 + i) * p.N] = p.f16 ? __half_as_ushort(__float2half_rn(f)) : __bfloat16_as_ushort(__float2bfloat16_rn(f));
                        }
                    }
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&acc_empty[acc]);
            }
        }
    }

    if constexpr (SPLIT) {
        // every CTA's MMAs are done (the warps that read tensor memory waited for them), so the rings are free for partial sums
        const Item t = item_of<BN>(p, first, s_off, s_blk, s_item);
        const int CW = 128 / S, n = (t.rows + 15) & ~15;
        __syncthreads();
        tc::cluster_sync();
        const bool alive = !*dead;
        float *part = reinterpret_cast<float *>(ring);   // [rank that sent it][token][channel of mine]
        if (warp >= 2 && alive) {
            const int quad = warp & 3, c = quad * 32 + lane, owner = c / CW;
            const uint32_t to = tc::map_to_rank(part, owner) + (uint32_t)((rank * n) * CW + c % CW) * 4;
            for (int c0 = 0; c0 < t.rows; c0 += 32) {
                uint32_t v[32];
                tc::tmem_ld32(tmem + c0 + ((uint32_t)(quad * 32) << 16), v);
                tc::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (c0 + i < t.rows) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(to + (uint32_t)((c0 + i) * CW) * 4), "r"(v[i]) : "memory");
            }
        }
        __syncwarp();
        tc::cluster_sync();
        if (alive) {
            const float alpha = (p.w_scale ? p.w_scale[t.e] : 1.0f) * (p.x_scale ? *p.x_scale : 1.0f);
            for (int i = threadIdx.x; i < t.rows * CW; i += 192) {
                const int token = i / CW, c = i % CW;
                const int64_t ch = (int64_t)t.nb * 128 + rank * CW + c;
                float f = 0.0f;
                for (int s = 0; s < S; ++s) f += part[(s * n + token) * CW + c];
                f *= alpha;
                if (ch < p.N) p.y[(t.yrow + token) * p.N + ch] = p.f16 ? __half_as_ushort(__float2half_rn(f)) : __bfloat16_as_ushort(__float2bfloat16_rn(f));
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (*dead && threadIdx.x == 0)   // a wait gave up: copies in flight land before the shared memory goes away
        for (int i = it < ST ? 0 : it - ST; i < it; ++i) tc::mbar_wait(&full[i % ST], (i / ST) & 1, p.status, 52);
    if (warp == 1) {
        tc::tc_fence_after();
        tc::tmem_dealloc(tmem, 512);
    }
}

template <int FMT, int BN, bool SPLIT>
static cudaError_t launch(const GemmArgs &p, int S, int64_t items, unsigned grid, cudaStream_t st) {
    static std::atomic<uint64_t> done{0};
    const size_t smem = Shape<FMT, BN>::smem(p.E, p.offset != nullptr);
    const cudaError_t e = ensure_func_attr(fp4_gemm_kernel<FMT, BN, SPLIT>, done, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<FMT, BN>::smem(MAX_EXPERTS, true));
    if (e != cudaSuccess) return e;
    return launch_overlapped(fp4_gemm_kernel<FMT, BN, SPLIT>, dim3(grid), 192u, smem, st, SPLIT ? S : 1, true, p, S, items);
}

}  // namespace fp4

using namespace fp4;

cudaError_t launch_fp4_gemm(const void *w, const float *w_scale, const void *x, const float *x_scale, const int32_t *offset, int E, int fmt, uint16_t *y, int64_t M,
                            int64_t N, int64_t K, bool f16, int *status, cudaStream_t st) {
    GemmArgs p{};
    p.w = (const uint8_t *)w; p.x = (const uint8_t *)x; p.w_scale = w_scale; p.x_scale = x_scale; p.offset = offset; p.y = y; p.status = status;
    p.E = E; p.NB = (int)((N + 127) / 128); p.KT = (int)((K + KB - 1) / KB); p.steps = (int)((K + 63) / 64);
    p.M = (int)M; p.N = N; p.f16 = f16;
    const int64_t sms = sm_count();
    int S = 1, BN = (offset ? M / E : M) > 128 ? 256 : 128;
    if (!offset && M <= 256) {
        BN = M > 128 ? 256 : 128;
        while (S < 8 && 2 * S <= p.KT && 2 * S * p.NB <= sms) S *= 2;
    }
    p.token_tiles = (int)((M + BN - 1) / BN);
    p.band = 16;
    const int64_t items = (int64_t)p.NB * p.token_tiles;
    const unsigned grid = S > 1 ? (unsigned)(items * S) : (unsigned)(offset ? sms : items < sms ? items : sms);
    auto go = [&](auto f) {
        constexpr int F = decltype(f)::value;
        if (S > 1) return BN == 256 ? launch<F, 256, true>(p, S, items, grid, st) : launch<F, 128, true>(p, S, items, grid, st);
        return BN == 256 ? launch<F, 256, false>(p, 1, items, grid, st) : launch<F, 128, false>(p, 1, items, grid, st);
    };
    return fmt == MX ? go(std::integral_constant<int, MX>{}) : go(std::integral_constant<int, NV>{});
}

}  // namespace cq
