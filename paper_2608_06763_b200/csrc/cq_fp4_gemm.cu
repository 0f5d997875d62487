// y[M][N] = x[M][K] W[N][K]^T, both sides 4-bit floating point with block scales (cq_fp4.cuh): tcgen05.mma takes the codes from
// shared memory and the scales from tensor memory and applies them, so nothing is decoded on the way.
#include "cq_fp4.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"
#include "cq_tiles.cuh"

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
    int bt, token_tiles, band;   // rows of x to a tile; dense: tiles along the rows of x; how many of them are swept together
    int M;                   // rows of x
    int64_t N;
    bool f16, wide;          // wide: rows of y start on 16-byte boundaries
    bool early;              // launched right behind the quantiser of x: everything else may be read before that has ended
    const uint16_t *xr;      // FEW: rows of x in the model dtype, ldx apart
    int64_t ldx, K;
    __device__ __forceinline__ int rows_of_tile(int, int) const { return bt; }
};

// What a CTA computes.  ONE: 128 channels x up to 128 rows of x; TWO: a pair of CTAs 256 channels x up to 256 rows; FEW: 128 channels x up to 16
// rows, which it quantises itself and keeps in shared memory; SMALL: 128 channels x up to 64 rows.
enum { ONE = 0, TWO = 1, FEW = 2, SMALL = 3 };
// rows, and k tiles of them, that fit beside the ring
constexpr int FEW_ROWS = 16, FEW_TILES = 16;
// A CTA quantises rows x k tiles, sixteen of their product at a time (0.5 us), while its weights come; in front of it that is a launch.  Where the
// first costs no more.  us, by itself / in front, MXFP4: 32: 6.4 / 6.8 (8 rows, 4096 x 4096), 13.4 / 15.4 (2 rows, 28672 x 4096); 48: 6.9 / 6.9 (12 rows,
// 4096 x 4096), 6.6 / 6.8 (12, 8192 x 2048), 14.3 / 15.5 (3, 28672 x 4096); 52 to 64 with many rows: 7.4 / 7.0 (13 and 16, 4096 x 4096), 7.1 / 6.8
// (13 and 16, 8192 x 2048); with many k tiles, which take longer themselves: 10.8 / 11.5 (4, 4096 x 14336), 14.9 / 15.4 (4, 28672 x 4096), 7.1 / 7.6 (8,
// 2048 x 8192), 7.4 / 7.4 (8, 6144 x 4096); beyond 64: 11.3 / 11.2 (5, 4096 x 14336), 15.5 / 15.6 (5, 28672 x 4096), 12.1 / 11.5 (6, 4096 x 14336).
constexpr int few_most(int rows) { return rows <= 8 ? 64 : 48; }

// D[tmem] (+)= A B, codes by shared-memory descriptors, scales in tensor memory.  PAIR: by the tensor cores of two SMs, each with 128 of
// the 256 rows of A and half of the columns of B in its shared memory.
template <int FMT, bool PAIR>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
#define CQ_UMMA_FP4(group, kind)                                                                          \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"                                        \
                 "tcgen05.mma.cta_group::" group ".kind::" kind " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"  \
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory")
    if (FMT == MX) {
        if (PAIR) CQ_UMMA_FP4("2", "mxf4.block_scale.scale_vec::2X"); else CQ_UMMA_FP4("1", "mxf4.block_scale.scale_vec::2X");
    } else {
        if (PAIR) CQ_UMMA_FP4("2", "mxf4nvf4.block_scale.scale_vec::4X"); else CQ_UMMA_FP4("1", "mxf4nvf4.block_scale.scale_vec::4X");
    }
#undef CQ_UMMA_FP4
}
// 512 bytes of scales (32 rows of 16 bytes) to four columns of tensor memory, in all four groups of 32 lanes.  PAIR: in both SMs, each
// from its own shared memory.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    if (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// descriptor of such a piece: eight-row groups of 128 contiguous bytes, no swizzle
__device__ __forceinline__ uint64_t smem_desc_plain(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)8 << 16) | ((uint64_t)8 << 32) | ((uint64_t)1 << 46);
}
// Instruction descriptor: e2m1 both, scale type (bit 23: e8m0), M = 128 (a pair 256), N by the tile.  Bits 4 and 29 up, added where it is
// used: which scales of a 32-bit column an MXFP4 step takes (0: the first two, 2: the last two).
template <int FMT, bool PAIR>
__device__ __forceinline__ uint32_t idesc_fp4(uint32_t n) {
    return (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (FMT == MX ? 1u << 23 : 0u) | ((PAIR ? 2u : 1u) << 27);
}

__device__ __forceinline__ uint32_t pack_out(uint32_t lo, uint32_t hi, float alpha, bool f16) {
    const float a = __uint_as_float(lo) * alpha, b = __uint_as_float(hi) * alpha;
    if (f16) { const __half2 p = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t *>(&p); }
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&p);
}
template <int FMT, int MODE, bool SPLIT>
struct Shape {
    static constexpr bool PAIR = MODE == TWO;
    static constexpr int BN = MODE == TWO ? 256 : MODE == ONE ? 128 : MODE == SMALL ? 64 : FEW_ROWS, CTAS = PAIR ? 2 : 1;
    static constexpr int SB = scale_bytes(FMT), BLOCKS = PAIR ? 2 : 1;      // row blocks of x that a tile may touch
    static constexpr int A_BYTES = CODE_BYTES + SB, B_BYTES = MODE == SMALL ? BN * 128 : CODE_BYTES;   // codes of x in this CTA: half of a pair's
    static constexpr int STAGE = A_BYTES + (MODE == FEW ? 0 : B_BYTES + BLOCKS * SB);
    static constexpr int STAGES = MODE == FEW ? 8 : MODE == SMALL ? 6 : MODE == ONE && SPLIT ? 4 : 5;
    static constexpr int ACCS = PAIR ? 1 : 2, ACC_COLS = BN < 32 ? 32 : BN;   // accumulators: while one is read the next tile fills the other
    static constexpr int ATOMS = SB / 512;                       // scale pieces of a row block and stage
    static constexpr int SF_COLS = ATOMS * 4 * (1 + BLOCKS);     // scale columns of a stage; each stage has its own
    // Up to 64 rows a stage's MMAs are short, and what bounds the stage is the warp that issues them (waiting, fencing, eight or twelve instructions,
    // committing: 500 cycles).  Two warps take turns then, each with accumulators of its own, which are added at the end.
    static constexpr int MMAS = MODE == FEW || MODE == SMALL ? 2 : 1;
    static constexpr int SF0 = ACCS * MMAS * ACC_COLS;
    static constexpr int PITCH = 272;                            // bytes of a row of the staged output: 128 channels and a gap against bank conflicts
    static constexpr int X_CODES = FEW_ROWS * 128, X_BYTES = MODE == FEW ? FEW_TILES * (X_CODES + SB) : 0;   // FEW: codes of a k tile; all k tiles
    static constexpr int OUT_BYTES = SPLIT ? 128 * (BN + 4) * 4 : (MODE == FEW ? 32 : 64) * PITCH;   // SPLIT: partial sums [run][channel][row of x, and a gap]
    // A stage of the ring always has the same one of them: a warp that passed over a stage in one round cannot tell from the parity of its
    // barrier, in the next, whether that round has come.
    static_assert(STAGES % MMAS == 0, "a stage belongs to one issuing warp");
    static_assert(SF0 + STAGES * SF_COLS <= 512, "tensor memory");
    static constexpr size_t smem(int E, bool routed) { return (size_t)STAGES * STAGE + X_BYTES + OUT_BYTES + 256 + (routed ? 3 * (size_t)(E + 1) * 4 : 0); }
    static_assert(STAGES * STAGE + X_BYTES + OUT_BYTES + 256 + (MODE == FEW ? 0 : 12 * (MAX_EXPERTS + 1)) <= 232448, "shared memory");
};

// SPLIT, the eight warps that write y: this CTA's partial sums to the CTAs that add them, then its own 128 / S channels of all runs, in their
// order.  Sums arrive counted on a barrier, so nobody waits for the whole cluster in between.  Few rows are sent from the registers;
// more go through the ring, which nobody needs any more, and from there in one copy to each CTA (128 rows: 6000 cycles in pieces of
// sixteen bytes, 2500 so).
// gave_up: the accumulator did not come.  Such a CTA sends zeros, and waits like the others for what is sent to it: a CTA whose sums have not all
// come may not leave, since they would land in shared memory that is no longer its own.  After a wait that ran out it waits once more; the
// status tells that y is not valid.
template <class SH>
__device__ __forceinline__ void send_and_add(const GemmArgs &p, const Item &t, int lgS, int run, int k_tiles, int warp, int lane, uint8_t *ring, uint8_t *part, uint64_t *sums,
                                             volatile int *dead, bool gave_up) {
    constexpr bool COPY = SH::BN > 16;
    const int lgCW = 7 - lgS, CW = 1 << lgCW, pitch = ((t.rows + 15) & ~15) + 4;
    const int quad = warp & 3, c = quad * 32 + lane, owner = c >> lgCW, tid = threadIdx.x - 128;
    const uint32_t bytes_of_run = (uint32_t)(pitch << lgCW) * 4u;
    if (tid == 0) tc::mbar_arrive_expect_tx(sums, COPY ? ((1u << lgS) - 1) * bytes_of_run : 128u * (uint32_t)((t.rows + 3) & ~3) * 4u);
    tc::tc_fence_after();
    __syncwarp();
    if (!COPY) cluster_wait();   // the others have started, and their barriers exist
    const uint32_t to = COPY ? tc::smem_u32(ring) + (uint32_t)c * pitch * 4 : tc::map_to_rank(part, owner) + (uint32_t)((run << lgCW) + (c & (CW - 1))) * pitch * 4;
    const uint32_t bar = COPY ? 0 : tc::map_to_rank(sums, owner);
    for (int c0 = (warp - 4) / 4 * 32; c0 < t.rows; c0 += 64) {
        uint32_t v[32];
        tc::tmem_ld32(c0 + ((uint32_t)(quad * 32) << 16), v);
        if (SH::MMAS == 2 && k_tiles > 1) {   // the sums of the other k tiles
            uint32_t v1[32];
            tc::tmem_ld32(SH::ACC_COLS + c0 + ((uint32_t)(quad * 32) << 16), v1);
            tc::tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(v1[i]));
        } else {
            tc::tmem_ld_wait();
        }
        if (gave_up) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 4)
            if (c0 + i < t.rows) {
                if (COPY) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + (uint32_t)(c0 + i) * 4), "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]) : "memory");
                else send(to + (uint32_t)(c0 + i) * 4, bar, v[i], v[i + 1], v[i + 2], v[i + 3]);
            }
    }
    if (COPY) {
        tc::fence_proxy_async();
        epilogue_sync();
        cluster_wait();   // the others have started, and their barriers exist
        if (tid < 1 << lgS && tid != run)
            asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(tc::map_to_rank(part, tid) + run * bytes_of_run), "r"(tc::smem_u32(ring) + tid * bytes_of_run), "r"(bytes_of_run), "r"(tc::map_to_rank(sums, tid)) : "memory");
        __syncwarp();
    } else {
        __syncwarp();
        cluster_arrive();
    }
    const float alpha = (p.w_scale ? p.w_scale[t.e] : 1.0f) * (p.x_scale ? *p.x_scale : 1.0f);
    const bool ok = tc::mbar_wait(sums, 0, p.status, 58, tc::WAIT_LIMIT_CYCLES, gave_up ? nullptr : dead);
    if (!ok) {
        *dead = 1;
        tc::mbar_wait(sums, 0, p.status, 58);
    }
    __syncwarp();
    if (COPY) cluster_arrive();   // what was copied from here has been received when all have arrived
    if (!ok || gave_up) return;
    // two channels of four rows a thread
    const int mine = 2 * (tid & (CW / 2 - 1));
    const int64_t ch = (int64_t)t.nb * 128 + (run << lgCW) + mine;
    uint16_t *out = p.y + (int64_t)t.yrow * p.N + ch;
    for (int r = (tid >> (lgCW - 1)) * 4; r < t.rows; r += (512 >> lgCW) * 4) {
        float f[2][4];
        for (int s = 0; s < 1 << lgS; ++s) {
            const uint8_t *from = COPY && s == run ? ring + s * bytes_of_run : part + s * bytes_of_run;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = *reinterpret_cast<const float4 *>(from + ((mine + j) * pitch + r) * 4);
                if (s == 0) { f[j][0] = v.x; f[j][1] = v.y; f[j][2] = v.z; f[j][3] = v.w; }
                else { f[j][0] += v.x; f[j][1] += v.y; f[j][2] += v.z; f[j][3] += v.w; }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (r + i >= t.rows) break;
            const uint16_t a = round_out(f[0][i] * alpha, p.f16), b = round_out(f[1][i] * alpha, p.f16);
            uint16_t *at = out + (int64_t)(r + i) * p.N;
            if (p.wide && ch < p.N) *reinterpret_cast<uint32_t *>(at) = a | (uint32_t)b << 16;   // N even: both are inside
            else {
                if (ch < p.N) at[0] = a;
                if (ch + 1 < p.N) at[1] = b;
            }
        }
    }
}

// Warps 0 and 2 bring tiles (bulk copies: 0 those of W, 2 those of x), warp 1 issues the MMAs (in the second CTA of a pair it tells the first
// that its tiles are there), warp 3 those of every second stage of small tiles, having read the offsets of routed rows, warps 4 to 11 write y.
// SPLIT: 2^lgS CTAs of a cluster share one output tile, each a run of its k tiles; the partial sums meet in the shared memory of the
// cluster, where each CTA adds 128 / S channels in the order of the runs.  One tile a CTA then; else CTAs (pairs) take tiles in turn.
// What bounds it.  256 x 256 tiles of pairs: a stage of 256 k is 512 cycles of the tensor core at its rate, and takes 640 with everything
// around it (issuing 14 to 18 instructions a stage, a tile's accumulators read before the next tile starts); 57344 x 8192, 4096 rows 650 to 820 us, 4.7 to
// 5.9 PFLOP/s, by what the power limit leaves of the clock; 8192 x 8192, 4096 rows 100 us in a burst with the tensor pipe 78 % active.  Copies come
// as they are stored, a contiguous run each.  One CTA of 128 x 128 is bound by its SM's port to L2 (36.9 KB a stage, 600 cycles), small tiles by
// memory: 28672 x 4096, 13 rows 13.1 us for 63 MB, of which some three are the launch, the first copies' way and the last tile's output, and
// one and a half the second round of tiles, which 76 of 148 SMs have.
// FEW: warps 4 to 11 first quantise the rows for this CTA's k tiles, while the first weights are on their way.
template <int FMT, int MODE, bool SPLIT>
__global__ void __launch_bounds__(384, 1) fp4_gemm_kernel(const GemmArgs p, int lgS, int n_items) {
    using SH = Shape<FMT, MODE, SPLIT>;
    constexpr bool PAIR = SH::PAIR;
    static_assert(!(PAIR && SPLIT), "pairs take whole tiles");
    constexpr int ST = SH::STAGES, SB = SH::SB, ACCS = SH::ACCS, BN = SH::BN, CTAS = SH::CTAS, ACC_COLS = SH::ACC_COLS, MMAS = SH::MMAS;
    constexpr uint32_t TMEM = 0;   // a CTA takes all of tensor memory: its first column is column 0
    extern __shared__ __align__(1024) uint8_t ring[];   // the swizzle counts address bits from 1024 on
    uint8_t *x_codes = ring + ST * SH::STAGE, *x_scales = x_codes + FEW_TILES * SH::X_CODES;
    uint8_t *staged = x_codes + SH::X_BYTES;
    uint64_t *full = reinterpret_cast<uint64_t *>(staged + SH::OUT_BYTES), *empty = full + ST, *acc_full = empty + ST, *acc_empty = acc_full + ACCS;
    uint64_t *drained = acc_empty + ACCS, *x_ready = drained + MMAS, *sums = x_ready + 1;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(sums + 1);
    volatile int *dead = reinterpret_cast<volatile int *>(s_tmem + 1);
    int *s_off = reinterpret_cast<int *>(staged + SH::OUT_BYTES + 256), *s_blk = s_off + p.E + 1, *s_item = s_blk + p.E + 1;
    static_assert((2 * ST + 2 * ACCS + MMAS + 2) * 8 + 8 <= 256, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // From the block's number, not the cluster's registers, and by shifts: what branches and addresses of the issuing warp hang on is uniform.
    const int lgC = PAIR ? 1 : SPLIT ? lgS : 0, cluster_rank = blockIdx.x & ((1 << lgC) - 1), unit = blockIdx.x >> lgC, units = gridDim.x >> lgC;
    const int half = PAIR ? cluster_rank : 0, run = SPLIT ? cluster_rank : 0;   // which 128 channels of the pair; which run of k
    const int k0 = SPLIT ? p.KT * run >> lgS : 0, k1 = SPLIT ? p.KT * (run + 1) >> lgS : p.KT;   // this CTA's k tiles

    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) { tc::mbar_init(&full[i], MODE == FEW ? 1 : PAIR && half == 0 ? 3 : 2); tc::mbar_init(&empty[i], 1); }   // a pair's first CTA also waits for the other's tiles
        for (int i = 0; i < ACCS; ++i) { tc::mbar_init(&acc_full[i], MMAS); tc::mbar_init(&acc_empty[i], 8 * CTAS); }
        for (int i = 0; i < MMAS; ++i) tc::mbar_init(&drained[i], 1);
        tc::mbar_init(x_ready, 8);
        tc::mbar_init(sums, 1);
        *dead = 0;
        tc::fence_barrier_init();
    }
    if (warp == 1) {
        if (PAIR) tc::tmem_alloc_pair(s_tmem, 512);
        else { tc::tmem_alloc(s_tmem, 512); tc::tmem_relinquish(); }
    }
    if (!p.offset && !p.early && threadIdx.x == 0 && unit < n_items) {   // the first weights on their way to L2, which sees what the kernel in front may still write
        const int nb = min(item_of<PAIR>(p, unit, nullptr, nullptr, nullptr).nb * CTAS + half, p.NB - 1);
        for (int kt = k0; kt < k1 && kt < k0 + ST; ++kt) tc::prefetch_l2(p.w + ((int64_t)nb * p.KT + kt) * tile_bytes(FMT), SH::A_BYTES);
    }
    tc::tc_fence_before();
    __syncthreads();
    if (PAIR) tc::cluster_sync();   // the partner's barriers exist before anything arrives on them
    if (SPLIT) cluster_arrive();
    tc::tc_fence_after();
    // From here on the next kernel may start: this one holds its tensor memory, which a kernel that waits for this one might else take.
    // Behind the quantiser of this call only the layout that it writes has to be waited for (by the warp that reads it, and in every CTA): the
    // quantiser lets this kernel start once all kernels in front of itself have ended, those that wrote weights, scales and offsets among them.
    if (p.early) launch_dependents();
    else tc::wait_for_previous_kernel();
    if (p.offset) {
        if (warp == 3) scan_groups(p.offset, p.E, p.M, s_off, s_blk, s_item, p.bt, PAIR ? (p.NB + 1) >> 1 : p.NB);
        __syncthreads();
    }
    const int items = p.offset ? __reduce_max_sync(~0u, s_item[p.E]) : n_items;   // (a reduction's result is uniform)
    const int stride = SPLIT ? items : units;   // split: one tile

    Tiles<PAIR, GemmArgs> tiles{p, unit, stride, items, s_off, s_blk, s_item, {}};
    int it = 0;   // stages filled (warps 0 and 2) or used (warp 1) so far
    if (warp == 0 || (warp == 2 && MODE != FEW)) {
        // A lane for each piece of a stage: warp 0 the weights, warp 2 its rows of codes (from one row block or two) and the scales of all
        // rows of the tile.  One lane issuing all of them took 530 cycles a stage, more than the tensor core; five lanes of one warp 290.
        const int64_t block = (int64_t)p.KT * tile_bytes(FMT);   // from a row block to the next
        uint32_t s = 0, phase = 1;
        bool ok = true;
        if (warp == 2 && p.early) wait_for_quantiser();
        for (int local = 0; ok && tiles.has(local); ++local) {
            const Item t = tiles.at(local);
            const int n = columns_of<PAIR>(t.rows), mine = n / CTAS, nb = min(t.nb * CTAS + half, p.NB - 1);   // an odd last pair reads a block twice
            const int r0 = t.off + half * mine, b0 = r0 / ROWS, in0 = r0 % ROWS, n0 = min(mine, ROWS - in0), n1 = mine - n0;
            const bool two = t.off + n > ROWS;
            const uint8_t *xt = p.x + ((int64_t)t.xblk * p.KT + k0) * tile_bytes(FMT), *src = xt;
            uint32_t to = 0, bytes = 0, all = SH::A_BYTES;
            if (warp == 0) {
                if (lane == 0) { src = p.w + (((int64_t)t.e * p.NB + nb) * p.KT + k0) * tile_bytes(FMT); bytes = SH::A_BYTES; }
            } else {
                all = (uint32_t)mine * 128 + (two ? 2 * SB : SB);
                if (lane == 0) { src = xt + b0 * block + in0 * 128; to = SH::A_BYTES; bytes = (uint32_t)n0 * 128; }
                else if (lane == 1) { src = xt + CODE_BYTES; to = SH::A_BYTES + SH::B_BYTES; bytes = SB; }
                else if (lane == 2) { src = xt + block + CODE_BYTES; to = SH::A_BYTES + SH::B_BYTES + SB; bytes = two ? SB : 0; }
                else if (lane == 3) { src = xt + (b0 + 1) * block; to = SH::A_BYTES + n0 * 128; bytes = (uint32_t)n1 * 128; }
            }
            for (int kt = k0; kt < k1; ++kt, ++it, src += tile_bytes(FMT)) {
                ok = uniform_wait(&empty[s], phase, p.status, 51, dead);   // the first round passes at once
                if (!ok) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&full[s], all);
                __syncwarp();
                if (bytes) tc::bulk_load(ring + s * SH::STAGE + to, src, bytes, &full[s]);
                if (++s == ST) { s = 0; phase ^= 1; }
            }
        }
        if (!ok && lane == 0) *dead = 1;
        __syncwarp();
    } else if (warp == 1 || (warp == 3 && MMAS == 2)) {
        // The whole warp walks the loops and one lane issues: what the instructions take stays in uniform registers (a stage takes twice
        // as long where a lane of its own does it all).
        const uint32_t odd = warp >> 1;   // MMAS == 2: which stages are this warp's, every second k tile of an output tile
        uint32_t s = 0, phase = 0;
        bool ok = MODE != FEW || uniform_wait(x_ready, 0, p.status, 57, dead);
        for (int local = 0; ok && tiles.has(local); ++local) {
            const Item t = tiles.at(local);
            const uint32_t n = MODE == FEW ? FEW_ROWS : __reduce_max_sync(~0u, columns_of<PAIR>(t.rows)), sf_row = PAIR || MODE == SMALL ? __reduce_max_sync(~0u, t.off / 32) : 0;   // a tile may start inside a row block
            const int acc = local & (ACCS - 1);
            const uint32_t d = TMEM + (acc * MMAS + odd) * ACC_COLS, desc = idesc_fp4<FMT, PAIR>(n);
            if (half == 0 && local >= ACCS) ok = uniform_wait(&acc_empty[acc], (local / ACCS - 1) & 1, p.status, 53, dead);
            tc::tc_fence_after();
            bool idle = true;
            for (int kt = k0; kt < k1 && ok; ++kt) {
                if (MMAS == 1 || (s & 1) == odd) {
                    idle = false;
                    ok = uniform_wait(&full[s], phase, p.status, 54, dead);
                    if (!ok) break;
                    if (PAIR && half == 1) {
                        if (lane == 0) tc::mbar_arrive_cluster(tc::map_to_rank(&full[s], cluster_rank & ~1));
                    } else {
                        tc::tc_fence_after();
                        const uint32_t a = tc::smem_u32(ring) + s * SH::STAGE, sfa = TMEM + SH::SF0 + s * SH::SF_COLS, sfb = sfa + SH::ATOMS * 4, sfn = sfb + sf_row;
                        const uint64_t da = tc::smem_desc_sw128(a), dsa = smem_desc_plain(a + CODE_BYTES);
                        const uint64_t db = MODE == FEW ? tc::smem_desc_sw128(tc::smem_u32(x_codes) + (kt - k0) * SH::X_CODES) : da + SH::A_BYTES / 16;
                        const uint64_t dsb = MODE == FEW ? smem_desc_plain(tc::smem_u32(x_scales) + (kt - k0) * SB) : dsa + (SB + SH::B_BYTES) / 16;
                        const int steps = p.steps - 4 * kt;
                        if (tc::elect_one()) {
#pragma unroll
                            for (int j = 0; j < SH::ATOMS; ++j) {
                                copy_scales<PAIR>(sfa + j * 4, dsa + j * 32);
#pragma unroll
                                for (int h = 0; h < SH::BLOCKS; ++h) copy_scales<PAIR>(sfb + (j * SH::BLOCKS + h) * 4, dsb + j * 32 + h * (SB / 16));
                            }
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int atom = FMT == MX ? j / 2 : j;
                                const uint32_t sf = FMT == MX ? (j & 1) * 2 : 0;
                                if (j == 0 || j < steps)
                                    umma_fp4<FMT, PAIR>(d, da + 2 * j, db + 2 * j, desc | sf << 4 | sf << 29, sfa + atom * 4, sfn + atom * 4 * SH::BLOCKS, j > 0 || kt >= k0 + MMAS);
                            }
                            if (PAIR) commit_to_pair(&empty[s], cluster_rank);
                            else tc::umma_commit(&empty[s]);
                            if (kt >= k1 - MMAS) {
                                if (PAIR) commit_to_pair(&acc_full[acc], cluster_rank);
                                else tc::umma_commit(&acc_full[acc]);
                            }
                        }
                        __syncwarp();
                    }
                }
                if (++s == ST) { s = 0; phase ^= 1; }
            }
            if (MMAS == 2 && ok && idle && lane == 0) tc::mbar_arrive(&acc_full[acc]);   // one k tile, and it was the other warp's
        }
        if (!ok && lane == 0) *dead = 1;
        if (!ok && half == 0) {   // what was issued completes before tensor memory is given back
            if (tc::elect_one()) {
                if (PAIR) commit_to_pair(&drained[odd], cluster_rank);
                else tc::umma_commit(&drained[odd]);
            }
            __syncwarp();
            tc::mbar_wait(&drained[odd], 0, p.status, 55);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // Tensor memory is emptied into registers first, already in the type of y, so that the next tile's MMAs wait for no store;
        // then 64 rows of y at a time go through shared memory, where the 8x8 matrices are turned round, and out as whole rows.
        if constexpr (MODE == FEW) {
            const int tid = threadIdx.x - 128, units = (k1 - k0) * p.M * 16, KU = (int)(p.K >> 4);
            const float g = FMT == NV && p.x_scale ? *p.x_scale : 1.0f;
            const float r = __fdiv_rn(1.0f, g);
            struct Unit { int kt, row; bool live, inside; uint4 a, b; };
            const int u = tid & 15;
            auto load = [&](int i) {   // the i-th unit of sixteen k of all rows
                Unit q;
                const int line = i >> 4;
                q.kt = line / p.M;
                q.row = line - q.kt * p.M;
                const int unit = (k0 + q.kt) * 16 + u;
                q.live = i < units;
                q.inside = unit < KU;
                const uint16_t *src = p.xr + q.row * p.ldx + (int64_t)unit * 16;
                const bool read = q.live && q.inside;
                q.a = read ? load16(src) : make_uint4(0, 0, 0, 0);
                q.b = read ? load16(src + 8) : make_uint4(0, 0, 0, 0);
                return q;
            };
            Unit next = load(tid);
            for (int i0 = 0; i0 < units; i0 += 256) {   // whole warps: they exchange scales
                const Unit q = next;
                if (i0 + 256 < units) next = load(i0 + 256 + tid);
                uint32_t scale;
                const uint2 codes = p.f16 ? quantize_unit<FMT, DT_F16>(q.a, q.b, r, scale) : quantize_unit<FMT, DT_BF16>(q.a, q.b, r, scale);
                if (!q.inside) scale = 0;   // behind K
                // a tile's scales and codes as in the layout, the codes of sixteen rows alone
                const uint32_t word = gather_scales<FMT>(scale);
                if (q.live) {
                    *reinterpret_cast<uint2 *>(x_codes + q.kt * SH::X_CODES + code_offset(q.row, u * 8)) = codes;
                    uint8_t *sc = x_scales + q.kt * SB + scale_offset(q.row, FMT == NV ? u : u >> 1) - CODE_BYTES;
                    if ((lane & (FMT == NV ? 3 : 7)) == 0) *reinterpret_cast<uint32_t *>(sc) = word;
                }
            }
            tc::fence_proxy_async();   // the tensor core reads through the async proxy
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(x_ready);
        }
        const int quad = warp & 3, part = (warp - 4) >> 2;   // the 32 lanes of tensor memory that a warp may read; its half of 64 columns
        for (int local = 0; tiles.has(local); ++local) {
            const Item t = tiles.at(local);
            const int acc = local & (ACCS - 1);
            const bool ok = tc::mbar_wait(&acc_full[acc], (local / ACCS) & 1, p.status, 56, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead);
            const bool gave_up = epilogue_any(!ok);
            if (gave_up) *dead = 1;
            if constexpr (SPLIT) {
                send_and_add<SH>(p, t, lgS, run, k1 - k0, warp, lane, ring, staged, sums, dead, gave_up);
                break;
            }
            if (gave_up) break;
            tc::tc_fence_after();
            const float alpha = (p.w_scale ? p.w_scale[t.e] : 1.0f) * (p.x_scale ? *p.x_scale : 1.0f);
            const int nb = t.nb * CTAS + half;
            constexpr int GROUPS = (BN + 63) / 64;
            uint32_t out16[GROUPS][16];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g * 64 + part * 32 < t.rows) {
                    uint32_t lo[16], hi[16];
                    // one k tile: it is in the accumulators of the warp whose stage it came in
                    const uint32_t from = TMEM + (acc * MMAS + (MMAS == 2 && k1 - k0 == 1 ? local & 1 : 0)) * ACC_COLS + g * 64 + part * 32 + ((uint32_t)(quad * 32) << 16);
                    tmem_ld_16x32(from, lo);
                    tmem_ld_16x32(from + (16u << 16), hi);
                    if (MMAS == 2 && k1 - k0 > 1) {   // the sums of the other k tiles
                        uint32_t lo1[16], hi1[16];
                        tmem_ld_16x32(from + ACC_COLS, lo1);
                        tmem_ld_16x32(from + ACC_COLS + (16u << 16), hi1);
                        tc::tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            lo[i] = __float_as_uint(__uint_as_float(lo[i]) + __uint_as_float(lo1[i]));
                            hi[i] = __float_as_uint(__uint_as_float(hi[i]) + __uint_as_float(hi1[i]));
                        }
                    } else {
                        tc::tmem_ld_wait();
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        out16[g][4 * i] = pack_out(lo[4 * i], lo[4 * i + 1], alpha, p.f16);
                        out16[g][4 * i + 1] = pack_out(lo[4 * i + 2], lo[4 * i + 3], alpha, p.f16);
                        out16[g][4 * i + 2] = pack_out(hi[4 * i], hi[4 * i + 1], alpha, p.f16);
                        out16[g][4 * i + 3] = pack_out(hi[4 * i + 2], hi[4 * i + 3], alpha, p.f16);
                    }
                }
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR && half == 1) tc::mbar_arrive_cluster(tc::map_to_rank(&acc_empty[acc], cluster_rank & ~1));
                else tc::mbar_arrive(&acc_empty[acc]);
            }
            const int chans = (int)min((int64_t)128, p.N - (int64_t)nb * 128);   // none or fewer in a last block without a partner
            const int tid = threadIdx.x - 128;
            const uint32_t at = tc::smem_u32(staged) + (part * 32 + (lane & 7)) * SH::PITCH + quad * 64 + (lane >> 3) * 16;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g * 64 >= t.rows) break;
                if (g * 64 + part * 32 < t.rows) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) stmatrix_trans(at + 8 * i * SH::PITCH, out16[g][4 * i], out16[g][4 * i + 1], out16[g][4 * i + 2], out16[g][4 * i + 3]);
                }
                epilogue_sync();
                const int count = min(64, t.rows - g * 64);
                uint16_t *out = p.y + ((int64_t)t.yrow + g * 64) * p.N + (int64_t)nb * 128;
                if (p.wide) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {   // sixteen threads a row
                        const int r = i * 16 + (tid >> 4), c = (tid & 15) * 8;
                        if (r < count && c < chans) *reinterpret_cast<uint4 *>(out + (int64_t)r * p.N + c) = *reinterpret_cast<const uint4 *>(staged + r * SH::PITCH + c * 2);
                    }
                } else {
                    for (int r = warp - 4; r < count; r += 8)
                        for (int c = lane; c < chans; c += 32) out[(int64_t)r * p.N + c] = *reinterpret_cast<const uint16_t *>(staged + r * SH::PITCH + c * 2);
                }
                epilogue_sync();   // read before it is written again
            }
        }
    }

    if (SPLIT && warp < 4) {   // the others have done so on their way
        __syncwarp();
        cluster_wait();
        cluster_arrive();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (*dead && (warp == 0 || warp == 2))   // a wait gave up: copies in flight land before the shared memory goes away
        for (int i = it < ST ? 0 : it - ST; i < it; ++i) tc::mbar_wait(&full[i % ST], (i / ST) & 1, p.status, 52);
    __syncwarp();
    if (PAIR) tc::cluster_sync();   // nothing of the pair is in flight towards a CTA that has left
    if (SPLIT) cluster_wait();      // nor are partial sums
    if (warp == 1) {
        tc::tc_fence_after();
        if (PAIR) tc::tmem_dealloc_pair(TMEM, 512);
        else tc::tmem_dealloc(TMEM, 512);
    }
}

template <int FMT, int MODE, bool SPLIT>
static cudaError_t launch(const GemmArgs &p, int lgS, int64_t items, unsigned grid, cudaStream_t st) {
    using SH = Shape<FMT, MODE, SPLIT>;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = ensure_func_attr(fp4_gemm_kernel<FMT, MODE, SPLIT>, done, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SH::smem(MAX_EXPERTS, MODE != FEW));
    if (e != cudaSuccess) return e;
    return launch_overlapped(fp4_gemm_kernel<FMT, MODE, SPLIT>, dim3(grid), 384u, SH::smem(p.E, p.offset != nullptr), st, SH::CTAS << (SPLIT ? lgS : 0), true, p, lgS, (int)items);
}

}  // namespace fp4

using namespace fp4;

// Runs of k that an output tile of few row blocks is cut into, while the GPU has places for them.  Eight CTAs to a cluster leave SMs
// without a cluster that fits (4096 x 4096, one row: 14.6 us with eight, 5.9 with four).
static int lg_runs_of(int tiles, int KT, int places) {
    int lg = 0;
    while (lg < 2 && 2 << lg <= KT && (int64_t)(2 << lg) * tiles <= places) ++lg;
    return lg;
}
static GemmArgs args_of(const void *w, const float *w_scale, const float *x_scale, uint16_t *y, int64_t M, int64_t N, int64_t K, bool f16, int *status) {
    GemmArgs p{};
    p.w = (const uint8_t *)w; p.w_scale = w_scale; p.x_scale = x_scale; p.y = y; p.status = status;
    p.E = 1; p.NB = (int)((N + 127) / 128); p.KT = (int)((K + KB - 1) / KB); p.steps = (int)((K + 63) / 64);
    p.M = (int)M; p.N = N; p.K = K; p.f16 = f16; p.wide = N % 8 == 0;
    p.band = 16;
    return p;
}

// What computes a product of more than sixteen rows: kind of tile, rows to a tile, runs of k (log2).  Costs in microseconds, from tiles forced in
// turn.  A k tile of one CTA takes as long as an SM's port to L2 does for its bytes (113 bytes a nanosecond) but no less than its
// MMAs take to issue; a pair's, 0.27 to 0.36.  Cutting k saves k tiles and costs a cluster's launch and the exchange.  Measured with quantised rows, two,
// four and six rounds of pairs with 256 rows, K 1024 to 8192: 0.34 (MXFP4) to 0.355 (NVFP4) a k tile and 1.25 a tile on top (its only
// accumulators are emptied before the next tile's first MMA): at K = 2048 31 % of a tile.
//   4096 x 14336, 200 rows: SMALL 16.6, ONE 20.3 (two runs 16.3), TWO 20.5 to 22.2;  4096 x 4096, 64 rows: SMALL 6.4 (two runs 7.4), ONE 7.7, TWO 8.7;
//   128 rows: SMALL 6.5, ONE 8.4;  512 rows: ONE 9.1, TWO 10.4 to 11.5;  6144 x 4096, 1024 rows: ONE 19.0, TWO 16.0 with 192 rows to a tile, 17.8 with 256;
//   2048 x 8192, 400 rows: ONE in two runs 12.8, whole 17.3, TWO 14.1;  28672 x 4096, 512 rows: ONE 45.6, TWO 33.6 to 38.4
struct Plan { int mode, bt, lg; };
static Plan dense_plan(int64_t M, int NB, int KT, int fmt) {
    static const Plan kinds[] = {{SMALL, 64, 0}, {SMALL, 64, 1}, {ONE, 128, 0}, {ONE, 128, 1}, {TWO, 128, 0}, {TWO, 192, 0}, {TWO, 256, 0}};
    const double a_kb = tile_bytes(fmt) / 1000.0, sb_kb = scale_bytes(fmt) / 1000.0;
    const int sms = sm_count();
    Plan best = kinds[2];
    double least = 1e30;
    for (const Plan &k : kinds) {
        const int ctas = k.mode == TWO ? 2 : 1, S = 1 << k.lg, nbu = (NB + ctas - 1) / ctas, places = sms / ctas;
        if (S > KT) continue;
        const int64_t tiles = (M + k.bt - 1) / k.bt, items = nbu * tiles;
        if (k.lg && items * S > places) continue;   // one round, or the runs of several tiles wait for one another's places
        const double n = M < k.bt ? (double)M : (double)k.bt, rounds = (double)((items * S + places - 1) / places);
        double per_kt, tail, base;
        if (k.mode == TWO) { per_kt = 0.18 + 0.18 * n / 256; tail = 1.5 * n / 256; base = 3.2; }
        else {
            per_kt = (a_kb + sb_kb + 0.128 * n) / 113.0;
            const double issue = k.mode == SMALL ? 0.15 : 0.27;
            if (per_kt < issue) per_kt = issue;
            tail = 0.5; base = 2.4 + (k.lg ? (k.mode == SMALL ? 3.0 : 4.5) : 0.0);
        }
        const double cost = base + rounds * ((KT + S - 1) / S * per_kt + tail);
        if (cost < least) { least = cost; best = k; }
    }
    return best;
}
// Routed rows: the loads are on the GPU, so the mean decides.  Sixteen matrices of 2816 x 2048, us with SMALL / ONE / TWO: 24 rows on average
// 12.8 / 13.5 / 14.6, 64: 14.6 / 14.6 / 17.1, 150: 20.5 / 19.2 / 20.6, 512: 53 / 40 / 33.
static Plan routed_plan(int64_t mean) { return mean > 256 ? Plan{TWO, 256, 0} : mean > 48 ? Plan{ONE, 128, 0} : Plan{SMALL, 64, 0}; }

bool fp4_few_ok(int64_t M, int64_t N, int64_t K) {
    if (M > FEW_ROWS) return false;
    const int NB = (int)((N + 127) / 128), KT = (int)((K + KB - 1) / KB), S = 1 << lg_runs_of(NB, KT, sm_count()), most = (KT + S - 1) / S;
    return most <= FEW_TILES && M * most <= few_most((int)M);
}
// what launch_fp4_few (own) or launch_fp4_gemm takes for M rows; routed: of E matrices
static Plan plan_of(int64_t E, bool routed, int64_t M, int64_t N, int64_t K, int fmt) {
    const int NB = (int)((N + 127) / 128), KT = (int)((K + KB - 1) / KB);
    if (routed) return routed_plan(M / E);
    return M <= FEW_ROWS ? Plan{SMALL, 64, lg_runs_of(NB, KT, sm_count())} : dense_plan(M, NB, KT, fmt);
}
Fp4Plan fp4_plan(int64_t E, bool routed, int64_t M, int64_t N, int64_t K, int fmt, bool own) {
    if (own) return Fp4Plan{128, FEW_ROWS, 1 << lg_runs_of((int)((N + 127) / 128), (int)((K + KB - 1) / KB), sm_count())};
    const Plan q = plan_of(E, routed, M, N, K, fmt);
    return Fp4Plan{q.mode == TWO ? 256 : 128, q.bt, 1 << q.lg};
}
cudaError_t launch_fp4_few(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, const float *x_scale, int fmt, uint16_t *y, int64_t M, int64_t N, int64_t K,
                           bool f16, int *status, cudaStream_t st) {
    GemmArgs p = args_of(w, w_scale, x_scale, y, M, N, K, f16, status);
    p.xr = x; p.ldx = ldx; p.bt = FEW_ROWS; p.token_tiles = 1;
    const int places = sm_count(), lg = lg_runs_of(p.NB, p.KT, places);
    const unsigned grid = (unsigned)(lg ? p.NB << lg : p.NB < places ? p.NB : places);
    if (fmt == MX) return lg ? launch<MX, FEW, true>(p, lg, p.NB, grid, st) : launch<MX, FEW, false>(p, 0, p.NB, grid, st);
    return lg ? launch<NV, FEW, true>(p, lg, p.NB, grid, st) : launch<NV, FEW, false>(p, 0, p.NB, grid, st);
}

cudaError_t launch_fp4_gemm(const void *w, const float *w_scale, const void *x, const float *x_scale, const int32_t *offset, int E, int fmt, uint16_t *y, int64_t M,
                            int64_t N, int64_t K, bool f16, bool early, int *status, cudaStream_t st) {
    GemmArgs p = args_of(w, w_scale, x_scale, y, M, N, K, f16, status);
    p.early = early;
    p.x = (const uint8_t *)x; p.offset = offset; p.E = E;
    const Plan q = plan_of(E, offset != nullptr, M, N, K, fmt);
    p.bt = q.bt;
    p.token_tiles = (int)((M + q.bt - 1) / q.bt);
    const int ctas = q.mode == TWO ? 2 : 1, nbu = (p.NB + ctas - 1) / ctas, places = sm_count() / ctas;
    const int64_t items = (int64_t)nbu * p.token_tiles;
    const unsigned grid = (unsigned)(q.lg ? items << q.lg : offset ? places : items < places ? items : places) * ctas;
    auto go = [&](auto f) {
        constexpr int F = decltype(f)::value;
        if (q.mode == TWO) return launch<F, TWO, false>(p, 0, items, grid, st);
        if (q.mode == ONE) return q.lg ? launch<F, ONE, true>(p, q.lg, items, grid, st) : launch<F, ONE, false>(p, 0, items, grid, st);
        return q.lg ? launch<F, SMALL, true>(p, q.lg, items, grid, st) : launch<F, SMALL, false>(p, 0, items, grid, st);
    };
    return fmt == MX ? go(std::integral_constant<int, MX>{}) : go(std::integral_constant<int, NV>{});
}

}  // namespace cq
