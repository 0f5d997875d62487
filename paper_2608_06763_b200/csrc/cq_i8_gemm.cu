// y[M][N] = x[M][K] W[N][K]^T, both sides 8-bit integers with a scale for each row (cq_i8.cuh): tcgen05.mma adds up the products of codes in
// 32-bit integers, exactly, and the two scales are applied once, to the sum.
#include "cq_i8.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"
#include "cq_tiles.cuh"

#include <algorithm>

namespace cq {
namespace i8 {

struct GemmArgs {
    const uint8_t *w, *x;
    const float *w_scale, *x_scale;   // [E][N]; [M] (FEW: formed here)
    const int32_t *offset;   // routed: first rows of the groups
    uint16_t *y;
    int *status;
    int E, NB, KT, steps;    // matrices; row blocks of W; k tiles; 32-wide steps of the tensor core that K has
    int bt, token_tiles, band;   // rows of x to a tile; dense: tiles along the rows of x; how many of them are swept together
    int M;                   // rows of x
    int64_t N;
    bool f16, wide;          // wide: rows of y start on 16-byte boundaries
    bool longest;            // K is MOST_K
    bool early;              // launched right behind the quantiser of x: everything else may be read before that has ended
    const uint16_t *xr;      // FEW: rows of x in the model dtype, ldx apart
    int64_t ldx, K;
    // a group's rows in even tiles: 300 rows as 160 and 140, not as 256 and 44
    __device__ __forceinline__ int rows_of_tile(int rows, int tiles) const { return offset ? ((rows + tiles - 1) / tiles + 31) & ~31 : bt; }
};

// What a CTA computes.  ONE: 128 channels x up to 128 rows of x; TWO: a pair of CTAs 256 channels x up to 256 rows; FEW: 128 channels x up to 16
// rows, which it quantises itself and keeps in shared memory; SMALL: 128 channels x up to 64 rows; WIDE: 128 channels x up to 240 rows, in several runs of k.
enum { ONE = 0, TWO = 1, FEW = 2, SMALL = 3, WIDE = 4 };
// rows, and k tiles of them, that fit beside the ring
constexpr int FEW_ROWS = 16, FEW_TILES = 32;

// D[tmem] (+)= A B, 32-bit integers.  PAIR: by the tensor cores of two SMs, each with 128 of the 256 rows of A and half of the columns of B in its
// shared memory.
template <bool PAIR>
__device__ __forceinline__ void umma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (!PAIR) { tc::umma_i8(d, a, b, idesc, accumulate); return; }
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// instruction descriptor: D int32, A and B signed, both K-major, M = 128 (a pair 256), N by the tile
template <bool PAIR>
__device__ __forceinline__ uint32_t idesc_of(uint32_t n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | ((PAIR ? 16u : 8u) << 24); }
// a sum times both scales: one rounding for the sum (beyond 2^24), one for the scales' product, one for theirs
__device__ __forceinline__ float value_of_sum(uint32_t sum, float s) { return (float)(int32_t)sum * s; }
// Sums of the longest K lie in (-2^31, 2^31]: the bits of -2^31 are those of +2^31, 2^17 products of -128 and -128, and 2^31 - 1 rounds to the same float.  (For every K at
// the conversion it cost the output of large products 1 to 6 %.)
__device__ __forceinline__ uint32_t largest_sum(uint32_t sum) { return sum == 0x80000000u ? 0x7FFFFFFFu : sum; }
__device__ __forceinline__ uint32_t pack_out(uint32_t lo, uint32_t hi, float s_lo, float s_hi, bool f16) {
    const float a = value_of_sum(lo, s_lo), b = value_of_sum(hi, s_hi);
    return f16 ? pack16<DT_F16>(a, b) : pack16<DT_BF16>(a, b);
}

template <int MODE, bool SPLIT>
struct Shape {
    static constexpr bool PAIR = MODE == TWO;
    static constexpr bool ALIAS = MODE == WIDE;   // partial sums are exchanged within the ring
    static constexpr int BN = MODE == TWO ? 256 : MODE == WIDE ? 240 : MODE == ONE ? 128 : MODE == SMALL ? 64 : FEW_ROWS, CTAS = PAIR ? 2 : 1;
    // A stage of the ring has DEEP k tiles.  Waiting, fencing and committing for each k tile takes 240 ns, more than its MMAs or its copy from L2 (150 for 64 rows).  With two
    // to a stage 512 rows of 4096 x 4096 take 10.5 us as ONE instead of 11.9; a pair's copies take longer than that, and a deeper ring of single tiles serves it better.
    static constexpr int DEEP = PAIR || MODE == WIDE ? 1 : 2;
    static constexpr int B_TILE = MODE == FEW ? 0 : BN / CTAS * 128;   // codes of x in this CTA: half of a pair's
    static constexpr int A_BYTES = DEEP * TILE_BYTES, B_BYTES = DEEP * B_TILE, STAGE = A_BYTES + B_BYTES;
    static constexpr int STAGES = PAIR ? 6 : MODE == ONE ? (SPLIT ? 2 : 3) : MODE == SMALL && SPLIT ? 3 : 4;
    static constexpr int ACCS = 2, ACC_COLS = BN < 32 ? 32 : BN > 128 ? 256 : BN;   // accumulators: while one is read the next tile fills the other
    static constexpr int PITCH = 272;                              // bytes of a row of the staged output: 128 channels and a gap against bank conflicts
    static constexpr int X_CODES = FEW_ROWS * 128, X_BYTES = MODE == FEW ? FEW_TILES * X_CODES : 0;   // FEW: codes of a k tile; all k tiles
    // SPLIT: partial sums [run][channel][row of x, and a gap]; ALIAS: what those that are sent and three quarters of those that come take beyond the ring
    static constexpr int SUMS = 128 * (BN + 4) * 4;
    static constexpr int OUT_BYTES = ALIAS ? SUMS / 4 * 7 - STAGES * STAGE : SPLIT ? SUMS : (MODE == FEW ? 32 : 64) * PITCH;
    static constexpr int SCALE_BYTES = BN * 4, BAR_BYTES = 256 + FEW_ROWS * 4;   // scales of the rows of a tile; barriers and what FEW gathers maxima in
    static constexpr size_t smem(int E, bool routed) {
        return (size_t)STAGES * STAGE + X_BYTES + OUT_BYTES + SCALE_BYTES + BAR_BYTES + (routed ? 3 * (size_t)(E + 1) * 4 : 0);
    }
    static_assert(STAGES * STAGE + X_BYTES + OUT_BYTES + SCALE_BYTES + BAR_BYTES + (MODE == FEW ? 0 : 12 * (MAX_EXPERTS + 1)) <= 232448, "shared memory");
    static_assert(ACCS * ACC_COLS <= 512, "tensor memory");
};

// A row of up to 128 values from shared memory to anywhere, by sixteen threads: sixteen bytes each where they are aligned in global memory, of which two neighbouring pieces
// of the row are shifted together; up to eight values before and behind singly.  4096 rows of 8191 x 2048 68.6 us with all values stored singly, 45.8 for rows of 8192.
__device__ __forceinline__ void store_row(uint16_t *to, const uint8_t *row, int j, int chans) {
    const int m = (int)(reinterpret_cast<uintptr_t>(to) >> 1) & 7;   // values in front of the row's first in its piece
    const uint16_t *values = reinterpret_cast<const uint16_t *>(row);
    const int c = 8 * j - m;   // this thread's piece: values c to c + 7
    if (c >= 0 && c + 8 <= chans) {
        const uint4 b = *reinterpret_cast<const uint4 *>(row + j * 16), a = m ? *reinterpret_cast<const uint4 *>(row + j * 16 - 16) : b;
        const int by = (8 - m) & 7;   // values of a that are left out
        uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int k = 0; k < 6; ++k) w[k] = by & 4 ? w[k + 2] : w[k];
#pragma unroll
        for (int k = 0; k < 5; ++k) w[k] = by & 2 ? w[k + 1] : w[k];
        const uint32_t odd = by & 1 ? 16u : 0u;
        *reinterpret_cast<uint4 *>(to + c) = make_uint4(__funnelshift_r(w[0], w[1], odd), __funnelshift_r(w[1], w[2], odd), __funnelshift_r(w[2], w[3], odd), __funnelshift_r(w[3], w[4], odd));
    } else if (c >= 0) {   // of a last block that has not all 128
        for (int k = c; k < min(c + 8, chans); ++k) to[k] = values[k];
    }
    const int edge = j < 8 - m ? j : 120 + j;   // before the first whole piece, behind the last of 128
    if (m && j < 8 && edge < chans) to[edge] = values[edge];
}
// SPLIT, the eight warps that write y: this CTA's partial sums to the CTAs that add them, then its own 128 / S channels of all runs.  Sums arrive
// counted on a barrier, so nobody waits for the whole cluster in between.  Few rows are sent from the registers; more go through the ring,
// which nobody needs any more, and from there in one copy to each CTA.  ALIAS: those of the others land in the ring too, once all rings are free.
// gave_up: the accumulator did not come.  Such a CTA sends zeros, and waits like the others for what is sent to it: a CTA whose sums have not all come may not leave, since
// they would land in shared memory that is no longer its own.  After a wait that ran out it waits once more; the status tells that y is not valid.
template <class SH>
__device__ __forceinline__ void send_and_add(const GemmArgs &p, const Item &t, int lgS, int run, int warp, int lane, uint8_t *ring, uint8_t *part, const float *x_scale, uint64_t *sums,
                                             volatile int *dead, bool gave_up) {
    constexpr bool COPY = SH::BN > 16;
    const int lgCW = 7 - lgS, CW = 1 << lgCW, pitch = ((t.rows + 15) & ~15) + 4;
    const int quad = warp & 3, c = quad * 32 + lane, owner = c >> lgCW, tid = threadIdx.x - 128;
    const uint32_t bytes_of_run = (uint32_t)(pitch << lgCW) * 4u;
    if (tid == 0) tc::mbar_arrive_expect_tx(sums, COPY ? ((1u << lgS) - 1) * bytes_of_run : 128u * (uint32_t)((t.rows + 3) & ~3) * 4u);
    tc::tc_fence_after();
    __syncwarp();
    if (SH::ALIAS) { cluster_arrive(); part = ring + 128 * pitch * 4; }   // this ring is free
    if (!COPY) cluster_wait();   // the others have started, and their barriers exist
    const uint32_t to = COPY ? tc::smem_u32(ring) + (uint32_t)c * pitch * 4 : tc::map_to_rank(part, owner) + (uint32_t)((run << lgCW) + (c & (CW - 1))) * pitch * 4;
    const uint32_t bar = COPY ? 0 : tc::map_to_rank(sums, owner);
    for (int c0 = (warp - 4) / 4 * 32; c0 < t.rows; c0 += 64) {
        uint32_t v[32];
        tc::tmem_ld32(c0 + ((uint32_t)(quad * 32) << 16), v);
        tc::tmem_ld_wait();
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
        cluster_wait();   // the others have started, and their barriers exist (ALIAS: their rings are free)
        if (tid < 1 << lgS && tid != run)
            asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(tc::map_to_rank(part, tid) + (run - (run > tid)) * bytes_of_run), "r"(tc::smem_u32(ring) + tid * bytes_of_run), "r"(bytes_of_run), "r"(tc::map_to_rank(sums, tid)) : "memory");
        __syncwarp();
    } else {
        __syncwarp();
        cluster_arrive();
    }
    // two channels of four rows a thread
    const int mine = 2 * (tid & (CW / 2 - 1));
    const int64_t ch = (int64_t)t.nb * 128 + (run << lgCW) + mine;
    const float w0 = ch < p.N ? p.w_scale[ch] : 0.0f, w1 = ch + 1 < p.N ? p.w_scale[ch + 1] : 0.0f;
    const bool ok = tc::mbar_wait(sums, 0, p.status, 68, tc::WAIT_LIMIT_CYCLES, gave_up ? nullptr : dead);
    if (!ok) {
        *dead = 1;
        tc::mbar_wait(sums, 0, p.status, 68);
    }
    __syncwarp();
    if (COPY) cluster_arrive();   // what was copied from here has been received when all have arrived
    if (!ok || gave_up) return;
    uint16_t *out = p.y + (int64_t)t.yrow * p.N + ch;
    const uint8_t *own = (COPY ? ring : part) + run * bytes_of_run;
    const int step = (512 >> lgCW) * 4;
    for (int r = (tid >> (lgCW - 1)) * 4; r < t.rows; r += step) {
        const int at = (mine * pitch + r) * 4, next = pitch * 4;
        uint4 f[2];   // modulo 2^32, as the tensor core adds
#pragma unroll
        for (int j = 0; j < 2; ++j) f[j] = *reinterpret_cast<const uint4 *>(own + at + j * next);
#pragma unroll
        for (int s = 1; s < 4; ++s)
            if (s < 1 << lgS) {
                const int other = run ^ s;
                const uint8_t *from = part + (COPY && other > run ? other - 1 : other) * bytes_of_run + at;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(from + j * next);
                    f[j].x += v.x; f[j].y += v.y; f[j].z += v.z; f[j].w += v.w;
                }
            }
        if (COPY && p.longest) {   // (what quantises itself has no -128)
#pragma unroll
            for (int j = 0; j < 2; ++j) f[j] = make_uint4(largest_sum(f[j].x), largest_sum(f[j].y), largest_sum(f[j].z), largest_sum(f[j].w));
        }
        const float4 xs = *reinterpret_cast<const float4 *>(x_scale + r);   // of what lies behind the rows nothing is stored
        const float x4[4] = {xs.x, xs.y, xs.z, xs.w};
        const uint32_t lo[4] = {f[0].x, f[0].y, f[0].z, f[0].w}, hi[4] = {f[1].x, f[1].y, f[1].z, f[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t v = pack_out(lo[i], hi[i], w0 * x4[i], w1 * x4[i], p.f16);
            uint16_t *to = out + (int64_t)(r + i) * p.N;
            if (r + i < t.rows) {
                if (p.wide) {   // N even: both are inside
                    if (ch < p.N) *reinterpret_cast<uint32_t *>(to) = v;
                } else {
                    if (ch < p.N) to[0] = (uint16_t)v;
                    if (ch + 1 < p.N) to[1] = (uint16_t)(v >> 16);
                }
            }
        }
    }
}

// FEW, the eight warps that write y later: the scales of the rows (over all of K) and this CTA's k tiles of their codes, into shared memory.
template <int DT>
__device__ __forceinline__ void quantize_here(const GemmArgs &p, int k0, int k1, uint32_t *s_top, float *x_scale, uint8_t *x_codes) {
    const int tid = threadIdx.x - 128, lane = tid & 31, KU = (int)(p.K >> 4), all = p.M * KU;
    for (int i0 = 0; i0 < all; i0 += 4 * 256) {
        uint4 a[4], b[4];
        int row[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + j * 256 + tid;
            row[j] = i < all ? i / KU : -1;
            const uint16_t *src = p.xr + row[j] * p.ldx + (int64_t)(i - row[j] * KU) * 16;
            a[j] = i < all ? load16(src) : make_uint4(0, 0, 0, 0);
            b[j] = i < all ? load16(src + 8) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w[8] = {a[j].x, a[j].y, a[j].z, a[j].w, b[j].x, b[j].y, b[j].z, b[j].w};
            const uint32_t top = top_of_16bit<DT>(w);
            if (__all_sync(~0u, row[j] == __shfl_sync(~0u, row[j], 0))) {
                const uint32_t m = __reduce_max_sync(~0u, top);
                if (lane == 0 && row[j] >= 0) atomicMax(&s_top[row[j]], m);
            } else if (row[j] >= 0) {
                atomicMax(&s_top[row[j]], top);
            }
        }
    }
    epilogue_sync();
    if (tid < p.M) x_scale[tid] = row_scale(s_top[tid]);
    const int units = (k1 - k0) * p.M * 8, u = tid & 7;
    for (int i = tid; i < units; i += 256) {
        const int line = i >> 3, kt = line / p.M, row = line - kt * p.M, unit = (k0 + kt) * 8 + u;
        uint4 c = make_uint4(0, 0, 0, 0);   // behind K
        if (unit < KU) {
            const uint16_t *src = p.xr + row * p.ldx + (int64_t)unit * 16;
            const uint4 a = load16(src), b = load16(src + 8);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            const float d = row_scale(s_top[row]);
            c = codes_of_16bit<DT>(w, d, __fdiv_rn(1.0f, d));
        }
        *reinterpret_cast<uint4 *>(x_codes + kt * (FEW_ROWS * 128) + piece_offset(row, u)) = c;
    }
    tc::fence_proxy_async();   // the tensor core reads through the async proxy
}

// Warps 0 and 2 bring tiles (bulk copies: 0 those of W, 2 those of x), warp 1 issues the MMAs (in the second CTA of a pair it tells the first
// that its tiles are there), warp 3 reads the offsets of routed rows, warps 4 to 11 write y.
// SPLIT: 2^lgS CTAs of a cluster share one output tile, each a run of its k tiles; the partial sums meet in the shared memory of the
// cluster, where each CTA adds 128 / S channels.  One tile a CTA then; else CTAs (pairs) take tiles in turn.
// FEW: warps 4 to 11 first quantise the rows for this CTA's k tiles, while the first weights are on their way.
// Measured: 4096 rows of 57344 x 8192 1.1 ms, 3.5 POP/s (tensor pipe 92 % active, the power limit); 1024 of 6144 x 4096 20.8 us, 2.5 POP/s (two rounds of pairs, their fill and the last
// output); 200 of 4096 x 14336 17.9, 3.3 TB/s of weights (what an SM takes from L2, and the exchange); one of 28672 x 4096 21.5 and of 57344 x 8192 79, 5.5 and 6.0 TB/s (memory);
// one of 4096 x 4096 6.5, of which setting up takes one, the rows two, the k tiles one and a half, exchange and output one.
template <int MODE, bool SPLIT>
__global__ void __launch_bounds__(384, 1) i8_gemm_kernel(const GemmArgs p, int lgS, int n_items) {
    using SH = Shape<MODE, SPLIT>;
    constexpr bool PAIR = SH::PAIR;
    static_assert(!(PAIR && SPLIT), "pairs take whole tiles");
    constexpr int ST = SH::STAGES, ACCS = SH::ACCS, BN = SH::BN, CTAS = SH::CTAS, ACC_COLS = SH::ACC_COLS;
    constexpr uint32_t TMEM = 0;   // a CTA takes all of tensor memory: its first column is column 0
    extern __shared__ __align__(1024) uint8_t ring[];   // the swizzle counts address bits from 1024 on
    uint8_t *x_codes = ring + ST * SH::STAGE;
    uint8_t *staged = x_codes + SH::X_BYTES;
    float *x_scale = reinterpret_cast<float *>(staged + SH::OUT_BYTES);
    uint64_t *full = reinterpret_cast<uint64_t *>(staged + SH::OUT_BYTES + SH::SCALE_BYTES), *empty = full + ST, *acc_full = empty + ST, *acc_empty = acc_full + ACCS;
    uint64_t *drained = acc_empty + ACCS, *x_ready = drained + 1, *sums = x_ready + 1;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(sums + 1);
    volatile int *dead = reinterpret_cast<volatile int *>(s_tmem + 1);
    int *s_off = reinterpret_cast<int *>(staged + SH::OUT_BYTES + SH::SCALE_BYTES + SH::BAR_BYTES), *s_blk = s_off + p.E + 1, *s_item = s_blk + p.E + 1;
    static_assert((2 * ST + 2 * ACCS + 3) * 8 + 8 <= 256, "barriers");
    uint32_t *s_top = reinterpret_cast<uint32_t *>(staged + SH::OUT_BYTES + SH::SCALE_BYTES + 256);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // From the block's number, not the cluster's registers, and by shifts: what branches and addresses of the issuing warp hang on is uniform.
    const int lgC = PAIR ? 1 : SPLIT ? lgS : 0, cluster_rank = blockIdx.x & ((1 << lgC) - 1), unit = blockIdx.x >> lgC, units = gridDim.x >> lgC;
    const int half = PAIR ? cluster_rank : 0, run = SPLIT ? cluster_rank : 0;   // which 128 channels of the pair; which run of k
    const int k0 = SPLIT ? p.KT * run >> lgS : 0, k1 = SPLIT ? p.KT * (run + 1) >> lgS : p.KT;   // this CTA's k tiles

    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) { tc::mbar_init(&full[i], MODE == FEW ? 1 : PAIR && half == 0 ? 3 : 2); tc::mbar_init(&empty[i], 1); }   // a pair's first CTA also waits for the other's tiles
        for (int i = 0; i < ACCS; ++i) { tc::mbar_init(&acc_full[i], 1); tc::mbar_init(&acc_empty[i], 8 * CTAS); }
        tc::mbar_init(drained, 1);
        tc::mbar_init(x_ready, 8);
        tc::mbar_init(sums, 1);
        *dead = 0;
        tc::fence_barrier_init();
    }
    if (MODE == FEW && threadIdx.x < FEW_ROWS) s_top[threadIdx.x] = 0;
    if (warp == 1) {
        if (PAIR) tc::tmem_alloc_pair(s_tmem, 512);
        else { tc::tmem_alloc(s_tmem, 512); tc::tmem_relinquish(); }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (PAIR) tc::cluster_sync();   // the partner's barriers exist before anything arrives on them
    if (SPLIT && !SH::ALIAS) cluster_arrive();
    tc::tc_fence_after();
    Tiles<PAIR, GemmArgs> tiles{p, unit, SPLIT ? n_items : units, n_items, s_off, s_blk, s_item, {}};   // split: one tile
    if (!p.offset) {   // what needs no other kernel: the first tiles' places, and the first weights on their way to L2, which sees what the kernel in front may still write
        tiles.look(0);
        tiles.ahead = true;
        if (warp == 3 && !p.early && tiles.has(0)) {
            const int nb = min(tiles.at(0).nb * CTAS + half, p.NB - 1);
            if (lane < SH::STAGES * SH::DEEP && k0 + lane < k1) tc::prefetch_l2(p.w + ((int64_t)nb * p.KT + k0 + lane) * TILE_BYTES, TILE_BYTES);
            __syncwarp();
        }
    }
    // From here on the next kernel may start: this one holds its tensor memory, which a kernel that waits for this one might else take.
    // Behind the quantiser of this call only the layout and the scales that it writes have to be waited for (by the warps that read them, and in every
    // CTA): the quantiser lets this kernel start once all kernels in front of itself have ended, those that wrote weights and offsets among them.
    if (p.early) launch_dependents();
    else tc::wait_for_previous_kernel();
    if (p.offset) {
        if (warp == 3) scan_groups(p.offset, p.E, p.M, s_off, s_blk, s_item, p.bt, PAIR ? (p.NB + 1) >> 1 : p.NB);
        __syncthreads();
    }
    if (p.offset) tiles.items = __reduce_max_sync(~0u, s_item[p.E]);   // (a reduction's result is uniform)

    int it = 0;   // stages filled (warps 0 and 2) so far
    if (warp == 0 || (warp == 2 && MODE != FEW)) {
        // warp 0 the weights, warp 2 its rows of codes, from one row block or several (a lane for each)
        const int64_t block = (int64_t)p.KT * TILE_BYTES;   // from a row block to the next
        uint32_t s = 0, phase = 1;
        bool ok = true;
        if (warp == 2 && p.early) wait_for_quantiser();
        for (int local = 0; ok && tiles.has(local); ++local) {
            const Item t = tiles.at(local);
            const int n = columns_of<PAIR>(t.rows), mine = n / CTAS, nb = min(t.nb * CTAS + half, p.NB - 1);   // an odd last pair reads a block twice
            const int r0 = t.off + half * mine, b0 = r0 / ROWS, in0 = r0 % ROWS;
            const uint8_t *xt = p.x + ((int64_t)t.xblk * p.KT + k0) * TILE_BYTES, *src = xt;
            // warp 0: one piece, neighbouring k tiles are neighbours in memory; warp 2: lanes 4 j to 4 j + 2 the rows of k tile j of a stage, a row block each
            const int mine_kt = warp == 0 ? 0 : lane >> 2, piece = lane & 3, lo = piece ? piece * ROWS - in0 : 0, hi = min(mine, (piece + 1) * ROWS - in0);
            uint32_t to = 0, bytes = 0, all = TILE_BYTES;
            if (warp == 0) {
                if (lane == 0) { src = p.w + (((int64_t)t.e * p.NB + nb) * p.KT + k0) * TILE_BYTES; bytes = TILE_BYTES; }
            } else {
                all = (uint32_t)mine * 128;
                if (mine_kt < SH::DEEP && lo < hi) {
                    src = xt + (b0 + piece) * block + (piece ? 0 : in0 * 128) + mine_kt * TILE_BYTES;
                    to = SH::A_BYTES + mine_kt * SH::B_TILE + lo * 128;
                    bytes = (uint32_t)(hi - lo) * 128;
                }
            }
            for (int kt = k0; kt < k1; kt += SH::DEEP, ++it, src += SH::DEEP * TILE_BYTES) {
                const uint32_t count = min(SH::DEEP, k1 - kt);
                ok = uniform_wait(&empty[s], phase, p.status, 61, dead);   // the first round passes at once
                if (!ok) break;
                if (lane == 0) tc::mbar_arrive_expect_tx(&full[s], all * count);
                __syncwarp();
                if (bytes && mine_kt < (int)count) tc::bulk_load(ring + s * SH::STAGE + to, src, warp == 0 ? bytes * count : bytes, &full[s]);
                if (++s == ST) { s = 0; phase ^= 1; }
            }
        }
        if (!ok && lane == 0) *dead = 1;
        __syncwarp();
    } else if (warp == 1) {
        // The whole warp walks the loops and one lane issues: what the instructions take stays in uniform registers.
        uint32_t s = 0, phase = 0;
        bool ok = MODE != FEW || uniform_wait(x_ready, 0, p.status, 67, dead);
        for (int local = 0; ok && tiles.has(local); ++local) {
            const uint32_t n = MODE == FEW ? FEW_ROWS : __reduce_max_sync(~0u, columns_of<PAIR>(tiles.at(local).rows));
            const int acc = local & (ACCS - 1);
            const uint32_t d = TMEM + acc * ACC_COLS, desc = idesc_of<PAIR>(n);
            if (half == 0 && local >= ACCS) ok = uniform_wait(&acc_empty[acc], (local / ACCS - 1) & 1, p.status, 63, dead);
            tc::tc_fence_after();
            for (int kt = k0; kt < k1 && ok; kt += SH::DEEP) {
                ok = uniform_wait(&full[s], phase, p.status, 64, dead);
                if (!ok) break;
                if (PAIR && half == 1) {
                    if (lane == 0) tc::mbar_arrive_cluster(tc::map_to_rank(&full[s], cluster_rank & ~1));
                } else {
                    tc::tc_fence_after();
                    const uint64_t da = tc::smem_desc_sw128(tc::smem_u32(ring) + s * SH::STAGE);
                    const uint64_t db = MODE == FEW ? tc::smem_desc_sw128(tc::smem_u32(x_codes) + (kt - k0) * SH::X_CODES) : da + SH::A_BYTES / 16;
                    constexpr int B_STEP = (MODE == FEW ? SH::X_CODES : SH::B_TILE) / 16;
                    const int steps = p.steps - 4 * kt, most = 4 * (k1 - kt);
                    if (tc::elect_one()) {
#pragma unroll
                        for (int j = 0; j < 4 * SH::DEEP; ++j)
                            if (j == 0 || (j < steps && (SH::DEEP == 1 || j < most)))
                                umma_i8<PAIR>(d, da + j / 4 * (TILE_BYTES / 16) + 2 * (j % 4), db + j / 4 * B_STEP + 2 * (j % 4), desc, j > 0 || kt > k0);
                        if (PAIR) commit_to_pair(&empty[s], cluster_rank);
                        else tc::umma_commit(&empty[s]);
                        if (kt + SH::DEEP >= k1) {
                            if (PAIR) commit_to_pair(&acc_full[acc], cluster_rank);
                            else tc::umma_commit(&acc_full[acc]);
                        }
                    }
                    __syncwarp();
                }
                if (++s == ST) { s = 0; phase ^= 1; }
            }
        }
        if (!ok && lane == 0) *dead = 1;
        if (!ok && half == 0) {   // what was issued completes before tensor memory is given back
            if (tc::elect_one()) {
                if (PAIR) commit_to_pair(drained, cluster_rank);
                else tc::umma_commit(drained);
            }
            __syncwarp();
            tc::mbar_wait(drained, 0, p.status, 65);
        }
        __syncwarp();
    } else if (warp >= 4) {
        // Tensor memory is emptied into registers first, already in the type of y, so that the next tile's MMAs wait for no store;
        // then 64 rows of y at a time go through shared memory, where the 8x8 matrices are turned round, and out as whole rows.
        const int quad = warp & 3, part = (warp - 4) >> 2, tid = threadIdx.x - 128;   // the 32 lanes of tensor memory that a warp may read; its half of 64 columns
        if constexpr (MODE == FEW) {
            if (p.f16) quantize_here<DT_F16>(p, k0, k1, s_top, x_scale, x_codes);
            else quantize_here<DT_BF16>(p, k0, k1, s_top, x_scale, x_codes);
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(x_ready);
        } else if (p.early) {
            wait_for_quantiser();
        }
        for (int local = 0; tiles.has(local); ++local) {
            const Item t = tiles.at(local);
            const int acc = local & (ACCS - 1), nb = t.nb * CTAS + half;
            // scales: of the rows to shared memory, of the four channels that a lane has of a group of columns to registers
            if (MODE != FEW && tid < t.rows) x_scale[tid] = p.x_scale[t.yrow + tid];
            float ws[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t ch = (int64_t)nb * 128 + quad * 32 + (lane >> 2) + 8 * i;
                ws[i] = !SPLIT && ch < p.N ? p.w_scale[(int64_t)t.e * p.N + ch] : 0.0f;
            }
            const bool ok = tc::mbar_wait(&acc_full[acc], (local / ACCS) & 1, p.status, 66, tc::WAIT_LIMIT_CYCLES, (volatile int *)dead);
            const bool gave_up = epilogue_any(!ok);
            if (gave_up) *dead = 1;
            if constexpr (SPLIT) {
                send_and_add<SH>(p, t, lgS, run, warp, lane, ring, staged, x_scale, sums, dead, gave_up);
                break;
            }
            if (gave_up) break;
            tc::tc_fence_after();
            constexpr int GROUPS = (BN + 63) / 64;
            uint32_t out16[GROUPS][16];
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int c0 = g * 64 + part * 32;
                if (c0 < t.rows) {
                    uint32_t lo[16], hi[16];
                    const uint32_t from = TMEM + acc * ACC_COLS + c0 + ((uint32_t)(quad * 32) << 16);
                    tmem_ld_16x32(from, lo);
                    tmem_ld_16x32(from + (16u << 16), hi);
                    tc::tmem_ld_wait();
                    if (MODE != FEW && p.longest) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) { lo[i] = largest_sum(lo[i]); hi[i] = largest_sum(hi[i]); }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 xs = BN >= 32 || c0 + 8 * i < BN ? *reinterpret_cast<const float2 *>(x_scale + c0 + 8 * i + 2 * (lane & 3)) : make_float2(0.0f, 0.0f);
                        out16[g][4 * i] = pack_out(lo[4 * i], lo[4 * i + 1], ws[0] * xs.x, ws[0] * xs.y, p.f16);
                        out16[g][4 * i + 1] = pack_out(lo[4 * i + 2], lo[4 * i + 3], ws[1] * xs.x, ws[1] * xs.y, p.f16);
                        out16[g][4 * i + 2] = pack_out(hi[4 * i], hi[4 * i + 1], ws[2] * xs.x, ws[2] * xs.y, p.f16);
                        out16[g][4 * i + 3] = pack_out(hi[4 * i + 2], hi[4 * i + 3], ws[3] * xs.x, ws[3] * xs.y, p.f16);
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
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 16 + (tid >> 4);
                        if (r < count) store_row(out + (int64_t)r * p.N, staged + r * SH::PITCH, tid & 15, chans);
                    }
                }
                epilogue_sync();   // read before it is written again, and so are the scales of the rows
            }
        }
    }

    if (SPLIT && warp < 4) {   // the others have done so on their way
        __syncwarp();
        if (SH::ALIAS) cluster_arrive();
        cluster_wait();
        cluster_arrive();
    }
    tc::tc_fence_before();
    __syncthreads();
    if (*dead && (warp == 0 || warp == 2))   // a wait gave up: copies in flight land before the shared memory goes away
        for (int i = it < ST ? 0 : it - ST; i < it; ++i) tc::mbar_wait(&full[i % ST], (i / ST) & 1, p.status, 62);
    __syncwarp();
    if (PAIR) tc::cluster_sync();   // nothing of the pair is in flight towards a CTA that has left
    if (SPLIT) cluster_wait();      // nor are partial sums
    if (warp == 1) {
        tc::tc_fence_after();
        if (PAIR) tc::tmem_dealloc_pair(TMEM, 512);
        else tc::tmem_dealloc(TMEM, 512);
    }
}

template <int MODE, bool SPLIT>
static cudaError_t allow_smem() {
    static std::atomic<uint64_t> done{0};
    return ensure_func_attr(i8_gemm_kernel<MODE, SPLIT>, done, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<MODE, SPLIT>::smem(MAX_EXPERTS, MODE != FEW));
}
template <int MODE, bool SPLIT>
static cudaError_t launch(const GemmArgs &p, int lgS, int64_t items, unsigned grid, cudaStream_t st) {
    using SH = Shape<MODE, SPLIT>;
    const cudaError_t e = allow_smem<MODE, SPLIT>();
    if (e != cudaSuccess) return e;
    return launch_overlapped(i8_gemm_kernel<MODE, SPLIT>, dim3(grid), 384u, SH::smem(p.E, p.offset != nullptr), st, SH::CTAS << (SPLIT ? lgS : 0), true, p, lgS, (int)items);
}

}  // namespace i8

using namespace i8;

// Clusters of four CTAs that the GPU takes at once: fewer than a quarter of its SMs, which are not in groups of four.  One cluster more waits for all others: 4352 x 4096 with 13 rows 9.9 us
// in four runs, 5.9 with one row block less, 6.0 in two.
static int clusters_of_four() {
    static std::atomic<int> cached[64];
    constexpr int USUAL = 33;   // of 148 SMs
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { (void)cudaGetLastError(); return USUAL; }
    if ((n = cached[dev].load(std::memory_order_relaxed)) > 0) return n;
    cudaLaunchAttribute four{};
    four.id = cudaLaunchAttributeClusterDimension;
    four.val.clusterDim.x = 4; four.val.clusterDim.y = four.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(4 * sm_count()); cfg.blockDim = dim3(384); cfg.dynamicSmemBytes = Shape<SMALL, true>::smem(1, false); cfg.attrs = &four; cfg.numAttrs = 1;
    if (allow_smem<SMALL, true>() != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, i8_gemm_kernel<SMALL, true>, &cfg) != cudaSuccess || n <= 0) { (void)cudaGetLastError(); return USUAL; }
    cached[dev].store(n, std::memory_order_relaxed);
    return n;
}
// Runs of k (log2) that an output tile of few row blocks is cut into, while the GPU has places for them.
static bool has_places(int64_t tiles, int lg) { return lg == 0 || (tiles << lg <= sm_count() && (lg < 2 || tiles <= clusters_of_four())); }
static int lg_runs_of(int tiles, int KT) {
    int lg = 0;
    while (lg < 2 && 2 << lg <= KT && has_places(tiles, lg + 1)) ++lg;
    return lg;
}
static GemmArgs args_of(const void *w, const float *w_scale, const float *x_scale, uint16_t *y, int64_t M, int64_t N, int64_t K, bool f16, int *status) {
    GemmArgs p{};
    p.w = (const uint8_t *)w; p.w_scale = w_scale; p.x_scale = x_scale; p.y = y; p.status = status;
    p.E = 1; p.NB = (int)((N + 127) / 128); p.KT = (int)((K + KB - 1) / KB); p.steps = (int)((K + 31) / 32);
    p.M = (int)M; p.N = N; p.K = K; p.f16 = f16; p.wide = N % 8 == 0; p.longest = K == MOST_K;
    p.band = 16;
    return p;
}

// What computes a product of more than sixteen rows: kind of tile, rows to a tile, runs of k (log2).  Costs in microseconds, from tiles forced in turn.  A k
// tile of one CTA takes as long as an SM's port to L2 does for its bytes (145 bytes a nanosecond); a pair's, its copies at least and for many rows its MMAs.  Cutting k saves
// k tiles and costs a cluster's launch and the exchange.
//   4096 x 4096, 200 rows: SMALL 8.9, ONE 10.0 (two runs 10.0), WIDE 11.7, TWO 10.6;  300: SMALL 14.3, ONE 10.2, TWO 11.4;  512: ONE 10.5, TWO 11.7;  700: ONE 17.3, TWO 12.8
//   4096 x 14336, 100 rows: SMALL 22.1, in two runs 15.1, ONE 24.6 / 18.7, in four 13.9, TWO 26.2;  200: SMALL 22.6, ONE 25.5, in two runs 19.7, WIDE in two 22.2, in four 17.8, TWO 26.6
//   8192 x 8192, 160 rows: ONE 16.9, WIDE in two runs 15.2, TWO 17.9;  4096 x 8192, 300 rows: ONE 16.6, WIDE in two 15.0, TWO 18.0;  925 x 12800, 1120 rows: ONE 26.1, in two runs 19.3, TWO 26.8
//   440 x 2912, 22 rows: SMALL 6.5, in two runs 5.6, in four 5.0;  3031 x 1664, 55 rows: 6.5 / 6.1 / 5.9
//   28672 x 4096, 40 rows: SMALL 20.8, TWO 22.8;  128: SMALL 28.7, ONE 24.8, TWO 25;  6144 x 4096, 1024 rows: ONE 24.9, TWO 20.3
//   11176 x 22368, 341 rows: SMALL 124, ONE 88.6, TWO 84.0 / 96.2 / 113.6 with 128 / 192 / 256 rows
// Tried and dropped, sums through L2 where integers may be added in any order: even runs of all k tiles for each CTA (4096 x 4096, one row 11.0 us
// where whole tiles then took 7.8, 28672 x 4096 as before, 57344 x 8192 79.7 where they took 84.2), the last round's pairs cut along K (200 rows of 4096 x 14336 21.5, 1024 of
// 6144 x 4096 28.8): an exchange there takes some four microseconds of fences, counting and reading back, and each run has two ends.
struct Plan { int mode, bt, lg; };
static int even_rows(int64_t M, int64_t tiles) { return (int)((M + tiles - 1) / tiles + 15) & ~15; }   // WIDE: rows of its tiles
static Plan dense_plan(int64_t M, int NB, int KT) {
    static const Plan kinds[] = {{SMALL, 64, 0}, {SMALL, 64, 1}, {SMALL, 64, 2}, {ONE, 128, 0}, {ONE, 128, 1}, {ONE, 128, 2}, {WIDE, 240, 1}, {WIDE, 240, 2}, {TWO, 128, 0}, {TWO, 192, 0}, {TWO, 256, 0}};
    const int sms = sm_count();
    Plan best = kinds[3];
    double least = 1e30;
    for (const Plan &k : kinds) {
        const int ctas = k.mode == TWO ? 2 : 1, S = 1 << k.lg, nbu = (NB + ctas - 1) / ctas, places = sms / ctas;
        if (S > KT || (k.mode == WIDE && M <= 128) || (k.mode == ONE && M <= 64)) continue;
        const int64_t tiles = (M + k.bt - 1) / k.bt, items = nbu * tiles;
        if (!has_places(items, k.lg)) continue;   // one round, or the runs of several tiles wait for one another's places
        const double n = k.mode == WIDE ? (double)even_rows(M, tiles) : M < k.bt ? (double)M : (double)k.bt, rounds = (double)((items * S + places - 1) / places);
        double per_kt, tail, base;
        if (k.mode == TWO) { per_kt = std::max(0.205, 0.13 + 0.15 * n / 256); tail = 0.5 * n / 256; base = 4.4; }
        else {
            per_kt = (16.4 + 0.128 * n) / 145.0;
            const double exchange = k.mode == SMALL ? (k.lg == 1 ? 0.4 + 0.017 * n : 0.6 + 0.026 * n) : k.mode == WIDE && k.lg == 2 ? 6.1 : 4.1;
            tail = k.lg ? 0.5 : 0.0094 * n; base = 2.8 + (k.lg ? exchange : 0.0);
        }
        const double cost = base + rounds * ((KT + S - 1) / S * per_kt + tail);
        if (cost < least) { least = cost; best = k; }
    }
    return best;
}
// Up to sixteen rows.  A CTA's own quantising takes 0.25 us for each row of 4096 (a call of its own in front is hidden but for the host's part, some two microseconds): us on the
// GPU, by itself / in front: 4096 x 4096, rows 1 to 4: 7.1 / 7.0, 7.4 / 7.1, 7.6 / 7.2, 7.8 / 7.2, 6: 9.6 / 7.3;  8192 x 2048, 4: 7.3 / 7.1, 8: 9.5 / 7.6;  4096 x 14336, 1: 10.2 / 11.2, 2: 12.2 /
// 11.4;  28672 x 4096, 1: 21.5 / 22.4, 3: 23.4 / 22.9.  FEW_MOST: rows x k tiles of 128.
constexpr int FEW_MOST = 128;
bool i8_few_ok(int64_t M, int64_t N, int64_t K) {
    if (M > FEW_ROWS) return false;
    const int NB = (int)((N + 127) / 128), KT = (int)((K + KB - 1) / KB), S = 1 << lg_runs_of(NB, KT), most = (KT + S - 1) / S;
    return most <= FEW_TILES && M * KT <= FEW_MOST;
}
// What launch_i8_gemm takes for M rows.  Routed rows: the loads are on the GPU, and pairs with 256 rows serve all of them.  Sixteen matrices of 2816 x 2048, us with SMALL / ONE /
// TWO: 2 rows on average 11.0 / 11.1 / 10.7, 24: 16.2 / 16.3 / 15.4, 64: 21.3 / 18.9 / 17.3, 256: 50.4 / 37.3 / 30.1, 512: 98.5 / 59.8 / 45.0.
static Plan plan_of(bool routed, int64_t M, int64_t N, int64_t K) {
    const int NB = (int)((N + 127) / 128), KT = (int)((K + KB - 1) / KB);
    if (routed) return {TWO, 256, 0};
    return M <= FEW_ROWS ? Plan{SMALL, 64, lg_runs_of(NB, KT)} : dense_plan(M, NB, KT);
}
I8Plan i8_plan(bool routed, int64_t M, int64_t N, int64_t K, bool own) {
    if (own) return I8Plan{128, FEW_ROWS, 1 << lg_runs_of((int)((N + 127) / 128), (int)((K + KB - 1) / KB))};
    const Plan q = plan_of(routed, M, N, K);
    return I8Plan{q.mode == TWO ? 256 : 128, q.bt, 1 << q.lg};
}
cudaError_t launch_i8_few(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, uint16_t *y, int64_t M, int64_t N, int64_t K, bool f16, int *status, cudaStream_t st) {
    GemmArgs p = args_of(w, w_scale, nullptr, y, M, N, K, f16, status);
    p.xr = x; p.ldx = ldx; p.bt = FEW_ROWS; p.token_tiles = 1;
    const int places = sm_count(), lg = lg_runs_of(p.NB, p.KT);
    const unsigned grid = (unsigned)(lg ? p.NB << lg : p.NB < places ? p.NB : places);
    return lg ? launch<FEW, true>(p, lg, p.NB, grid, st) : launch<FEW, false>(p, 0, p.NB, grid, st);
}

cudaError_t launch_i8_gemm(const void *w, const float *w_scale, const void *x, const float *x_scale, const int32_t *offset, int E, uint16_t *y, int64_t M, int64_t N, int64_t K,
                           bool f16, bool early, int *status, cudaStream_t st) {
    GemmArgs p = args_of(w, w_scale, x_scale, y, M, N, K, f16, status);
    p.early = early;
    p.x = (const uint8_t *)x; p.offset = offset; p.E = E;
    const Plan q = plan_of(offset != nullptr, M, N, K);
    p.token_tiles = (int)((M + q.bt - 1) / q.bt);
    p.bt = q.mode == WIDE ? even_rows(M, p.token_tiles) : q.bt;
    if (q.mode == WIDE) p.token_tiles = (int)((M + p.bt - 1) / p.bt);   // rounded up, the rows of many tiles may fit fewer
    const int ctas = q.mode == TWO ? 2 : 1, nbu = (p.NB + ctas - 1) / ctas, places = sm_count() / ctas;
    const int64_t items = (int64_t)nbu * p.token_tiles;
    const unsigned grid = (unsigned)(q.lg ? items << q.lg : offset ? places : items < places ? items : places) * ctas;
    if (q.mode == TWO) return launch<TWO, false>(p, 0, items, grid, st);
    if (q.mode == WIDE) return launch<WIDE, true>(p, q.lg, items, grid, st);
    if (q.mode == ONE) return q.lg ? launch<ONE, true>(p, q.lg, items, grid, st) : launch<ONE, false>(p, 0, items, grid, st);
    return q.lg ? launch<SMALL, true>(p, q.lg, items, grid, st) : launch<SMALL, false>(p, 0, items, grid, st);
}

}  // namespace cq
