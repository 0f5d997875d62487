// What the products of two stored operands share (cq_fp4_gemm.cu, cq_i8_gemm.cu): the order of their output tiles, the way of accumulators to
// y, waits and arrivals within a CTA, a pair, a cluster.
// Args, the arguments of a product, has: offset (routed: first rows of the groups), E, NB (row blocks of W), M (rows of x), bt (rows of x to a tile at most), token_tiles
// (dense: tiles along the rows of x), band (how many of them are swept together), rows_of_tile(rows, tiles): what a tile has of so many rows that fill so many tiles.
#pragma once
#include "cq_rows.cuh"
#include "cq_tc_ptx.cuh"

namespace cq {
namespace rows {

// accumulators to registers in the order of 8x8 matrices: lane l has row l / 4 (+ 8), columns 8 i + 2 (l % 4) and the next
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void stmatrix_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint16_t round_out(float v, bool f16) { return f16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

// the MMAs issued so far arrive on this barrier in both CTAs of the pair (cluster ranks r & ~1 and the next) when they have completed
__device__ __forceinline__ void commit_to_pair(uint64_t *bar, int cluster_rank) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(tc::smem_u32(bar)), "h"((uint16_t)(3 << (cluster_rank & ~1))) : "memory");
}
// a bounded wait of a whole warp, whose answer all lanes share
__device__ __forceinline__ bool uniform_wait(uint64_t *bar, uint32_t parity, int *status, int code, volatile int *dead) {
    if (__all_sync(~0u, tc::mbar_try_wait(bar, parity))) return true;
    return __all_sync(~0u, tc::mbar_wait(bar, parity, status, code, tc::WAIT_LIMIT_CYCLES, dead));
}
// the eight warps that write y: a barrier, and whether any thread brings a true (what one of them decides alone would leave the others waiting)
__device__ __forceinline__ bool epilogue_any(bool v) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.or.pred q, 1, 256, p;\n\tselp.b32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)v) : "memory");
    return r != 0;
}
__device__ __forceinline__ void wait_for_quantiser() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// sixteen bytes into the shared memory of a CTA of the cluster, counted there on `bar`
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d), "r"(bar) : "memory");
}
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

struct Item { int e, nb, rows, xblk, off, yrow; };   // matrix; row block (pair of them); rows of the tile; first row block of x and row in it; row of y

// The idx-th output tile.  Token tiles run fastest within a band of them, so that the CTAs that work at the same time share the
// weights of few row blocks and the activations of one band; both then come from L2.
template <bool PAIR, class Args>
__device__ __forceinline__ Item item_of(const Args &p, int idx, const int *s_off, const int *s_blk, const int *s_item) {
    Item t;
    int rows = p.M, tiles = p.token_tiles, first_blk = 0, first_row = 0;
    t.e = 0;
    if (p.offset) {
        t.e = find_group(s_item, p.E, idx);
        idx -= s_item[t.e];
        first_row = s_off[t.e];
        rows = s_off[t.e + 1] - s_off[t.e];
        first_blk = s_blk[t.e];
        tiles = (rows + p.bt - 1) / p.bt;
    }
    const int nbu = PAIR ? (p.NB + 1) >> 1 : p.NB;
    const int per_band = nbu * p.band, g = idx / per_band, rem = idx - g * per_band;
    const int wide = min(p.band, tiles - g * p.band);
    t.nb = rem / wide;
    const int tt = g * p.band + rem - t.nb * wide;
    const int bt = p.rows_of_tile(rows, tiles), row0 = tt * bt;
    t.rows = min(bt, rows - row0);
    t.xblk = first_blk + row0 / ROWS;
    t.off = row0 % ROWS;
    t.yrow = first_row + row0;
    return t;
}
// The tiles of a CTA, unit + i * stride, as each warp goes through them: 32 at a time, a lane for each, since the divisions of one by one
// took as long as two stages of the tensor core.
template <bool PAIR, class Args>
struct Tiles {
    const Args &p;
    const int unit, stride;
    int items;
    const int *s_off, *s_blk, *s_item;
    Item mine;
    bool ahead = false;   // `look` has been called for the first 32
    __device__ __forceinline__ bool has(int i) const { return unit + (int64_t)i * stride < items; }
    __device__ __forceinline__ void look(int i) {
        const int64_t idx = unit + (int64_t)(i + (int)(threadIdx.x & 31)) * stride;
        if (idx < items) mine = item_of<PAIR>(p, (int)idx, s_off, s_blk, s_item);
        __syncwarp();
    }
    __device__ __forceinline__ Item at(int i) {   // i = 0, 1, 2 ..; the whole warp
        if ((i & 31) == 0 && !(i == 0 && ahead)) look(i);
        Item t;
        const int packed = __shfl_sync(~0u, mine.rows << 8 | mine.off, i & 31);
        t.e = __shfl_sync(~0u, mine.e, i & 31);
        t.nb = __shfl_sync(~0u, mine.nb, i & 31);
        t.xblk = __shfl_sync(~0u, mine.xblk, i & 31);
        t.yrow = __shfl_sync(~0u, mine.yrow, i & 31);
        t.rows = packed >> 8;
        t.off = packed & 255;
        return t;
    }
};
template <bool PAIR> __device__ __forceinline__ int columns_of(int rows) { return PAIR ? (rows + 31) & ~31 : (rows + 15) & ~15; }

}  // namespace rows
}  // namespace cq
