// Quantisers to 4-bit floating point with block scales (layout and formats: cq_fp4.cuh), their inverse, and the exchange with the
// form that checkpoints store.  All of them move bytes: a thread takes sixteen consecutive k of one row.
#include "cq_fp4.cuh"
#include "cq_gated.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"

namespace cq {
namespace fp4 {

// ---------------------------------------------------------------- which rows, and where they go
struct Rows {
    const int32_t *route_token;   // routed: the row of x that row r takes (null: r itself)
    const int32_t *offset;        // routed: first rows of the groups, on the device (null: rows are dense)
    int E;                        // groups, or matrices of `per` rows each
    int64_t per, rows, T;         // rows of one matrix; all rows; rows that x has
};
// the row among the padded rows of the layout of dense rows
__device__ __forceinline__ int64_t padded_row(const Rows &q, int64_t r) {
    if (q.E == 1) return r;
    const int64_t e = r / q.per;
    return e * ((q.per + ROWS - 1) / ROWS * ROWS) + (r - e * q.per);
}
__device__ __forceinline__ void scan_if_routed(const Rows &q, int *s_off, int *s_blk) {
    if (!q.offset) return;
    if (threadIdx.x < 32) scan_groups(q.offset, q.E, (int)q.rows, s_off, s_blk);
    __syncthreads();
}

// The quantisers' work is cut into pieces of 32 rows x 256 k of a tile; a block of 256 threads takes them in turn.  Sixteen threads hold the
// 256 k of a row, a thread sixteen k of two rows, so that what depends on the place is worked out once a piece: with a flat
// index a value cost sixteen instructions, most of them for its address.
constexpr int PIECE = 32;
struct Piece { int64_t first; int blk, kt, from, rows, e; };   // first row of the row block; row block, k tile; first row of the piece in it; rows that the row block has; matrix
__device__ __forceinline__ int64_t pieces_of(const Rows &q, int KT, const int *s_blk) {
    const int64_t blocks = q.offset ? s_blk[q.E] : q.E * ((q.per + ROWS - 1) / ROWS);
    return blocks * KT * (ROWS / PIECE);
}
__device__ __forceinline__ Piece piece_at(const Rows &q, int KT, int64_t i, const int *s_off, const int *s_blk) {
    Piece c;
    const int64_t line = i <= 0xFFFFFFFFll ? (int64_t)((uint32_t)i / (uint32_t)KT) : i / KT;
    c.kt = (int)(i - line * KT);
    c.blk = (int)(line / (ROWS / PIECE));
    c.from = (int)(line % (ROWS / PIECE)) * PIECE;
    if (q.offset) {
        c.e = find_group(s_blk, q.E, c.blk);
        const int in = (c.blk - s_blk[c.e]) * ROWS;
        c.first = s_off[c.e] + in;
        c.rows = min(ROWS, s_off[c.e + 1] - s_off[c.e] - in);
    } else {
        const int per = (int)((q.per + ROWS - 1) / ROWS);
        c.e = q.E == 1 ? 0 : c.blk / per;
        const int64_t in = (int64_t)(c.blk - c.e * per) * ROWS;
        c.first = c.e * q.per + in;
        c.rows = (int)min((int64_t)ROWS, q.per - in);
    }
    return c;
}

// Sixteen codes of (row r, unit u of sixteen k) of a tile and their scales.  All lanes take part in the exchange of the scale
// bytes: four scales of a row are neighbours in memory and are written as one word.
template <int FMT>
__device__ __forceinline__ void store_unit(uint8_t *tile, int r, int u, bool live, uint2 codes, uint32_t scale) {
    const int lane = threadIdx.x & 31;
    const uint32_t word = gather_scales<FMT>(scale);
    if (!live) return;
    *reinterpret_cast<uint2 *>(tile + code_offset(r, u * 8)) = codes;
    if (FMT == NV) {
        if ((lane & 3) == 0) *reinterpret_cast<uint32_t *>(tile + scale_offset(r, u)) = word;
    } else if ((lane & 7) == 0) {
        *reinterpret_cast<uint32_t *>(tile + scale_offset(r, u >> 1)) = word;
    }
}
// NVFP4: what values are multiplied by under each scale byte, r / scale (the byte of NaN: 0), in shared memory
__device__ __forceinline__ void fill_factors(float *s_factor, float r) {
    if (threadIdx.x < 128) s_factor[threadIdx.x] = threadIdx.x < 127 ? __fdiv_rn(r, from_e4m3(threadIdx.x)) : 0.0f;
}

// ---------------------------------------------------------------- the quantiser
// Bound by memory and, for 16-bit values, by instructions alike: 2 (4) bytes read and 0.53 or 0.56 written a value, eleven instructions.  Measured:
// 14336 x 4096 fp32 to MXFP4 44.6 us (6.0 TB/s, 0.91 of the copy rate), 4096 x 8192 bf16 to NVFP4 19.3 us (4.5 TB/s; issue slots 64 % used), to MXFP4
// 18.6 us, a row of 4096 2.6 us, most of it the way to memory and back.  A loop over single units with more threads at a time was 10 % slower.
template <int FMT, int DT>
__global__ void __launch_bounds__(256) quantize_kernel(const void *x, int64_t ldx, Rows q, int64_t K, int KT, const float *tensor_scale, uint8_t *layout) {
    extern __shared__ int s_tab[];
    __shared__ float s_factor[128];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const int u = threadIdx.x & 15, KU = (int)(K >> 4);
    const int64_t pieces = pieces_of(q, KT, s_blk);
    int scaled_for = -1;   // the matrix that r and the factors belong to
    float r = 1.0f;
    for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
        const Piece c = piece_at(q, KT, i, s_off, s_blk);
        if (c.from >= c.rows) continue;
        const int e = q.offset ? 0 : c.e;
        const int unit = c.kt * 16 + u;
        uint8_t *tile = layout + ((int64_t)c.blk * KT + c.kt) * tile_bytes(FMT);
        uint4 raw[2][DT == DT_F32 ? 4 : 2];
        bool live[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = c.from + (threadIdx.x >> 4) + 16 * j;
            live[j] = row < c.rows;
            int64_t src = c.first + row;
            bool read = live[j] && unit < KU;
            if (read && q.route_token) {
                src = q.route_token[src];
                read = src >= 0 && src < q.T;   // any other token is a row of zeros
            }
            const uint8_t *p = reinterpret_cast<const uint8_t *>(x) + (src * ldx + (int64_t)unit * 16) * (DT == DT_F32 ? 4 : 2);
#pragma unroll
            for (int k = 0; k < (DT == DT_F32 ? 4 : 2); ++k) raw[j][k] = read ? load16(p + 16 * k) : make_uint4(0, 0, 0, 0);
        }
        if (FMT == NV && e != scaled_for) {
            if (scaled_for >= 0) __syncthreads();
            if (tensor_scale) r = __fdiv_rn(1.0f, tensor_scale[e]);
            fill_factors(s_factor, r);
            __syncthreads();
            scaled_for = e;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if (c.from + 16 * j >= c.rows) break;
            float v[16];
            uint32_t top;
            if (DT == DT_F32) {
                top = 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint4 w = raw[j][DT == DT_F32 ? k : 0];
                    v[4 * k] = __uint_as_float(w.x); v[4 * k + 1] = __uint_as_float(w.y);
                    v[4 * k + 2] = __uint_as_float(w.z); v[4 * k + 3] = __uint_as_float(w.w);
                }
#pragma unroll
                for (int k = 0; k < 16; ++k) top = max(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
            } else {
                const uint32_t w[8] = {raw[j][0].x, raw[j][0].y, raw[j][0].z, raw[j][0].w, raw[j][1].x, raw[j][1].y, raw[j][1].z, raw[j][1].w};
                top = top_of_16bit<DT>(w);
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = value_of<DT>(w, k);
            }
            float factor;
            uint32_t scale = block_scale<FMT>(top_of_block<FMT>(top), r, s_factor, factor);
            uint2 codes = round_codes(v, factor);
            if (factor == 0.0f) codes = make_uint2(0, 0);   // a block with a NaN or an infinity: what counts is its scale
            if (unit >= KU) scale = 0;                      // behind K
            store_unit<FMT>(tile, c.from + (threadIdx.x >> 4) + 16 * j, u, live[j], codes, scale);
        }
    }
}

// ---------------------------------------------------------------- gated activation and quantiser
// act = silu(gate) * up, rounded to the model dtype (cq_gated.cuh), then quantised; the activation itself reaches no memory.  A code changes when
// that rounding falls on the other side of a border between two codes, so it has to be right.  In a unit of sixteen with a value whose
// rounding 32 bits leave open the candidates on both sides are quantised, and only where a scale or a code differs is the activation formed in 64 bits.
// 25 instructions an activation, in pairs where the GPU has paired fp32 operations; the issue slots are 72 % used.  4096 x 14336 to MXFP4 60.7 us
// (4.4 TB/s); with expf and no pairs 102, with the 64-bit evaluation by single lanes 72.  13 x 14336 3.6 us.  Looking for infinities is 0.8 of the 60.7.
template <int FMT, int DT>
__global__ void __launch_bounds__(256, 4) swiglu_quantize_kernel(const uint16_t *h, int64_t ldh, Rows q, int64_t I, int KT, const float *tensor_scale, uint8_t *layout) {
    extern __shared__ int s_tab[];
    __shared__ float s_factor[128];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    const float r = FMT == NV && tensor_scale ? __fdiv_rn(1.0f, *tensor_scale) : 1.0f;
    if (FMT == NV) fill_factors(s_factor, r);
    scan_if_routed(q, s_off, s_blk);
    __syncthreads();
    const int u = threadIdx.x & 15, KU = (int)(I >> 4);
    const int64_t pieces = pieces_of(q, KT, s_blk);
    for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
        const Piece c = piece_at(q, KT, i, s_off, s_blk);
        if (c.from >= c.rows) continue;
        const int unit = c.kt * 16 + u;
        uint8_t *tile = layout + ((int64_t)c.blk * KT + c.kt) * tile_bytes(FMT);
#pragma unroll 1
        for (int j = 0; j < 2 && c.from + 16 * j < c.rows; ++j) {   // one unit at a time: its registers leave room for the threads that hide the loads
            const int row = c.from + (threadIdx.x >> 4) + 16 * j;
            const bool live = row < c.rows, read = live && unit < KU;
            const uint16_t *pg = h + (c.first + row) * ldh + (int64_t)unit * 16, *pu = pg + I;
            uint32_t gw[8] = {}, uw[8] = {};
            if (read) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint4 a = load16(pg + 8 * k), b = load16(pu + 8 * k);
                    gw[4 * k] = a.x; gw[4 * k + 1] = a.y; gw[4 * k + 2] = a.z; gw[4 * k + 3] = a.w;
                    uw[4 * k] = b.x; uw[4 * k + 1] = b.y; uw[4 * k + 2] = b.z; uw[4 * k + 3] = b.w;
                }
            }
            uint32_t act[8], near = ~0u;
            float y[16], small = 1.0f;
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
                gated_in_32_bits(value_of<DT>(gw, k), value_of<DT>(gw, k + 1), value_of<DT>(uw, k), value_of<DT>(uw, k + 1), y[k], y[k + 1]);
                near = nearer<DT>(near, y[k], y[k + 1]);
                act[k / 2] = pack16<DT>(y[k], y[k + 1]);
                if (DT == DT_F16) small = fminf(small, fminf(y[k] == 0.0f ? 1.0f : fabsf(y[k]), y[k + 1] == 0.0f ? 1.0f : fabsf(y[k + 1])));   // subnormal halves have their borders elsewhere
            }
            constexpr uint32_t WIDE = 2 * BAND * (DT == DT_BF16 ? 1 : 8);
            const uint32_t largest = top_of_16bit<DT>(act);
            const bool far = top_of_16bit<DT>(gw) > 0x42700000u || largest >= 0x7F800000u;   // 60; infinities and NaN
            const bool open = (near & 0xFFFFu) <= WIDE || (near >> 16) <= WIDE || far || (DT == DT_F16 && small < 6.103515625e-05f);
            uint32_t top = top_of_block<FMT>(largest);
            if (__any_sync(~0u, open)) {
                uint32_t a0[8], a1[8];   // a unit without open values has one candidate
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    a0[k] = open ? pack16<DT>(ulps_away(y[2 * k], -BAND), ulps_away(y[2 * k + 1], -BAND)) : act[k];
                    a1[k] = open ? pack16<DT>(ulps_away(y[2 * k], BAND), ulps_away(y[2 * k + 1], BAND)) : act[k];
                }
                float f0, f1, v0[16], v1[16];
                const uint32_t s0 = block_scale<FMT>(top_of_block<FMT>(top_of_16bit<DT>(a0)), r, s_factor, f0);
                const uint32_t s1 = block_scale<FMT>(top_of_block<FMT>(top_of_16bit<DT>(a1)), r, s_factor, f1);
#pragma unroll
                for (int k = 0; k < 16; ++k) { v0[k] = value_of<DT>(a0, k); v1[k] = value_of<DT>(a1, k); }
                const uint2 c0 = round_codes(v0, f0), c1 = round_codes(v1, f1);
                settle_in_64_bits<DT>(open && (far || s0 != s1 || c0.x != c1.x || c0.y != c1.y), gw, uw, act);
                top = top_of_block<FMT>(top_of_16bit<DT>(act));
            }
            float factor, v[16];
            uint32_t scale = block_scale<FMT>(top, r, s_factor, factor);
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = value_of<DT>(act, k);
            uint2 codes = round_codes(v, factor);
            if (factor == 0.0f) codes = make_uint2(0, 0);
            if (unit >= KU) scale = 0;
            store_unit<FMT>(tile, row, u, live, codes, scale);
        }
    }
}

// ---------------------------------------------------------------- back to values
// code * fl32(scale * g), rounded once to the type asked for.  Reads what the layout stores, writes 2 or 4 bytes a value: a thread takes
// eight values, so that a warp's stores are one run of memory (sixteen a thread, half of each run at a time: 51 us for 58.7 M values in
// bfloat16; 30.3 so, 4.9 TB/s, eleven instructions a value).
template <int FMT, int DT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *layout, Rows q, int64_t K, int KT, const float *tensor_scale, void *y) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const int u = threadIdx.x & 31, KU = (int)(K >> 3);
    const int64_t pieces = pieces_of(q, KT, s_blk);
    for (int64_t i = blockIdx.x; i < pieces; i += gridDim.x) {
        const Piece c = piece_at(q, KT, i, s_off, s_blk);
        if (c.from >= c.rows || c.kt * 32 + u >= KU) continue;
        const uint8_t *tile = layout + ((int64_t)c.blk * KT + c.kt) * tile_bytes(FMT);
        const float g = FMT == NV && tensor_scale ? tensor_scale[q.offset ? 0 : c.e] : 1.0f;
        uint32_t codes[4], scales[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = c.from + (threadIdx.x >> 5) + 8 * j;   // what lies behind the last row is inside the tile too
            codes[j] = *reinterpret_cast<const uint32_t *>(tile + code_offset(r, u * 4));
            scales[j] = tile[scale_offset(r, FMT == NV ? u >> 1 : u >> 2)];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = c.from + (threadIdx.x >> 5) + 8 * j;
            if (r >= c.rows) break;
            const float s = FMT == NV ? __fmul_rn(from_e4m3(scales[j]), g) : from_e8m0(scales[j]);
            float v[8];
            from_e2m1x8(codes[j], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= s;
            const int64_t at = (c.first + r) * K + c.kt * KB + u * 8;
            if (DT == DT_F32) {
                float4 *p = reinterpret_cast<float4 *>(reinterpret_cast<float *>(y) + at);
                p[0] = make_float4(v[0], v[1], v[2], v[3]);
                p[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(y) + at) = make_uint4(pack16<DT>(v[0], v[1]), pack16<DT>(v[2], v[3]), pack16<DT>(v[4], v[5]), pack16<DT>(v[6], v[7]));
            }
        }
    }
}

// ---------------------------------------------------------------- checkpoints (once for each matrix of a model): codes [rows][K / 2], scales [rows][K / block]
template <int FMT, bool IN>
__global__ void __launch_bounds__(256) exchange_kernel(uint8_t *codes, uint8_t *scales, Rows q, int64_t K, int KT, uint8_t *layout) {
    const int KU = KT * 16, block = block_of(FMT);
    const int64_t total = q.rows * KU;
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = idx / KU;
        const int unit = (int)(idx - row * KU), u = unit & 15;
        const int64_t k = (int64_t)unit * 16, prow = padded_row(q, row);
        const int r = (int)(prow & (ROWS - 1));
        uint8_t *tile = layout + ((prow >> 7) * KT + (unit >> 4)) * (int64_t)tile_bytes(FMT);
        uint2 *at = reinterpret_cast<uint2 *>(tile + code_offset(r, u * 8));
        uint8_t *sat = tile + scale_offset(r, (u * 16) / block);
        const bool inside = k < K, first = (u * 16) % block == 0;
        uint2 *cp = reinterpret_cast<uint2 *>(codes + row * (K / 2) + k / 2);   // K a multiple of 16: 8-byte pieces
        uint8_t *sp = scales + row * (K / block) + k / block;
        if (IN) {
            *at = inside ? *cp : make_uint2(0, 0);
            if (first) *sat = inside ? *sp : (uint8_t)0;
        } else if (inside) {
            *cp = *at;
            if (first) *sp = *sat;
        }
    }
}

// ---------------------------------------------------------------- launchers
// Enough blocks to fill the SMs eight deep; the rest follows in a loop (the tables of a block are filled once).
static unsigned grid_of(int64_t blocks) {
    const int64_t most = 8 * (int64_t)sm_count();
    return (unsigned)(blocks < most ? blocks : most);
}
static unsigned grid_for(int64_t units) { return grid_of((units + 255) / 256); }
// pieces of all row blocks that may have rows (routed: every group may end a block early); of the last row block of a single matrix only those that have
static unsigned grid_for_pieces(const Rows &q, int KT) {
    const int64_t per = q.offset ? (q.rows + (ROWS - 1) * (q.E < q.rows ? q.E : q.rows)) / ROWS * ROWS : q.E == 1 ? q.rows : (q.per + ROWS - 1) / ROWS * ROWS * q.E;
    return grid_of((per + PIECE - 1) / PIECE * KT);
}
static size_t table_bytes(const Rows &q) { return q.offset ? 2 * (size_t)(q.E + 1) * sizeof(int) : 0; }
static Rows rows_of(const Fp4Rows &s) { return Rows{s.route_token, s.offset, s.E, s.per, s.rows, s.T}; }
static int kt_of(int64_t K) { return (int)((K + KB - 1) / KB); }

}  // namespace fp4

using namespace fp4;

cudaError_t launch_fp4_quantize(const void *x, int dtype, int64_t ldx, const Fp4Rows &s, int fmt, int64_t K, const float *tensor_scale, void *layout, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(K);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_for_pieces(q, KT)), 256u, table_bytes(q), st, 1, true, x, ldx, q, K, KT, tensor_scale, (uint8_t *)layout);
    };
    if (fmt == MX) return dtype == DT_BF16 ? go(quantize_kernel<MX, DT_BF16>) : dtype == DT_F16 ? go(quantize_kernel<MX, DT_F16>) : go(quantize_kernel<MX, DT_F32>);
    return dtype == DT_BF16 ? go(quantize_kernel<NV, DT_BF16>) : dtype == DT_F16 ? go(quantize_kernel<NV, DT_F16>) : go(quantize_kernel<NV, DT_F32>);
}

cudaError_t launch_fp4_swiglu_quantize(const void *h, int dtype, int64_t ldh, const Fp4Rows &s, int fmt, int64_t I, const float *tensor_scale, void *layout, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(I);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_for_pieces(q, KT)), 256u, table_bytes(q), st, 1, true, (const uint16_t *)h, ldh, q, I, KT, tensor_scale, (uint8_t *)layout);
    };
    if (fmt == MX) return dtype == DT_BF16 ? go(swiglu_quantize_kernel<MX, DT_BF16>) : go(swiglu_quantize_kernel<MX, DT_F16>);
    return dtype == DT_BF16 ? go(swiglu_quantize_kernel<NV, DT_BF16>) : go(swiglu_quantize_kernel<NV, DT_F16>);
}

cudaError_t launch_fp4_dequantize(const void *layout, const Fp4Rows &s, int fmt, int64_t K, const float *tensor_scale, void *y, int dtype, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(K);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_for_pieces(q, KT)), 256u, table_bytes(q), st, 1, true, (const uint8_t *)layout, q, K, KT, tensor_scale, y);
    };
    if (fmt == MX) return dtype == DT_BF16 ? go(dequantize_kernel<MX, DT_BF16>) : dtype == DT_F16 ? go(dequantize_kernel<MX, DT_F16>) : go(dequantize_kernel<MX, DT_F32>);
    return dtype == DT_BF16 ? go(dequantize_kernel<NV, DT_BF16>) : dtype == DT_F16 ? go(dequantize_kernel<NV, DT_F16>) : go(dequantize_kernel<NV, DT_F32>);
}

cudaError_t launch_fp4_exchange(uint8_t *codes, uint8_t *scales, const Fp4Rows &s, int fmt, int64_t K, void *layout, bool in, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(K);
    const unsigned grid = grid_for(q.rows * KT * 16);
    if (fmt == MX) {
        if (in) exchange_kernel<MX, true><<<grid, 256, 0, st>>>(codes, scales, q, K, KT, (uint8_t *)layout);
        else exchange_kernel<MX, false><<<grid, 256, 0, st>>>(codes, scales, q, K, KT, (uint8_t *)layout);
    } else {
        if (in) exchange_kernel<NV, true><<<grid, 256, 0, st>>>(codes, scales, q, K, KT, (uint8_t *)layout);
        else exchange_kernel<NV, false><<<grid, 256, 0, st>>>(codes, scales, q, K, KT, (uint8_t *)layout);
    }
    return cudaGetLastError();
}

}  // namespace cq
