// Quantisers to 4-bit floating point with block scales (layout and formats: cq_fp4.cuh), their inverse, and the exchange with the
// form that checkpoints store.  All of them move bytes: a thread takes sixteen consecutive k of one row.
#include "cq_fp4.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"

namespace cq {
namespace fp4 {

// ---------------------------------------------------------------- sixteen values of a row
struct Raw16 { uint4 v[2]; };
__device__ __forceinline__ uint4 load16(const void *p) { return *reinterpret_cast<const uint4 *>(p); }
template <int DT>
__device__ __forceinline__ float value_of(const uint32_t *w, int i) {
    const uint32_t h = (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
    return DT == DT_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
// bits of the largest magnitude of sixteen 16-bit values; NaN counts as the largest
template <int DT>
__device__ __forceinline__ uint32_t top_of_16bit(const uint32_t *w) {
    if (DT == DT_BF16) {
        __nv_bfloat162 m = __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w[0]));
#pragma unroll
        for (int i = 1; i < 8; ++i) m = __hmax2_nan(m, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i])));
        const uint32_t b = *reinterpret_cast<uint32_t *>(&m) & 0x7FFF7FFFu;
        return max(b << 16, b & 0xFFFF0000u);
    }
    __half2 m = __habs2(*reinterpret_cast<const __half2 *>(&w[0]));
#pragma unroll
    for (int i = 1; i < 8; ++i) m = __hmax2_nan(m, __habs2(*reinterpret_cast<const __half2 *>(&w[i])));
    return max(__float_as_uint(__low2float(m)) & 0x7FFFFFFFu, __float_as_uint(__high2float(m)) & 0x7FFFFFFFu);
}

template <int FMT>
__device__ __forceinline__ uint32_t top_of_block(uint32_t top) {   // MXFP4: two threads hold a block
    return FMT == MX ? max(top, __shfl_xor_sync(~0u, top, 1)) : top;
}

// ---------------------------------------------------------------- where a row goes
struct Rows {
    const int32_t *route_token;   // routed: the row of x that row r takes (null: r itself)
    const int32_t *offset;        // routed: first rows of the groups, on the device (null: rows are dense)
    int E;                        // groups, or matrices of `per` rows each
    int64_t per, rows, T;         // rows of one matrix; all rows; rows that x has
};
// the row among the padded rows of the layout, or -1
__device__ __forceinline__ int64_t padded_row(const Rows &q, int64_t r, const int *s_off, const int *s_blk) {
    if (r >= q.rows) return -1;
    if (q.offset) {
        if (r >= s_off[q.E]) return -1;
        const int e = find_group(s_off, q.E, (int)r);
        return (int64_t)s_blk[e] * ROWS + ((int)r - s_off[e]);
    }
    if (q.E == 1) return r;
    const int64_t e = r / q.per;
    return e * ((q.per + ROWS - 1) / ROWS * ROWS) + (r - e * q.per);
}

// Sixteen codes of (row, unit of 16 k) and their scales into the layout.  All lanes take part in the exchange of the scale
// bytes: four scales of a row are neighbours in memory and are written as one word.
template <int FMT>
__device__ __forceinline__ void store_unit(uint8_t *layout, int64_t prow, int unit, int KT, uint2 codes, uint32_t scale) {
    const int lane = threadIdx.x & 31;
    uint32_t word;
    if (FMT == NV) {
        word = scale << (8 * (lane & 3));
        word |= __shfl_xor_sync(~0u, word, 1);
        word |= __shfl_xor_sync(~0u, word, 2);
    } else {
        word = scale << (8 * ((lane >> 1) & 3));
        word |= __shfl_xor_sync(~0u, word, 2);
        word |= __shfl_xor_sync(~0u, word, 4);
    }
    if (prow < 0) return;
    const int r = (int)(prow & (ROWS - 1)), u = unit & 15;
    uint8_t *tile = layout + ((prow >> 7) * KT + (unit >> 4)) * (int64_t)tile_bytes(FMT);
    *reinterpret_cast<uint2 *>(tile + code_offset(r, u * 8)) = codes;
    if (FMT == NV) {
        if ((lane & 3) == 0) *reinterpret_cast<uint32_t *>(tile + scale_offset(r, u)) = word;
    } else if ((lane & 7) == 0) {
        *reinterpret_cast<uint32_t *>(tile + scale_offset(r, u >> 1)) = word;
    }
}

template <int FMT>
__device__ __forceinline__ uint2 round_codes(const float *v, float factor) {
    float u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __fmul_rn(v[i], factor);
    return make_uint2(to_e2m1x8(u), to_e2m1x8(u + 8));
}

__device__ __forceinline__ void scan_if_routed(const Rows &q, int *s_off, int *s_blk) {
    if (!q.offset) return;
    if (threadIdx.x < 32) scan_groups(q.offset, q.E, (int)q.rows, s_off, s_blk);
    __syncthreads();
}

// ---------------------------------------------------------------- the quantiser
// Bound by memory: 2 (4) bytes read and 0.53 or 0.56 written a value.
template <int FMT, int DT>
__global__ void __launch_bounds__(256) quantize_kernel(const void *x, int64_t ldx, Rows q, int64_t K, int KT, const float *tensor_scale, uint8_t *layout) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const uint32_t U = (uint32_t)KT * 16u, KU = (uint32_t)(K >> 4);
    const int64_t total = q.rows * U;
    for (int64_t base = (int64_t)blockIdx.x * 256; base < total; base += (int64_t)gridDim.x * 256) {   // whole warps stay together
        const int64_t idx = base + threadIdx.x;
        const int64_t row = total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)idx / U) : idx / U;
        const uint32_t unit = (uint32_t)(idx - row * U);
        const int64_t prow = idx < total ? padded_row(q, row, s_off, s_blk) : -1;
        int64_t src = row;
        bool read = prow >= 0 && unit < KU;
        if (read && q.route_token) {
            src = q.route_token[row];
            read = src >= 0 && src < q.T;   // any other token is a row of zeros
        }
        const float r = FMT == NV ? (tensor_scale ? __fdiv_rn(1.0f, tensor_scale[q.offset || q.E == 1 || row >= q.rows ? 0 : row / q.per]) : 1.0f) : 1.0f;
        float v[16];
        uint32_t top;
        if (DT == DT_F32) {
            const float *p = reinterpret_cast<const float *>(x) + src * ldx + (int64_t)unit * 16;
            top = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = read ? load16(p + 4 * i) : make_uint4(0, 0, 0, 0);
                v[4 * i] = __uint_as_float(w.x); v[4 * i + 1] = __uint_as_float(w.y);
                v[4 * i + 2] = __uint_as_float(w.z); v[4 * i + 3] = __uint_as_float(w.w);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        } else {
            const uint16_t *p = reinterpret_cast<const uint16_t *>(x) + src * ldx + (int64_t)unit * 16;
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (read) { a = load16(p); b = load16(p + 8); }
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            top = top_of_16bit<DT>(w);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = value_of<DT>(w, i);
        }
        float factor;
        uint32_t scale = block_scale<FMT>(top_of_block<FMT>(top), r, factor);
        uint2 codes = round_codes<FMT>(v, factor);
        if (factor == 0.0f) codes = make_uint2(0, 0);   // a block with a NaN or an infinity: what counts is its scale
        if (unit >= KU) scale = 0;                      // behind K
        store_unit<FMT>(layout, prow, (int)unit, KT, codes, scale);
    }
}

// ---------------------------------------------------------------- gated activation and quantiser
// act = silu(gate) * up = gate up / (1 + exp(-gate)), rounded to the model dtype, then quantised; the activation itself reaches no memory.
// A code changes when a rounding to the model dtype falls on the other side of a border between two codes, so that rounding has to
// be right, and 32 bits leave it open where the value lies next to a border of the model dtype.  gate * up is exact in 32 bits, exp
// is off by 1 ulp, the sum by half, the division by 2: four ulps.  Where no value lies within BAND = 8 ulps of a border
// the roundings stand; in a unit where one does (one in 180 in bfloat16, one in 23 in binary16), its two candidates are
// quantised both ways, and only when the scale or a code differ is the value formed in 64 bits.  Far negative gates
// (exp(60) is still finite in 32 bits, with room) go that way at once.
constexpr int BAND = 8;
template <int DT>
__device__ __forceinline__ uint32_t round16(float v) {
    return DT == DT_BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)) : (uint32_t)__half_as_ushort(__float2half_rn(v));
}
template <int DT>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (DT == DT_BF16) { const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const uint32_t *>(&p); }
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}
template <int DT>
__device__ __noinline__ uint32_t gated_in_64_bits(float g, float u) {
    const double y = (double)g * (double)u / (1.0 + exp(-(double)g));
    return round16<DT>((float)y);
}
__device__ __forceinline__ float ulps_away(float v, int n) { return __uint_as_float(__float_as_uint(v) + n); }   // n > 0: away from zero

template <int FMT, int DT>
__global__ void __launch_bounds__(256) swiglu_quantize_kernel(const uint16_t *h, int64_t ldh, Rows q, int64_t I, int KT, const float *tensor_scale, uint8_t *layout) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const uint32_t U = (uint32_t)KT * 16u, KU = (uint32_t)(I >> 4);
    const int64_t total = q.rows * U;
    const float r = FMT == NV && tensor_scale ? __fdiv_rn(1.0f, *tensor_scale) : 1.0f;
    for (int64_t base = (int64_t)blockIdx.x * 256; base < total; base += (int64_t)gridDim.x * 256) {
        const int64_t idx = base + threadIdx.x;
        const int64_t row = total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)idx / U) : idx / U;
        const uint32_t unit = (uint32_t)(idx - row * U);
        const int64_t prow = idx < total ? padded_row(q, row, s_off, s_blk) : -1;
        const bool read = prow >= 0 && unit < KU;
        const uint16_t *pg = h + row * ldh + (int64_t)unit * 16, *pu = pg + I;
        uint32_t gw[8] = {}, uw[8] = {}, act[8];
        if (read) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 a = load16(pg + 8 * i), b = load16(pu + 8 * i);
                gw[4 * i] = a.x; gw[4 * i + 1] = a.y; gw[4 * i + 2] = a.z; gw[4 * i + 3] = a.w;
                uw[4 * i] = b.x; uw[4 * i + 1] = b.y; uw[4 * i + 2] = b.z; uw[4 * i + 3] = b.w;
            }
        }
        float y[16];
        // least distance to a border of the model dtype, in ulps, less BAND; borders lie in the middle of the bits that are dropped
        constexpr uint32_t DROP = DT == DT_BF16 ? 0xFFFFu : 0x1FFFu, HALF = DT == DT_BF16 ? 0x8000u : 0x1000u;
        uint32_t near = ~0u;
        float least = 0.0f, small = 1.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float g = value_of<DT>(gw, i), u = value_of<DT>(uw, i);
            y[i] = __fdividef(__fmul_rn(g, u), 1.0f + expf(-g));
            near = min(near, (__float_as_uint(y[i]) - HALF + BAND) & DROP);
            least = fminf(least, g);
            if (DT == DT_F16) small = fminf(small, y[i] == 0.0f ? 1.0f : fabsf(y[i]));   // subnormal halves have their borders elsewhere
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) act[i] = pack16<DT>(y[2 * i], y[2 * i + 1]);
        const bool far = least < -60.0f;
        const bool open = near <= 2 * BAND || far || (DT == DT_F16 && small < 6.103515625e-05f);
        uint32_t top = top_of_block<FMT>(top_of_16bit<DT>(act));
        if (__any_sync(~0u, open)) {
            // the candidates on both sides: a unit without open values has the same ones
            uint32_t a0[8], a1[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                a0[i] = pack16<DT>(ulps_away(y[2 * i], -BAND), ulps_away(y[2 * i + 1], -BAND));
                a1[i] = pack16<DT>(ulps_away(y[2 * i], BAND), ulps_away(y[2 * i + 1], BAND));
                if (!open) a0[i] = a1[i] = act[i];
            }
            const uint32_t t0 = top_of_block<FMT>(top_of_16bit<DT>(a0)), t1 = top_of_block<FMT>(top_of_16bit<DT>(a1));
            float f0, f1, v0[16], v1[16];
            const uint32_t s0 = block_scale<FMT>(t0, r, f0), s1 = block_scale<FMT>(t1, r, f1);
#pragma unroll
            for (int i = 0; i < 16; ++i) { v0[i] = value_of<DT>(a0, i); v1[i] = value_of<DT>(a1, i); }
            const uint2 c0 = round_codes<FMT>(v0, f0), c1 = round_codes<FMT>(v1, f1);
            const bool differ = open && (far || s0 != s1 || c0.x != c1.x || c0.y != c1.y);
            if (differ) {
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    const uint32_t g2 = gw[i], u2 = uw[i];
                    uint32_t lo = gated_in_64_bits<DT>(value_of<DT>(&g2, 0), value_of<DT>(&u2, 0));
                    act[i] = lo | gated_in_64_bits<DT>(value_of<DT>(&g2, 1), value_of<DT>(&u2, 1)) << 16;
                }
            }
            top = top_of_block<FMT>(top_of_16bit<DT>(act));
        }
        float factor, v[16];
        uint32_t scale = block_scale<FMT>(top, r, factor);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = value_of<DT>(act, i);
        uint2 codes = round_codes<FMT>(v, factor);
        if (factor == 0.0f) codes = make_uint2(0, 0);
        if (unit >= KU) scale = 0;
        store_unit<FMT>(layout, prow, (int)unit, KT, codes, scale);
    }
}

// ---------------------------------------------------------------- back to values
// code * fl32(scale * g), rounded once to the type asked for.  Reads what the layout stores, writes 2 or 4 bytes a value.
template <int FMT, int DT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *layout, Rows q, int64_t K, int KT, const float *tensor_scale, void *y) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const uint32_t KU = (uint32_t)(K >> 4);
    const int64_t total = q.rows * KU;
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)idx / KU) : idx / KU;
        const int unit = (int)(idx - row * KU), u = unit & 15;
        const int64_t prow = padded_row(q, row, s_off, s_blk);
        if (prow < 0) continue;
        const int r = (int)(prow & (ROWS - 1));
        const uint8_t *tile = layout + ((prow >> 7) * KT + (unit >> 4)) * (int64_t)tile_bytes(FMT);
        const uint2 codes = *reinterpret_cast<const uint2 *>(tile + code_offset(r, u * 8));
        float s;
        if (FMT == NV) {
            s = from_e4m3(tile[scale_offset(r, u)]);
            if (tensor_scale) s = __fmul_rn(s, tensor_scale[q.offset || q.E == 1 ? 0 : row / q.per]);
        } else {
            s = from_e8m0(tile[scale_offset(r, u >> 1)]);
        }
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = from_e2m1((i < 8 ? codes.x : codes.y) >> (4 * (i & 7))) * s;
        const int64_t at = row * K + (int64_t)unit * 16;
        if (DT == DT_F32) {
            float4 *p = reinterpret_cast<float4 *>(reinterpret_cast<float *>(y) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack16<DT>(v[2 * i], v[2 * i + 1]);
            uint4 *p = reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(y) + at);
            p[0] = make_uint4(w[0], w[1], w[2], w[3]);
            p[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

// ---------------------------------------------------------------- checkpoints: codes [rows][K / 2], scales [rows][K / block]
template <int FMT, bool IN>
__global__ void __launch_bounds__(256) exchange_kernel(uint8_t *codes, uint8_t *scales, Rows q, int64_t K, int KT, uint8_t *layout) {
    const int KU = KT * 16, block = block_of(FMT);
    const int64_t total = q.rows * KU;
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = idx / KU;
        const int unit = (int)(idx - row * KU), u = unit & 15;
        const int64_t k = (int64_t)unit * 16, prow = padded_row(q, row, nullptr, nullptr);
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
// Enough blocks to fill the SMs eight deep; the rest of the rows follow in a loop (the table of the groups is read once a block).
static unsigned grid_for(int64_t units) {
    const int64_t blocks = (units + 255) / 256, most = 8 * (int64_t)sm_count();
    return (unsigned)(blocks < most ? blocks : most);
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
        return launch_overlapped(kern, dim3(grid_for(q.rows * KT * 16)), 256u, table_bytes(q), st, 1, true, x, ldx, q, K, KT, tensor_scale, (uint8_t *)layout);
    };
    if (fmt == MX) return dtype == DT_BF16 ? go(quantize_kernel<MX, DT_BF16>) : dtype == DT_F16 ? go(quantize_kernel<MX, DT_F16>) : go(quantize_kernel<MX, DT_F32>);
    return dtype == DT_BF16 ? go(quantize_kernel<NV, DT_BF16>) : dtype == DT_F16 ? go(quantize_kernel<NV, DT_F16>) : go(quantize_kernel<NV, DT_F32>);
}

cudaError_t launch_fp4_swiglu_quantize(const void *h, int dtype, int64_t ldh, const Fp4Rows &s, int fmt, int64_t I, const float *tensor_scale, void *layout, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(I);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_for(q.rows * KT * 16)), 256u, table_bytes(q), st, 1, true, (const uint16_t *)h, ldh, q, I, KT, tensor_scale, (uint8_t *)layout);
    };
    if (fmt == MX) return dtype == DT_BF16 ? go(swiglu_quantize_kernel<MX, DT_BF16>) : go(swiglu_quantize_kernel<MX, DT_F16>);
    return dtype == DT_BF16 ? go(swiglu_quantize_kernel<NV, DT_BF16>) : go(swiglu_quantize_kernel<NV, DT_F16>);
}

cudaError_t launch_fp4_dequantize(const void *layout, const Fp4Rows &s, int fmt, int64_t K, const float *tensor_scale, void *y, int dtype, cudaStream_t st) {
    const Rows q = rows_of(s);
    const int KT = kt_of(K);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_for(q.rows * (K / 16))), 256u, table_bytes(q), st, 1, true, (const uint8_t *)layout, q, K, KT, tensor_scale, y);
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
