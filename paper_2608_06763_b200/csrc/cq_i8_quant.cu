// Quantisers to 8-bit integers with a scale for each row (layout: cq_i8.cuh), their inverse, and the exchange with the form that checkpoints
// store.
#include "cq_gated.cuh"
#include "cq_i8.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"

namespace cq {
namespace i8 {

// A row belongs to a team of threads, 32 to 512 of them, each with units of sixteen neighbouring k; a block has one team or several.
constexpr int HELD = 4;   // units of a row that a thread keeps in registers until the row's scale is known
struct Rows {
    const int32_t *route_token;   // routed: the row of x that row r takes (null: r itself)
    const int32_t *offset;        // routed: first rows of the groups, on the device (null: rows are dense)
    int E;                        // groups, or matrices of `per` rows each
    int64_t per, rows, T;         // rows of one matrix; all rows; rows that x has
    int team;                     // threads to a row
};
struct Place { int64_t src, at; bool live, read; };   // row of x; row among the padded rows of the layout; whether it is one; whether x has it
__device__ __forceinline__ void scan_if_routed(const Rows &q, int *s_off, int *s_blk) {
    if (!q.offset) return;
    if (threadIdx.x < 32) scan_groups(q.offset, q.E, (int)q.rows, s_off, s_blk);
    __syncthreads();
}
__device__ __forceinline__ Place place_of(const Rows &q, int64_t r, const int *s_off, const int *s_blk) {
    Place p{r, r, r < q.rows, r < q.rows};
    if (q.offset) {
        p.live = p.live && r >= s_off[0] && r < s_off[q.E];
        p.read = p.live;
        if (p.live) {
            const int e = find_group(s_off, q.E, (int)r);
            p.at = (int64_t)s_blk[e] * ROWS + (r - s_off[e]);
            if (q.route_token) {
                p.src = q.route_token[r];
                p.read = p.src >= 0 && p.src < q.T;   // any other token is a row of zeros
            }
        }
    } else if (q.E > 1 && p.live) {
        const int64_t e = r / q.per;
        p.at = e * ((q.per + ROWS - 1) / ROWS * ROWS) + (r - e * q.per);
    }
    return p;
}
// the largest of a team's values; `red` has a word for each warp of the block, and is not written again before the next but one of these
__device__ __forceinline__ uint32_t team_max(uint32_t v, int team, uint32_t *red) {
    v = __reduce_max_sync(~0u, v);
    if (team == 32) return v;
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
    const int first = threadIdx.x / team * (team / 32), lane = threadIdx.x & 31;
    return __reduce_max_sync(~0u, lane < team / 32 ? red[first + lane] : 0u);
}

// ---------------------------------------------------------------- where sixteen values of a row come from
// rows of x as they are
template <int DT>
struct Plain {
    static constexpr int WORDS = DT == DT_F32 ? 16 : 8;
    const void *x;
    int64_t ldx;
    __device__ __forceinline__ uint32_t get(int64_t row, int64_t unit, bool read, uint32_t *w) const {
        const uint8_t *p = reinterpret_cast<const uint8_t *>(x) + (row * ldx + unit * 16) * (DT == DT_F32 ? 4 : 2);
#pragma unroll
        for (int k = 0; k < WORDS / 4; ++k) {
            const uint4 q = read ? load16(p + 16 * k) : make_uint4(0, 0, 0, 0);
            w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
        }
        uint32_t top = 0;
        if (DT == DT_F32) {
#pragma unroll
            for (int k = 0; k < WORDS; ++k) top = max(top, w[k] & 0x7FFFFFFFu);
        } else {
            top = top_of_16bit<DT>(w);
        }
        return top;
    }
    __device__ __forceinline__ uint4 codes(const uint32_t *w, float d, float r) const {
        if (DT != DT_F32) return codes_of_16bit<DT == DT_F32 ? DT_BF16 : DT>(w, d, r);
        float v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(w[k % WORDS]);
        return codes_of(v, d, r);
    }
};
// silu(gate) * up of rows of h (gate | up), rounded to their type (cq_gated.cuh); what 32 bits leave open is formed in 64
template <int DT>
struct Gated {
    static constexpr int WORDS = 8;
    const uint16_t *h;
    int64_t ldh, I;
    __device__ __forceinline__ uint32_t get(int64_t row, int64_t unit, bool read, uint32_t *act) const {
        const uint16_t *pg = h + row * ldh + unit * 16, *pu = pg + I;
        uint32_t gw[8] = {}, uw[8] = {};
        if (read) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint4 a = load16(pg + 8 * k), b = load16(pu + 8 * k);
                gw[4 * k] = a.x; gw[4 * k + 1] = a.y; gw[4 * k + 2] = a.z; gw[4 * k + 3] = a.w;
                uw[4 * k] = b.x; uw[4 * k + 1] = b.y; uw[4 * k + 2] = b.z; uw[4 * k + 3] = b.w;
            }
        }
        uint32_t near = ~0u;
        float small = 1.0f;
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            float y0, y1;
            gated_in_32_bits(value_of<DT>(gw, k), value_of<DT>(gw, k + 1), value_of<DT>(uw, k), value_of<DT>(uw, k + 1), y0, y1);
            near = nearer<DT>(near, y0, y1);
            act[k / 2] = pack16<DT>(y0, y1);
            if (DT == DT_F16) small = fminf(small, fminf(y0 == 0.0f ? 1.0f : fabsf(y0), y1 == 0.0f ? 1.0f : fabsf(y1)));   // subnormal halves have their borders elsewhere
        }
        constexpr uint32_t BAND_BITS = 2 * BAND * (DT == DT_BF16 ? 1 : 8);
        const uint32_t largest = top_of_16bit<DT>(act);
        const bool far = top_of_16bit<DT>(gw) > 0x42700000u || largest >= 0x7F800000u;   // 60; infinities and NaN
        const bool open = read && ((near & 0xFFFFu) <= BAND_BITS || (near >> 16) <= BAND_BITS || far || (DT == DT_F16 && small < 6.103515625e-05f));
        if (!__any_sync(~0u, open)) return largest;
        settle_in_64_bits<DT>(open, gw, uw, act);
        return top_of_16bit<DT>(act);
    }
    __device__ __forceinline__ uint4 codes(const uint32_t *w, float d, float r) const { return codes_of_16bit<DT>(w, d, r); }
};

// ---------------------------------------------------------------- the quantisers
template <class From, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 3 : 1) quantize_kernel(const From from, Rows q, int64_t K, int KT, float *scale, uint8_t *layout) {
    extern __shared__ int s_tab[];
    __shared__ uint32_t red[2][THREADS / 32];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const int in = threadIdx.x & (q.team - 1), teams = blockDim.x / q.team, KU = (int)(K >> 4), units = KT * 8;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < q.rows; r0 += (int64_t)gridDim.x * teams, turn ^= 1) {
        const int64_t r = r0 + threadIdx.x / q.team;
        const Place p = place_of(q, r, s_off, s_blk);
        uint32_t w[HELD][From::WORDS], top = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int u = in + i * q.team;
            if (i == 0 || i * q.team < KU) top = max(top, from.get(p.src, u, p.read && u < KU, w[i]));   // whole warps
        }
        for (int u = in + HELD * q.team; u - in < KU; u += q.team) {
            uint32_t more[From::WORDS];
            top = max(top, from.get(p.src, u, p.read && u < KU, more));
        }
        const float d = row_scale(team_max(top, q.team, red[turn])), inverse = __fdiv_rn(1.0f, d);
        if (p.live && in == 0) scale[r] = d;
        uint8_t *line = layout + (p.at >> 7) * KT * (int64_t)TILE_BYTES;
        const int rr = (int)(p.at & (ROWS - 1));
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int u = in + i * q.team;
            if (u < units && p.live) {
                const uint4 c = u < KU ? from.codes(w[i], d, inverse) : make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(line + (int64_t)(u >> 3) * TILE_BYTES + piece_offset(rr, u & 7)) = c;
            }
        }
        for (int u = in + HELD * q.team; u - in < units; u += q.team) {   // of a long row: formed again
            uint32_t more[From::WORDS];
            from.get(p.src, u, p.read && u < KU, more);
            if (u < units && p.live) {
                const uint4 c = u < KU ? from.codes(more, d, inverse) : make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(line + (int64_t)(u >> 3) * TILE_BYTES + piece_offset(rr, u & 7)) = c;
            }
        }
    }
}

// ---------------------------------------------------------------- back to values
// code * scale, rounded once to the type asked for.  A thread takes eight values, so that a warp's stores are one run of memory.
template <int DT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *layout, Rows q, int64_t K, int KT, const float *scale, void *y) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const int in = threadIdx.x & (q.team - 1), teams = blockDim.x / q.team, units = (int)(K >> 3);
    for (int64_t r = (int64_t)blockIdx.x * teams + threadIdx.x / q.team; r < q.rows; r += (int64_t)gridDim.x * teams) {
        const Place p = place_of(q, r, s_off, s_blk);
        if (!p.live) continue;
        const float s = scale[r];
        const uint8_t *line = layout + (p.at >> 7) * KT * (int64_t)TILE_BYTES;
        const int rr = (int)(p.at & (ROWS - 1));
#pragma unroll 4
        for (int u = in; u < units; u += q.team) {
            const uint2 c = *reinterpret_cast<const uint2 *>(line + (int64_t)(u >> 4) * TILE_BYTES + piece_offset(rr, (u >> 1) & 7) + (u & 1) * 8);
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (float)(int8_t)((k < 4 ? c.x : c.y) >> (8 * (k & 3)) & 0xFFu) * s;
            const int64_t at = r * K + (int64_t)u * 8;
            if (DT == DT_F32) {
                float4 *o = reinterpret_cast<float4 *>(reinterpret_cast<float *>(y) + at);
                o[0] = make_float4(v[0], v[1], v[2], v[3]);
                o[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                constexpr int D = DT == DT_F32 ? DT_BF16 : DT;
                *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(y) + at) = make_uint4(pack16<D>(v[0], v[1]), pack16<D>(v[2], v[3]), pack16<D>(v[4], v[5]), pack16<D>(v[6], v[7]));
            }
        }
    }
}

// ---------------------------------------------------------------- checkpoints (once for each matrix of a model): codes [rows][K]
template <bool IN>
__global__ void __launch_bounds__(256) exchange_kernel(uint8_t *codes, Rows q, int64_t K, int KT, uint8_t *layout) {
    const int64_t units = (int64_t)KT * 8, total = q.rows * units;
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t row = idx / units, u = idx - row * units;
        const Place p = place_of(q, row, nullptr, nullptr);
        uint4 *at = reinterpret_cast<uint4 *>(layout + ((p.at >> 7) * KT + (u >> 3)) * (int64_t)TILE_BYTES + piece_offset((int)(p.at & (ROWS - 1)), (int)(u & 7)));
        uint4 *c = reinterpret_cast<uint4 *>(codes + row * K + u * 16);
        const bool inside = u * 16 < K;
        if (IN) *at = inside ? *c : make_uint4(0, 0, 0, 0);
        else if (inside) *c = *at;
    }
}

// ---------------------------------------------------------------- launchers
static Rows rows_of(const I8Rows &s, int team) { return Rows{s.route_token, s.offset, s.E, s.per, s.rows, s.T, team}; }
static int kt_of(int64_t K) { return (int)((K + KB - 1) / KB); }
static size_t table_bytes(const I8Rows &s) { return s.offset ? 2 * (size_t)(s.E + 1) * sizeof(int) : 0; }
// Threads to a row: one unit each where there are few rows and latency counts, else four.
static int team_of(int64_t rows, int units, int most) {
    const int want = rows <= 2 * sm_count() ? units : (units + HELD - 1) / HELD;
    int team = 32;
    while (team < want && team < most) team *= 2;
    return team;
}
static unsigned grid_of(int64_t rows, int teams, int per_sm) {
    const int64_t blocks = (rows + teams - 1) / teams, most = (int64_t)per_sm * sm_count();
    return (unsigned)(blocks < most ? blocks : most);
}
template <class From>
static cudaError_t quantize(const From &from, const I8Rows &s, int64_t K, float *scale, void *layout, cudaStream_t st) {
    const int KT = kt_of(K), team = team_of(s.rows, KT * 8, s.rows <= 2 * sm_count() ? 512 : 256), threads = team < 256 ? 256 : team;
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_of(s.rows, threads / team, 4)), (unsigned)threads, table_bytes(s), st, 1, true, from, rows_of(s, team), K, KT, scale, (uint8_t *)layout);
    };
    return threads == 256 ? go(quantize_kernel<From, 256>) : go(quantize_kernel<From, 512>);
}

}  // namespace i8

using namespace i8;

cudaError_t launch_i8_quantize(const void *x, int dtype, int64_t ldx, const I8Rows &s, int64_t K, float *scale, void *layout, cudaStream_t st) {
    if (dtype == DT_BF16) return quantize(Plain<DT_BF16>{x, ldx}, s, K, scale, layout, st);
    if (dtype == DT_F16) return quantize(Plain<DT_F16>{x, ldx}, s, K, scale, layout, st);
    return quantize(Plain<DT_F32>{x, ldx}, s, K, scale, layout, st);
}
cudaError_t launch_i8_swiglu_quantize(const void *h, int dtype, int64_t ldh, const I8Rows &s, int64_t I, float *scale, void *layout, cudaStream_t st) {
    if (dtype == DT_BF16) return quantize(Gated<DT_BF16>{(const uint16_t *)h, ldh, I}, s, I, scale, layout, st);
    return quantize(Gated<DT_F16>{(const uint16_t *)h, ldh, I}, s, I, scale, layout, st);
}
cudaError_t launch_i8_dequantize(const void *layout, const I8Rows &s, int64_t K, const float *scale, void *y, int dtype, cudaStream_t st) {
    const int KT = kt_of(K), team = team_of(s.rows, (int)(K >> 3), 256);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_of(s.rows, 256 / team, 8)), 256u, table_bytes(s), st, 1, true, (const uint8_t *)layout, rows_of(s, team), K, KT, scale, y);
    };
    return dtype == DT_BF16 ? go(dequantize_kernel<DT_BF16>) : dtype == DT_F16 ? go(dequantize_kernel<DT_F16>) : go(dequantize_kernel<DT_F32>);
}
cudaError_t launch_i8_exchange(uint8_t *codes, const I8Rows &s, int64_t K, void *layout, bool in, cudaStream_t st) {
    const int KT = kt_of(K);
    const unsigned grid = grid_of((s.rows * KT * 8 + 255) / 256, 1, 8);
    if (in) exchange_kernel<true><<<grid, 256, 0, st>>>(codes, rows_of(s, 32), K, KT, (uint8_t *)layout);
    else exchange_kernel<false><<<grid, 256, 0, st>>>(codes, rows_of(s, 32), K, KT, (uint8_t *)layout);
    return cudaGetLastError();
}

}  // namespace cq
