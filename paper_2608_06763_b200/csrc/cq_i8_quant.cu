// Quantisers to 8-bit integers with a scale for each row (layout: cq_i8.cuh), their inverse, and the exchange with the form that checkpoints
// store.
#include "cq_gated.cuh"
#include "cq_i8.cuh"
#include "cq_internal.h"
#include "cq_tc_ptx.cuh"
#include "cq_tiles.cuh"

namespace cq {
namespace i8 {

// A row belongs to a team of threads, 32 to 512 of them, which take units of sixteen neighbouring k in turn; a block has one team or several.
// What a thread has read (formed) stays in shared memory until the row's scale is known; of a row beyond that room the rest is formed again.
constexpr int ROOM = 40 << 10;   // bytes of shared memory for that
constexpr int MOST_SPREAD = 8;
struct Rows {
    const int32_t *route_token;   // routed: the row of x that row r takes (null: r itself)
    const int32_t *offset;        // routed: first rows of the groups, on the device (null: rows are dense)
    int E;                        // groups, or matrices of `per` rows each
    int64_t per, rows, T;         // rows of one matrix; all rows; rows that x has
    int team, held;               // threads to a row; units of a row that are kept, a multiple of `team`
    const int32_t *route_row;     // SCATTER: rows are tokens, [rows][top] the routes of each (-1: none); `routes` of all
    int top, routes;
    int lg_spread, part;          // SPREAD: blocks to a row (log2), units of each
};
struct Place { int64_t src, at; bool live, read; };   // row of x; row among the padded rows of the layout; whether it is one; whether x has it
__device__ __forceinline__ void scan_if_routed(const Rows &q, int *s_off, int *s_blk) {
    if (!q.offset) return;
    if (threadIdx.x < 32) scan_groups(q.offset, q.E, q.route_row ? q.routes : (int)q.rows, s_off, s_blk);
    __syncthreads();
}
// the row of x that row r takes; known before the groups are
__device__ __forceinline__ int64_t source_of(const Rows &q, int64_t r) { return q.route_token && r < q.rows ? q.route_token[r] : r; }
__device__ __forceinline__ Place place_of(const Rows &q, int64_t r, int64_t source, const int *s_off, const int *s_blk) {
    Place p{source, r, r < q.rows, r < q.rows};
    if (q.offset) {
        p.live = p.live && r >= s_off[0] && r < s_off[q.E];
        p.read = p.live;
        if (p.live) {
            const int e = find_group(s_off, q.E, (int)r);
            p.at = (int64_t)s_blk[e] * ROWS + (r - s_off[e]);
            if (q.route_token) p.read = source >= 0 && source < q.T;   // any other token is a row of zeros
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
    const int mine = threadIdx.x / team, lane = threadIdx.x & 31;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "r"(team) : "memory");
    return __reduce_max_sync(~0u, lane < team / 32 ? red[mine * (team / 32) + lane] : 0u);
}
// ---------------------------------------------------------------- where sixteen values of a row come from
// Units of a row in shared memory: 16-byte pieces of one unit `step` apart, so that a warp's accesses have no conflicts.
struct Store {
    uint4 *at;
    int step;
    __device__ __forceinline__ uint4 &piece(int slot, int k) const { return at[k * step + slot]; }
};
// rows of x as they are
template <int DT>
struct Plain {
    static constexpr int PIECES = DT == DT_F32 ? 4 : 2, AHEAD = DT == DT_F32 ? 2 : 4;   // units whose loads are on their way together
    const void *x;
    int64_t ldx;
    static constexpr int UNIT = 16 * PIECES;   // bytes of a unit
    struct Raw { uint4 q[PIECES]; };
    __device__ __forceinline__ const uint8_t *unit(int64_t row, int u) const { return reinterpret_cast<const uint8_t *>(x) + row * ldx * (DT == DT_F32 ? 4 : 2) + (int64_t)u * UNIT; }
    __device__ __forceinline__ Raw load(const uint8_t *p, bool read) const {
        Raw r;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) r.q[k] = read ? load16(p + 16 * k) : make_uint4(0, 0, 0, 0);
        return r;
    }
    // to a slot of the store; the largest magnitude.  The whole warp.
    __device__ __forceinline__ void keep(const Raw &r, const uint8_t *, bool, const Store &s, int slot, uint32_t &largest) const {
        uint32_t w[4 * PIECES], top = 0;
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            s.piece(slot, k) = r.q[k];
            w[4 * k] = r.q[k].x; w[4 * k + 1] = r.q[k].y; w[4 * k + 2] = r.q[k].z; w[4 * k + 3] = r.q[k].w;
        }
        if constexpr (DT != DT_F32) {
            top = top_of_16bit<DT>(w);
        } else {
#pragma unroll
            for (int k = 0; k < 4 * PIECES; ++k) top = max(top, w[k] & 0x7FFFFFFFu);
        }
        largest = max(largest, top);
    }
    __device__ __forceinline__ uint4 codes(const Store &s, int slot, float d, float r) const {
        uint32_t w[4 * PIECES];
#pragma unroll
        for (int k = 0; k < PIECES; ++k) {
            const uint4 q = s.piece(slot, k);
            w[4 * k] = q.x; w[4 * k + 1] = q.y; w[4 * k + 2] = q.z; w[4 * k + 3] = q.w;
        }
        if constexpr (DT != DT_F32) {
            return codes_of_16bit<DT>(w, d, r);
        } else {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = __uint_as_float(w[k]);
            return codes_of(v, d, r);
        }
    }
};
__device__ __forceinline__ float largest_of(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// silu(gate) * up of rows of h (gate | up), rounded to their type (cq_gated.cuh).  Values whose rounding 32 bits leave open are formed in 64, each
// lane one of its own at a time: in binary16 three warps of four have one in every step, but few lanes: 4096 x 14336 take 109 us, in bfloat16 72.  (Kept with a bit that says
// so, and formed only where the row's largest or a code hangs on them: one in fifty does, but telling them costs more than forming them, 126 us.  Noted by a warp, and up to 32
// of a row formed together: 117.)
template <int DT>
struct Gated {
    static constexpr int AHEAD = 1, PIECES = 2, UNIT = 32;
    const uint16_t *h;
    int64_t ldh, I;
    struct Raw { uint4 g[2], u[2]; };
    __device__ __forceinline__ const uint8_t *unit(int64_t row, int u) const { return reinterpret_cast<const uint8_t *>(h + row * ldh) + (int64_t)u * UNIT; }
    __device__ __forceinline__ Raw load(const uint8_t *p, bool read) const {
        const uint8_t *pu = p + I * 2;
        Raw r;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            r.g[k] = read ? load16(p + 16 * k) : make_uint4(0, 0, 0, 0);
            r.u[k] = read ? load16(pu + 16 * k) : make_uint4(0, 0, 0, 0);
        }
        return r;
    }
    // value k of a unit in 64 bits
    __device__ __forceinline__ void settle(const uint8_t *p, int k, const Store &s, int slot) const {
        const uint16_t *pg = reinterpret_cast<const uint16_t *>(p) + k;
        const uint32_t g = pg[0], u = pg[I];
        const float y = gated_in_64_bits(value_of<DT>(&g, 0), value_of<DT>(&u, 0));
        reinterpret_cast<uint16_t *>(&s.piece(slot, k >> 3))[k & 7] = (uint16_t)pack16<DT>(y, 0.0f);
    }
    __device__ __forceinline__ uint32_t top_of(const Store &s, int slot) const {
        const uint4 a = s.piece(slot, 0), b = s.piece(slot, 1);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        return top_of_16bit<DT>(w);
    }
    __device__ __forceinline__ void keep(const Raw &r, const uint8_t *p, bool read, const Store &s, int slot, uint32_t &largest) const {
        const uint32_t gw[8] = {r.g[0].x, r.g[0].y, r.g[0].z, r.g[0].w, r.g[1].x, r.g[1].y, r.g[1].z, r.g[1].w};
        const uint32_t uw[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[1].x, r.u[1].y, r.u[1].z, r.u[1].w};
        uint32_t act[8], low[8], near = ~0u, least = ~0u;
        float gate = 0.0f, most = 0.0f;   // the largest magnitudes; NaN counts as the largest
        constexpr uint32_t LEAST = 0x0400u, ENDLESS = DT == DT_BF16 ? 0x7F80u : 0x7C00u, FAR = DT == DT_BF16 ? 0x4270u : 0x5380u;   // the least normal half, infinity, 60
#pragma unroll
        for (int k = 0; k < 16; k += 2) {
            const float g0 = value_of<DT>(gw, k), g1 = value_of<DT>(gw, k + 1);
            float y0, y1;
            gated_in_32_bits(g0, g1, value_of<DT>(uw, k), value_of<DT>(uw, k + 1), y0, y1);
            gate = largest_of(gate, g0, g1);
            most = largest_of(most, y0, y1);
            low[k / 2] = dropped<DT>(y0, y1);
            near = nearer<DT>(near, low[k / 2]);
            act[k / 2] = pack16<DT>(y0, y1);
            if (DT == DT_F16) least = __viaddmin_u32(__float_as_uint(y0) & 0x7FFFFFFFu, ~0u, __viaddmin_u32(__float_as_uint(y1) & 0x7FFFFFFFu, ~0u, least));   // less one: 0 is exact, and becomes the largest
        }
        constexpr uint32_t WIDE = 2 * BAND * (DT == DT_BF16 ? 1 : 8);
        const uint32_t rounded = pack16<DT>(most, 0.0f);
        uint32_t top = __float_as_uint(value_of<DT>(&rounded, 0)) & 0x7FFFFFFFu;
        // far gates, what is not finite, and subnormal halves, which have their borders elsewhere
        const bool odd = read && (!(gate <= 60.0f) || top >= 0x7F800000u || (DT == DT_F16 && least < 0x38800000u - 1));   // 2^-14
        const bool open = read && ((near & 0xFFFFu) <= WIDE || (near >> 16) <= WIDE);
        s.piece(slot, 0) = make_uint4(act[0], act[1], act[2], act[3]);
        s.piece(slot, 1) = make_uint4(act[4], act[5], act[6], act[7]);
        if (open || odd) {
            uint32_t mask = 0;   // value 2 k at bit k, value 2 k + 1 at bit 16 + k
#pragma unroll
            for (int k = 0; k < 8; ++k) {   // the top bit of a half is set where its distance is at most WIDE
                const uint32_t far = __viaddmin_u16x2(low[k], ABOVE<DT> << 16 | ABOVE<DT>, (WIDE + 1) << 16 | (WIDE + 1));
                mask |= (((0x7FFFu + WIDE + 1) << 16 | (0x7FFFu + WIDE + 1)) - far & 0x80008000u) >> (15 - k);
            }
            if (odd) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const uint32_t a = (k & 1 ? act[k / 2] >> 16 : act[k / 2]) & 0x7FFFu, g = (k & 1 ? gw[k / 2] >> 16 : gw[k / 2]) & 0x7FFFu;
                    if (g > FAR || a >= ENDLESS || (DT == DT_F16 && a < LEAST)) mask |= 1u << (k / 2 + 16 * (k & 1));
                }
            }
            for (; mask; mask &= mask - 1) {
                const int b = __ffs(mask) - 1;
                settle(p, 2 * (b & 15) + (b >> 4), s, slot);
            }
            top = top_of(s, slot);
        }
        largest = max(largest, top);
    }
    __device__ __forceinline__ uint4 codes(const Store &s, int slot, float d, float r) const {
        const uint4 a = s.piece(slot, 0), b = s.piece(slot, 1);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        return codes_of_16bit<DT>(w, d, r);
    }
};

// ---------------------------------------------------------------- the quantisers
// Two passes over a row, of which the second reads shared memory: the row's largest magnitude gives its scale, the scale its codes.  Bound by issue slots: 4096 x 8192 rows of
// bfloat16 in 27 us (300 warp instructions for 32 units, a third of them for codes next to a border, which ties among bfloat16 values make common), gated 4096 x 14336 in 74 (510;
// 71 % of the slots taken), in binary16 in 109 (700); the bytes would take 16 and 46.  Two blocks of 512 threads or more smaller ones fit an SM: 64 registers hold a unit of both operands.
// SCATTER: a token's codes go to all of its routes, formed once.
struct Copy { uint8_t *line; int row; };   // the row block of a route, the row in it
// SPREAD: few long rows, each by a cluster of blocks, which tell one another the largest value of their parts.
template <class From, bool SCATTER, bool SPREAD>
__global__ void __launch_bounds__(512, 2) quantize_kernel(const From from, Rows q, int64_t K, int KT, float *scale, uint8_t *layout) {
    extern __shared__ uint4 s_store[];
    __shared__ uint32_t red[2][16], s_parts[MOST_SPREAD];
    if (SPREAD) cluster_arrive();
    tc::wait_for_previous_kernel();
    const int in = threadIdx.x & (q.team - 1), teams = blockDim.x / q.team, mine = threadIdx.x / q.team;
    const int lg = SPREAD ? q.lg_spread : 0, rank = blockIdx.x & ((1 << lg) - 1), base = SPREAD ? rank * q.part : 0;   // this block's first unit
    const int KU = SPREAD ? min((int)(K >> 4) - base, q.part) : (int)(K >> 4), units = SPREAD ? min(KT * 8 - base, q.part) : KT * 8;
    const int slots = q.held < KU ? q.held + q.team : q.held;   // a row that is longer has a slot for each thread besides
    const Store s{s_store + mine * From::PIECES * slots, slots};
    Copy *s_copy = reinterpret_cast<Copy *>(s_store + teams * From::PIECES * slots);   // SCATTER: [teams][two rows in turn][top]
    int *s_off = reinterpret_cast<int *>(s_copy + (SCATTER ? 2 * teams * q.top : 0)), *s_blk = s_off + q.E + 1;
    const int64_t stride = (int64_t)(gridDim.x >> lg) * teams;
    int64_t r = (int64_t)(blockIdx.x >> lg) * teams + mine, next = source_of(q, r);
    scan_if_routed(q, s_off, s_blk);
    int turn = 0;
    for (; r - mine < q.rows; r += stride, turn ^= 1) {
        const Place p = SCATTER ? Place{r, 0, r < q.rows, r < q.rows} : place_of(q, r, next, s_off, s_blk);
        Copy *copies = s_copy + (2 * mine + turn) * q.top;   // read until the next row's barrier, written again behind it
        if (SCATTER) {
            for (int j = in; j < q.top; j += q.team) {
                const int route = p.live ? q.route_row[r * q.top + j] : -1;
                const bool there = route >= s_off[0] && route < s_off[q.E];
                const int e = there ? find_group(s_off, q.E, route) : 0, at = there ? s_blk[e] * ROWS + (route - s_off[e]) : 0;
                copies[j] = Copy{there ? layout + (int64_t)(at >> 7) * KT * TILE_BYTES : nullptr, at & (ROWS - 1)};
            }
            __syncwarp();
        } else {
            next = source_of(q, r + stride);
        }
        uint32_t top = 0;
        const uint8_t *first = from.unit(p.src, base + in), *src = first;
        const int64_t step = (int64_t)q.team * From::UNIT;
        for (int u0 = in; u0 - in < KU; u0 += From::AHEAD * q.team, src += From::AHEAD * step) {   // whole warps
            typename From::Raw raw[From::AHEAD];
#pragma unroll
            for (int i = 0; i < From::AHEAD; ++i) raw[i] = from.load(src + i * step, p.read && u0 + i * q.team < KU);
#pragma unroll
            for (int i = 0; i < From::AHEAD; ++i) {
                const int u = u0 + i * q.team;
                if (u - in >= KU) break;
                from.keep(raw[i], src + i * step, p.read && u < KU, s, u < q.held ? u : q.held + in, top);
            }
        }
        top = team_max(top, q.team, red[turn]);
        if (SPREAD) {   // a row to a block: once
            cluster_wait();   // the others have started
            if (in < 1 << lg) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(tc::map_to_rank(&s_parts[rank], in)), "r"(top) : "memory");
            __syncwarp();
            cluster_arrive();
            cluster_wait();
            for (int j = 0; j < 1 << lg; ++j) top = max(top, s_parts[j]);
        }
        const float d = row_scale(top), inverse = __frcp_rn(d);
        if (SCATTER) {
            for (int j = in; j < q.top; j += q.team)
                if (copies[j].line) scale[q.route_row[r * q.top + j]] = d;
        } else if (p.live && base + in == 0) {
            scale[r] = d;
        }
        // a unit's place in its tile is that of the thread, 8 units a tile
        uint8_t *dst = layout + ((p.at >> 7) * KT + ((base + in) >> 3)) * (int64_t)TILE_BYTES + piece_offset((int)(p.at & (ROWS - 1)), in & 7);
        const int64_t dst_step = (int64_t)(q.team >> 3) * TILE_BYTES;
        src = first;
#pragma unroll 1
        for (int u = in; u - in < units; u += q.team, src += step, dst += dst_step) {
            const int slot = u < q.held ? u : q.held + in;
            if (u >= q.held && u - in < KU) from.keep(from.load(src, p.read && u < KU), src, p.read && u < KU, s, slot, top);   // formed again
            if (u < units && p.live) {
                const uint4 c = u < KU ? from.codes(s, slot, d, inverse) : make_uint4(0, 0, 0, 0);
                if (SCATTER) {
                    for (int j = 0; j < q.top; ++j) {
                        const Copy to = copies[j];
                        if (to.line) *reinterpret_cast<uint4 *>(to.line + (int64_t)(u >> 3) * TILE_BYTES + piece_offset(to.row, in & 7)) = c;
                    }
                } else {
                    *reinterpret_cast<uint4 *>(dst) = c;
                }
            }
        }
    }
}

// ---------------------------------------------------------------- back to values
// code * scale in fp32, and from there to the type asked for (in 16 bits a second rounding).  A thread reads sixteen codes; in 16 bits neighbouring threads exchange halves, so that each
// of a warp's two stores fills whole sectors.  Bound by memory and its own instructions alike: 4096 x 14336 in 30 us, 5.8 TB/s with the codes still in L2 (without the exchange 38).
template <int DT>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t *layout, Rows q, int64_t K, int KT, const float *scale, void *y) {
    extern __shared__ int s_tab[];
    tc::wait_for_previous_kernel();
    int *s_off = s_tab, *s_blk = s_tab + q.E + 1;
    scan_if_routed(q, s_off, s_blk);
    const int in = threadIdx.x & (q.team - 1), teams = blockDim.x / q.team, units = (int)(K >> 4), odd = threadIdx.x & 1;
    for (int64_t r = (int64_t)blockIdx.x * teams + threadIdx.x / q.team; r < q.rows; r += (int64_t)gridDim.x * teams) {
        const Place p = place_of(q, r, r, s_off, s_blk);
        if (!p.live) continue;
        const float s = scale[r];
        const uint8_t *line = layout + (p.at >> 7) * KT * (int64_t)TILE_BYTES;
        const int rr = (int)(p.at & (ROWS - 1));
#pragma unroll 4
        for (int u = in; u - in < units; u += q.team) {   // whole warps
            uint4 c = make_uint4(0, 0, 0, 0);
            if (u < units) c = load16(line + (int64_t)(u >> 3) * TILE_BYTES + piece_offset(rr, u & 7));
            uint32_t w[4] = {c.x, c.y, c.z, c.w};
            if (DT != DT_F32) {   // the even thread has the first halves of both units then, the odd one the second halves
                const uint32_t x = __shfl_xor_sync(~0u, odd ? c.x : c.z, 1), y = __shfl_xor_sync(~0u, odd ? c.y : c.w, 1);
                w[0] = odd ? x : c.x; w[1] = odd ? y : c.y;
                w[2] = odd ? c.z : x; w[3] = odd ? c.w : y;
            }
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = (float)(int8_t)(w[k >> 2] >> (8 * (k & 3)) & 0xFFu) * s;
            if (DT == DT_F32) {
                float4 *o = reinterpret_cast<float4 *>(reinterpret_cast<float *>(y) + r * K + (int64_t)u * 16);
                if (u < units) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
                }
            } else {
                constexpr int D = DT == DT_F32 ? DT_BF16 : DT;
                const int even = u & ~1;
                uint4 *o = reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(y) + r * K + (int64_t)even * 16) + odd;
                if (even < units) o[0] = make_uint4(pack16<D>(v[0], v[1]), pack16<D>(v[2], v[3]), pack16<D>(v[4], v[5]), pack16<D>(v[6], v[7]));
                if (even + 1 < units) o[2] = make_uint4(pack16<D>(v[8], v[9]), pack16<D>(v[10], v[11]), pack16<D>(v[12], v[13]), pack16<D>(v[14], v[15]));
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
        const Place p = place_of(q, row, row, nullptr, nullptr);
        uint4 *at = reinterpret_cast<uint4 *>(layout + ((p.at >> 7) * KT + (u >> 3)) * (int64_t)TILE_BYTES + piece_offset((int)(p.at & (ROWS - 1)), (int)(u & 7)));
        uint4 *c = reinterpret_cast<uint4 *>(codes + row * K + u * 16);
        const bool inside = u * 16 < K;
        if (IN) *at = inside ? *c : make_uint4(0, 0, 0, 0);
        else if (inside) *c = *at;
    }
}

// ---------------------------------------------------------------- launchers
static Rows rows_of(const I8Rows &s, int team, int held) { return Rows{s.route_token, s.offset, s.E, s.per, s.rows, s.T, team, held, s.route_row, s.top, (int)s.routes}; }
static int kt_of(int64_t K) { return (int)((K + KB - 1) / KB); }
static size_t table_bytes(const I8Rows &s) { return s.offset ? 2 * (size_t)(s.E + 1) * sizeof(int) : 0; }
// Threads to a row: a unit each while all fit the GPU at once and latency counts, then two, then four.  us with 64 / 128 / 256 threads: 400 x 4096 7.0 / 4.6 /
// 4.2, 1024 x 4096 8.4 / 6.7 / 6.9, 2048 x 4096 11.3 / 10.3 / 11.6, 4096 x 8192 34.5 / 29.1 / 32.8; with 32 / 64 / 128: 4096 x 2048 11.0 / 10.1 / 11.5, 8192 x 1408
// 12.9 / 15.2 / 19.4 (a GPU on the slow side).
static int team_of(int64_t rows, int units, int most) {
    const int64_t all = rows * units;
    const int each = all <= 200000 ? 1 : all <= 600000 ? 2 : 4, want = (units + each - 1) / each;
    int team = 32;
    while (team < want && team < most) team *= 2;
    return team;
}
// per_sm: blocks of an SM at most, which take rows in turn (routed rows, whose tables each block fills first); 0: as many as there are rows for
static unsigned grid_of(int64_t rows, int teams, int per_sm) {
    const int64_t blocks = (rows + teams - 1) / teams, most = per_sm ? (int64_t)per_sm * sm_count() : blocks;
    return (unsigned)(blocks < most ? blocks : most);
}
// Blocks to a row (log2).  A long row takes as long as its SM takes to issue it, a cluster half a microsecond: us with 1 / 2 / 4 / 8, gated (as they are) 1 x 4096 2.7 / 3.1 / 3.1 / 3.0,
// 1 x 8192 3.3 / 3.4 / 3.1 / 3.0, 13 x 14336 4.9 / 4.8 / 3.8 / 3.6 (4.0 / 4.0 / 3.2 / 3.0), 64 x 14336 5.3 / 4.7 / 4.6 / 4.6, 64 x 28672 12.8 / 7.7 / 6.4 / 6.3 (8.8 / 6.1 / 5.5 / 5.2), 148 x 14336 6.7 /
// 6.4 / 8.3 / 8.3.
static int lg_spread_of(int64_t rows, int units) {
    int lg = 0;
    while (units >= 512 && 2 << lg <= MOST_SPREAD && rows << (lg + 1) <= 2 * sm_count() && units >> (lg + 1) >= 112) ++lg;
    return lg;
}
template <bool SCATTER = false, class From>
static cudaError_t quantize(const From &from, const I8Rows &s, int64_t K, float *scale, void *layout, cudaStream_t st) {
    const int KT = kt_of(K), lg = SCATTER ? 0 : lg_spread_of(s.rows, (int)(K >> 4)), part = ((KT + (1 << lg) - 1) >> lg) * 8;   // whole tiles
    const int KU = lg ? part : (int)(K >> 4), team = team_of(s.rows, KU, s.rows <= 2 * sm_count() ? 512 : 256), threads = lg || team >= 256 ? team : 256, teams = threads / team;
    const int all = (KU + team - 1) / team * team, room = ROOM / (teams * From::PIECES * 16) / team * team;
    const int held = all <= room ? all : room - team;
    const size_t smem = (size_t)teams * From::PIECES * 16 * (held < all ? held + team : held) + (SCATTER ? 2 * (size_t)teams * s.top * sizeof(Copy) : 0) + table_bytes(s);
    Rows q = rows_of(s, team, held);
    q.lg_spread = lg; q.part = part;
    const unsigned grid = lg ? (unsigned)s.rows << lg : grid_of(s.rows, teams, s.offset ? 1024 / threads : 0);
    auto go = [&](auto kern) { return launch_overlapped(kern, dim3(grid), (unsigned)threads, smem, st, 1 << lg, true, from, q, K, KT, scale, (uint8_t *)layout); };
    if constexpr (SCATTER) return go(quantize_kernel<From, true, false>);
    else return lg ? go(quantize_kernel<From, false, true>) : go(quantize_kernel<From, false, false>);
}

}  // namespace i8

using namespace i8;

cudaError_t launch_i8_quantize(const void *x, int dtype, int64_t ldx, const I8Rows &s, int64_t K, float *scale, void *layout, cudaStream_t st) {
    if (s.route_row) return dtype == DT_BF16 ? quantize<true>(Plain<DT_BF16>{x, ldx}, s, K, scale, layout, st) : quantize<true>(Plain<DT_F16>{x, ldx}, s, K, scale, layout, st);
    if (dtype == DT_BF16) return quantize(Plain<DT_BF16>{x, ldx}, s, K, scale, layout, st);
    if (dtype == DT_F16) return quantize(Plain<DT_F16>{x, ldx}, s, K, scale, layout, st);
    return quantize(Plain<DT_F32>{x, ldx}, s, K, scale, layout, st);
}
cudaError_t launch_i8_swiglu_quantize(const void *h, int dtype, int64_t ldh, const I8Rows &s, int64_t I, float *scale, void *layout, cudaStream_t st) {
    if (dtype == DT_BF16) return quantize(Gated<DT_BF16>{(const uint16_t *)h, ldh, I}, s, I, scale, layout, st);
    return quantize(Gated<DT_F16>{(const uint16_t *)h, ldh, I}, s, I, scale, layout, st);
}
cudaError_t launch_i8_dequantize(const void *layout, const I8Rows &s, int64_t K, const float *scale, void *y, int dtype, cudaStream_t st) {
    const int KT = kt_of(K), team = team_of(s.rows, (int)(K >> 4), 256);
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3(grid_of(s.rows, 256 / team, s.offset ? 8 : 0)), 256u, table_bytes(s), st, 1, true, (const uint8_t *)layout, rows_of(s, team, 0), K, KT, scale, y);
    };
    return dtype == DT_BF16 ? go(dequantize_kernel<DT_BF16>) : dtype == DT_F16 ? go(dequantize_kernel<DT_F16>) : go(dequantize_kernel<DT_F32>);
}
cudaError_t launch_i8_exchange(uint8_t *codes, const I8Rows &s, int64_t K, void *layout, bool in, cudaStream_t st) {
    const int KT = kt_of(K);
    const unsigned grid = grid_of((s.rows * KT * 8 + 255) / 256, 1, 8);
    if (in) exchange_kernel<true><<<grid, 256, 0, st>>>(codes, rows_of(s, 32, 0), K, KT, (uint8_t *)layout);
    else exchange_kernel<false><<<grid, 256, 0, st>>>(codes, rows_of(s, 32, 0), K, KT, (uint8_t *)layout);
    return cudaGetLastError();
}

}  // namespace cq
