// The gated activation silu(gate) * up: its exact value rounded to fp32, and that to the model dtype.
#pragma once
#include "cq_rows.cuh"

namespace cq {
namespace rows {

// act = gate up / (1 + exp(-gate)).  (Of bfloat16 activations some ten in a million, of binary16 ones eight times as many, become halfway values by the first rounding, and the second
// takes the even neighbour, wherever the exact value lay.)  32 bits leave its rounding open where it lies next to a border of the model dtype.  In units of 2^-24 of
// the value: gate * up is exact; exp(-g) = 2^h (1 + l ln 2), h + l = -g log2(e) with the constant in two parts, ex2.approx 4 and the two products 2;
// the sum 1, the reciprocal 2, the last product 1: ten.  Where no value lies within BAND = 12 units of the last place (each at least such a unit)
// of a border, the roundings stand; in a unit of sixteen one does in 170 in bfloat16, in 22 in binary16.  Gates beyond 60
// either way are open in any case (exp(60) leaves room in 32 bits for the denominator and its reciprocal), and so is a unit with an
// activation that is not finite: gate * up is exact within the range of fp32 alone, and leaves it where silu(gate) * up need not.
constexpr int BAND = 12;
__device__ __forceinline__ float gated_in_64_bits(float g, float u) { return (float)((double)g * (double)u / (1.0 + exp(-(double)g))); }
// The units of the lanes that ask for it, one after another: a lane for each of the sixteen activations (a lane by itself would take
// sixteen times as long, and the rest of its warp would wait).
template <int DT>
__device__ __forceinline__ void settle_in_64_bits(bool ask, const uint32_t *gw, const uint32_t *uw, uint32_t *act) {
    const int lane = threadIdx.x & 31, mine = (lane & 15) >> 1;
    for (uint32_t left = __ballot_sync(~0u, ask); left; left &= left - 1) {
        const int from = __ffs(left) - 1;
        uint32_t g = 0, u = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __shfl_sync(~0u, gw[i], from), b = __shfl_sync(~0u, uw[i], from);
            if (mine == i) { g = a; u = b; }
        }
        if (lane & 1) { g >>= 16; u >>= 16; }
        const float y = gated_in_64_bits(value_of<DT>(&g, 0), value_of<DT>(&u, 0));
        const uint32_t both = pack16<DT>(y, __shfl_down_sync(~0u, y, 1));   // in the even lanes
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t t = __shfl_sync(~0u, both, 2 * i);
            if (lane == from) act[i] = t;
        }
    }
}
__device__ __forceinline__ float ulps_away(float v, int n) { return __uint_as_float(__float_as_uint(v) + n); }   // n > 0: away from zero
// two activations
__device__ __forceinline__ void gated_in_32_bits(float g0, float g1, float u0, float u1, float &y0, float &y1) {
    const Pair g = pair_of(g0, g1), major = pair_of(1.44269502f, 1.44269502f), minor = pair_of(-1.92596303e-8f, -1.92596303e-8f);   // log2(e) = major - minor
    const Pair h = mul2(g, major);   // -h: its sign is taken off where it is used
    float h0, h1, d0, d1;
    unpair(h, h0, h1);
    const Pair l = fma2(g, minor, fma2(g, pair_of(-1.44269502f, -1.44269502f), h));
    float e0, e1;
    asm("{\n\t.reg .f32 h;\n\tneg.f32 h, %1;\n\tex2.approx.ftz.f32 %0, h;\n\t}" : "=f"(e0) : "f"(h0));
    asm("{\n\t.reg .f32 h;\n\tneg.f32 h, %1;\n\tex2.approx.ftz.f32 %0, h;\n\t}" : "=f"(e1) : "f"(h1));
    const Pair e = pair_of(e0, e1);
    unpair(add2(fma2(e, mul2(l, pair_of(0.693147181f, 0.693147181f)), e), pair_of(1.0f, 1.0f)), d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(d0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(d1));
    unpair(mul2(mul2(g, pair_of(u0, u1)), pair_of(e0, e1)), y0, y1);
}
// The bits that rounding two values to the model dtype drops (binary16: in their eighths), and how they become a distance: bits + ABOVE is
// bits - border + BAND, at most 2 BAND (in such units) next to a border; borders lie in the middle of these bits.
template <int DT> constexpr uint32_t ABOVE = (0x8000u + BAND * (DT == DT_BF16 ? 1u : 8u)) & 0xFFFFu;
template <int DT>
__device__ __forceinline__ uint32_t dropped(float y0, float y1) {
    const uint32_t low = __byte_perm(__float_as_uint(y0), __float_as_uint(y1), 0x5410);
    return DT == DT_BF16 ? low : (low & 0x1FFF1FFFu) * 8u;
}
// the least distance of what was dropped of two values and of those before
template <int DT>
__device__ __forceinline__ uint32_t nearer(uint32_t near, uint32_t bits) { return __viaddmin_u16x2(bits, ABOVE<DT> << 16 | ABOVE<DT>, near); }
template <int DT>
__device__ __forceinline__ uint32_t nearer(uint32_t near, float y0, float y1) { return nearer<DT>(near, dropped<DT>(y0, y1)); }

}  // namespace rows
}  // namespace cq
