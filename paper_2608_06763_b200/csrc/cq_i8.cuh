// 8-bit integers with a scale for each row: the device layout, the rounding of values to codes.
//
// A value is an int8 code times the fp32 scale of its row (weights: a channel; activations: a token).
//
// Device layout: rows are padded to 128 and k to 128; tile (row block rb, k block kt) of 128 rows x 128 k, 16384 bytes, is stored at
// (rb * KT + kt) * 16384: 128 bytes a row, the 16-byte pieces of row r exchanged by piece ^= r & 7, the 128-byte swizzle of a K-major
// MMA operand, so that one bulk copy brings what the tensor core reads.  Several matrices of one shape (the experts of a layer)
// follow one another.  Activations of routed rows keep each group in row blocks of its own.  Codes behind K are zeros; rows behind the last
// are never written, and what they hold reaches no result.  Scales lie beside the layout, one for each row that there is.
#pragma once
#include "cq_rows.cuh"

namespace cq {
namespace i8 {

using namespace rows;

constexpr int KB = 128;                     // k of a tile
constexpr int TILE_BYTES = ROWS * KB;
constexpr int64_t MOST_K = 1 << 17;         // sums of so many products of codes have 32 bits to themselves: from -2^17 * 128 * 127 > -2^31 to 2^17 * 128 * 128 = 2^31

// byte of a tile that holds piece u (sixteen k) of row r
__host__ __device__ inline int piece_offset(int r, int u) { return r * 128 + ((u ^ (r & 7)) << 4); }

// The scale of a row, from the bits of its largest |x|: d = max(top, 1e-10) / 127; NaN for a row that holds an infinity or a NaN.
__device__ __forceinline__ float row_scale(uint32_t top) {
    return top >= 0x7F800000u ? __uint_as_float(0x7FFFFFFFu) : __fdiv_rn(fmaxf(__uint_as_float(top), 1e-10f), 127.0f);
}
// Codes: x / d (a quotient rounded to fp32) to the nearest integer, halves away from zero; a row without a finite scale: zeros.
// The product with r = 1 / d is off by less than 127 * 3 * 2^-24 of the quotient, so where no product lies within BORDER of a half, its nearest
// integer is that of the quotient.  Adding 1.5 * 2^23 rounds to an integer and leaves it in the low bits.  Elsewhere (a unit in 800) the quotient is
// compared with the half h that it lies next to: rounded to fp32 it reaches h if |x| / d >= h - e, e half the distance of h from the fp32 number
// below (a tie goes to h, the even one of the two).  |x| - h d is exact in fp32 (a multiple of half a unit of d, less than 2^18 of them) and so is d e.
constexpr float BORDER = 4e-5f;
static_assert(127.0f * 3.0f / 16777216.0f < BORDER, "the product's error");
// the code of one value v >= 0
__device__ __forceinline__ int code_of(float v, float d, float r) {
    const float q = v * r, n = rintf(q), off = q - n;
    if (fabsf(off) <= 0.5f - BORDER) return (int)n;
    const float h = n + copysignf(0.5f, off), e = 0.5f * (h - __uint_as_float(__float_as_uint(h) - 1u));
    return (int)h + (fmaf(-h, d, v) >= -(d * e));
}
// sixteen codes
__device__ __forceinline__ uint4 codes_of(const float *v, float d, float r) {
    constexpr float MAGIC = 12582912.0f;
    const Pair rr = pair_of(r, r), up = pair_of(MAGIC, MAGIC), down = pair_of(-MAGIC, -MAGIC), minus = pair_of(-1.0f, -1.0f);
    uint32_t b[16];
    float far = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; k += 2) {
        const Pair q = mul2(pair_of(v[k], v[k + 1]), rr), s = add2(q, up), off = fma2(add2(s, down), minus, q);
        float s0, s1, o0, o1;
        unpair(s, s0, s1);
        unpair(off, o0, o1);
        b[k] = __float_as_uint(s0);
        b[k + 1] = __float_as_uint(s1);
        far = fmaxf(far, fmaxf(fabsf(o0), fabsf(o1)));
    }
    if (far > 0.5f - BORDER) {
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int m = code_of(fabsf(v[k]), d, r);
            b[k] = (uint32_t)(v[k] < 0.0f ? -m : m);
        }
    }
    uint32_t out[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = __byte_perm(__byte_perm(b[4 * k], b[4 * k + 1], 0x0040), __byte_perm(b[4 * k + 2], b[4 * k + 3], 0x0040), 0x5410);
    return d == d ? make_uint4(out[0], out[1], out[2], out[3]) : make_uint4(0, 0, 0, 0);
}
template <int DT>
__device__ __forceinline__ uint4 codes_of_16bit(const uint32_t *w, float d, float r) {
    float v[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = value_of<DT>(w, k);
    return codes_of(v, d, r);
}

}  // namespace i8
}  // namespace cq
