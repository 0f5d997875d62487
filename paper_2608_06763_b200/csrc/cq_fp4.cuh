// 4-bit floating point with block scales: formats, the device layout, conversions.
//
// A value is an e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) times the scale of its block of consecutive k:
//   CQ_MXFP4  blocks of 32, scale 2^(byte - 127)  (e8m0; 255 is NaN)
//   CQ_NVFP4  blocks of 16, scale in e4m3 (127 is NaN), and one fp32 factor for the whole matrix beside the layout
//
// Device layout: rows are padded to 128 and k to 256; tile (row block rb, k block kt) of 128 rows x 256 k is stored at
// (rb * KT + kt) * tile_bytes as  [codes 16384 B][scales 2048 B (NVFP4) or 1024 B (MXFP4)], so that one bulk copy brings what the
// tensor core reads, in the order in which it reads it:
//   codes   128 bytes a row, two codes a byte (even k in the low half), the 16-byte pieces of row r exchanged by
//           piece ^= r & 7: the 128-byte swizzle of a K-major MMA operand
//   scales  pieces of 512 bytes, each four scales along k (64 k of NVFP4, 128 k of MXFP4) of 128 rows:
//           row r, scale j at (r % 32) * 16 + (r / 32) * 4 + j, the order in which tcgen05.cp.32x128b moves scales to tensor memory
// Several matrices of one shape (the experts of a layer) follow one another.  Activations of routed rows keep each group in row
// blocks of its own.  Codes and scales behind K are written as zeros; rows behind the last are never written, and
// what they hold reaches no result (a row of an operand meets only its own row or column of the product).
#pragma once
#include "cq_rows.cuh"

namespace cq {
namespace fp4 {

using namespace rows;

constexpr int MX = 0, NV = 1;                 // CQ_MXFP4, CQ_NVFP4
constexpr int KB = 256;                       // a tile has ROWS rows and so many k
constexpr int CODE_BYTES = ROWS * KB / 2;

__host__ __device__ constexpr int block_of(int fmt) { return fmt == MX ? 32 : 16; }
__host__ __device__ constexpr int scale_bytes(int fmt) { return ROWS * KB / block_of(fmt); }
__host__ __device__ constexpr int tile_bytes(int fmt) { return CODE_BYTES + scale_bytes(fmt); }

// byte of a tile that holds the codes of k = 2 b, 2 b + 1 in row r
__host__ __device__ inline int code_offset(int r, int b) { return r * 128 + (((b >> 4) ^ (r & 7)) << 4) + (b & 15); }
// byte of a tile that holds scale j of row r, counted along k inside the tile
__host__ __device__ inline int scale_offset(int r, int j) { return CODE_BYTES + (j >> 2) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (j & 3); }

// ---- conversions ----------------------------------------------------------------------------
// eight values to eight codes, the first in the lowest four bits; nearest, ties to the even code, saturating at 6
__device__ __forceinline__ uint32_t to_e2m1x8(const float *v) {
    uint32_t out;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(out) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return out;
}
__device__ __forceinline__ uint32_t to_e4m3(float v) {   // v >= 0
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
    return r & 0xFFu;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
    return __half2float(__ushort_as_half((unsigned short)(h & 0xFFFFu)));
}
__device__ __forceinline__ float from_e8m0(uint32_t b) {
    return __uint_as_float(b == 255u ? 0x7FFFFFFFu : b == 0u ? 0x00400000u : b << 23);
}
// eight codes to values, exactly (the conversion goes through binary16, which holds them all)
__device__ __forceinline__ void from_e2m1x8(uint32_t c, float *v) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(c));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[i]));
        v[2 * i] = f.x; v[2 * i + 1] = f.y;
    }
}

// The scale byte of a block, and the factor its values are multiplied by before they are rounded to codes.  top: bits of the largest
// |x| (a NaN or an infinity makes the scale NaN and the factor 0).  NVFP4: r = 1 / g, factors: r / scale by scale byte (null: divided here).
template <int FMT>
__device__ __forceinline__ uint32_t block_scale(uint32_t top, float r, const float *factors, float &factor) {
    if (FMT == MX) {
        uint32_t b = (top >> 23) > 2u ? (top >> 23) - 2u : 0u;   // floor(log2 top) - 2, not below -127
        factor = __uint_as_float((254u - b) << 23);
        if (top >= 0x7F800000u) { factor = 0.0f; b = 255u; }
        return b;
    }
    // 2^-9 is the least scale that e4m3 has: a block of zeros or of less than that keeps a scale to be divided by
    const float s = fminf(fmaxf(__fdiv_rn(__fmul_rn(__uint_as_float(top), r), 6.0f), 0.001953125f), 448.0f);
    const uint32_t b = top >= 0x7F800000u ? 127u : to_e4m3(s);
    factor = factors ? factors[b] : b == 127u ? 0.0f : __fdiv_rn(r, from_e4m3(b));
    return b;
}

template <int FMT>
__device__ __forceinline__ uint32_t top_of_block(uint32_t top) {   // MXFP4: two threads hold a block
    return FMT == MX ? max(top, __shfl_xor_sync(~0u, top, 1)) : top;
}
__device__ __forceinline__ uint2 round_codes(const float *v, float factor) {
    float u[16];
    const Pair f = pair_of(factor, factor);
#pragma unroll
    for (int i = 0; i < 16; i += 2) unpair(mul2(pair_of(v[i], v[i + 1]), f), u[i], u[i + 1]);
    return make_uint2(to_e2m1x8(u), to_e2m1x8(u + 8));
}
// Four scales of a row, held by neighbouring lanes (a scale of MXFP4 by two), as they lie in memory.  All lanes take part.
template <int FMT>
__device__ __forceinline__ uint32_t gather_scales(uint32_t scale) {
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
    return word;
}
// Sixteen values of a row in a model dtype to codes and the scale of their block; r = 1 / g.  All lanes take part.
template <int FMT, int DT>
__device__ __forceinline__ uint2 quantize_unit(const uint4 &a, const uint4 &b, float r, uint32_t &scale) {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float v[16], factor;
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = value_of<DT>(w, k);
    scale = block_scale<FMT>(top_of_block<FMT>(top_of_16bit<DT>(w)), r, nullptr, factor);
    return factor == 0.0f ? make_uint2(0, 0) : round_codes(v, factor);
}

}  // namespace fp4
}  // namespace cq
