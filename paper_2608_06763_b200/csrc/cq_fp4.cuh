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
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cq {
namespace fp4 {

constexpr int MX = 0, NV = 1;                 // CQ_MXFP4, CQ_NVFP4
constexpr int DT_BF16 = 0, DT_F16 = 1, DT_F32 = 2;   // CQ_BF16, CQ_F16, CQ_F32
constexpr int ROWS = 128, KB = 256;           // a tile
constexpr int CODE_BYTES = ROWS * KB / 2;
constexpr int MAX_EXPERTS = 512;              // the offsets' tables in shared memory

__host__ __device__ constexpr int block_of(int fmt) { return fmt == MX ? 32 : 16; }
__host__ __device__ constexpr int scale_bytes(int fmt) { return ROWS * KB / block_of(fmt); }
__host__ __device__ constexpr int tile_bytes(int fmt) { return CODE_BYTES + scale_bytes(fmt); }

// byte of a tile that holds the codes of k = 2 b, 2 b + 1 in row r
__host__ __device__ inline int code_offset(int r, int b) { return r * 128 + (((b >> 4) ^ (r & 7)) << 4) + (b & 15); }
// byte of a tile that holds scale j of row r, counted along k inside the tile
__host__ __device__ inline int scale_offset(int r, int j) { return CODE_BYTES + (j >> 2) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (j & 3); }

// ---- groups of routed rows ------------------------------------------------------------------
// offset[e] .. offset[e + 1] are the rows of group e, as the router left them on the GPU.  What does not ascend, or leaves
// [0, R], is brought back into it: the largest value so far, at most R.  One warp writes the offsets and the first row
// block of each group (E + 1 values each); the block synchronises before it reads them.
__device__ __forceinline__ void scan_groups(const int32_t *offset, int E, int R, int *s_off, int *s_blk) {
    const int lane = threadIdx.x & 31;
    int top = 0, blk = 0;   // of what lies in front
    for (int e0 = 0; e0 <= E; e0 += 32) {
        const int e = e0 + lane;
        int o = e <= E ? min(max(offset[e], 0), R) : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(~0u, o, d);
            if (lane >= d) o = max(o, v);
        }
        o = max(o, top);
        int before = __shfl_up_sync(~0u, o, 1);
        if (lane == 0) before = e0 == 0 ? o : top;
        int b = (o - before + ROWS - 1) / ROWS;   // row blocks of the group that ends here
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(~0u, b, d);
            if (lane >= d) b += v;
        }
        b += blk;
        if (e <= E) { s_off[e] = o; s_blk[e] = b; }
        top = __shfl_sync(~0u, o, 31);
        blk = __shfl_sync(~0u, b, 31);
    }
}
// the group that a row or a tile belongs to: the last e with table[e] <= v (v < table[E])
__device__ __forceinline__ int find_group(const int *table, int E, int v) {
    int lo = 0, hi = E;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (table[mid] <= v) lo = mid; else hi = mid;
    }
    return lo;
}

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
// the magnitude of a code is 2 x + ... : read off a word of half values in 4-bit fields would cost more than this
__device__ __forceinline__ float from_e2m1(uint32_t c) {
    const uint32_t m = c & 7u;
    const float v = m < 2u ? 0.5f * (float)m : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
    return (c & 8u) ? -v : v;
}

// The scale byte of a block, and the factor its values are multiplied by before they are rounded to codes.  top: bits of the largest
// |x| (a NaN or an infinity makes the scale NaN); r = 1 / g (NVFP4).
template <int FMT>
__device__ __forceinline__ uint32_t block_scale(uint32_t top, float r, float &factor) {
    if (FMT == MX) {
        const uint32_t b = (top >> 23) > 2u ? (top >> 23) - 2u : 0u;   // floor(log2 top) - 2, not below -127
        factor = __uint_as_float((254u - b) << 23);
        if (top >= 0x7F800000u) { factor = 0.0f; return 255u; }
        return b;
    }
    // 2^-9 is the least scale that e4m3 has: a block of zeros or of less than that keeps a scale to be divided by
    const float s = fminf(fmaxf(__fdiv_rn(__fmul_rn(__uint_as_float(top), r), 6.0f), 0.001953125f), 448.0f);
    const uint32_t b = to_e4m3(s);
    factor = __fdiv_rn(r, from_e4m3(b));
    if (top >= 0x7F800000u) { factor = 0.0f; return 127u; }
    return b;
}

}  // namespace fp4
}  // namespace cq
