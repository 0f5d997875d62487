// What the operators on quantised rows share, whatever the codes are: groups of routed rows, the values of a row in 16 bits, paired
// fp32 arithmetic.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace cq {
namespace rows {

constexpr int DT_BF16 = 0, DT_F16 = 1, DT_F32 = 2;   // CQ_BF16, CQ_F16, CQ_F32
constexpr int ROWS = 128;                            // of a tile of an operand
constexpr int MAX_EXPERTS = 512;                     // the offsets' tables in shared memory

// ---- groups of routed rows ------------------------------------------------------------------
// offset[e] .. offset[e + 1] are the rows of group e, as the router left them on the GPU.  What does not ascend, or leaves
// [0, R], is brought back into it: the largest value so far, at most R.  One warp writes the offsets and the first row
// block of each group (E + 1 values each), and, for a product, its first tile (bt rows of x to a tile, `times` of them); the
// block synchronises before it reads them.
__device__ __forceinline__ void scan_groups(const int32_t *offset, int E, int R, int *s_off, int *s_blk, int *s_item = nullptr, int bt = 1, int times = 0) {
    const int lane = threadIdx.x & 31;
    int top = 0, blk = 0, item = 0;   // of what lies in front
    for (int e0 = 0; e0 <= E; e0 += 32) {
        const int e = e0 + lane;
        int o = max(e <= E ? min(max(offset[e], 0), R) : 0, top);
        int before = __shfl_up_sync(~0u, o, 1);
        if (lane == 0) before = e0 == 0 ? o : top;
        if (__any_sync(~0u, e <= E && o < before)) {   // not ascending
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int v = __shfl_up_sync(~0u, o, d);
                if (lane >= d) o = max(o, v);
            }
            before = __shfl_up_sync(~0u, o, 1);
            if (lane == 0) before = e0 == 0 ? o : top;
        }
        // behind E the counts mean nothing, and nobody reads them
        int b = (o - before + ROWS - 1) / ROWS, n = s_item ? (o - before + bt - 1) / bt : 0;   // row blocks and tiles of the group that ends here
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(~0u, b, d), u = __shfl_up_sync(~0u, n, d);
            if (lane >= d) { b += v; n += u; }
        }
        b += blk;
        n += item;
        if (e <= E) {
            s_off[e] = o;
            s_blk[e] = b;
            if (s_item) s_item[e] = n * times;
        }
        top = __shfl_sync(~0u, o, 31);
        blk = __shfl_sync(~0u, b, 31);
        item = __shfl_sync(~0u, n, 31);
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

// ---------------------------------------------------------------- two fp32 operations an instruction, each rounded by itself
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float a, float b) { Pair r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void unpair(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// ---------------------------------------------------------------- sixteen values of a row in 16 bits
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

template <int DT>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (DT == DT_BF16) { const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi); return *reinterpret_cast<const uint32_t *>(&p); }
    const __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&p);
}

}  // namespace rows
}  // namespace cq
