// C entries of 4-bit floating point with block scales (include/cubicquant.h): argument checks on the host, then launches.
#include "../../include/cubicquant.h"

#include <algorithm>

#include "cq_fp4.cuh"
#include "cq_internal.h"

using namespace cq;

namespace {

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
int wrap(cudaError_t e) {
    if (e == cudaSuccess) return CQ_OK;
    set_last_cuda_error(e);
    return CQ_ERR_CUDA;
}
int64_t blocks_of(int64_t rows) { return (rows + fp4::ROWS - 1) / fp4::ROWS; }
constexpr int64_t MOST = (int64_t)1 << 30;   // rows, channels, k: every index of a tile stays within 32 bits

int check_shape(int fmt, int64_t E, int64_t M, int64_t K) {
    if ((fmt != CQ_MXFP4 && fmt != CQ_NVFP4) || E <= 0 || M <= 0 || K <= 0) return CQ_ERR_INVALID_ARG;
    if (K % fp4::block_of(fmt) != 0 || M > MOST || K > MOST || E > MOST / blocks_of(M)) return CQ_ERR_UNSUPPORTED;
    return CQ_OK;
}
int check_groups(int64_t E, int64_t R) {
    if (E <= 0 || R <= 0) return CQ_ERR_INVALID_ARG;
    return E > fp4::MAX_EXPERTS ? CQ_ERR_UNSUPPORTED : CQ_OK;
}
// e8m0 scales carry the whole exponent range; a factor beside them is not part of that format
int check_scale(int fmt, const float *tensor_scale) { return fmt == CQ_MXFP4 && tensor_scale ? CQ_ERR_INVALID_ARG : CQ_OK; }
int check_rows(const void *x, int dtype, int64_t ldx, int64_t K) {
    if (dtype != CQ_BF16 && dtype != CQ_F16 && dtype != CQ_F32) return CQ_ERR_INVALID_ARG;
    if (ldx < K) return CQ_ERR_INVALID_ARG;
    return misaligned(x) || ldx % (dtype == CQ_F32 ? 4 : 8) != 0 ? CQ_ERR_ALIGNMENT : CQ_OK;
}
Fp4Rows dense(int64_t E, int64_t M) { return Fp4Rows{nullptr, nullptr, (int)E, M, E * M, E * M}; }
int64_t routed_blocks(int64_t E, int64_t R) { return (R + (fp4::ROWS - 1) * std::min(E, R)) / fp4::ROWS; }   // every group starts a block
size_t bytes_of(int fmt, int64_t blocks, int64_t K) { return (size_t)blocks * (size_t)((K + fp4::KB - 1) / fp4::KB) * (size_t)fp4::tile_bytes(fmt); }
constexpr size_t STATUS_BYTES = 512;

#define CQ_TRY(expr)                     \
    do {                                 \
        const int st_ = (expr);          \
        if (st_ != CQ_OK) return st_;    \
    } while (0)

int check_arch() {   // as for every product: tcgen05 needs a device of compute capability 10.x
    int dev = 0, major = 0;
    CQ_TRY(wrap(cudaGetDevice(&dev)));
    CQ_TRY(wrap(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)));
    return major == 10 ? CQ_OK : CQ_ERR_ARCH;
}

int64_t product_blocks(int64_t E, bool routed, int64_t M) { return routed ? routed_blocks(E, M) : blocks_of(M); }
int check_product(int fmt, int64_t E, bool routed, int64_t M, int64_t N, int64_t K) {
    CQ_TRY(check_shape(fmt, E, N, K));
    CQ_TRY(check_shape(fmt, 1, M, K));
    if (routed) CQ_TRY(check_groups(E, M));
    return blocks_of(N) * product_blocks(E, routed, M) > MOST / 2 ? CQ_ERR_UNSUPPORTED : CQ_OK;   // two tiles of 64 rows to a row block, counted in 32 bits
}
// x: the layout of quantised rows (ldx < 0), or rows in the model dtype, quantised into the workspace first
int product(const void *w, const float *w_scale, const void *x, int64_t ldx, int64_t T, const int32_t *route_token, const float *x_scale, const int32_t *offset, bool routed,
            int64_t E, int fmt, uint16_t *y, int act_f16, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    const bool quantised = ldx < 0;
    if (!w || !x || !y || !workspace || (routed && !offset) || (routed && !quantised && (!route_token || T <= 0))) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_product(fmt, E, routed, M, N, K));
    CQ_TRY(check_scale(fmt, w_scale));
    CQ_TRY(check_scale(fmt, x_scale));
    const int dtype = act_f16 ? CQ_F16 : CQ_BF16;
    if (!quantised) CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(w) || misaligned(x) || misaligned(y) || misaligned(workspace)) return CQ_ERR_ALIGNMENT;
    if (workspace_bytes < STATUS_BYTES + (quantised ? 0 : bytes_of(fmt, product_blocks(E, routed, M), K))) return CQ_ERR_WORKSPACE;
    CQ_TRY(check_arch());
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t *ws = (uint8_t *)workspace;
    if (!quantised && !routed && fp4_few_ok(M, N, K))
        return wrap(launch_fp4_few(w, w_scale, (const uint16_t *)x, ldx, x_scale, fmt, y, M, N, K, act_f16 != 0, (int *)ws, st));
    if (!quantised) {
        const Fp4Rows rows = routed ? Fp4Rows{route_token, offset, (int)E, M, M, T} : dense(1, M);
        CQ_TRY(wrap(launch_fp4_quantize(x, dtype, ldx, rows, fmt, K, x_scale, ws + STATUS_BYTES, st)));
        x = ws + STATUS_BYTES;
    }
    return wrap(launch_fp4_gemm(w, w_scale, x, x_scale, offset, (int)E, fmt, y, M, N, K, act_f16 != 0, !quantised, (int *)ws, st));
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t cq_fp4_layout_bytes(int fmt, int64_t E, int64_t M, int64_t K) {
    return check_shape(fmt, E, M, K) == CQ_OK ? bytes_of(fmt, E * blocks_of(M), K) : 0;
}
size_t cq_fp4_routed_layout_bytes(int fmt, int64_t E, int64_t R, int64_t K) {
    return check_shape(fmt, 1, R, K) == CQ_OK && check_groups(E, R) == CQ_OK ? bytes_of(fmt, routed_blocks(E, R), K) : 0;
}
size_t cq_fp4_workspace_bytes(int fmt, int64_t M, int64_t K) {
    const size_t b = cq_fp4_layout_bytes(fmt, 1, M, K);
    return b ? STATUS_BYTES + b : 0;
}
size_t cq_fp4_routed_workspace_bytes(int fmt, int64_t E, int64_t R, int64_t K) {
    const size_t b = cq_fp4_routed_layout_bytes(fmt, E, R, K);
    return b ? STATUS_BYTES + b : 0;
}

int cq_fp4_pack(const uint8_t *codes, const uint8_t *scales, int fmt, int64_t E, int64_t M, int64_t K, void *layout, void *stream) {
    if (!codes || !scales || !layout) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, E, M, K));
    if (misaligned(layout) || misaligned(codes)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_fp4_exchange(const_cast<uint8_t *>(codes), const_cast<uint8_t *>(scales), dense(E, M), fmt, K, layout, true, (cudaStream_t)stream));
}
int cq_fp4_unpack(const void *layout, int fmt, int64_t E, int64_t M, int64_t K, uint8_t *codes, uint8_t *scales, void *stream) {
    if (!codes || !scales || !layout) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, E, M, K));
    if (misaligned(layout) || misaligned(codes)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_fp4_exchange(codes, scales, dense(E, M), fmt, K, const_cast<void *>(layout), false, (cudaStream_t)stream));
}

int cq_fp4_quantize(const void *x, int dtype, int64_t ldx, int fmt, int64_t E, int64_t M, int64_t K, const float *tensor_scale, void *layout, void *stream) {
    if (!x || !layout) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, E, M, K));
    CQ_TRY(check_scale(fmt, tensor_scale));
    CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(layout)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_fp4_quantize(x, dtype, ldx, dense(E, M), fmt, K, tensor_scale, layout, (cudaStream_t)stream));
}
int cq_fp4_quantize_routed(const void *x, int dtype, int64_t ldx, int64_t T, const int32_t *route_token, const int32_t *expert_offset, int64_t E, int64_t R, int fmt,
                           int64_t K, const float *tensor_scale, void *layout, void *stream) {
    if (!x || !layout || !route_token || !expert_offset || T <= 0) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, 1, R, K));
    CQ_TRY(check_groups(E, R));
    CQ_TRY(check_scale(fmt, tensor_scale));
    CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(layout)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_fp4_quantize(x, dtype, ldx, Fp4Rows{route_token, expert_offset, (int)E, R, R, T}, fmt, K, tensor_scale, layout, (cudaStream_t)stream));
}
int cq_fp4_swiglu_quantize(const void *h, int dtype, int64_t ldh, int fmt, int64_t M, int64_t I, const int32_t *expert_offset, int64_t E, const float *tensor_scale,
                           void *layout, void *stream) {
    if (!h || !layout || (dtype != CQ_BF16 && dtype != CQ_F16)) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, 1, M, I));
    if (expert_offset) CQ_TRY(check_groups(E, M));
    CQ_TRY(check_scale(fmt, tensor_scale));
    CQ_TRY(check_rows(h, dtype, ldh, 2 * I));
    if (misaligned(layout) || I % 8 != 0) return CQ_ERR_ALIGNMENT;
    const Fp4Rows rows = expert_offset ? Fp4Rows{nullptr, expert_offset, (int)E, M, M, M} : dense(1, M);
    return wrap(launch_fp4_swiglu_quantize(h, dtype, ldh, rows, fmt, I, tensor_scale, layout, (cudaStream_t)stream));
}
int cq_fp4_dequantize(const void *layout, int fmt, int64_t E, int64_t M, int64_t K, const int32_t *expert_offset, const float *tensor_scale, void *y, int dtype, void *stream) {
    if (!layout || !y || (dtype != CQ_BF16 && dtype != CQ_F16 && dtype != CQ_F32)) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(fmt, expert_offset ? 1 : E, M, K));
    if (expert_offset) CQ_TRY(check_groups(E, M));
    CQ_TRY(check_scale(fmt, tensor_scale));
    if (misaligned(layout) || misaligned(y)) return CQ_ERR_ALIGNMENT;
    const Fp4Rows rows = expert_offset ? Fp4Rows{nullptr, expert_offset, (int)E, M, M, M} : dense(E, M);
    return wrap(launch_fp4_dequantize(layout, rows, fmt, K, tensor_scale, y, dtype, (cudaStream_t)stream));
}

int cq_fp4_gemm(const void *w, const float *w_scale, const void *x, const float *x_scale, int fmt, uint16_t *y, int act_f16, int64_t M, int64_t N, int64_t K,
                void *workspace, size_t workspace_bytes, void *stream) {
    return product(w, w_scale, x, -1, 0, nullptr, x_scale, nullptr, false, 1, fmt, y, act_f16, M, N, K, workspace, workspace_bytes, stream);
}
int cq_fp4_linear(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, const float *x_scale, int fmt, uint16_t *y, int act_f16, int64_t M, int64_t N,
                  int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    if (ldx < 0) return CQ_ERR_INVALID_ARG;
    return product(w, w_scale, x, ldx, 0, nullptr, x_scale, nullptr, false, 1, fmt, y, act_f16, M, N, K, workspace, workspace_bytes, stream);
}
int cq_fp4_gemm_routed(const void *w, const float *w_scale, const void *x, const float *x_scale, const int32_t *expert_offset, int64_t E, int fmt, uint16_t *y, int act_f16,
                       int64_t R, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    return product(w, w_scale, x, -1, 0, nullptr, x_scale, expert_offset, true, E, fmt, y, act_f16, R, N, K, workspace, workspace_bytes, stream);
}
int cq_fp4_linear_routed(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, int64_t T, const int32_t *route_token, const float *x_scale,
                         const int32_t *expert_offset, int64_t E, int fmt, uint16_t *y, int act_f16, int64_t R, int64_t N, int64_t K, void *workspace,
                         size_t workspace_bytes, void *stream) {
    if (ldx < 0) return CQ_ERR_INVALID_ARG;
    return product(w, w_scale, x, ldx, T, route_token, x_scale, expert_offset, true, E, fmt, y, act_f16, R, N, K, workspace, workspace_bytes, stream);
}

int cq_debug_fp4_plan(int fmt, int64_t E, int64_t M, int64_t N, int64_t K, int quantised, int64_t *plan) {
    if (!plan || E < 0) return CQ_ERR_INVALID_ARG;
    const bool routed = E > 0;
    CQ_TRY(check_product(fmt, routed ? E : 1, routed, M, N, K));
    const bool own = !quantised && !routed && fp4_few_ok(M, N, K);
    const Fp4Plan p = fp4_plan(E, routed, M, N, K, fmt, own);
    plan[0] = p.channels; plan[1] = p.rows; plan[2] = p.runs; plan[3] = own;
    return CQ_OK;
}

}  // extern "C"
#pragma GCC visibility pop
