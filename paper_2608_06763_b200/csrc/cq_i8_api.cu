// C entries of routing to experts and of 8-bit integers with a scale for each row (include/cubicquant.h): argument checks on the host, then launches.
#include "../../include/cubicquant.h"

#include <algorithm>

#include "cq_i8.cuh"
#include "cq_internal.h"

using namespace cq;

namespace {

bool misaligned(const void *p, uintptr_t to = 16) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
int wrap(cudaError_t e) {
    if (e == cudaSuccess) return CQ_OK;
    set_last_cuda_error(e);
    return CQ_ERR_CUDA;
}
int64_t blocks_of(int64_t rows) { return (rows + i8::ROWS - 1) / i8::ROWS; }
constexpr int64_t MOST = (int64_t)1 << 30;   // rows, channels, routes: every index of a tile stays within 32 bits
constexpr int MOST_TOP = 32;                 // choices of a token: a lane of a warp for each

#define CQ_TRY(expr)                     \
    do {                                 \
        const int st_ = (expr);          \
        if (st_ != CQ_OK) return st_;    \
    } while (0)

int check_shape(int64_t E, int64_t M, int64_t K) {
    if (E <= 0 || M <= 0 || K <= 0) return CQ_ERR_INVALID_ARG;
    return K % 16 != 0 || K > i8::MOST_K || M > MOST || E > MOST / blocks_of(M) ? CQ_ERR_UNSUPPORTED : CQ_OK;
}
int check_groups(int64_t E, int64_t R) {
    if (E <= 0 || R <= 0) return CQ_ERR_INVALID_ARG;
    return E > i8::MAX_EXPERTS ? CQ_ERR_UNSUPPORTED : CQ_OK;
}
int check_rows(const void *x, int dtype, int64_t ldx, int64_t K) {
    if (dtype != CQ_BF16 && dtype != CQ_F16 && dtype != CQ_F32) return CQ_ERR_INVALID_ARG;
    if (ldx < K) return CQ_ERR_INVALID_ARG;
    return misaligned(x) || ldx % (dtype == CQ_F32 ? 4 : 8) != 0 ? CQ_ERR_ALIGNMENT : CQ_OK;
}
I8Rows dense(int64_t E, int64_t M) { return I8Rows{nullptr, nullptr, (int)E, M, E * M, E * M}; }
I8Rows routed_rows(const int32_t *route_token, const int32_t *offset, int64_t E, int64_t R, int64_t T) { return I8Rows{route_token, offset, (int)E, R, R, T}; }
int64_t routed_blocks(int64_t E, int64_t R) { return (R + (i8::ROWS - 1) * std::min(E, R)) / i8::ROWS; }   // every group starts a block
size_t bytes_of(int64_t blocks, int64_t K) { return (size_t)blocks * (size_t)((K + i8::KB - 1) / i8::KB) * (size_t)i8::TILE_BYTES; }
size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }
constexpr size_t STATUS_BYTES = 512;

int check_arch() {   // as for every product: tcgen05 needs a device of compute capability 10.x
    int dev = 0, major = 0;
    CQ_TRY(wrap(cudaGetDevice(&dev)));
    CQ_TRY(wrap(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)));
    return major == 10 ? CQ_OK : CQ_ERR_ARCH;
}

int64_t product_blocks(int64_t E, bool routed, int64_t M) { return routed ? routed_blocks(E, M) : blocks_of(M); }
int check_product(int64_t E, bool routed, int64_t M, int64_t N, int64_t K) {
    CQ_TRY(check_shape(E, N, K));
    CQ_TRY(check_shape(1, M, K));
    if (routed) CQ_TRY(check_groups(E, M));
    return blocks_of(N) * product_blocks(E, routed, M) > MOST / 2 ? CQ_ERR_UNSUPPORTED : CQ_OK;   // two tiles of 64 rows to a row block, counted in 32 bits
}
size_t workspace_of(int64_t blocks, int64_t M, int64_t K) { return STATUS_BYTES + padded((size_t)M * sizeof(float)) + bytes_of(blocks, K); }

// x: the layout of quantised rows (ldx < 0) and their scales, or rows in the model dtype, quantised into the workspace first
int product(const void *w, const float *w_scale, const void *x, int64_t ldx, const float *x_scale, int64_t T, const int32_t *route_token, const int32_t *offset, bool routed,
            int64_t E, uint16_t *y, int act_f16, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    const bool quantised = ldx < 0;
    if (!w || !w_scale || !x || !y || !workspace || (quantised && !x_scale) || (routed && !offset) || (routed && !quantised && (!route_token || T <= 0))) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_product(E, routed, M, N, K));
    const int dtype = act_f16 ? CQ_F16 : CQ_BF16;
    if (!quantised) CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(w) || misaligned(x) || misaligned(y) || misaligned(workspace) || misaligned(w_scale, 4) || misaligned(x_scale, 4)) return CQ_ERR_ALIGNMENT;
    if (workspace_bytes < (quantised ? STATUS_BYTES : workspace_of(product_blocks(E, routed, M), M, K))) return CQ_ERR_WORKSPACE;
    CQ_TRY(check_arch());
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t *ws = (uint8_t *)workspace;
    if (!quantised && !routed && i8_few_ok(M, N, K)) return wrap(launch_i8_few(w, w_scale, (const uint16_t *)x, ldx, y, M, N, K, act_f16 != 0, (int *)ws, st));
    if (!quantised) {
        float *scale = (float *)(ws + STATUS_BYTES);
        uint8_t *layout = ws + STATUS_BYTES + padded((size_t)M * sizeof(float));
        CQ_TRY(wrap(launch_i8_quantize(x, dtype, ldx, routed ? routed_rows(route_token, offset, E, M, T) : dense(1, M), K, scale, layout, st)));
        x = layout;
        x_scale = scale;
    }
    return wrap(launch_i8_gemm(w, w_scale, x, x_scale, offset, (int)E, y, M, N, K, act_f16 != 0, !quantised, (int *)ws, st));
}

// the workspace of cq_i8_moe: offsets of its parts
struct MoePlan { size_t x_scale, x, h, a_scale, a, total; };
MoePlan moe_plan(int64_t E, int64_t R, int64_t H, int64_t I) {
    MoePlan p;
    const int64_t blocks = routed_blocks(E, R);
    p.x_scale = STATUS_BYTES;
    p.a_scale = p.x_scale + padded((size_t)R * sizeof(float));
    p.x = p.a_scale + padded((size_t)R * sizeof(float));
    p.a = p.x + bytes_of(blocks, H);
    p.h = p.a + bytes_of(blocks, I);
    p.total = p.h + padded((size_t)R * (size_t)std::max(2 * I, H) * 2);   // gate | up, and, when that has been read, the outputs of the routes
    return p;
}
int check_moe(int64_t E, int64_t T, int top, int64_t H, int64_t I) {
    if (T <= 0 || top <= 0 || H <= 0 || I <= 0) return CQ_ERR_INVALID_ARG;
    if (top > MOST_TOP || T > MOST / top) return CQ_ERR_UNSUPPORTED;
    CQ_TRY(check_product(E, true, T * top, 2 * I, H));
    return check_product(E, true, T * top, H, I);
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t cq_route_workspace_bytes(int64_t T, int64_t E) { return T > 0 && T <= MOST && E > 0 && E <= i8::MAX_EXPERTS ? route_count_bytes(T, E) : 0; }

int cq_route(const void *logits, int dtype, int64_t ldl, int64_t T, int64_t E, int top, int score, const float *bias, int groups, int groups_kept, int group_best, int renormalise,
             float scale, int32_t *expert, float *weight, int32_t *route_token, int32_t *expert_offset, int32_t *route_row, void *workspace, size_t workspace_bytes, void *stream) {
    if (!logits || !expert || !weight || !route_token || !expert_offset || !route_row || !workspace || T <= 0 || E <= 0 || top <= 0) return CQ_ERR_INVALID_ARG;
    if ((score != CQ_SOFTMAX && score != CQ_SIGMOID) || (dtype != CQ_BF16 && dtype != CQ_F16 && dtype != CQ_F32) || ldl < E) return CQ_ERR_INVALID_ARG;
    if (groups <= 0 || groups_kept <= 0 || groups_kept > groups || (group_best != 1 && group_best != 2) || E % groups != 0) return CQ_ERR_INVALID_ARG;
    if (top > E / groups * groups_kept) return CQ_ERR_INVALID_ARG;
    if (E > i8::MAX_EXPERTS || groups > 32 || top > MOST_TOP || T > MOST / top) return CQ_ERR_UNSUPPORTED;
    if (misaligned(logits, dtype == CQ_F32 ? 4 : 2) || misaligned(bias, 4) || misaligned(expert, 4) || misaligned(weight, 4) || misaligned(route_token, 4) ||
        misaligned(expert_offset, 4) || misaligned(route_row, 4) || misaligned(workspace))
        return CQ_ERR_ALIGNMENT;
    if (workspace_bytes < route_count_bytes(T, E)) return CQ_ERR_WORKSPACE;
    RouteCall c{};
    c.logits = logits; c.dtype = dtype; c.ldl = ldl; c.T = T; c.E = (int)E; c.groups = groups; c.kept = groups_kept; c.best = group_best; c.top = top; c.bias = bias;
    c.sigmoid = score == CQ_SIGMOID; c.renormalise = renormalise != 0; c.scale = scale;
    c.expert = expert; c.row = route_row; c.token = route_token; c.offset = expert_offset; c.weight = weight; c.counts = (int32_t *)workspace;
    return wrap(launch_route(c, (cudaStream_t)stream));
}

int cq_combine(const uint16_t *y_routes, int64_t ldr, int64_t R, const float *weight, const int32_t *route_row, int64_t T, int top, int64_t N, const uint16_t *add, int64_t lda,
               uint16_t *y, int64_t ldy, int act_f16, void *stream) {
    if (!y_routes || !weight || !route_row || !y || R <= 0 || T <= 0 || top <= 0 || N <= 0 || ldr < N || ldy < N || (add && lda < N)) return CQ_ERR_INVALID_ARG;
    if (top > MOST_TOP || T > MOST / top || N > MOST || R > MOST) return CQ_ERR_UNSUPPORTED;
    if (misaligned(y_routes, 2) || misaligned(weight, 4) || misaligned(route_row, 4) || misaligned(add, 2) || misaligned(y, 2)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_combine(y_routes, ldr, R, weight, route_row, T, top, N, add, lda, y, ldy, act_f16 != 0, (cudaStream_t)stream));
}

size_t cq_i8_layout_bytes(int64_t E, int64_t M, int64_t K) { return check_shape(E, M, K) == CQ_OK ? bytes_of(E * blocks_of(M), K) : 0; }
size_t cq_i8_routed_layout_bytes(int64_t E, int64_t R, int64_t K) {
    return check_shape(1, R, K) == CQ_OK && check_groups(E, R) == CQ_OK ? bytes_of(routed_blocks(E, R), K) : 0;
}
size_t cq_i8_workspace_bytes(int64_t M, int64_t K) { return check_shape(1, M, K) == CQ_OK ? workspace_of(blocks_of(M), M, K) : 0; }
size_t cq_i8_routed_workspace_bytes(int64_t E, int64_t R, int64_t K) {
    return check_shape(1, R, K) == CQ_OK && check_groups(E, R) == CQ_OK ? workspace_of(routed_blocks(E, R), R, K) : 0;
}

int cq_i8_pack(const int8_t *codes, int64_t E, int64_t M, int64_t K, void *layout, void *stream) {
    if (!codes || !layout) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(E, M, K));
    if (misaligned(layout) || misaligned(codes)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_exchange(reinterpret_cast<uint8_t *>(const_cast<int8_t *>(codes)), dense(E, M), K, layout, true, (cudaStream_t)stream));
}
int cq_i8_unpack(const void *layout, int64_t E, int64_t M, int64_t K, int8_t *codes, void *stream) {
    if (!codes || !layout) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(E, M, K));
    if (misaligned(layout) || misaligned(codes)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_exchange(reinterpret_cast<uint8_t *>(codes), dense(E, M), K, const_cast<void *>(layout), false, (cudaStream_t)stream));
}

int cq_i8_quantize(const void *x, int dtype, int64_t ldx, int64_t E, int64_t M, int64_t K, void *layout, float *scale, void *stream) {
    if (!x || !layout || !scale) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(E, M, K));
    CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(layout) || misaligned(scale, 4)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_quantize(x, dtype, ldx, dense(E, M), K, scale, layout, (cudaStream_t)stream));
}
int cq_i8_quantize_routed(const void *x, int dtype, int64_t ldx, int64_t T, const int32_t *route_token, const int32_t *expert_offset, int64_t E, int64_t R, int64_t K, void *layout,
                          float *scale, void *stream) {
    if (!x || !layout || !scale || !route_token || !expert_offset || T <= 0) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(1, R, K));
    CQ_TRY(check_groups(E, R));
    CQ_TRY(check_rows(x, dtype, ldx, K));
    if (misaligned(layout) || misaligned(scale, 4)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_quantize(x, dtype, ldx, routed_rows(route_token, expert_offset, E, R, T), K, scale, layout, (cudaStream_t)stream));
}
int cq_i8_swiglu_quantize(const void *h, int dtype, int64_t ldh, int64_t M, int64_t I, const int32_t *expert_offset, int64_t E, void *layout, float *scale, void *stream) {
    if (!h || !layout || !scale || (dtype != CQ_BF16 && dtype != CQ_F16)) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(1, M, I));
    if (expert_offset) CQ_TRY(check_groups(E, M));
    CQ_TRY(check_rows(h, dtype, ldh, 2 * I));
    if (misaligned(layout) || misaligned(scale, 4)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_swiglu_quantize(h, dtype, ldh, expert_offset ? routed_rows(nullptr, expert_offset, E, M, M) : dense(1, M), I, scale, layout, (cudaStream_t)stream));
}
int cq_i8_dequantize(const void *layout, const float *scale, int64_t E, int64_t M, int64_t K, const int32_t *expert_offset, void *y, int dtype, void *stream) {
    if (!layout || !scale || !y || (dtype != CQ_BF16 && dtype != CQ_F16 && dtype != CQ_F32)) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_shape(expert_offset ? 1 : E, M, K));
    if (expert_offset) CQ_TRY(check_groups(E, M));
    if (misaligned(layout) || misaligned(y) || misaligned(scale, 4)) return CQ_ERR_ALIGNMENT;
    return wrap(launch_i8_dequantize(layout, expert_offset ? routed_rows(nullptr, expert_offset, E, M, M) : dense(E, M), K, scale, y, dtype, (cudaStream_t)stream));
}

int cq_i8_gemm(const void *w, const float *w_scale, const void *x, const float *x_scale, uint16_t *y, int act_f16, int64_t M, int64_t N, int64_t K, void *workspace,
               size_t workspace_bytes, void *stream) {
    return product(w, w_scale, x, -1, x_scale, 0, nullptr, nullptr, false, 1, y, act_f16, M, N, K, workspace, workspace_bytes, stream);
}
int cq_i8_linear(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, uint16_t *y, int act_f16, int64_t M, int64_t N, int64_t K, void *workspace, size_t workspace_bytes,
                 void *stream) {
    if (ldx < 0) return CQ_ERR_INVALID_ARG;
    return product(w, w_scale, x, ldx, nullptr, 0, nullptr, nullptr, false, 1, y, act_f16, M, N, K, workspace, workspace_bytes, stream);
}
int cq_i8_gemm_routed(const void *w, const float *w_scale, const void *x, const float *x_scale, const int32_t *expert_offset, int64_t E, uint16_t *y, int act_f16, int64_t R, int64_t N,
                      int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    return product(w, w_scale, x, -1, x_scale, 0, nullptr, expert_offset, true, E, y, act_f16, R, N, K, workspace, workspace_bytes, stream);
}
int cq_i8_linear_routed(const void *w, const float *w_scale, const uint16_t *x, int64_t ldx, int64_t T, const int32_t *route_token, const int32_t *expert_offset, int64_t E, uint16_t *y,
                        int act_f16, int64_t R, int64_t N, int64_t K, void *workspace, size_t workspace_bytes, void *stream) {
    if (ldx < 0) return CQ_ERR_INVALID_ARG;
    return product(w, w_scale, x, ldx, nullptr, T, route_token, expert_offset, true, E, y, act_f16, R, N, K, workspace, workspace_bytes, stream);
}

size_t cq_i8_moe_workspace_bytes(int64_t E, int64_t T, int top, int64_t H, int64_t I) { return check_moe(E, T, top, H, I) == CQ_OK ? moe_plan(E, T * top, H, I).total : 0; }
int cq_i8_moe(const void *gate_up, const float *gate_up_scale, const void *down, const float *down_scale, int64_t E, const uint16_t *x, int64_t ldx, int64_t T, int top,
              const int32_t *expert_offset, const int32_t *route_row, const float *weight, const uint16_t *add, int64_t lda, uint16_t *y, int64_t ldy,
              int act_f16, int64_t H, int64_t I, void *workspace, size_t workspace_bytes, void *stream) {
    if (!gate_up || !gate_up_scale || !down || !down_scale || !x || !expert_offset || !route_row || !weight || !y || !workspace) return CQ_ERR_INVALID_ARG;
    CQ_TRY(check_moe(E, T, top, H, I));
    const int dtype = act_f16 ? CQ_F16 : CQ_BF16;
    CQ_TRY(check_rows(x, dtype, ldx, H));
    if (ldy < H || (add && lda < H)) return CQ_ERR_INVALID_ARG;
    if (misaligned(gate_up) || misaligned(down) || misaligned(workspace) || misaligned(gate_up_scale, 4) || misaligned(down_scale, 4) || misaligned(weight, 4) ||
        misaligned(expert_offset, 4) || misaligned(route_row, 4) || misaligned(add, 2) || misaligned(y, 2))
        return CQ_ERR_ALIGNMENT;
    const int64_t R = T * top;
    const MoePlan p = moe_plan(E, R, H, I);
    if (workspace_bytes < p.total) return CQ_ERR_WORKSPACE;
    CQ_TRY(check_arch());
    cudaStream_t st = (cudaStream_t)stream;
    uint8_t *ws = (uint8_t *)workspace;
    float *xs = (float *)(ws + p.x_scale), *as = (float *)(ws + p.a_scale);
    uint16_t *h = (uint16_t *)(ws + p.h);
    const bool f16 = act_f16 != 0;
    // a token is quantised once, whatever the number of its routes
    CQ_TRY(wrap(launch_i8_quantize(x, dtype, ldx, I8Rows{nullptr, expert_offset, (int)E, T, T, T, route_row, top, R}, H, xs, ws + p.x, st)));
    CQ_TRY(wrap(launch_i8_gemm(gate_up, gate_up_scale, ws + p.x, xs, expert_offset, (int)E, h, R, 2 * I, H, f16, true, (int *)ws, st)));
    CQ_TRY(wrap(launch_i8_swiglu_quantize(h, dtype, 2 * I, routed_rows(nullptr, expert_offset, E, R, R), I, as, ws + p.a, st)));
    CQ_TRY(wrap(launch_i8_gemm(down, down_scale, ws + p.a, as, expert_offset, (int)E, h, R, H, I, f16, true, (int *)ws, st)));
    return wrap(launch_combine(h, H, R, weight, route_row, T, top, H, add, lda, y, ldy, f16, st));
}

int cq_debug_i8_plan(int64_t E, int64_t M, int64_t N, int64_t K, int quantised, int64_t *plan) {
    if (!plan || E < 0) return CQ_ERR_INVALID_ARG;
    const bool routed = E > 0;
    CQ_TRY(check_product(routed ? E : 1, routed, M, N, K));
    const bool own = !quantised && !routed && i8_few_ok(M, N, K);
    const I8Plan p = i8_plan(routed, M, N, K, own);
    plan[0] = p.channels; plan[1] = p.rows; plan[2] = p.runs; plan[3] = own;
    return CQ_OK;
}

}  // extern "C"
#pragma GCC visibility pop
