// Routing to experts and back: the choice of experts from router logits with the map of their routes grouped by expert, and the weighted
// sum of a token's routes.  What lies between them are the products of routed rows.
#include <math_constants.h>

#include <type_traits>

#include "cq_internal.h"
#include "cq_rows.cuh"
#include "cq_tc_ptx.cuh"

namespace cq {
namespace route {

using namespace rows;

struct Args {
    const void *logits;
    int64_t ldl;
    const float *bias;               // for the choice alone, or null
    int T, E, groups, per, kept, best, top;   // per: experts of a group; best: choice scores that make its score
    int lanes, each;                 // lanes to a group, experts to a lane
    bool sigmoid, renormalise;
    float scale;
    int32_t *expert, *row, *token, *offset;
    float *weight;
    int32_t *counts;                 // [blocks][E]: routes of each block's tokens
    int per_block;                   // tokens of a block
};

// Floats to integers of the same order, none of them 0, which stands for "not to be chosen".
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ uint64_t ordered(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return b ^ ((uint64_t)((int64_t)b >> 63) | 0x8000000000000000ull);
}
__device__ __forceinline__ uint64_t warp_max(uint64_t v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const uint64_t u = __shfl_xor_sync(~0u, v, o);
        if (u > v) v = u;
    }
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
template <int DT>
__device__ __forceinline__ float one_logit(const void *logits, int64_t at) {
    float v;
    if (DT == DT_F32) v = reinterpret_cast<const float *>(logits)[at];
    else if (DT == DT_BF16) v = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(logits)[at] << 16);
    else v = __half2float(reinterpret_cast<const __half *>(logits)[at]);
    return v;
}
// NaN becomes -inf (not to be chosen), +inf the largest number, -0 becomes 0 (equal logits have equal bits)
__device__ __forceinline__ float clean(float v) { return v > -CUDART_INF_F ? fminf(v, 3.402823466e38f) + 0.0f : -CUDART_INF_F; }

// A warp has a token, a lane `each` neighbouring experts of one group: group lane / lanes, from (lane % lanes) * each on.
struct Mine { int first, count; };   // expert, how many
__device__ __forceinline__ Mine mine_of(const Args &p, int lane) {
    const int g = lane / p.lanes, in = (lane - g * p.lanes) * p.each;
    return {g * p.per + in, g < p.groups ? max(0, min(p.each, p.per - in)) : 0};
}

// Which groups stay: a lane's group by its score (-inf: it has no expert to choose); `open` where the least that stays and the best that does not
// are closer than `margin`.
template <class F>
__device__ __forceinline__ bool group_stays(const Args &p, int lane, F total, F margin, bool &open) {
    const int own = lane / p.lanes;
    int ahead = 0;
    for (int g = 0; g < p.groups; ++g) {
        const F t = __shfl_sync(~0u, total, g * p.lanes);
        ahead += t > total || (t == total && g < own);
    }
    const bool any = own < p.groups && total > -CUDART_INF_F, stays = any && ahead < p.kept;
    F least = stays ? total : (F)CUDART_INF_F, most = any && !stays ? total : (F)-CUDART_INF_F;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        least = min(least, __shfl_xor_sync(~0u, least, o));
        most = max(most, __shfl_xor_sync(~0u, most, o));
    }
    open = most > -CUDART_INF_F && !(least - most > margin);
    return stays;
}
// the best two of a group, from those of its lanes
template <class F>
__device__ __forceinline__ F group_total(const Args &p, F first, F second) {
    for (int o = 1; o < p.lanes; o <<= 1) {
        const F a = __shfl_xor_sync(~0u, first, o), b = __shfl_xor_sync(~0u, second, o);
        second = max(min(first, a), max(second, b));
        first = max(first, a);
    }
    return p.best == 2 && second > -CUDART_INF_F ? first + second : first;
}

// The choice in 64 bits, for rows that 32 bits leave open.  Lane j returns the j-th expert (-1: none).
template <int V, int DT>
__device__ __noinline__ int choose_in_64_bits(const Args &p, int64_t t) {
    const int lane = threadIdx.x & 31;
    const Mine m = mine_of(p, lane);
    float l[V];
    double c[V];
    float top = -CUDART_INF_F;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        l[i] = i < m.count ? clean(one_logit<DT>(p.logits, t * p.ldl + m.first + i)) : -CUDART_INF_F;
        top = fmaxf(top, l[i]);
    }
    top = unordered(__reduce_max_sync(~0u, ordered(top)));
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        c[i] = l[i] == -CUDART_INF_F ? 0.0 : p.sigmoid ? 1.0 / (1.0 + exp(-(double)l[i])) : exp((double)l[i] - (double)top);
        sum += c[i];
    }
    sum = warp_sum(sum);
    double first = -CUDART_INF, second = -CUDART_INF;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (!p.sigmoid) c[i] /= sum;
        if (p.bias && i < m.count) c[i] += (double)p.bias[m.first + i];
        if (!(l[i] > -CUDART_INF_F && c[i] > -CUDART_INF)) c[i] = -CUDART_INF;
        second = max(second, min(first, c[i]));
        first = max(first, c[i]);
    }
    bool stays = true;
    if (p.groups > 1) {
        bool open;
        stays = group_stays<double>(p, lane, group_total<double>(p, first, second), 0.0, open);
    }
    uint32_t left = 0;   // experts that may still be taken
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (stays && c[i] > -CUDART_INF) left |= 1u << i;
    int chosen = -1;
    for (int j = 0; j < p.top; ++j) {
        uint64_t k = 0;
        uint32_t by = 0;
        int at = -1;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint64_t ki = ordered(c[i] + 0.0);
            const uint32_t li = ordered(l[i]);
            if ((left >> i & 1) && (ki > k || (ki == k && li > by))) { k = ki; by = li; at = i; }
        }
        const uint64_t best = warp_max(k);
        if (best == 0) break;
        const uint32_t logit = __reduce_max_sync(~0u, k == best ? by : 0u);
        const int from = __ffs(__ballot_sync(~0u, k == best && by == logit)) - 1;
        const int e = __shfl_sync(~0u, m.first + at, from);
        if (lane == j) chosen = e;
        if (lane == from) left &= ~(1u << at);
    }
    return chosen;
}

// The choice of one token by one warp: lane j returns the j-th expert (-1: none) and its weight.
//
// Without a bias experts are in the order of their logits, which is exact.  Else choice scores are formed in 32 bits; where two that
// follow one another among the best `top` + 1 are closer than both may be off, the row is decided in 64 bits.  How far off, in 2^-24:
// a sigmoid, of itself: expf 4, the sum 1, the division 1.  A softmax: l - max rounds by z = max - l of e^-z, at most 0.37 of the whole, expf
// 4, the sum of E terms V + 5 <= 37 and the mean of their z <= ln E = 6.2 and expf's 4, the division 1: 53.  The bias adds |c| / 2.
template <int V, int DT, bool WIDE>
__device__ __forceinline__ int choose(const Args &p, int64_t t, const float *bias, float &weight) {
    const int lane = threadIdx.x & 31;
    const Mine m = mine_of(p, lane);
    float l[V];
    if (WIDE) {   // `each` is V, and the rows allow it
        constexpr int BYTES = V * (DT == DT_F32 ? 4 : 2), WORDS = BYTES / 4;
        uint32_t w[WORDS];
        const uint8_t *src = reinterpret_cast<const uint8_t *>(p.logits) + (t * p.ldl + m.first) * (DT == DT_F32 ? 4 : 2);
        if (m.count) {
            if (BYTES >= 16) {
#pragma unroll
                for (int i = 0; i < WORDS; i += 4) {
                    const uint4 q = load16(src + 4 * i);
                    w[i] = q.x; w[(i + 1) % WORDS] = q.y; w[(i + 2) % WORDS] = q.z; w[(i + 3) % WORDS] = q.w;
                }
            } else if (BYTES == 8) {
                const uint2 q = *reinterpret_cast<const uint2 *>(src);
                w[0] = q.x; w[1 % WORDS] = q.y;
            } else {
                w[0] = *reinterpret_cast<const uint32_t *>(src);
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = m.count ? clean(DT == DT_F32 ? __uint_as_float(w[i % WORDS]) : value_of<DT == DT_F32 ? DT_BF16 : DT>(w, DT == DT_F32 ? 0 : i)) : -CUDART_INF_F;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) l[i] = i < m.count ? clean(one_logit<DT>(p.logits, t * p.ldl + m.first + i)) : -CUDART_INF_F;
    }
    float top = l[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, l[i]);
    top = unordered(__reduce_max_sync(~0u, ordered(top)));
    weight = 0.0f;
    if (top == -CUDART_INF_F) return -1;

    const bool scores = p.bias || p.groups > 1, whole = !p.sigmoid && (scores || !p.renormalise);
    float sum = 1.0f;
    uint32_t key[V];
    bool stays = true, open = false;
    float rest = 0.0f;   // how far two choice scores may be off, but for the part that grows with them
    if (scores || whole) {
        float s[V];
        if (p.sigmoid) {
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = __fdiv_rn(1.0f, 1.0f + expf(-l[i]));
            rest = 16.0f * 5.9604645e-8f;
        } else {
            sum = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) { s[i] = expf(l[i] - top); sum += s[i]; }
            sum = warp_sum(sum);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = __fdiv_rn(s[i], sum);
            rest = 128.0f * 5.9604645e-8f;
        }
        if (scores) {
            float first = -CUDART_INF_F, second = -CUDART_INF_F;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (bias && i < m.count) s[i] += bias[m.first + i];
                if (!(l[i] > -CUDART_INF_F && s[i] > -CUDART_INF_F)) s[i] = -CUDART_INF_F;
                second = fmaxf(second, fminf(first, s[i]));
                first = fmaxf(first, s[i]);
            }
            if (p.groups > 1) {
                const float total = group_total<float>(p, first, second);
                // each of four choice scores is off by |c| / 2 more, their sums by as much again: 8 |c| in units of 2^-24
                const float a = fabsf(first), b = fabsf(second);
                const float large = unordered(__reduce_max_sync(~0u, ordered(fmaxf(a < CUDART_INF_F ? a : 0.0f, b < CUDART_INF_F ? b : 0.0f))));
                stays = group_stays<float>(p, lane, total, 2.0f * rest + 4.7683716e-7f * large, open);
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = stays && (!scores || s[i] > -CUDART_INF_F) ? ordered(bias ? s[i] + 0.0f : l[i]) : 0u;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = ordered(l[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) if (l[i] == -CUDART_INF_F) key[i] = 0u;

    int chosen = -1;
    uint32_t got = 0, best = 0;   // lane j: the key of the j-th; the best key that this lane still has
    float logit = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) best = max(best, key[i]);
    const int rounds = p.bias ? min(p.top + 1, 32) : p.top;   // one more, to see how far it is from the last
    for (int j = 0; j < rounds; ++j) {
        const uint32_t k = __reduce_max_sync(~0u, best);
        if (k == 0) break;
        const int from = __ffs(__ballot_sync(~0u, best == k)) - 1;
        int at = 0;
        float lv = 0.0f;
#pragma unroll
        for (int i = V - 1; i >= 0; --i) if (key[i] == k) { at = i; lv = l[i]; }
        const int e = __shfl_sync(~0u, m.first + at, from);
        lv = __shfl_sync(~0u, lv, from);
        if (lane == j) { chosen = e; got = k; logit = lv; }
        if (lane == from) {
            best = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i == at) key[i] = 0;
                best = max(best, key[i]);
            }
        }
    }
    if (p.bias) {
        // equal logits with equal biases are equal, and the lower index is first
        const int next = __shfl_down_sync(~0u, chosen, 1);
        const uint32_t after = __shfl_down_sync(~0u, got, 1);
        const float l1 = __shfl_down_sync(~0u, logit, 1);
        if (lane + 1 < rounds && chosen >= 0 && next >= 0) {
            const float a = unordered(got), b = unordered(after);
            const bool equal = logit == l1 && bias[chosen] == bias[next];
            open |= !equal && !(a - b > rest + 2.3841858e-7f * fmaxf(fabsf(a), fabsf(b)));
        }
        // all of 32 were wanted: what follows the last is in nobody's hands
        if (rounds == p.top) open |= __reduce_max_sync(~0u, best) != 0;
    }
    if (__any_sync(~0u, open)) {
        chosen = choose_in_64_bits<V, DT>(p, t);
        if (chosen >= 0) logit = clean(one_logit<DT>(p.logits, t * p.ldl + chosen));
    }
    const bool there = lane < p.top && chosen >= 0;
    if (!there) chosen = -1;
    // weights: over the sum of the chosen they do not depend on a common factor, so the largest logit is taken out where scores would vanish
    if (p.renormalise) {
        float large = unordered(__reduce_max_sync(~0u, there ? ordered(logit) : 0u));
        float w = 0.0f;
        if (p.sigmoid) {
            large = fminf(large, 0.0f);
            if (there) w = logit < 0.0f ? __fdiv_rn(expf(logit - large), 1.0f + expf(logit)) : __fdiv_rn(expf(-large), 1.0f + expf(-logit));
        } else if (there) {
            w = expf(logit - large);
        }
        const float all = warp_sum(w);
        if (there) weight = __fdiv_rn(w, all) * p.scale;
    } else if (there) {
        weight = (p.sigmoid ? __fdiv_rn(1.0f, 1.0f + expf(-logit)) : __fdiv_rn(expf(logit - top), sum)) * p.scale;
    }
    return chosen;
}

// ---------------------------------------------------------------- the map
// A block has `per_block` neighbouring tokens and takes CHUNK of them at a time, a warp one after another.  A bit for each token that chose an expert
// tells a route's place among those of its expert: the routes of tokens in front, in this chunk by counting bits, before it by a running
// count.  Nothing depends on the order in which warps come.  The places among all blocks' routes are added by place_kernel, or, where one block has
// all tokens, at once.
constexpr int CHUNK = 64, THREADS = 512;
static_assert(CHUNK % 32 == 0, "words of bits");

// first route of each expert (E + 1 values), from their counts; the first warp of the block, all of it
__device__ __forceinline__ void scan_counts(const int *counts, int E, int *first) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int n = e0 + lane < E ? counts[e0 + lane] : 0;
        int s = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int u = __shfl_up_sync(~0u, s, o);
            if (lane >= o) s += u;
        }
        if (e0 + lane < E) first[e0 + lane] = before + s - n;
        before += __shfl_sync(~0u, s, 31);
    }
    if (lane == 0) first[E] = before;
}

template <int V, int DT, bool WIDE>
__global__ void __launch_bounds__(THREADS) route_kernel(const Args p) {
    extern __shared__ int s_mem[];
    constexpr int W = CHUNK / 32;
    uint32_t *s_bits = reinterpret_cast<uint32_t *>(s_mem);          // [E][W]
    int *s_run = s_mem + p.E * W, *s_first = s_run + p.E;            // [E], [E + 1]
    float *s_bias = reinterpret_cast<float *>(s_first + p.E + 1);    // [E]
    int16_t *s_chosen = reinterpret_cast<int16_t *>(s_bias + p.E);   // [CHUNK][top]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = THREADS / 32;
    const int from = blockIdx.x * p.per_block, to = min(p.T, from + p.per_block);
    for (int i = threadIdx.x; i < p.E * W; i += THREADS) s_bits[i] = 0;
    for (int i = threadIdx.x; i < p.E; i += THREADS) s_run[i] = 0;
    tc::wait_for_previous_kernel();
    if (p.bias) for (int i = threadIdx.x; i < p.E; i += THREADS) s_bias[i] = p.bias[i];
    __syncthreads();
    for (int t0 = from; t0 < to; t0 += CHUNK) {
        const int n = min(CHUNK, to - t0);
        for (int i = warp; i < n; i += warps) {
            const int64_t t = t0 + i;
            float weight;
            const int e = choose<V, DT, WIDE>(p, t, p.bias ? s_bias : nullptr, weight);
            if (lane < p.top) {
                p.expert[t * p.top + lane] = e;
                p.weight[t * p.top + lane] = weight;
                s_chosen[i * p.top + lane] = (int16_t)e;
                if (e >= 0) atomicOr(&s_bits[e * W + (i >> 5)], 1u << (i & 31));
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n * p.top; i += THREADS) {
            const int tl = i / p.top, e = s_chosen[i];
            int at = -1;
            if (e >= 0) {
                at = s_run[e] + __popc(s_bits[e * W + (tl >> 5)] & ((1u << (tl & 31)) - 1u));
                for (int w = 0; w < tl >> 5; ++w) at += __popc(s_bits[e * W + w]);
            }
            p.row[(int64_t)t0 * p.top + i] = at;   // among this block's routes of the expert
        }
        __syncthreads();
        for (int e = threadIdx.x; e < p.E; e += THREADS) {
            int c = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) { c += __popc(s_bits[e * W + w]); s_bits[e * W + w] = 0; }
            s_run[e] += c;
        }
        __syncthreads();
    }
    if (gridDim.x > 1) {
        for (int e = threadIdx.x; e < p.E; e += THREADS) p.counts[(int64_t)blockIdx.x * p.E + e] = s_run[e];
        return;
    }
    if (warp == 0) scan_counts(s_run, p.E, s_first);
    __syncthreads();
    for (int e = threadIdx.x; e <= p.E; e += THREADS) p.offset[e] = s_first[e];
    const int R = p.T * p.top, last = s_first[p.E];
    for (int i = threadIdx.x; i < R; i += THREADS) {
        const int e = p.expert[i];   // of this block's own writes
        if (e >= 0) {
            const int at = s_first[e] + p.row[i];
            p.row[i] = at;
            p.token[at] = i / p.top;
        }
        if (i >= last) p.token[i] = -1;
    }
}

__global__ void __launch_bounds__(THREADS) place_kernel(const Args p) {
    extern __shared__ int s_mem[];
    int *s_all = s_mem, *s_before = s_all + p.E, *s_first = s_before + p.E;   // [E], [E], [E + 1]
    for (int i = threadIdx.x; i < 2 * p.E; i += THREADS) s_mem[i] = 0;
    tc::wait_for_previous_kernel();
    __syncthreads();
    // parts of the blocks by `slices` teams of threads, an expert to a thread
    const int width = (p.E + 31) / 32 * 32, slices = max(1, THREADS / width), blocks = gridDim.x;
    for (int e = threadIdx.x % width, s = threadIdx.x / width; s < slices && e < p.E; e += width) {
        const int b0 = (int)((int64_t)blocks * s / slices), b1 = (int)((int64_t)blocks * (s + 1) / slices);
        int all = 0, before = 0;
#pragma unroll 8
        for (int b = b0; b < b1; ++b) {
            const int c = p.counts[(int64_t)b * p.E + e];
            all += c;
            before += b < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&s_all[e], all);
        atomicAdd(&s_before[e], before);
    }
    __syncthreads();
    if (threadIdx.x < 32) scan_counts(s_all, p.E, s_first);
    __syncthreads();
    if (blockIdx.x == 0) for (int e = threadIdx.x; e <= p.E; e += THREADS) p.offset[e] = s_first[e];
    const int64_t from = (int64_t)blockIdx.x * p.per_block * p.top, to = min((int64_t)p.T * p.top, from + (int64_t)p.per_block * p.top);
    const int last = s_first[p.E];
    for (int64_t i = from + threadIdx.x; i < to; i += THREADS) {
        const int e = p.expert[i];
        if (e >= 0) {
            const int at = s_first[e] + s_before[e] + p.row[i];
            p.row[i] = at;
            p.token[at] = (int)(i / p.top);
        }
        if (i >= last) p.token[i] = -1;
    }
}

// ---------------------------------------------------------------- the routes of a token together
// y[t] = add[t] + sum over j of weight[t][j] routes[row[t][j]], in fp32 and in the order of j, rounded once.  A thread takes eight (one) values of a token.
// Rows outside [0, R) are no routes and are not read.  `add` may be y.
template <bool F16, bool WIDE>
__global__ void __launch_bounds__(256) combine_kernel(const uint16_t *routes, int64_t ldr, int64_t R, const float *weight, const int32_t *row, int64_t T, int top, int64_t N,
                                                      const uint16_t *add, int64_t lda, uint16_t *y, int64_t ldy) {
    tc::wait_for_previous_kernel();
    constexpr int DT = F16 ? DT_F16 : DT_BF16, BATCH = 4;
    const int64_t per = WIDE ? N / 8 : N, total = T * per;
    for (int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x; idx < total; idx += (int64_t)gridDim.x * 256) {
        const int64_t t = idx / per, c = idx - t * per;
        const int32_t *rows_of = row + t * top;
        const float *weights = weight + t * top;
        if (WIDE) {
            float f[8];
            uint4 a = make_uint4(0, 0, 0, 0);
            if (add) a = load16(add + t * lda + c * 8);
            const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = add ? value_of<DT>(aw, k) : 0.0f;
            for (int j0 = 0; j0 < top; j0 += BATCH) {
                uint4 v[BATCH];
                float w[BATCH];
                bool live[BATCH];
#pragma unroll
                for (int j = 0; j < BATCH; ++j) {
                    const int64_t r = j0 + j < top ? rows_of[j0 + j] : -1;
                    live[j] = r >= 0 && r < R;
                    v[j] = live[j] ? load16(routes + r * ldr + c * 8) : make_uint4(0, 0, 0, 0);
                    w[j] = live[j] ? weights[j0 + j] : 0.0f;
                }
#pragma unroll
                for (int j = 0; j < BATCH; ++j)
                    if (live[j]) {
                        const uint32_t vw[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] = fmaf(w[j], value_of<DT>(vw, k), f[k]);
                    }
            }
            *reinterpret_cast<uint4 *>(y + t * ldy + c * 8) = make_uint4(pack16<DT>(f[0], f[1]), pack16<DT>(f[2], f[3]), pack16<DT>(f[4], f[5]), pack16<DT>(f[6], f[7]));
        } else {
            float f = 0.0f;
            if (add) { const uint32_t w = add[t * lda + c]; f = value_of<DT>(&w, 0); }
            for (int j = 0; j < top; ++j) {
                const int64_t r = rows_of[j];
                if (r >= 0 && r < R) { const uint32_t w = routes[r * ldr + c]; f = fmaf(weights[j], value_of<DT>(&w, 0), f); }
            }
            y[t * ldy + c] = (uint16_t)pack16<DT>(f, 0.0f);
        }
    }
}

}  // namespace route

using namespace route;

// Tokens of a block, and blocks: all SMs have some; one block has all where there are few.
static int blocks_of(int64_t T) {
    if (T <= CHUNK) return 1;
    const int64_t b = (T + 31) / 32, most = sm_count();
    return (int)(b < most ? b : most);
}
size_t route_count_bytes(int64_t T, int64_t E) {
    const int64_t most = (T + 31) / 32 < 148 ? (T + 31) / 32 : sm_count() > 148 ? sm_count() : 148;
    return (size_t)(most * E) * sizeof(int32_t);
}

cudaError_t launch_route(const RouteCall &c, cudaStream_t st) {
    Args p{};
    p.logits = c.logits; p.ldl = c.ldl; p.bias = c.bias;
    p.T = (int)c.T; p.E = c.E; p.groups = c.groups; p.per = c.E / c.groups; p.kept = c.kept; p.best = c.best; p.top = c.top;
    p.sigmoid = c.sigmoid; p.renormalise = c.renormalise; p.scale = c.scale;
    p.expert = c.expert; p.row = c.row; p.token = c.token; p.offset = c.offset; p.weight = c.weight; p.counts = c.counts;
    p.lanes = 32;
    while (p.lanes > 1 && p.lanes * c.groups > 32) p.lanes >>= 1;
    p.each = (p.per + p.lanes - 1) / p.lanes;
    const int blocks = blocks_of(c.T);
    p.per_block = (int)((c.T + blocks - 1) / blocks);
    const int V = p.each <= 2 ? 2 : p.each <= 4 ? 4 : p.each <= 8 ? 8 : p.each <= 16 ? 16 : 32;
    const int size = c.dtype == DT_F32 ? 4 : 2, bytes = V * size, unit = bytes < 16 ? bytes : 16;
    const bool wide = V <= 8 && p.each == V && p.per == p.lanes * V && reinterpret_cast<uintptr_t>(c.logits) % unit == 0 && c.ldl * size % unit == 0;
    const size_t smem = ((size_t)c.E * (CHUNK / 32 + 3) + 1) * 4 + (size_t)CHUNK * c.top * 2;
    auto go = [&](auto kern) { return launch_overlapped(kern, dim3(blocks), (unsigned)THREADS, smem, st, 1, true, p); };
    auto with = [&](auto v, auto dt) {
        constexpr int VV = decltype(v)::value, DT = decltype(dt)::value;
        return wide ? go(route_kernel<VV, DT, VV <= 8>) : go(route_kernel<VV, DT, false>);
    };
    auto of = [&](auto v) {
        return c.dtype == DT_F32 ? with(v, std::integral_constant<int, DT_F32>{}) : c.dtype == DT_F16 ? with(v, std::integral_constant<int, DT_F16>{})
                                                                                                      : with(v, std::integral_constant<int, DT_BF16>{});
    };
    cudaError_t e;
    switch (V) {
        case 2: e = of(std::integral_constant<int, 2>{}); break;
        case 4: e = of(std::integral_constant<int, 4>{}); break;
        case 8: e = of(std::integral_constant<int, 8>{}); break;
        case 16: e = of(std::integral_constant<int, 16>{}); break;
        default: e = of(std::integral_constant<int, 32>{}); break;
    }
    if (e != cudaSuccess || blocks == 1) return e;
    return launch_overlapped(place_kernel, dim3(blocks), (unsigned)THREADS, (size_t)(3 * c.E + 1) * 4, st, 1, true, p);
}

cudaError_t launch_combine(const uint16_t *routes, int64_t ldr, int64_t R, const float *weight, const int32_t *row, int64_t T, int top, int64_t N, const uint16_t *add,
                           int64_t lda, uint16_t *y, int64_t ldy, bool f16, cudaStream_t st) {
    const auto odd = [](const void *q, int64_t ld) { return (reinterpret_cast<uintptr_t>(q) & 15u) != 0 || ld % 8 != 0; };
    const bool wide = N % 8 == 0 && !odd(routes, ldr) && !odd(y, ldy) && !(add && odd(add, lda));
    const int64_t blocks = (T * (wide ? N / 8 : N) + 255) / 256, most = 16 * (int64_t)sm_count();
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3((unsigned)(blocks < most ? blocks : most)), 256u, 0, st, 1, true, routes, ldr, R, weight, row, T, top, N, add, lda, y, ldy);
    };
    if (f16) return wide ? go(combine_kernel<true, true>) : go(combine_kernel<true, false>);
    return wide ? go(combine_kernel<false, true>) : go(combine_kernel<false, false>);
}

}  // namespace cq
