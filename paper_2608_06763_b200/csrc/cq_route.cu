// Routing to experts and back: the choice of experts from router logits with the map of their routes grouped by expert, and the weighted
// sum of a token's routes.  What lies between them are the products of routed rows.
#include <math_constants.h>

#include <algorithm>
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
    int lg_lanes, each;              // lanes to a group (log2), experts to a lane
    bool sigmoid, renormalise;
    float scale;
    int32_t *expert, *row, *token, *offset;
    float *weight;
    int32_t *counts;                 // [blocks][pitch]: routes of each block's tokens
    int pitch;                       // E, to a multiple of four
    int per_block;                   // tokens of a block
};

// Floats to integers of the same order, none of them 0, which stands for "not to be chosen".
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
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
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ int sum_up(int v) {   // of this lane and those in front
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(~0u, v, o);
        if ((int)(threadIdx.x & 31) >= o) v += u;
    }
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
__device__ __forceinline__ float clean(float v) { return fminf(fmaxf(v, -CUDART_INF_F), 3.402823466e38f) + 0.0f; }

// A warp has a token, a lane `each` neighbouring experts of one group.
struct Mine { int first, count; };   // expert, how many
__device__ __forceinline__ Mine mine_of(const Args &p, int lane) {
    const int g = lane >> p.lg_lanes, in = (lane & ((1 << p.lg_lanes) - 1)) * p.each, count = g < p.groups ? max(0, min(p.each, p.per - in)) : 0;
    return {count ? g * p.per + in : 0, count};
}

// the best two of a group, from those of its lanes
template <class F>
__device__ __forceinline__ void best_two_of_group(const Args &p, F &first, F &second) {
    for (int o = 1; o < 1 << p.lg_lanes; o <<= 1) {
        const F a = __shfl_xor_sync(~0u, first, o), b = __shfl_xor_sync(~0u, second, o);
        second = max(min(first, a), max(second, b));
        first = max(first, a);
    }
}

// What a warp puts its candidates into, in ascending order of experts, and the best of them in order.
constexpr int CANDIDATES = 32;
struct Candidates { float key[CANDIDATES]; uint32_t expert[CANDIDATES], best[CANDIDATES]; float logit[CANDIDATES]; double score[CANDIDATES]; };
// Where a value reaches the limit: it and its expert to the next place of `key` and `expert`, and a place further.
__device__ __forceinline__ void put(uint32_t &at, float key, float limit, uint32_t expert) {
    static_assert(CANDIDATES * 4 == 128, "from key to expert");
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ge.f32 p, %1, %2;\n\t@p st.shared.f32 [%0], %1;\n\t@p st.shared.u32 [%0 + 128], %3;\n\t@p add.u32 %0, %0, 4;\n\t}"
                 : "+r"(at) : "f"(key), "f"(limit), "r"(expert) : "memory");
}

// Choice scores in 64 bits, -inf of what may not be chosen; top: the row's largest logit.  The whole warp.
template <int V, int DT>
__device__ __forceinline__ void scores_in_64_bits(const Args &p, int64_t t, float top, float (&l)[V], double (&c)[V]) {
    const Mine m = mine_of(p, threadIdx.x & 31);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        l[i] = i < m.count ? clean(one_logit<DT>(p.logits, t * p.ldl + m.first + i)) : -CUDART_INF_F;
        c[i] = l[i] == -CUDART_INF_F ? 0.0 : p.sigmoid ? 1.0 / (1.0 + exp(-(double)l[i])) : exp((double)l[i] - (double)top);
        sum += c[i];
    }
    sum = warp_sum(sum);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (!p.sigmoid) c[i] /= sum;
        if (p.bias && i < m.count) c[i] += (double)p.bias[m.first + i];
        if (!(l[i] > -CUDART_INF_F && c[i] > -CUDART_INF)) c[i] = -CUDART_INF;
    }
}
// The choice in 64 bits among all experts of the groups that stay, for rows with more equals than there is room for.  Lane j returns the j-th
// expert (-1: none).
template <int V, int DT>
__device__ __noinline__ int choose_in_64_bits(const Args &p, int64_t t, float top, bool stays) {
    const int lane = threadIdx.x & 31;
    const Mine m = mine_of(p, lane);
    float l[V];
    double c[V];
    scores_in_64_bits<V, DT>(p, t, top, l, c);
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
// The candidates' choice scores in 64 bits, s.score, and their logits, s.logit; top: the row's largest logit.  The whole warp, a candidate to a lane.
template <int V, int DT>
__device__ __forceinline__ void score_candidates(const Args &p, int64_t t, float top, int all, Candidates &s) {
    const int lane = threadIdx.x & 31;
    const float l = lane < all ? clean(one_logit<DT>(p.logits, t * p.ldl + s.expert[lane])) : 0.0f;
    double c;
    if (p.sigmoid) {
        c = 1.0 / (1.0 + exp(-(double)l));
    } else {
        const Mine m = mine_of(p, lane);
        double sum = 0.0;
        for (int i = 0; i < m.count; ++i) {
            const float v = clean(one_logit<DT>(p.logits, t * p.ldl + m.first + i));
            if (v > -CUDART_INF_F) sum += exp((double)v - (double)top);
        }
        c = exp((double)l - (double)top) / warp_sum(sum);
    }
    if (lane < all) {
        s.score[lane] = p.bias ? c + (double)p.bias[s.expert[lane]] : c;
        s.logit[lane] = l;
    }
    __syncwarp();
}
// Their order in 64 bits, s.best, for rows whose choice among them 32 bits leave open.
template <int V, int DT>
__device__ __noinline__ void settle_in_64_bits(const Args &p, int64_t t, float top, int all, Candidates &s) {
    const int lane = threadIdx.x & 31;
    score_candidates<V, DT>(p, t, top, all, s);
    const double c = lane < all ? s.score[lane] : 0.0;
    const float l = lane < all ? s.logit[lane] : 0.0f;
    int ahead = 0;
    for (int j = 0; j < all; ++j) {
        const double cj = s.score[j];
        const float lj = s.logit[j];
        ahead += cj > c || (cj == c && (lj > l || (lj == l && j < lane)));
    }
    if (lane < all) s.best[ahead] = lane;
    __syncwarp();
}
// Whether a lane's group is among the `kept` best, from the totals of lanes g < groups in 64 bits.
__device__ __forceinline__ bool own_group_stays(const Args &p, double total) {
    const int lane = threadIdx.x & 31;
    int ahead = 0;
    for (int g = 0; g < p.groups; ++g) {
        const double o = __shfl_sync(~0u, total, g);
        ahead += o > total || (o == total && g < lane);
    }
    return __ballot_sync(~0u, lane < p.groups && total > -CUDART_INF && ahead < p.kept) >> (lane >> p.lg_lanes) & 1;
}
// The same for rows whose groups 32 bits leave open: the candidates hold all that may be among the best two of a group.
template <int V, int DT>
__device__ __noinline__ bool group_stays_by_candidates(const Args &p, int64_t t, float top, int all, Candidates &s) {
    const int lane = threadIdx.x & 31;
    score_candidates<V, DT>(p, t, top, all, s);
    double first = -CUDART_INF, second = -CUDART_INF;
    for (int j = 0; j < all; ++j)
        if ((int)s.expert[j] / p.per == lane) {
            second = max(second, min(first, s.score[j]));
            first = max(first, s.score[j]);
        }
    __syncwarp();
    return own_group_stays(p, p.best == 2 && second > -CUDART_INF ? first + second : first);
}
// Or all of them, where there are too many.
template <int V, int DT>
__device__ __noinline__ bool group_stays_in_64_bits(const Args &p, int64_t t, float top) {
    float l[V];
    double c[V], first = -CUDART_INF, second = -CUDART_INF;
    scores_in_64_bits<V, DT>(p, t, top, l, c);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        second = max(second, min(first, c[i]));
        first = max(first, c[i]);
    }
    best_two_of_group<double>(p, first, second);
    const double total = p.best == 2 && second > -CUDART_INF ? first + second : first;
    return own_group_stays(p, __shfl_sync(~0u, total, ((threadIdx.x & 31) << p.lg_lanes) & 31));
}

__device__ __forceinline__ float exp2_approx(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float reciprocal_approx(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }

// The choice of one token by one warp: lane j returns the j-th expert (-1: none) and its weight.
//
// Without a bias experts are in the order of their logits, which is exact.  Else choice scores are formed in 32 bits; where two that
// follow one another among the best `top` + 1 are closer than both may be off, the row is decided in 64 bits.  How far off, in u = 2^-24, with
// ex2.approx 4, rcp.approx 2 and log2(e) and its product 2 of the exponent: a sigmoid, s = 1 / (1 + e): of s (1 - s) 2 |l| + 4, which is 1.5 at most,
// and 3 for the sum and the reciprocal: 4.5.  A softmax, z = max - l: 3 z of e^-z, 1.1 at most, and, of itself, 4, the sum of E terms V + 5 <= 37
// with 3 times the mean of z <= ln E = 6.2 and 4, the reciprocal and the product 3: 68.  Adding the bias is off by |c| more, half a step of the sum.  Two choice scores are then
// out of order by 9 + 2 |c| or 136 + 2 |c| at most; what is taken, 16 + 4 |c| and 160 + 4 |c|, leaves room for the rounding of the comparison itself.
//
// The best: the (top + 1)-th largest of the lanes' largest is not above the (top + 1)-th largest of all, so what reaches it are candidates; hardly
// more than that many, since few lanes have two.  Each finds its place by counting those in front of it.  Many equals, or a large
// `top`, leave more candidates than there is room for: then the largest is taken out time and again.  8192 tokens to 8 of 256: 20 us, 36 with the latter alone.
// The logits of one lane as they are stored.  WIDE: `each` is V, and the rows allow wide loads.
template <int V, int DT, bool WIDE>
struct Raw {
    static constexpr int BYTES = V * (DT == DT_F32 ? 4 : 2), WORDS = WIDE ? BYTES / 4 : V;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const Args &p, int64_t t, const Mine &m) {
        const uint8_t *src = reinterpret_cast<const uint8_t *>(p.logits) + (t * p.ldl + m.first) * (DT == DT_F32 ? 4 : 2);
        constexpr uint32_t NONE = DT == DT_F32 ? 0xFF800000u : DT == DT_BF16 ? 0xFF80FF80u : 0xFC00FC00u;   // -inf
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = NONE;
        if constexpr (WIDE) {
            if (!m.count) return;
            if constexpr (BYTES >= 16) {
#pragma unroll
                for (int i = 0; i < WORDS; i += 4) {
                    const uint4 q = load16(src + 4 * i);
                    w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
                }
            } else if constexpr (BYTES == 8) {
                const uint2 q = *reinterpret_cast<const uint2 *>(src);
                w[0] = q.x; w[1] = q.y;
            } else {
                w[0] = *reinterpret_cast<const uint32_t *>(src);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < m.count) w[i] = DT == DT_F32 ? reinterpret_cast<const uint32_t *>(src)[i] : (uint32_t)reinterpret_cast<const uint16_t *>(src)[i];
        }
    }
    __device__ __forceinline__ float logit(int i) const {
        if constexpr (DT == DT_F32) return clean(__uint_as_float(w[i]));
        else return clean(WIDE ? value_of<DT>(w, i) : value_of<DT>(&w[i % WORDS], 0));
    }
};

template <int V, int DT, bool WIDE>
__device__ __forceinline__ int choose(const Args &p, int64_t t, const Mine &m, const float *bias, Candidates &s, float &weight) {
    const int lane = threadIdx.x & 31;
    constexpr float U = 5.9604645e-8f, LOG2E = 1.44269504f, LEAST = -3.402823466e38f;
    const float NONE = -CUDART_INF_F;   // not to be chosen; LEAST: the least of those that may be
    const bool scores = bias || p.groups > 1;
    float l[V], key[V], top, sum, rest;   // rest: how far two choice scores may be off, but for the part that grows with them
    bool stays;
    // Once; a second time where 32 bits left the groups open (whatever the first time had in registers need not outlive the call that decides).
    for (uint32_t decided = 0;;) {   // lanes whose groups stay
        {
            Raw<V, DT, WIDE> raw;
            raw.load(p, t, m);
#pragma unroll
            for (int i = 0; i < V; ++i) l[i] = raw.logit(i);
        }
        top = l[0];
#pragma unroll
        for (int i = 1; i < V; ++i) top = fmaxf(top, l[i]);
        top = warp_max(top);
        weight = 0.0f;
        if (top == NONE) return -1;

        sum = 1.0f; rest = 0.0f;
        stays = true;
        float c[V];
        if (scores || (!p.sigmoid && !p.renormalise)) {
            if (p.sigmoid) {
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] = reciprocal_approx(1.0f + exp2_approx(-LOG2E * l[i]));
                rest = 16.0f * U;
            } else {
                sum = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) { c[i] = exp2_approx(LOG2E * (l[i] - top)); sum += c[i]; }
                sum = warp_sum(sum);
                const float part = reciprocal_approx(sum);
#pragma unroll
                for (int i = 0; i < V; ++i) c[i] *= part;
                rest = 160.0f * U;
            }
        }
        if (scores) {
            if (bias) {   // has V values behind the last
                const float *mine = bias + m.first;
                if constexpr (WIDE && V % 4 == 0) {
#pragma unroll
                    for (int i = 0; i < V; i += 4) {
                        const float4 b = *reinterpret_cast<const float4 *>(mine + i);
                        c[i] += b.x; c[i + 1] += b.y; c[i + 2] += b.z; c[i + 3] += b.w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) c[i] += mine[i];
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) c[i] = l[i] > NONE ? c[i] : NONE;
            if (p.groups > 1 && decided) {
                stays = decided >> lane & 1;
            } else if (p.groups > 1) {
                float first = NONE, second = NONE;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    second = fmaxf(second, fminf(first, c[i]));
                    first = fmaxf(first, c[i]);
                }
                const float a = fabsf(first), b = fabsf(second);
                const float large = warp_max(fmaxf(a < CUDART_INF_F ? a : 0.0f, b < CUDART_INF_F ? b : 0.0f));
                best_two_of_group<float>(p, first, second);
                const float total = p.best == 2 ? 0.5f * first + (second > NONE ? 0.5f * second : 0.0f) : first;   // halves: the sum of two lowest numbers is none
                float left = lane < p.groups << p.lg_lanes ? total : NONE, least = NONE;
                stays = false;
                for (int g = 0; g < p.kept; ++g) {   // the best of those that are left; of equals the first
                    const float k = warp_max(left);
                    if (k == NONE) break;
                    least = k;
                    const int from = __ffs(__ballot_sync(~0u, left == k)) - 1;
                    if ((uint32_t)(lane - from) < 1u << p.lg_lanes) { stays = true; left = NONE; }
                }
                // Each of four halves is off by |c| / 2 (single scores by |c|), either sum by |c| again: 4 |c| for two groups, all that is taken, besides
                // what their scores are off (`rest` leaves room there).  What stays has to be that far above what does not.
                const float most = warp_max(left);
                if (most > NONE && !(least - most > rest + 4.0f * U * large)) {
                    const float near = fmaxf((p.best == 2 && second > NONE ? second : first) - rest - 4.0f * U * large, LEAST);
                    int count = 0;
#pragma unroll
                    for (int i = 0; i < V; ++i) count += c[i] >= near;
                    const int behind = sum_up(count), all = __shfl_sync(~0u, behind, 31);
                    if (all <= CANDIDATES) {
                        uint32_t at = tc::smem_u32(&s.key[behind - count]);
#pragma unroll
                        for (int i = 0; i < V; ++i) put(at, c[i], near, m.first + i);
                        __syncwarp();
                        stays = group_stays_by_candidates<V, DT>(p, t, top, all, s);
                    } else {
                        stays = group_stays_in_64_bits<V, DT>(p, t, top);
                    }
                    decided = __ballot_sync(~0u, stays);
                    continue;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = !stays ? NONE : bias ? c[i] : l[i];
        break;
    }

    const int rounds = bias ? min(p.top + 1, 32) : p.top;   // one more, to see how far it is from the last
    int chosen = -1, count = 0;
    bool open = false;
    float got = NONE, best = key[0], limit = NONE, logit = 0.0f;   // lane j: the key of the j-th; the best key that this lane still has
#pragma unroll
    for (int i = 1; i < V; ++i) best = fmaxf(best, key[i]);
    {
        float left = best;
#pragma unroll 4
        for (int j = 0; j < rounds; ++j) {
            limit = warp_max(left);
            if (left == limit) left = NONE;
        }
        if (bias) limit -= 2.0f * rest + 8.0f * U * fabsf(limit);   // and what may belong in front of the last
        limit = fmaxf(limit, LEAST);   // fewer lanes than that have any
    }
#pragma unroll
    for (int i = 0; i < V; ++i) count += key[i] >= limit;
    const int behind = sum_up(count), all = __shfl_sync(~0u, behind, 31);
    if (all <= CANDIDATES) {
        uint32_t at = tc::smem_u32(&s.key[behind - count]);
#pragma unroll
        for (int i = 0; i < V; ++i) put(at, key[i], limit, m.first + i);
        if (lane < 3 && all + lane < CANDIDATES) s.key[all + lane] = NONE;
        __syncwarp();
        const float mine = lane < all ? s.key[lane] : NONE;
        int ahead = __popc(__match_any_sync(~0u, __float_as_uint(mine)) & ((1u << lane) - 1u));   // of equals those in front: lower experts
        for (int j = 0; j < all; j += 4) {   // what lies behind the last is not larger
            const float4 k = *reinterpret_cast<const float4 *>(&s.key[j]);
            ahead += (k.x > mine) + (k.y > mine) + (k.z > mine) + (k.w > mine);
        }
        if (lane < all) s.best[ahead] = lane;
        __syncwarp();
        if (lane < min(all, rounds)) {
            const uint32_t from = s.best[lane];
            chosen = s.expert[from]; got = s.key[from];
            logit = bias ? clean(one_logit<DT>(p.logits, t * p.ldl + chosen)) : got;
        }
    } else {
        for (int j = 0; j < rounds; ++j) {
            const float k = warp_max(best);
            if (k == NONE) break;
            const int from = __ffs(__ballot_sync(~0u, best == k)) - 1;
            int which = 0;
            float lv = 0.0f;
#pragma unroll
            for (int i = V - 1; i >= 0; --i) if (key[i] == k) { which = i; lv = l[i]; }
            const int e = __shfl_sync(~0u, m.first + which, from);
            lv = __shfl_sync(~0u, lv, from);
            if (lane == j) { chosen = e; got = k; logit = lv; }
            if (lane == from) {
                best = NONE;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (i == which) key[i] = NONE;
                    best = fmaxf(best, key[i]);
                }
            }
        }
        if (bias) {   // of what is left none may lie in front of the last that is chosen
            const int last = __shfl_sync(~0u, chosen, p.top - 1);
            const float of_last = __shfl_sync(~0u, got, p.top - 1), logit_of_last = __shfl_sync(~0u, logit, p.top - 1);
            if (last >= 0) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    open |= key[i] > NONE && !(of_last - key[i] > rest + 4.0f * U * fmaxf(fabsf(of_last), fabsf(key[i]))) && !(l[i] == logit_of_last && bias[m.first + i] == bias[last]);
            }
        }
    }
    if (bias) {
        // Equal logits with equal biases are equal, and the lower index is first.  Where that holds of the last that is chosen and the first that is not, another one
        // behind them, as near or nearer, may lie in front of both.
        bool tied = false;
        const int next = __shfl_down_sync(~0u, chosen, 1);
        const float after = __shfl_down_sync(~0u, got, 1);
        const float l1 = __shfl_down_sync(~0u, logit, 1);
        if (lane + 1 < rounds && chosen >= 0 && next >= 0) {
            const bool equal = logit == l1 && bias[chosen] == bias[next];
            open |= !equal && !(got - after > rest + 4.0f * U * fmaxf(fabsf(got), fabsf(after)));
            tied = equal && lane + 1 == p.top;
        }
        if (all <= CANDIDATES && __any_sync(~0u, tied)) {   // with more of them that has been seen to
            const int last = __shfl_sync(~0u, chosen, p.top - 1);
            const float of_last = __shfl_sync(~0u, got, p.top - 1), logit_of_last = __shfl_sync(~0u, logit, p.top - 1);
            if (lane < all) {
                const int e = s.expert[lane];
                const float k = s.key[lane];
                open |= !(fabsf(of_last - k) > rest + 4.0f * U * fmaxf(fabsf(of_last), fabsf(k))) &&
                        !(clean(one_logit<DT>(p.logits, t * p.ldl + e)) == logit_of_last && bias[e] == bias[last]);
            }
        }
    }
    if (__any_sync(~0u, open)) {
        if (all <= CANDIDATES) {
            settle_in_64_bits<V, DT>(p, t, top, all, s);
            if (lane < min(all, p.top)) { chosen = s.expert[s.best[lane]]; logit = s.logit[s.best[lane]]; }
        } else {
            chosen = choose_in_64_bits<V, DT>(p, t, top, stays);
            if (chosen >= 0) logit = clean(one_logit<DT>(p.logits, t * p.ldl + chosen));
        }
    }
    __syncwarp();   // the candidates may be replaced
    const bool there = lane < p.top && chosen >= 0;
    if (!there) chosen = -1;
    // weights: over the sum of the chosen they do not depend on a common factor, so the largest logit is taken out where scores would vanish
    if (p.renormalise) {
        float large = warp_max(there ? logit : NONE);
        float w = 0.0f;
        if (p.sigmoid) {
            large = fminf(large, 0.0f);
            if (there) w = __fdividef(logit < 0.0f ? expf(logit - large) : 1.0f, 1.0f + expf(-fabsf(logit)));   // large is 0 where a logit is not negative
        } else if (there) {
            w = expf(logit - large);
        }
        const float all = warp_sum(w);
        if (there) weight = __fdividef(w, all) * p.scale;
    } else if (there) {
        weight = (p.sigmoid ? __fdividef(logit < 0.0f ? expf(logit) : 1.0f, 1.0f + expf(-fabsf(logit))) : __fdividef(expf(logit - top), sum)) * p.scale;
    }
    return chosen;
}

// ---------------------------------------------------------------- the map
// A block has `per_block` neighbouring tokens and takes CHUNK of them at a time, a warp one after another.  A bit for each token that chose an expert
// tells a route's place among those of its expert: the routes of tokens in front, in this chunk by counting bits, before it by a running
// count.  Nothing depends on the order in which warps come.  The places among all blocks' routes are added by place_kernel, or, where one block has
// all tokens, at once.
// Bound by latency: a token is 980 warp instructions (256 experts in groups), most of them in a chain of reductions, of which 28 warps hide half (55 % of the issue slots are taken).  8192
// tokens are 56 to a block, two for each warp one after the other: 19 to 20 us, some 10 of them in normal blocks; a row that 64 bits have to settle (six of them do) holds its block up by one to four, the
// second kernel takes four.  Their bytes would take 0.8.
constexpr int CHUNK = 128, PLACED = 2;   // PLACED: blocks of tokens whose routes one block of place_kernel places
// At least as many as there are experts.  More warps hide more of a token's 3 us, until registers get short: 256 experts, 8192 / 65536 tokens with 768 threads 20.0 / 85, 896 19.1 / 84.
constexpr int threads_for(int V) { return V <= 4 ? 1024 : V == 8 ? 896 : 512; }
static_assert(CHUNK % 32 == 0 && MAX_EXPERTS <= 512, "words of bits; a thread for each expert");

// Thread e's `count` routes: how many the experts in front have.  The whole block, at least E threads of it; all: of all experts; `sums`: 16 words of shared memory.
__device__ __forceinline__ int in_front(int count, int E, int *sums, int &all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (E + 31) >> 5;
    const int s = sum_up(count);
    if (lane == 31 && warp < warps) sums[warp] = s;
    __syncthreads();
    const int of = lane < warps ? sums[lane] : 0;
    all = __reduce_add_sync(~0u, of);
    return s - count + __reduce_add_sync(~0u, lane < warp ? of : 0);
}
static_assert(MAX_EXPERTS <= 16 * 32, "sums of the warps");

template <int V, int DT, bool WIDE>
__global__ void __launch_bounds__(threads_for(V)) route_kernel(const Args p) {
    extern __shared__ __align__(16) int s_mem[];
    __shared__ int s_sums[16];
    constexpr int W = CHUNK / 32, THREADS = threads_for(V), WARPS = THREADS / 32;
    Candidates *s_candidates = reinterpret_cast<Candidates *>(s_mem);   // [WARPS]
    uint32_t *s_bits = reinterpret_cast<uint32_t *>(s_candidates + WARPS);   // [E][W]
    float *s_bias = reinterpret_cast<float *>(s_bits + p.E * W);     // [E + V], 16-byte aligned
    int *s_run = reinterpret_cast<int *>(s_bias + p.E + V);          // [E]
    int16_t *s_chosen = reinterpret_cast<int16_t *>(s_run + p.E);    // [CHUNK][top]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int from = blockIdx.x * p.per_block, to = min(p.T, from + p.per_block);
    const Mine m = mine_of(p, lane);
    for (int i = threadIdx.x; i < p.E * W; i += THREADS) s_bits[i] = 0;
    for (int i = threadIdx.x; i < p.E; i += THREADS) s_run[i] = 0;
    tc::wait_for_previous_kernel();
    if (p.bias)
        for (int i = threadIdx.x; i < p.E; i += THREADS) s_bias[i] = fmaxf(p.bias[i], -CUDART_INF_F);   // NaN excludes as -inf does
    __syncthreads();
    for (int t0 = from; t0 < to; t0 += CHUNK) {
        const int n = min(CHUNK, to - t0);
        for (int i = warp; i < n; i += WARPS) {
            const int t = t0 + i;
            float weight;
            const int e = choose<V, DT, WIDE>(p, t, m, p.bias ? s_bias : nullptr, s_candidates[warp], weight);
            if (lane < p.top) {
                p.expert[t * p.top + lane] = e;
                p.weight[t * p.top + lane] = weight;
                s_chosen[i * p.top + lane] = (int16_t)e;
                if (e >= 0) atomicOr(&s_bits[e * W + (i >> 5)], 1u << (i & 31));
            }
        }
        __syncthreads();
        // where one block has all tokens, s_run becomes the first routes of the experts
        const int own = threadIdx.x;
        int mine = 0, last = 0;
        if (own < p.E) {
#pragma unroll
            for (int w = 0; w < W; ++w) mine += __popc(s_bits[own * W + w]);
        }
        if (gridDim.x == 1) {
            const int first = in_front(mine, p.E, s_sums, last);
            if (own < p.E) p.offset[own] = s_run[own] = first;
            if (own == 0) p.offset[p.E] = last;
            __syncthreads();
        }
        for (int i = threadIdx.x; i < n * p.top; i += THREADS) {
            const int tl = i / p.top, e = s_chosen[i];
            int at = -1;
            if (e >= 0) {
                at = s_run[e] + __popc(s_bits[e * W + (tl >> 5)] & ((1u << (tl & 31)) - 1u));
#pragma unroll
                for (int w = 0; w + 1 < W; ++w) at += w < tl >> 5 ? __popc(s_bits[e * W + w]) : 0;
                if (gridDim.x == 1) p.token[at] = t0 + tl;
            }
            p.row[t0 * p.top + i] = at;   // among this block's routes of the expert, or among all
            if (gridDim.x == 1 && i >= last) p.token[i] = -1;
        }
        if (gridDim.x == 1) return;
        __syncthreads();
        if (own < p.E) {
            s_run[own] += mine;
#pragma unroll
            for (int w = 0; w < W; ++w) s_bits[own * W + w] = 0;
        }
        __syncthreads();
    }
    for (int e = threadIdx.x; e < p.E; e += THREADS) p.counts[(int64_t)blockIdx.x * p.pitch + e] = s_run[e];
}

// The places of PLACED blocks' routes among all: those of experts in front, of the expert's in blocks in front, of the expert's in this block.
constexpr int SLICES = 16;
__global__ void __launch_bounds__(1024) place_kernel(const Args p, int blocks) {
    extern __shared__ __align__(16) int s_mem[];
    __shared__ int s_sums[16];
    // four experts to a thread, the blocks shared among `slices` of them
    const int quads = p.pitch / 4, slices = min(SLICES, 1024 / quads), quad = threadIdx.x % quads, slice = threadIdx.x / quads;
    int *s_all = s_mem, *s_before = s_all + slices * p.pitch, *s_base = s_before + slices * p.pitch;   // [slices][pitch] twice, [PLACED][pitch]
    tc::wait_for_previous_kernel();
    const int b0 = blockIdx.x * PLACED, own = min(PLACED, blocks - b0);
    const int of_block = p.per_block * p.top, from = b0 * of_block, to = min(p.T * p.top, from + own * of_block);   // routes: 2^30 at most, and blocks of 148 or more parts of them
    int i = from + threadIdx.x;
    int e = i < to ? p.expert[i] : -1, in = i < to ? p.row[i] : 0;   // on their way while the counts are added
    int mine[PLACED];
#pragma unroll
    for (int g = 0; g < PLACED; ++g) mine[g] = g + 1 < own && (int)threadIdx.x < p.E ? p.counts[(int64_t)(b0 + g) * p.pitch + threadIdx.x] : 0;
    if (slice < slices) {
        int4 all = make_int4(0, 0, 0, 0), before = all;
#pragma unroll 10
        for (int b = slice; b < blocks; b += slices) {
            const int4 c = *reinterpret_cast<const int4 *>(p.counts + (int64_t)b * p.pitch + quad * 4);
            all.x += c.x; all.y += c.y; all.z += c.z; all.w += c.w;
            if (b < b0) { before.x += c.x; before.y += c.y; before.z += c.z; before.w += c.w; }
        }
        *reinterpret_cast<int4 *>(s_all + slice * p.pitch + quad * 4) = all;
        *reinterpret_cast<int4 *>(s_before + slice * p.pitch + quad * 4) = before;
    }
    __syncthreads();
    int all = 0, base = 0, last;
    if ((int)threadIdx.x < p.E)
        for (int k = 0; k < slices; ++k) { all += s_all[k * p.pitch + threadIdx.x]; base += s_before[k * p.pitch + threadIdx.x]; }
    const int first = in_front(all, p.E, s_sums, last);
    base += first;
    if ((int)threadIdx.x < p.E) {
        if (blockIdx.x == 0) p.offset[threadIdx.x] = first;
#pragma unroll
        for (int g = 0; g < PLACED; ++g) { s_base[g * p.pitch + threadIdx.x] = base; base += mine[g]; }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offset[p.E] = last;
    __syncthreads();
    while (i < to) {
        if (e >= 0) {
            const int at = s_base[(PLACED == 2 ? i - from >= of_block : (i - from) / of_block) * p.pitch + e] + in;
            p.row[i] = at;
            p.token[at] = i / p.top;
        }
        if (i >= last) p.token[i] = -1;
        i += 1024;
        if (i < to) { e = p.expert[i]; in = p.row[i]; }
    }
}

// ---------------------------------------------------------------- the routes of a token together
// y[t] = add[t] + sum over j of weight[t][j] routes[row[t][j]], in fp32 and in the order of j, rounded once.  A thread takes VALUES neighbouring values of a token (as many as
// one load brings of rows that are so aligned), UNITS times; the loads of four routes are on their way together.  Rows outside [0, R) are no routes and are not read.  `add` may be
// y.  Bound by memory: 4096 tokens of 4096 values and eight routes 46.4 us, 6.5 TB/s (with divisions of a flat index by the row's length 49.5); of 4094 values 53.  Of 4095 79,
// bound by instructions: one value to a load, 55 M warp instructions where wide loads need 25, 64 % of the issue slots taken by 24 warps to an SM (their registers).
template <int VALUES> struct Some;
template <> struct Some<8> { using T = uint4; };
template <> struct Some<2> { using T = uint32_t; };
template <> struct Some<1> { using T = uint32_t; };
template <int VALUES>
__device__ __forceinline__ typename Some<VALUES>::T load_if(bool there, const uint16_t *p) {
    if constexpr (VALUES == 1) {   // as one predicated load: 16-bit registers would be packed in pairs, each load waited for
        uint32_t v;
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b16 h;\n\tsetp.ne.u32 p, %2, 0;\n\tmov.b16 h, 0;\n\t@p ld.global.b16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v) : "l"(p), "r"((uint32_t)there));
        return v;
    } else {
        using T = typename Some<VALUES>::T;
        return there ? *reinterpret_cast<const T *>(p) : T{};
    }
}
constexpr int units_for(int values) { return 8 / values; }
template <bool F16, int VALUES>
__global__ void __launch_bounds__(256) combine_kernel(const uint16_t *routes, int64_t ldr, int R, const float *weight, const int32_t *row, int T, int top, int N, const uint16_t *add, int64_t lda,
                                                      uint16_t *y, int64_t ldy) {
    tc::wait_for_previous_kernel();
    using S = typename Some<VALUES>::T;
    constexpr int DT = F16 ? DT_F16 : DT_BF16, BATCH = 4, UNITS = units_for(VALUES);
    const auto value = [](const S &s, int k) {
        if constexpr (VALUES == 8) { const uint32_t w[4] = {s.x, s.y, s.z, s.w}; return value_of<DT>(w, k); }
        else { const uint32_t w = s; return value_of<DT>(&w, k); }
    };
    const int t = blockIdx.x * blockDim.y + threadIdx.y;   // blocks of one token, or of several short ones
    if (t >= T) return;
    const int32_t *rows_of = row + t * top;
    const float *weights = weight + t * top;
    const int apart = blockDim.x * VALUES;   // from a unit to the next
    for (int c0 = threadIdx.x * VALUES; c0 < N; c0 += apart * UNITS) {
        float f[UNITS][VALUES];
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const bool with = add && c0 + u * apart < N;
            const S a = load_if<VALUES>(with, add + t * lda + c0 + u * apart);
#pragma unroll
            for (int k = 0; k < VALUES; ++k) f[u][k] = with ? value(a, k) : 0.0f;
        }
        for (int j0 = 0; j0 < top; j0 += BATCH) {
            S v[BATCH][UNITS];
            float w[BATCH];
            bool live[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int r = j0 + j < top ? rows_of[j0 + j] : -1;
                live[j] = r >= 0 && r < R;
                const uint16_t *from = routes + r * ldr + c0;
#pragma unroll
                for (int u = 0; u < UNITS; ++u) v[j][u] = load_if<VALUES>(live[j] && c0 + u * apart < N, from + u * apart);
                w[j] = live[j] ? weights[j0 + j] : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j)
                if (live[j]) {
#pragma unroll
                    for (int u = 0; u < UNITS; ++u)
#pragma unroll
                        for (int k = 0; k < VALUES; ++k) f[u][k] = fmaf(w[j], value(v[j][u], k), f[u][k]);
                }
        }
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (c0 + u * apart >= N) break;
            uint16_t *to = y + t * ldy + c0 + u * apart;
            if constexpr (VALUES == 8) *reinterpret_cast<uint4 *>(to) = make_uint4(pack16<DT>(f[u][0], f[u][1]), pack16<DT>(f[u][2], f[u][3]), pack16<DT>(f[u][4], f[u][5]), pack16<DT>(f[u][6], f[u][7]));
            else if constexpr (VALUES == 2) *reinterpret_cast<uint32_t *>(to) = pack16<DT>(f[u][0], f[u][1]);
            else *to = (uint16_t)pack16<DT>(f[u][0], 0.0f);
        }
    }
}

}  // namespace route

using namespace route;

// Blocks of tokens.  One block has all where there are few, and its launch is the only one: a round of its warps takes 4 us more the fuller it is, the
// second launch 3 (256 experts in groups, us alone / in two launches: 16 tokens 5.1 / 7.7, 32: 8.4 / 7.6, 64: 12.3 / 7.7).  Else as many blocks as SMs, of four tokens or more.
constexpr int ALONE = 16;
static_assert(ALONE <= CHUNK, "one chunk");
static int blocks_of(int64_t T) {
    if (T <= ALONE) return 1;
    const int64_t b = (T + 3) / 4, most = sm_count();
    return (int)(b < most ? b : most);
}
static int pitch_of(int64_t E) { return (int)((E + 3) / 4 * 4); }
size_t route_count_bytes(int64_t T, int64_t E) {
    const int64_t most = (T + 3) / 4 < 148 ? (T + 3) / 4 : sm_count() > 148 ? sm_count() : 148;
    return (size_t)(most * pitch_of(E)) * sizeof(int32_t);
}

cudaError_t launch_route(const RouteCall &c, cudaStream_t st) {
    Args p{};
    p.logits = c.logits; p.ldl = c.ldl; p.bias = c.bias;
    p.T = (int)c.T; p.E = c.E; p.groups = c.groups; p.per = c.E / c.groups; p.kept = c.kept; p.best = c.best; p.top = c.top;
    p.sigmoid = c.sigmoid; p.renormalise = c.renormalise; p.scale = c.scale;
    p.expert = c.expert; p.row = c.row; p.token = c.token; p.offset = c.offset; p.weight = c.weight; p.counts = c.counts; p.pitch = pitch_of(c.E);
    p.lg_lanes = 5;
    while (p.lg_lanes > 0 && c.groups << p.lg_lanes > 32) --p.lg_lanes;
    const int lanes = 1 << p.lg_lanes;
    p.each = (p.per + lanes - 1) / lanes;
    const int blocks = blocks_of(c.T);
    p.per_block = (int)((c.T + blocks - 1) / blocks);
    const int V = p.each <= 2 ? 2 : p.each <= 4 ? 4 : p.each <= 8 ? 8 : p.each <= 16 ? 16 : 32;
    const int size = c.dtype == DT_F32 ? 4 : 2, bytes = V * size, unit = bytes < 16 ? bytes : 16;
    const bool wide = V <= 8 && p.each == V && p.per == lanes * V && reinterpret_cast<uintptr_t>(c.logits) % unit == 0 && c.ldl * size % unit == 0;
    const unsigned threads = (unsigned)threads_for(V);
    const size_t smem = threads / 32 * sizeof(Candidates) + ((size_t)c.E * (CHUNK / 32 + 2) + V) * 4 + (size_t)CHUNK * c.top * 2;
    auto go = [&](auto kern) { return launch_overlapped(kern, dim3(blocks), threads, smem, st, 1, true, p); };
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
    return launch_overlapped(place_kernel, dim3((blocks + PLACED - 1) / PLACED), 1024u, (size_t)(2 * std::min(SLICES, 4096 / p.pitch) + PLACED) * p.pitch * 4, st, 1, true, p, blocks);
}

cudaError_t launch_combine(const uint16_t *routes, int64_t ldr, int64_t R, const float *weight, const int32_t *row, int64_t T, int top, int64_t N, const uint16_t *add,
                           int64_t lda, uint16_t *y, int64_t ldy, bool f16, cudaStream_t st) {
    const auto fits = [&](int values) {
        const auto row = [&](const void *q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % (2 * values) == 0 && ld % values == 0; };
        return N % values == 0 && row(routes, ldr) && row(y, ldy) && (!add || row(add, lda));
    };
    const int values = fits(8) ? 8 : fits(2) ? 2 : 1;
    const int64_t per = (N / values + units_for(values) - 1) / units_for(values);
    const int64_t rounds = (per + 255) / 256;   // even ones, of whole warps
    const unsigned across = (unsigned)((per + rounds - 1) / rounds + 31) / 32 * 32, tokens = 256 / across;
    auto go = [&](auto kern) {
        return launch_overlapped(kern, dim3((unsigned)((T + tokens - 1) / tokens)), dim3(across, tokens), 0, st, 1, true, routes, ldr, (int)R, weight, row, (int)T, top, (int)N, add, lda, y, ldy);
    };
    if (f16) return values == 8 ? go(combine_kernel<true, 8>) : values == 2 ? go(combine_kernel<true, 2>) : go(combine_kernel<true, 1>);
    return values == 8 ? go(combine_kernel<false, 8>) : values == 2 ? go(combine_kernel<false, 2>) : go(combine_kernel<false, 1>);
}

}  // namespace cq
