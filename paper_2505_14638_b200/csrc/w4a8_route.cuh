// Routing of tokens to experts: the choice of top_k experts from router logits, their weights, and the order of the rows by
// expert that the experts' products read.
//
// Two launches (one where a single CTA holds all tokens).  route_choose_kernel: a warp per token, V = experts / 32 keys per lane;
// the CTA then counts its tokens' experts and numbers the rows of each expert in the order of the tokens.  route_place_kernel:
// every CTA sums the counts of the CTAs before it (at most kRouteChunks rows of counts, from L2) and turns the numbers into
// rows.  No atomics on global memory: the order never varies.
//
// The choice: without a bias and with groups judged by their best expert, scores have the order of the logits, whose 32 bits are
// the keys.  Otherwise a key is score + bias in FP64: in FP32 two experts whose keys differ by less than a rounding would
// change places.
#pragma once

#include <cuda_bf16.h>

#include "w4a8_common.cuh"
#include "w4a8_ptx.cuh"

namespace w4a8 {

constexpr int kRouteMaxExperts = 512, kRouteMaxTopK = 32, kRouteMaxGroups = 32;
constexpr int kRouteWarps = 16;      // tokens that a CTA works on at a time
constexpr int kRouteChunks = 148;    // CTAs at most

struct RouteParams {
    const void* logits;
    int64_t ldl;
    const float* bias;
    int32_t *ids, *offsets, *slots;
    float* weights;
    uint32_t* counts;   // [chunks][E]
    int64_t M;
    int E, top_k, groups, top_groups, group_best, chunk, chunks;
    int logits_fp32, sigmoid, renormalize;
    float scale;
};

// Keys whose order as unsigned integers is that of the values; 0 is left for experts that cannot be chosen.
__device__ __forceinline__ uint64_t order_key(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // (-0 becomes 0)
    return b ^ ((b >> 63) ? 0xFFFFFFFFFFFFFFFFull : 0x8000000000000000ull);
}
__device__ __forceinline__ uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ double key_value(uint64_t k) {
    return __longlong_as_double((long long)(k ^ ((k >> 63) ? 0x8000000000000000ull : 0xFFFFFFFFFFFFFFFFull)));
}
__device__ __forceinline__ uint32_t warp_max(uint32_t k) { return __reduce_max_sync(0xFFFFFFFFu, k); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
    const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}

__device__ __forceinline__ float route_logit(const RouteParams& p, int64_t at) {
    return p.logits_fp32 ? __ldg(static_cast<const float*>(p.logits) + at)
                         : __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(p.logits) + at) << 16);
}

// exp(x - most), with x == most exact also at infinity.
__device__ __forceinline__ double route_exp(double x, double most) { return x == most ? 1.0 : exp(x - most); }

// Row offsets of the experts from their counts, exclusive, by the first warp; total[e] in, first[e] out, first[E] = all rows.
__device__ __forceinline__ void route_offsets(const uint32_t* total, uint32_t* first, int E) {
    const int lane = threadIdx.x & 31;
    uint32_t base = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const uint32_t own = e0 + lane < E ? total[e0 + lane] : 0u;
        uint32_t sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += before;
        }
        if (e0 + lane < E) first[e0 + lane] = base + sum - own;
        base += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    if (lane == 0) first[E] = base;
}

template <int V, typename Key>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_choose_kernel(const RouteParams p) {
    constexpr bool WIDE = sizeof(Key) == 8;
    __shared__ uint32_t count[kRouteMaxExperts], first[kRouteMaxExperts + 1];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int E = p.E, k = p.top_k, size = E / p.groups;
    const int64_t m0 = (int64_t)blockIdx.x * p.chunk, m1 = min(p.M, m0 + p.chunk);
    for (int e = threadIdx.x; e < E; e += kRouteWarps * 32) count[e] = 0u;

    for (int64_t m = m0 + warp; m < m1; m += kRouteWarps) {
        float x[V];
        float most = -INFINITY;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = lane + 32 * i;
            x[i] = e < E ? route_logit(p, m * p.ldl + e) : -INFINITY;
            if (x[i] != x[i]) x[i] = -INFINITY;   // (a NaN is never chosen and has no part in the others' scores)
            most = fmaxf(most, x[i]);
        }
        float sum = 0.0f;
        double sum64 = 0.0;
        if (!p.sigmoid) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        }
        Key key[V];
        if constexpr (WIDE) {
            double s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (p.sigmoid) {
                    s[i] = 1.0 / (1.0 + exp(-(double)x[i]));
                } else {
                    s[i] = x[i] == -INFINITY ? 0.0 : route_exp((double)x[i], (double)most);
                    sum64 += s[i];
                }
            }
            if (!p.sigmoid) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum64 += __shfl_xor_sync(0xFFFFFFFFu, sum64, o);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = lane + 32 * i;
                double v = p.sigmoid ? s[i] : s[i] / sum64;
                if (p.bias != nullptr && e < E) v += (double)__ldg(p.bias + e);
                key[i] = x[i] == -INFINITY || !(v > -(double)INFINITY) ? 0 : order_key(v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) key[i] = x[i] == -INFINITY ? 0 : order_key(x[i]);
            if (!p.sigmoid && !p.renormalize) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum += x[i] == -INFINITY ? 0.0f : (x[i] == most ? 1.0f : expf(x[i] - most));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                sum64 = sum;
            }
        }

        if (p.groups > 1) {
            // Lane g judges group g: the sum of the group_best highest keys, lowest where one of them cannot be chosen.
            Key score = 0;
            for (int g = 0; g < p.groups; ++g) {
                Key best = 0, second = 0;   // this lane's in the group
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int e = lane + 32 * i;
                    if (e < g * size || e >= (g + 1) * size) continue;
                    if (key[i] > best) {
                        second = best;
                        best = key[i];
                    } else if (key[i] > second) {
                        second = key[i];
                    }
                }
                const Key top = warp_max(best);
                Key mine = top;
                if constexpr (WIDE) {
                    if (p.group_best == 2 && size > 1) {
                        const unsigned holds = __ballot_sync(0xFFFFFFFFu, best == top);
                        const Key next = warp_max(lane == __ffs((int)holds) - 1 ? second : best);
                        mine = top == 0 || next == 0 ? 0 : order_key(key_value(top) + key_value(next));
                    }
                }
                if (lane == g) score = mine;
            }
            int before = 0;   // groups that come before this lane's
            for (int g = 0; g < p.groups; ++g) {
                const Key other = __shfl_sync(0xFFFFFFFFu, score, g);
                before += other > score || (other == score && g < lane) ? 1 : 0;
            }
            const unsigned kept = __ballot_sync(0xFFFFFFFFu, lane < p.groups && before < p.top_groups);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int e = lane + 32 * i;
                if (e < E && !(kept >> (e / size) & 1u)) key[i] = 0;
            }
        }

        int id = -1;   // lane j keeps the j-th choice
        for (int j = 0; j < k; ++j) {
            Key best = 0;
            int at = 0;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (key[i] > best) {
                    best = key[i];
                    at = i;
                }
            const Key top = warp_max(best);
            if (top == 0) break;
            const unsigned e = __reduce_min_sync(0xFFFFFFFFu, best == top ? (unsigned)(lane + 32 * at) : 0xFFFFFFFFu);
            if (lane == j) id = (int)e;
            if ((e & 31u) == (unsigned)lane) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (i == (int)(e >> 5)) key[i] = 0;
            }
        }

        // Weights of the chosen, in FP64 (one lane each), rounded once.
        double w = 0.0;
        if (id >= 0) {
            const double v = (double)route_logit(p, m * p.ldl + id);
            w = p.sigmoid ? 1.0 / (1.0 + exp(-v)) : route_exp(v, (double)most);
        }
        if (p.renormalize) {
            double all = w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
            w = all > 0.0 ? w / all : 0.0;
        } else if (!p.sigmoid) {
            w = sum64 > 0.0 ? w / sum64 : 0.0;
        }
        if (lane < k) {
            p.ids[m * k + lane] = id;
            p.weights[m * k + lane] = (float)(w * (double)p.scale);
        }
    }

    // Rows of each expert among this CTA's tokens, numbered in their order (the first warp, 32 choices at a time).
    __syncthreads();
    if (warp == 0) {
        const int64_t end = m1 * k;
        for (int64_t i0 = m0 * k; i0 < end; i0 += 32) {
            const int64_t i = i0 + lane;
            const int e = i < end ? __ldcg(p.ids + i) : -1;
            const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
            const uint32_t had = e >= 0 ? count[e] : 0u;
            if (i < end) p.slots[i] = e >= 0 ? (int32_t)(had + __popc(same & ((1u << lane) - 1u))) : -1;
            __syncwarp();
            if (e >= 0 && (same >> lane) == 1u) count[e] = had + __popc(same);   // (the last of them)
            __syncwarp();
        }
        if (p.chunks == 1) {
            route_offsets(count, first, E);
            __syncwarp();
        }
    }
    __syncthreads();
    if (p.chunks > 1) {
        for (int e = threadIdx.x; e < E; e += kRouteWarps * 32) p.counts[(int64_t)blockIdx.x * E + e] = count[e];
    } else {
        for (int e = threadIdx.x; e <= E; e += kRouteWarps * 32) p.offsets[e] = (int32_t)first[e];
        for (int64_t i = m0 * k + threadIdx.x; i < m1 * k; i += kRouteWarps * 32) {
            const int e = __ldcg(p.ids + i);
            if (e >= 0) p.slots[i] = __ldcg(p.slots + i) + (int32_t)first[e];
        }
    }
}

__global__ void __launch_bounds__(kRouteWarps * 32)
route_place_kernel(const RouteParams p) {
    __shared__ uint32_t total[kRouteMaxExperts], before[kRouteMaxExperts], first[kRouteMaxExperts + 1];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int E = p.E, k = p.top_k;
    for (int e = threadIdx.x; e < E; e += kRouteWarps * 32) {
        uint32_t all = 0, mine = 0;
#pragma unroll 16
        for (int c = 0; c < p.chunks; ++c) {
            const uint32_t n = __ldcg(p.counts + (int64_t)c * E + e);
            all += n;
            if (c < (int)blockIdx.x) mine += n;
        }
        total[e] = all;
        before[e] = mine;
    }
    __syncthreads();
    if (threadIdx.x < 32) route_offsets(total, first, E);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= E; e += kRouteWarps * 32) p.offsets[e] = (int32_t)first[e];
    const int64_t m0 = (int64_t)blockIdx.x * p.chunk, m1 = min(p.M, m0 + p.chunk);
    for (int64_t i = m0 * k + threadIdx.x; i < m1 * k; i += kRouteWarps * 32) {
        const int e = __ldcg(p.ids + i);
        if (e >= 0) p.slots[i] = __ldcg(p.slots + i) + (int32_t)(first[e] + before[e]);
    }
}

}  // namespace w4a8
