// Routing of tokens to experts: the choice of top_k experts from router logits, their weights, and the order of the rows by
// expert that the experts' products read.
//
// route_choose_kernel: a warp per token, V consecutive experts per lane; then the CTA counts its tokens' experts and numbers the rows
// of each expert in the order of the tokens.  Up to 128 tokens the CTAs are one cluster and read one another's counts: one launch.
// Above, route_place_kernel follows: every CTA sums the counts of the CTAs before it (at most kRouteChunks rows, from L2) and turns
// the numbers into rows.  No atomics: the order never varies.
//
// Nothing here is near the bound of its bytes (2 MB of logits: 0.4 us): what counts are launches and the length of the chain of
// dependent steps of a token -- load, keys, groups, top_k rounds of a warp-wide maximum, weights.  Hence: groups judged all
// at once by exchanges among the lanes that hold them; a maximum of 64-bit keys by their upper words, by the lower ones only
// where those are equal; weights in FP64 for as many of a warp's tokens at a time as fill its lanes; the next token's logits
// fetched ahead.
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
constexpr int kRouteCluster = 8;     // CTAs of the single launch
constexpr int kRouteLocalIds = 2048; // choices of a CTA that are kept in shared memory

struct RouteParams {
    const void* logits;
    int64_t ldl;
    const float* bias;
    int32_t *ids, *offsets, *slots;
    float* weights;
    uint32_t* counts;   // [chunks][E]
    int64_t M;
    int E, top_k, groups, top_groups, group_best, chunk, chunks;
    int logits_fp32, sigmoid, renormalize, clustered;
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

// Row offsets of the experts from their counts, exclusive, by all warps (one of them per 32 experts); `sums`: a word per warp.
// total[e] in, first[e] out, first[E] = all rows.
__device__ __forceinline__ void route_offsets(const uint32_t* total, uint32_t* first, uint32_t* sums, int E) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = threadIdx.x;
    const uint32_t own = e < E ? total[e] : 0u;
    uint32_t sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, sum, o);
        if (lane >= o) sum += before;
    }
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    uint32_t base = 0;
#pragma unroll
    for (int w = 0; w < kRouteWarps; ++w) base += w < warp ? sums[w] : 0u;
    if (e < E) first[e] = base + sum - own;
    if (e == E - 1) first[E] = base + sum;
    __syncthreads();
}
static_assert(kRouteMaxExperts <= kRouteWarps * 32, "a thread per expert");

// V consecutive logits of a row from `e` on; experts that are not there, and NaN, as -inf (a NaN is never chosen and has no part
// in the others' scores).
template <int V>
__device__ __forceinline__ void route_load(const RouteParams& p, int64_t m, int e, float (&x)[V]) {
    if (p.logits_fp32) {
        const float* src = static_cast<const float*>(p.logits) + m * p.ldl + e;
        if (V >= 4 && e + V <= p.E && (reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
#pragma unroll
            for (int i = 0; i + 3 < V; i += 4) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(src + i));
                x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = e + i < p.E ? __ldg(src + i) : -INFINITY;
        }
    } else {
        const uint16_t* src = static_cast<const uint16_t*>(p.logits) + m * p.ldl + e;
        if (V >= 4 && e + V <= p.E && (reinterpret_cast<uintptr_t>(src) & 7u) == 0) {
#pragma unroll
            for (int i = 0; i + 3 < V; i += 4) {
                const uint2 v = __ldg(reinterpret_cast<const uint2*>(src + i));
                x[i] = __uint_as_float(v.x << 16), x[i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                x[i + 2] = __uint_as_float(v.y << 16), x[i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = e + i < p.E ? __uint_as_float((uint32_t)__ldg(src + i) << 16) : -INFINITY;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (x[i] != x[i]) x[i] = -INFINITY;
}

template <int V, typename Key>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_choose_kernel(const RouteParams p) {
    constexpr bool WIDE = sizeof(Key) == 8;
    __shared__ uint32_t count[kRouteMaxExperts], total[kRouteMaxExperts], first[kRouteMaxExperts + 1], sums[kRouteWarps];
    __shared__ __align__(16) uint8_t warp_count[kRouteWarps][kRouteMaxExperts];
    __shared__ int16_t local_ids[kRouteLocalIds];
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e0 = lane * V;
    const int E = p.E, k = p.top_k, size = E / p.groups;
    const int64_t m0 = (int64_t)blockIdx.x * p.chunk, m1 = min(p.M, m0 + p.chunk);
    const bool local = (int64_t)p.chunk * k <= kRouteLocalIds;
    for (int e = threadIdx.x; e < E; e += kRouteWarps * 32) count[e] = 0u;
    // lanes of a group, where a group is a power of two of whole lanes; 0 otherwise
    const int span = size % V == 0 && ((size / V) & (size / V - 1)) == 0 ? size / V : 0;
    float bias[WIDE ? V : 1];
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = p.bias != nullptr && e0 + i < E ? __ldg(p.bias + e0 + i) : 0.0f;
    }
    // A warp's tokens are weighed `batch` at a time, each by kp lanes.
    const int kp = k <= 1 ? 1 : 1 << (32 - __clz(k - 1)), batch = 32 / kp, sub = lane / kp, j_mine = lane & (kp - 1);

    float ahead[V];
    if (m0 + warp < m1) route_load<V>(p, m0 + warp, e0, ahead);
    for (int64_t mb = m0 + warp; mb < m1; mb += (int64_t)batch * kRouteWarps) {
        int id = -1;                             // lane sub * kp + j: choice j of the batch's token sub
        float most_mine = 0.0f;                  // that token's largest logit
        double sum_mine = 0.0;                   // and the sum of its softmax
        for (int b = 0; b < batch; ++b) {
            const int64_t m = mb + (int64_t)b * kRouteWarps;
            if (m >= m1) break;
            float x[V];
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = ahead[i];
                most = fmaxf(most, x[i]);
            }
            if (m + kRouteWarps < m1) route_load<V>(p, m + kRouteWarps, e0, ahead);
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
                double scale = 1.0;
                if (!p.sigmoid) {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sum64 += __shfl_xor_sync(0xFFFFFFFFu, sum64, o);
                    scale = sum64;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const double v = (p.sigmoid ? s[i] : s[i] / scale) + (double)bias[i];
                    key[i] = x[i] == -INFINITY || !(v > -(double)INFINITY) ? 0 : order_key(v);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) key[i] = x[i] == -INFINITY ? 0 : order_key(x[i]);
                if (!p.sigmoid && !p.renormalize) {
                    float sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) sum += x[i] == -INFINITY ? 0.0f : (x[i] == most ? 1.0f : expf(x[i] - most));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
                    sum64 = sum;
                }
            }
            if (sub == b) {
                most_mine = most;
                sum_mine = sum64;
            }

            if (p.groups > 1) {
                // A group's key: the sum of the group_best highest, lowest where one of them cannot be chosen.
                auto judge = [&](Key top, Key next) -> Key {
                    if constexpr (WIDE) {
                        if (p.group_best == 2 && size > 1) return top == 0 || next == 0 ? 0 : order_key(key_value(top) + key_value(next));
                    }
                    return top;
                };
                unsigned kept = 0;
                if (span > 0) {
                    Key best = 0, second = 0;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const Key low = key[i] < best ? key[i] : best;
                        best = key[i] > best ? key[i] : best;
                        second = low > second ? low : second;
                    }
                    for (int o = 1; o < span; o <<= 1) {   // (lanes of one group exchange theirs)
                        const Key b2 = __shfl_xor_sync(0xFFFFFFFFu, best, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, second, o);
                        const Key low = b2 < best ? b2 : best;
                        best = b2 > best ? b2 : best;
                        second = second > s2 ? second : s2;
                        second = low > second ? low : second;
                    }
                    const Key score = judge(best, second);
                    const int mine = lane / span;
                    int before = 0;   // groups that come before this lane's
                    for (int g = 0; g < p.groups; ++g) {
                        const Key other = __shfl_sync(0xFFFFFFFFu, score, g * span);
                        before += other > score || (other == score && g < mine) ? 1 : 0;
                    }
                    if (mine >= p.groups || before >= p.top_groups) {
#pragma unroll
                        for (int i = 0; i < V; ++i) key[i] = 0;
                    }
                } else {
                    Key score = 0;   // lane g judges group g
                    for (int g = 0; g < p.groups; ++g) {
                        Key best = 0, second = 0;   // this lane's in the group
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            if (e0 + i < g * size || e0 + i >= (g + 1) * size) continue;
                            const Key low = key[i] < best ? key[i] : best;
                            best = key[i] > best ? key[i] : best;
                            second = low > second ? low : second;
                        }
                        const Key top = warp_max(best);
                        const unsigned holds = __ballot_sync(0xFFFFFFFFu, best == top);
                        const Key next = warp_max(lane == __ffs((int)holds) - 1 ? second : best);
                        if (lane == g) score = judge(top, next);
                    }
                    int before = 0;
                    for (int g = 0; g < p.groups; ++g) {
                        const Key other = __shfl_sync(0xFFFFFFFFu, score, g);
                        before += other > score || (other == score && g < lane) ? 1 : 0;
                    }
                    kept = __ballot_sync(0xFFFFFFFFu, lane < p.groups && before < p.top_groups);
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (e0 + i < E && !(kept >> ((e0 + i) / size) & 1u)) key[i] = 0;
                }
            }

            // The choices, highest first: the lane with the highest key of all gives it up and looks for its next one.
            Key best = 0;
            int at = 0;
            auto own_best = [&]() {
                best = 0;
                at = 0;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (key[i] > best) {
                        best = key[i];
                        at = i;
                    }
            };
            own_best();
            for (int j = 0; j < k; ++j) {
                unsigned holds;
                if constexpr (WIDE) {
                    const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(best >> 32));
                    holds = __ballot_sync(0xFFFFFFFFu, (uint32_t)(best >> 32) == hi);
                    if ((holds & (holds - 1u)) != 0u) {
                        const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (holds >> lane & 1u) ? (uint32_t)best : 0u);
                        holds = __ballot_sync(0xFFFFFFFFu, (holds >> lane & 1u) && (uint32_t)best == lo);
                    }
                } else {
                    const uint32_t top = __reduce_max_sync(0xFFFFFFFFu, best);
                    holds = __ballot_sync(0xFFFFFFFFu, best == top);
                }
                const int from = __ffs((int)holds) - 1;   // (equal keys: the lowest lane has the lowest index)
                const int e = __shfl_sync(0xFFFFFFFFu, best == 0 ? -1 : e0 + at, from);
                if (e < 0) break;
                if (lane == b * kp + j) id = e;
                if (lane == from) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i == at) key[i] = 0;
                    own_best();
                }
            }
        }

        // Weights of the batch's choices, in FP64 (one lane each), rounded once.
        const int64_t m = mb + (int64_t)sub * kRouteWarps;
        double w = 0.0;
        if (id >= 0) {
            const double v = (double)route_logit(p, m * p.ldl + id);
            w = p.sigmoid ? 1.0 / (1.0 + exp(-v)) : route_exp(v, (double)most_mine);
        }
        double by = p.sigmoid ? 1.0 : sum_mine;
        if (p.renormalize) {
            by = w;
            for (int o = kp >> 1; o > 0; o >>= 1) by += __shfl_xor_sync(0xFFFFFFFFu, by, o);
        }
        w = by > 0.0 ? w / by : 0.0;
        if (m < m1 && j_mine < k) {
            p.ids[m * k + j_mine] = id;
            p.weights[m * k + j_mine] = (float)(w * (double)p.scale);
            if (local) local_ids[(m - m0) * k + j_mine] = (int16_t)id;
        }
    }

    // Rows of each expert among this CTA's tokens, numbered in their order: 512 choices at a time, a warp's 32 among themselves and
    // then behind those of the warps before it.
    const int64_t begin = m0 * k, end = m1 * k;
    for (int64_t i0 = begin; i0 < end; i0 += kRouteWarps * 32) {
        for (int c = threadIdx.x; c < kRouteWarps * kRouteMaxExperts / 16; c += kRouteWarps * 32)
            reinterpret_cast<uint4*>(&warp_count[0][0])[c] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        const int64_t i = i0 + threadIdx.x;
        const int e = i < end ? (local ? (int)local_ids[i - begin] : __ldcg(p.ids + i)) : -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
        if (e >= 0 && (same >> lane) == 1u) warp_count[warp][e] = (uint8_t)__popc(same);   // (the last of them)
        __syncthreads();
        uint32_t rank = 0, had = 0;
        if (e >= 0) {
            rank = count[e] + __popc(same & ((1u << lane) - 1u));
            for (int w = 0; w < warp; ++w) rank += warp_count[w][e];
        }
        if ((int)threadIdx.x < E)
#pragma unroll
            for (int w = 0; w < kRouteWarps; ++w) had += warp_count[w][threadIdx.x];
        __syncthreads();
        if ((int)threadIdx.x < E) count[threadIdx.x] += had;
        if (i < end) p.slots[i] = e >= 0 ? (int32_t)rank : -1;
    }
    __syncthreads();
    if (!p.clustered) {
        for (int e = threadIdx.x; e < E; e += kRouteWarps * 32) p.counts[(int64_t)blockIdx.x * E + e] = count[e];
        return;
    }
    // One cluster: the counts of the CTAs before this one, and of all.
    if (p.chunks > 1) ptx::cluster_sync_all();
    uint32_t before = 0;
    if ((int)threadIdx.x < E) {
        uint32_t all = 0;
        for (int c = 0; c < p.chunks; ++c) {
            uint32_t n = count[threadIdx.x];
            if (p.chunks > 1) {
                const uint32_t from = ptx::map_to_cta(ptx::smem_addr(&count[threadIdx.x]), (uint32_t)c);
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n) : "r"(from) : "memory");
            }
            all += n;
            if (c < (int)blockIdx.x) before += n;
        }
        total[threadIdx.x] = all;
    }
    __syncthreads();
    route_offsets(total, first, sums, E);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= E; e += kRouteWarps * 32) p.offsets[e] = (int32_t)first[e];
    if ((int)threadIdx.x < E) total[threadIdx.x] = first[threadIdx.x] + before;
    __syncthreads();
    for (int64_t i = begin + threadIdx.x; i < end; i += kRouteWarps * 32) {   // (each thread its own numbers)
        const int e = local ? (int)local_ids[i - begin] : __ldcg(p.ids + i);
        if (e >= 0) p.slots[i] = __ldcg(p.slots + i) + (int32_t)total[e];
    }
    if (p.chunks > 1) ptx::cluster_sync_all();   // (nobody leaves while its counts may be read)
}

__global__ void __launch_bounds__(kRouteWarps * 32)
route_place_kernel(const RouteParams p) {
    __shared__ uint32_t total[kRouteMaxExperts], before[kRouteMaxExperts], first[kRouteMaxExperts + 1], sums[kRouteWarps];
    ptx::griddep_launch_dependents();
    const int E = p.E, k = p.top_k;
    if ((int)threadIdx.x < E) total[threadIdx.x] = before[threadIdx.x] = 0u;
    __syncthreads();
    ptx::griddep_wait();
    // threads / E threads share an expert, each with every so many of the rows of counts (whole numbers: sums in any order)
    const int parts = kRouteWarps * 32 / E, part = (int)threadIdx.x / E, mine = (int)threadIdx.x - part * E;
    if (part < parts) {
        uint32_t all = 0, earlier = 0;
#pragma unroll 16
        for (int c = part; c < p.chunks; c += parts) {
            const uint32_t n = __ldcg(p.counts + (int64_t)c * E + mine);
            all += n;
            if (c < (int)blockIdx.x) earlier += n;
        }
        atomicAdd(&total[mine], all);
        atomicAdd(&before[mine], earlier);
    }
    __syncthreads();
    route_offsets(total, first, sums, E);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= E; e += kRouteWarps * 32) p.offsets[e] = (int32_t)first[e];
    const int64_t m0 = (int64_t)blockIdx.x * p.chunk, m1 = min(p.M, m0 + p.chunk);
    for (int64_t i = m0 * k + threadIdx.x; i < m1 * k; i += kRouteWarps * 32) {
        const int e = __ldcg(p.ids + i);
        if (e >= 0) p.slots[i] = __ldcg(p.slots + i) + (int32_t)(first[e] + before[e]);
    }
}

}  // namespace w4a8
