// Routing of tokens to experts: the choice of top_k experts from router logits, their weights, and the order of the rows by
// expert that the experts' products read.
//
// route_choose_kernel: clusters of eight CTAs, a warp per token, V consecutive experts per lane; then a CTA counts its tokens'
// experts, numbers the rows of each expert in the order of the tokens and tells the other CTAs of the cluster its counts.  Up to
// 128 tokens that is all: one cluster, one launch.  Above, route_place_kernel follows: every CTA sums the counts of the clusters
// before its own (at most 32 rows, from L2) and turns the numbers into rows.  No atomics on global memory: the order never varies.
//
// Nothing here is near the bound of its bytes (2 MB of logits: 0.4 us): what counts are launches and the length of the chain of
// dependent steps of a token -- load, keys, groups, top_k rounds of a warp-wide maximum, weights.  Hence: a key carries its
// expert's index in its low bits, so that no two are equal and a maximum says whose it is; a lane sorts its keys once and
// gives up the first (looking for the next one among eight took 525 cycles a round, this takes 150); groups are ranked all at
// once by exchanges among the lanes that hold them; weights in FP64 (but for one sum, see there) for as many of a warp's tokens at a
// time as fill its lanes; the next token's logits are fetched ahead.  Measured: 64 tokens of 256 experts in 8 groups 7.3 us, 8192
// tokens of 128 experts 16.4 to 19.4 us on different GPUs.
//
// The choice: without a bias and with groups ranked by their best expert, scores have the order of the logits, whose 32 bits are
// the keys' upper words.  Otherwise (WIDE) a key is score + bias in FP64, cut to 43 bits of fraction: in FP32 two experts whose
// keys differ by less than a rounding would change places.
#pragma once

#include <cuda_bf16.h>

#include "w4a8_common.cuh"
#include "w4a8_ptx.cuh"

namespace w4a8 {

constexpr int kRouteMaxExperts = 512, kRouteMaxTopK = 32, kRouteMaxGroups = 32;
constexpr int kRouteWarps = 16;      // tokens that a CTA works on at a time
constexpr int kRouteCluster = 8;
// CTAs at most: 32 clusters are resident at two CTAs per SM, 36 took a second round.  Two CTAs per SM hold up to 128 experts; above,
// 98 to 128 registers of 512 threads leave one, and 256 CTAs are two rounds (4096 tokens of 256 experts in 8 groups 31.7 us).
constexpr int kRouteChunks = 256;
constexpr int kRouteLocalIds = 2048; // choices of a CTA that are kept in shared memory

struct RouteParams {
    const void* logits;
    int64_t ldl;
    const float* bias;
    int32_t *ids, *offsets, *slots;
    float* weights;
    uint32_t* counts;   // [clusters][E]
    int64_t M;
    int E, top_k, groups, top_groups, group_best, chunk, chunks;
    int logits_fp32, sigmoid, renormalize;
    float scale;
};

// Keys: their order as unsigned integers is that of the values, and for equal values the lower index comes first; 0 is left for
// experts that cannot be chosen.
constexpr uint64_t kRouteIndexBits = 511u;
static_assert(kRouteMaxExperts == kRouteIndexBits + 1, "an index fits the low bits");
__device__ __forceinline__ uint64_t order_bits(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v + 0.0);   // (-0 becomes 0)
    return b ^ ((b >> 63) ? 0xFFFFFFFFFFFFFFFFull : 0x8000000000000000ull);
}
__device__ __forceinline__ uint32_t order_bits(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ uint64_t route_key(double v, int e) { return (order_bits(v) & ~kRouteIndexBits) | (kRouteIndexBits - (uint64_t)e); }
__device__ __forceinline__ uint64_t route_key(float v, int e) { return (uint64_t)order_bits(v) << 32 | (kRouteIndexBits - (uint64_t)e); }
__device__ __forceinline__ int key_index(uint64_t k) { return (int)(kRouteIndexBits - (k & kRouteIndexBits)); }
__device__ __forceinline__ double key_value(uint64_t k) {
    k &= ~kRouteIndexBits;
    return __longlong_as_double((long long)(k ^ ((k >> 63) ? 0x8000000000000000ull : 0xFFFFFFFFFFFFFFFFull)));
}
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
    const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32));
    const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }

// Batcher's odd-even merge sort, descending (V a power of two, at most 16).
template <int V>
__device__ __forceinline__ void sort_keys(uint64_t (&k)[V]) {
#pragma unroll
    for (int p = 1; p < V; p <<= 1)
#pragma unroll
        for (int q = p; q >= 1; q >>= 1)
#pragma unroll
            for (int j = q % p; j + q < V; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i)
                    if (i + j + q < V && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
                        const uint64_t a = k[i + j], b = k[i + j + q];
                        k[i + j] = max64(a, b);
                        k[i + j + q] = min64(a, b);
                    }
}

__device__ __forceinline__ float route_logit(const RouteParams& p, int64_t at) {
    return p.logits_fp32 ? __ldg(static_cast<const float*>(p.logits) + at)
                         : __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(p.logits) + at) << 16);
}

// exp(x - most), with x == most exact also at infinity.
__device__ __forceinline__ double route_exp(double x, double most) { return x == most ? 1.0 : exp(x - most); }

// exp(t) and 1 / d in FP64 without a branch, so that a lane's V experts go through them side by side (the library's functions,
// each with a path for extreme arguments, one behind the other took 5700 of a token's 17900 cycles).  exp: t = n ln 2 + r with |r| at
// most half of ln 2 after Cody and Waite (ln 2 in two parts, the first of 32 bits, so that n times it is exact), the Taylor series
// of exp(r) to the twelfth power (the rest is below 2^-52), and 2^n as two factors, so that results run out to infinity and
// zero.  |t| at most 1000.
__device__ __forceinline__ double plain_exp(double t) {
    const double big = 6755399441055744.0;   // 1.5 * 2^52: adding it rounds to whole numbers, which its low word then holds
    const double shifted = fma(t, 1.4426950408889634, big);
    const int n = __double2loint(shifted);
    const double whole = shifted - big;
    double r = fma(whole, -0.693147180369123816490, t);
    r = fma(whole, -1.90821492927058770002e-10, r);
    double v = 1.0 / 479001600.0;
    v = fma(v, r, 1.0 / 39916800.0);
    v = fma(v, r, 1.0 / 3628800.0);
    v = fma(v, r, 1.0 / 362880.0);
    v = fma(v, r, 1.0 / 40320.0);
    v = fma(v, r, 1.0 / 5040.0);
    v = fma(v, r, 1.0 / 720.0);
    v = fma(v, r, 1.0 / 120.0);
    v = fma(v, r, 1.0 / 24.0);
    v = fma(v, r, 1.0 / 6.0);
    v = fma(v, r, 0.5);
    v = fma(v, r, 1.0);
    v = fma(v, r, 1.0);
    const int half = n >> 1;
    return v * __hiloint2double((1023 + half) << 20, 0) * __hiloint2double((1023 + n - half) << 20, 0);
}
// d from 1 to 2: an approximation of 20 bits, and two of Newton's steps.
__device__ __forceinline__ double plain_inverse(double d) {
    double y;
    asm("rcp.approx.ftz.f64 %0, %1;" : "=d"(y) : "d"(d));
    y = fma(y, fma(-d, y, 1.0), y);
    y = fma(y, fma(-d, y, 1.0), y);
    return y;
}

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

template <int V, bool WIDE>
__global__ void __launch_bounds__(kRouteWarps * 32)
route_choose_kernel(const RouteParams p) {
    __shared__ uint32_t count[kRouteMaxExperts], from[kRouteCluster][kRouteMaxExperts], first[kRouteMaxExperts + 1], sums[kRouteWarps];
    __shared__ __align__(16) uint8_t warp_count[kRouteWarps][kRouteMaxExperts];
    __shared__ int16_t local_ids[kRouteLocalIds];
    ptx::griddep_launch_dependents();
    ptx::cluster_arrive_relaxed();   // (waited for ahead of the first access to another CTA's shared memory: all have started by then)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e0 = lane * V;
    const int E = p.E, k = p.top_k, size = E / p.groups;
    const int64_t m0 = min(p.M, (int64_t)blockIdx.x * p.chunk), m1 = min(p.M, m0 + p.chunk);
    const bool local = (int64_t)p.chunk * k <= kRouteLocalIds;
    const uint32_t rank = ptx::cluster_ctarank();
    if ((int)threadIdx.x < E) count[threadIdx.x] = 0u;
    // lanes of a group, where a group is a power of two of whole lanes; 0 otherwise
    const int span = size % V == 0 && ((size / V) & (size / V - 1)) == 0 ? size / V : 0;
    // A warp's tokens are weighed `batch` at a time, each by kp lanes.
    const int kp = k <= 1 ? 1 : 1 << (32 - __clz(k - 1)), batch = 32 / kp, sub = lane / kp, j_mine = lane & (kp - 1);
    ptx::griddep_wait();
    float ahead[V], bias[WIDE ? V : 1];
    if (m0 + warp < m1) route_load<V>(p, m0 + warp, e0, ahead);
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = p.bias != nullptr && e0 + i < E ? __ldg(p.bias + e0 + i) : 0.0f;
    }
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
            uint64_t key[V];
            if constexpr (WIDE) {
                double s[V], inverse = 1.0;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (p.sigmoid) {
                        // (of exp(-|x|), so that scores keep their order down to FP64's least number, logits of -745)
                        const double z = plain_exp(fmax(-fabs((double)x[i]), -1000.0)), of_positive = plain_inverse(1.0 + z);
                        s[i] = x[i] < 0.0f ? z * of_positive : of_positive;
                    } else {
                        s[i] = x[i] == most ? 1.0 : plain_exp(fmax((double)x[i] - (double)most, -1000.0));   // (0 where x is -inf)
                        sum64 += s[i];
                    }
                }
                if (!p.sigmoid) {
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) sum64 += __shfl_xor_sync(0xFFFFFFFFu, sum64, o);
                    inverse = 1.0 / sum64;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const double v = s[i] * inverse + (double)bias[i];
                    key[i] = x[i] == -INFINITY || !(v > -(double)INFINITY) ? 0 : route_key(v, e0 + i);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) key[i] = x[i] == -INFINITY ? 0 : route_key(x[i], e0 + i);
                // The sum over all experts, which a renormalised softmax does without, in FP32.  Relative to it: every exp within 2 ulp
                // (2^-22); the differences in front of them 2^-24 of themselves, on average over the terms at most ln E = 6.3 times 2^-24;
                // E / 32 + 5 sums of 2^-24; the weight's own rounding: within (E / 32 + 17) 2^-24.  In FP64 it took the kernel 13 to 17 %
                // longer (64 tokens of 256 experts 5.8 -> 6.6 us, 8192 of 128 17.7 -> 20.7).
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
                // A group's key: the sum of the group_best highest, lowest where one of them cannot be chosen.  (An index in its low
                // bits does no harm: groups of equal value are taken in their order, which is that of their best experts' indices
                // as long as these are not compared; so they are taken off.)
                auto group_key = [&](uint64_t top, uint64_t next) -> uint64_t {
                    if (WIDE && p.group_best == 2 && size > 1) return top == 0 || next == 0 ? 0 : order_bits(key_value(top) + key_value(next));
                    return top == 0 ? 0 : top | kRouteIndexBits;
                };
                if (span > 0) {
                    uint64_t best = 0, second = 0;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        second = max64(second, min64(key[i], best));
                        best = max64(best, key[i]);
                    }
                    for (int o = 1; o < span; o <<= 1) {   // (lanes of one group exchange theirs)
                        const uint64_t b2 = __shfl_xor_sync(0xFFFFFFFFu, best, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, second, o);
                        second = max64(max64(second, s2), min64(best, b2));
                        best = max64(best, b2);
                    }
                    const uint64_t score = group_key(best, second);
                    const int mine = lane / span;
                    int before = 0;   // groups that come before this lane's
#pragma unroll 8
                    for (int g = 0; g < p.groups; ++g) {
                        const uint64_t other = __shfl_sync(0xFFFFFFFFu, score, g * span);
                        before += other > score || (other == score && g < mine) ? 1 : 0;
                    }
                    if (mine >= p.groups || before >= p.top_groups) {
#pragma unroll
                        for (int i = 0; i < V; ++i) key[i] = 0;
                    }
                } else {
                    uint64_t score = 0;   // lane g has the key of group g
                    for (int g = 0; g < p.groups; ++g) {
                        uint64_t best = 0, second = 0;   // this lane's in the group
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            if (e0 + i < g * size || e0 + i >= (g + 1) * size) continue;
                            second = max64(second, min64(key[i], best));
                            best = max64(best, key[i]);
                        }
                        const uint64_t top = warp_max(best), next = warp_max(best == top ? second : best);
                        if (lane == g) score = group_key(top, next);
                    }
                    int before = 0;
                    for (int g = 0; g < p.groups; ++g) {
                        const uint64_t other = __shfl_sync(0xFFFFFFFFu, score, g);
                        before += other > score || (other == score && g < lane) ? 1 : 0;
                    }
                    const unsigned kept = __ballot_sync(0xFFFFFFFFu, lane < p.groups && before < p.top_groups);
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (e0 + i < E && !(kept >> ((e0 + i) / size) & 1u)) key[i] = 0;
                }
            }

            // The choices, highest first.
            sort_keys<V>(key);
            for (int j = 0; j < k; ++j) {
                const uint64_t top = warp_max(key[0]);
                if (top == 0) break;
                if (lane == b * kp + j) id = key_index(top);
                if (key[0] == top) {
#pragma unroll
                    for (int i = 0; i + 1 < V; ++i) key[i] = key[i + 1];
                    key[V - 1] = 0;
                }
            }
        }

        // Weights of the batch's choices, in FP64 (one lane each) but for sum_mine of keys that are logits, rounded once.
        const int64_t m = mb + (int64_t)sub * kRouteWarps;
        double w = 0.0;
        if (id >= 0) {
            const double v = (double)route_logit(p, m * p.ldl + id);
            if (p.sigmoid) {
                const double z = exp(-fabs(v));
                w = (v < 0.0 ? z : 1.0) / (1.0 + z);
            } else {
                w = route_exp(v, (double)most_mine);
            }
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
    // then behind those of the warps before it.  The last (or only) round's numbers stay in registers.
    const int64_t begin = m0 * k, end = m1 * k;
    int e = -1;
    uint32_t number = 0;
    int64_t i0 = begin;
    while (true) {
        const int used = (int)min((int64_t)kRouteWarps, (end - i0 + 31) / 32);   // warps with choices
        if (warp < used) {
#pragma unroll
            for (int c = lane; c < kRouteMaxExperts / 16; c += 32) reinterpret_cast<uint4*>(warp_count[warp])[c] = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncthreads();
        const int64_t i = i0 + threadIdx.x;
        e = i < end ? (local ? (int)local_ids[i - begin] : __ldcg(p.ids + i)) : -1;
        const unsigned same = __match_any_sync(0xFFFFFFFFu, e);
        if (e >= 0 && (same >> lane) == 1u) warp_count[warp][e] = (uint8_t)__popc(same);   // (the last of them)
        __syncthreads();
        if (e >= 0) {
            number = count[e] + __popc(same & ((1u << lane) - 1u));
            for (int w = 0; w < warp; ++w) number += warp_count[w][e];
        }
        uint32_t had = 0;
        if ((int)threadIdx.x < E)
            for (int w = 0; w < used; ++w) had += warp_count[w][threadIdx.x];
        __syncthreads();
        if ((int)threadIdx.x < E) count[threadIdx.x] += had;
        if (i0 + kRouteWarps * 32 >= end) break;
        if (i < end) p.slots[i] = e >= 0 ? (int32_t)number : -1;
        i0 += kRouteWarps * 32;
    }
    __syncthreads();
    // Every CTA of the cluster gets every CTA's counts.
    ptx::cluster_wait();
    if ((int)threadIdx.x < E) {
#pragma unroll
        for (uint32_t c = 0; c < kRouteCluster; ++c)
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ptx::map_to_cta(ptx::smem_addr(&from[rank][threadIdx.x]), c)), "r"(count[threadIdx.x]) : "memory");
    }
    ptx::cluster_sync_all();
    uint32_t before = 0, all = 0;
    if ((int)threadIdx.x < E) {
#pragma unroll
        for (uint32_t c = 0; c < kRouteCluster; ++c) {
            all += from[c][threadIdx.x];
            if (c < rank) before += from[c][threadIdx.x];
        }
        count[threadIdx.x] = all;
    }
    __syncthreads();
    const bool only = gridDim.x == kRouteCluster;
    if (only) {
        route_offsets(count, first, sums, E);
        if (blockIdx.x == 0)
            for (int c = threadIdx.x; c <= E; c += kRouteWarps * 32) p.offsets[c] = (int32_t)first[c];
    } else if (rank == 0 && (int)threadIdx.x < E) {
        p.counts[(int64_t)(blockIdx.x / kRouteCluster) * E + threadIdx.x] = all;
    }
    // what comes before this CTA's rows of an expert: in the cluster, or in all
    if ((int)threadIdx.x < E) from[0][threadIdx.x] = before + (only ? first[threadIdx.x] : 0u);
    __syncthreads();
    const int64_t i = i0 + threadIdx.x;
    if (i < end) p.slots[i] = e >= 0 ? (int32_t)(number + from[0][e]) : -1;
    for (int64_t r = begin + threadIdx.x; r < i0; r += kRouteWarps * 32) {   // (each thread its own numbers of earlier rounds)
        const int er = local ? (int)local_ids[r - begin] : __ldcg(p.ids + r);
        if (er >= 0) p.slots[r] = __ldcg(p.slots + r) + (int32_t)from[0][er];
    }
}

__global__ void __launch_bounds__(kRouteWarps * 32)
route_place_kernel(const RouteParams p) {
    __shared__ uint32_t total[kRouteMaxExperts], before[kRouteMaxExperts], first[kRouteMaxExperts + 1], sums[kRouteWarps];
    ptx::griddep_launch_dependents();
    const int E = p.E, k = p.top_k;
    const int clusters = p.chunks / kRouteCluster, own = (int)blockIdx.x / kRouteCluster;
    if ((int)threadIdx.x < E) total[threadIdx.x] = before[threadIdx.x] = 0u;
    __syncthreads();
    ptx::griddep_wait();
    // threads / E threads share an expert, each with every so many of the rows of counts (whole numbers: sums in any order)
    const int parts = kRouteWarps * 32 / E, part = (int)threadIdx.x / E, mine = (int)threadIdx.x - part * E;
    if (part < parts) {
        uint32_t all = 0, earlier = 0;
#pragma unroll 16
        for (int c = part; c < clusters; c += parts) {
            const uint32_t n = __ldcg(p.counts + (int64_t)c * E + mine);
            all += n;
            if (c < own) earlier += n;
        }
        atomicAdd(&total[mine], all);
        atomicAdd(&before[mine], earlier);
    }
    __syncthreads();
    route_offsets(total, first, sums, E);
    if (blockIdx.x == 0)
        for (int e = threadIdx.x; e <= E; e += kRouteWarps * 32) p.offsets[e] = (int32_t)first[e];
    const int64_t m0 = min(p.M, (int64_t)blockIdx.x * p.chunk), m1 = min(p.M, m0 + p.chunk);
    for (int64_t i = m0 * k + threadIdx.x; i < m1 * k; i += kRouteWarps * 32) {
        const int e = __ldcg(p.ids + i);
        if (e >= 0) p.slots[i] = __ldcg(p.slots + i) + (int32_t)(first[e] + before[e]);
    }
}

}  // namespace w4a8
