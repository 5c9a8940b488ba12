// Activations to E4M3 with one scale per token and block of 128 columns (plain or gated, optionally written to the rows that
// the experts of each token read), and the weighted sum of the experts' outputs of each token.  Both are bound by HBM: (4096, 14336)
// gated 47.4 us in a graph (295 MB: 6.2 TB/s) and 48 to 55 as calls, the sum of 8 rows of 4096 values for each of 4096 tokens 49.7 us
// in a graph (302 MB: 6.1 TB/s) and 51.3 as calls; a few tokens take a launch, 2.2 us.
#pragma once

#include <cuda_bf16.h>

#include "w4a8_common.cuh"
#include "w4a8_ptx.cuh"

namespace w4a8 {

// Maxima below this count as this one, so that 448 / maximum stays finite.
constexpr float kBlockLeastMax = 7.888609052210118e-31f;   // 2^-100

// Scale and its inverse of a block whose largest magnitude is `amax` (Eq. 13 per block).
__device__ __forceinline__ void block_scale(float amax, float& s, float& inv) {
    const float a = fmaxf(amax, kBlockLeastMax);
    s = amax == 0.0f ? 1.0f : __fdiv_rn(a, kE4M3Max);
    inv = amax == 0.0f ? 1.0f : __fdiv_rn(kE4M3Max, a);
}

// Two values of g / (1 + exp(-g)) * u, two FP32 lanes per instruction where there is one: at 32 instructions a value the kernel was
// bound by their issue ((4096, 14336) 72.6 us).  exp(-g) = 2^t (1 + l ln 2) with t = -g log2(e) rounded and l what the rounding took,
// log2(e) in two parts; approximations of 2^t (2^-22) and of the reciprocal (2^-23), so that silu is within 2^-20.5.  Gates below -87
// give 0: there the reciprocal is below the normal numbers.  t stays finite, so that l does for every finite gate (gates above 2.36e38
// would have l = infinity, and 0 times it behind a 2^t of 0).  A gate that is NaN or infinite gives NaN.
__device__ __forceinline__ unsigned long long silu_mul(float g0, float g1, float u0, float u1) {
    constexpr float c_hi = -1.44269502162933349609375f, c_lo = -1.92596299e-8f, ln2 = 0.69314718056f;
    const unsigned long long g = pack_f32x2(g0, g1), low = pack_f32x2(fmaxf(g0, -88.0f), fmaxf(g1, -88.0f));
    float t0, t1, e0, e1;
    unpack_f32x2(mul_f32x2(low, pack_f32x2(c_hi, c_hi)), t0, t1);
    t0 = fmaxf(t0, -3.402823466e38f), t1 = fmaxf(t1, -3.402823466e38f);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e0) : "f"(t0));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e1) : "f"(t1));
    unsigned long long l = fma_f32x2(low, pack_f32x2(c_hi, c_hi), pack_f32x2(-t0, -t1));
    l = fma_f32x2(low, pack_f32x2(c_lo, c_lo), l);
    const unsigned long long e = pack_f32x2(e0, e1);
    // 1 + e + e l ln 2
    unsigned long long d = add_f32x2(e, pack_f32x2(1.0f, 1.0f));
    d = fma_f32x2(e, mul_f32x2(l, pack_f32x2(ln2, ln2)), d);
    float d0, d1, r0, r1;
    unpack_f32x2(d, d0, d1);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(d0));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(d1));
    return mul_f32x2(mul_f32x2(g, pack_f32x2(r0, r1)), pack_f32x2(u0, u1));
}

// Eight lanes hold a block, 16 consecutive columns each; a warp takes four consecutive blocks of a row.  K % 16 == 0, so a lane
// lies inside the row or outside.  The gated kind keeps silu(gate) * up in FP32: a rounding to BF16 in between would only add
// an error.
// top_k == 0: row m of the result is row m.  Otherwise it is written to the rows slots[m][0..top_k), entries outside [0, rows)
// skipped: a token is read and quantized once however many experts read it.
template <bool GATED>
__global__ void __launch_bounds__(256)
quantize_blocks_kernel(const uint16_t* __restrict__ x, int M, int K, int64_t ldx, const int32_t* __restrict__ slots, int top_k,
                       uint8_t* __restrict__ x8, int64_t rows, int64_t ldx8, float* __restrict__ s_x, int64_t lds) {
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int lane = threadIdx.x & 31;
    const int per_row = (K + 511) >> 9;   // warps' pieces of a row
    // (row and piece are carried along: a division each time took a tenth of the instructions)
    const int warps = gridDim.x * (blockDim.x >> 5), p0 = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int row_step = warps / per_row, piece_step = warps - row_step * per_row;
    int64_t m = p0 / per_row;
    int piece = p0 - (int)m * per_row;
    // The next piece's values are on their way while this one's are worked on (the gated kind: 59.5 us without).
    uint4 ahead[GATED ? 4 : 2];
    auto fetch = [&]() {
        const int col = piece * 512 + lane * 16;
        if (m < M && col < K) {
            const uint4* src = reinterpret_cast<const uint4*>(x + m * ldx + col);
            ahead[0] = __ldg(src);
            ahead[1] = __ldg(src + 1);
            if constexpr (GATED) {
                const uint4* up = reinterpret_cast<const uint4*>(x + m * ldx + K + col);
                ahead[2] = __ldg(up);
                ahead[3] = __ldg(up + 1);
            }
        }
    };
    fetch();
    while (m < M) {
        const int64_t row = m;
        const int col = piece * 512 + lane * 16;
        const bool have = col < K;
        uint4 now[GATED ? 4 : 2];
#pragma unroll
        for (int i = 0; i < (GATED ? 4 : 2); ++i) now[i] = ahead[i];
        m += row_step;
        piece += piece_step;
        if (piece >= per_row) {
            piece -= per_row;
            ++m;
        }
        fetch();
        float v[16];
        if (have) {
            const uint32_t w[8] = {now[0].x, now[0].y, now[0].z, now[0].w, now[1].x, now[1].y, now[1].z, now[1].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
            if constexpr (GATED) {
                const uint32_t u[8] = {now[2].x, now[2].y, now[2].z, now[2].w, now[3].x, now[3].y, now[3].z, now[3].w};
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    unpack_f32x2(silu_mul(v[2 * i], v[2 * i + 1], __uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u)), v[2 * i], v[2 * i + 1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0.0f;
        }
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(v[i]));
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
        float s, inv;
        block_scale(amax, s, inv);
#pragma unroll
        for (int i = 0; i < 16; i += 2) unpack_f32x2(mul_f32x2(pack_f32x2(v[i], v[i + 1]), pack_f32x2(inv, inv)), v[i], v[i + 1]);
        uint4 q;
        q.x = cvt_e4m3x4(v[0], v[1], v[2], v[3]);
        q.y = cvt_e4m3x4(v[4], v[5], v[6], v[7]);
        q.z = cvt_e4m3x4(v[8], v[9], v[10], v[11]);
        q.w = cvt_e4m3x4(v[12], v[13], v[14], v[15]);
        if (!have) continue;   // (no warp-wide step follows)
        if (top_k == 0) {
            *reinterpret_cast<uint4*>(x8 + row * ldx8 + col) = q;
            if ((lane & 7) == 0) s_x[row * lds + (col >> 7)] = s;
        } else {
            for (int j = 0; j < top_k; ++j) {
                const int64_t r = __ldg(slots + row * top_k + j);
                if (r < 0 || r >= rows) continue;
                *reinterpret_cast<uint4*>(x8 + r * ldx8 + col) = q;
                if ((lane & 7) == 0) s_x[r * lds + (col >> 7)] = s;
            }
        }
    }
}

// Eight consecutive values of a row as FP32.  READ_ONLY: of memory that the kernel does not write.
template <bool READ_ONLY>
__device__ __forceinline__ void load8(const void* base, int64_t at, bool fp32, float (&v)[8]) {
    if (fp32) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        float4 a, b;
        if constexpr (READ_ONLY) a = __ldg(p), b = __ldg(p + 1);
        else a = p[0], b = p[1];
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + at);
        uint4 a;
        if constexpr (READ_ONLY) a = __ldg(p);
        else a = *p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

__device__ __forceinline__ uint32_t bf16x2_bits(float lo, float hi) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
}

// out[m] = add[m] + sum_j weights[m][j] * y[slots[m][j]]: FP32 sums in ascending order of j behind the added row, rounded once.
// A thread holds eight columns of a token; the rows of four experts are in flight at a time.  `add` may be `out`: a thread reads its
// piece of the one before it writes that of the other, and no thread reads another's.
template <bool Y32, bool OUT32>
__global__ void __launch_bounds__(256)
combine_experts_kernel(const void* __restrict__ y, int64_t rows, int64_t ldy, const int32_t* __restrict__ slots,
                       const float* __restrict__ weights, int64_t M, int top_k, int N, const void* add, int64_t ldadd, void* out,
                       int64_t ldo) {
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int per_row = N >> 3;
    const int threads = gridDim.x * blockDim.x, p0 = blockIdx.x * blockDim.x + threadIdx.x;
    const int row_step = threads / per_row, piece_step = threads - row_step * per_row;
    int64_t m = p0 / per_row;
    for (int piece = p0 - (int)m * per_row; m < M; m += row_step, piece += piece_step) {
        if (piece >= per_row) {
            piece -= per_row;
            if (++m >= M) break;
        }
        const int col = piece * 8;
        float acc[8] = {};
        if (add != nullptr) load8<false>(add, m * ldadd + col, OUT32, acc);
        for (int j0 = 0; j0 < top_k; j0 += 4) {
            float v[4][8], w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t r = j0 + j < top_k ? (int64_t)__ldg(slots + m * top_k + j0 + j) : -1;
                const bool have = r >= 0 && r < rows;
                w[j] = have ? __ldg(weights + m * top_k + j0 + j) : 0.0f;
                if (have) {
                    load8<true>(y, r * ldy + col, Y32, v[j]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[j], v[j][i], acc[i]);
        }
        if constexpr (OUT32) {
            float4* o = reinterpret_cast<float4*>(static_cast<float*>(out) + m * ldo + col);
            o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + m * ldo + col) =
                make_uint4(bf16x2_bits(acc[0], acc[1]), bf16x2_bits(acc[2], acc[3]), bf16x2_bits(acc[4], acc[5]), bf16x2_bits(acc[6], acc[7]));
        }
    }
}

}  // namespace w4a8
