// FP8 linear layers with a scale per block of 128 (activations: one per token and 128 columns; weights: one per 128 x 128):
//   y[m][n] = sum_b s_x[m][b] * s_w[n / 128][b] * P_b[m][n],   P_b[m][n] = sum over the 128 columns of block b of x8 * w8,
// of one layer, or of several experts whose rows lie one behind the other.  P_b is one k-block's MMAs into a buffer of its own in
// tensor memory (FP32); warps fetch it and add s_x * s_w times it to sums in registers -- the scales change with every
// k-block, so the tensor cores cannot go on adding.
//
// linear_blocks_kernel (few tokens): a tile is up to 128 output channels x up to TMAX tokens.  The weights are the A operand, the
// tokens the B operand (N = the tile's tokens rounded up to 16), so that few tokens cost few columns; a thread sums one channel.
//
// Bound by the weight stream: a stage of the ring is a k-block of weights with its activations, loaded by TMA in the 128-byte
// swizzle.  The plan (w4a8_blocks_plan.h) takes as many channels per tile as make the tiles come out even over the SMs, and
// where there are too few, the CTAs of a cluster take a part of K each.  Sums go to the CTA that adds and writes their channels
// (itself where K is not cut) through distributed shared memory, to be added there in ascending order of K by two warps of
// their own, while the others are at the next tile: results repeat, no workspace is needed, so nothing of one call can meet
// another's, and outputs are written in pieces of 16 bytes.
//
// A stage's weights may be fewer than the 128 rows that an MMA reads: the other rows are whatever lies behind them, and give sums
// of channels that nothing looks at.
//
// Warps: 0 loads, 1 MMAs (and tensor memory's allocation), 2 and 3 outputs, then one group of four that adds, or two above 32 tokens
// (each half of the tokens: with one, 80 tokens were bound by it, 780 cycles a k-block).
//
// Measured: 512 rows of 120 of 128 experts, (4096, 4096) each (2.0 GB of weights), 289 to 302 us: 6.7 to 7.0 TB/s, more than a plain copy reaches
// (reads alone).  128 rows of 31 experts 102 us: DRAM reads are the weights' 521 MB, once.  Few weights are bound by what surrounds
// their stream -- launch, first loads, the sums' way, outputs: (77, 14336, 4096) 19.4 us, 3.3 TB/s (of its tiles' 80 tokens the first
// group that adds has 64); (1, 6144, 4096) 7.5 us, 3.3 TB/s; 8 rows of 8 experts 13.6 us, 3.4 TB/s.  Asking for the first weights ahead
// of the wait for the earlier kernel gained nothing.
#pragma once

#include <cuda_bf16.h>

#include "w4a8_blocks_plan.h"
#include "w4a8_common.cuh"
#include "w4a8_ptx.cuh"

namespace w4a8 {

constexpr int kBlocksMaxExperts = 512;

struct BlocksParams {
    const float *s_x, *s_w;
    const int32_t* offsets;   // [E + 1]; NULL: one layer, all rows
    void* y;
    int64_t lds, ldy, rows;
    int E, N, KB, NB;         // experts; channels; k-blocks; channel blocks
    int out_fp32;
    int tokens;               // tokens of a tile at most
    // linear_blocks_kernel
    int channels, row_tiles;  // channels of a tile (a multiple of 8), tiles of all channels
    int cut;                  // CTAs (a cluster) that share a tile's K
    int share;                // channels of a tile that each of them writes, at most
    int stages, xslot;        // ring: stages, bytes of a stage's activations (whole boxes of 32 tokens)
    int part_buffers;         // tiles whose sums may be on their way
    unsigned int* status;
};

// Where the experts' rows and token tiles begin, in shared memory.
struct ExpertTable {
    int32_t row[kBlocksMaxExperts + 1];    // first row; row[E] = end of the last
    int32_t tile[kBlocksMaxExperts + 1];   // token tiles of the experts before
    int32_t sums[8];
};

// All threads of the block (256 of them work) fill the table; a barrier ends it.  Offsets are taken into [0, rows] and in ascending
// order, whatever they hold.
__device__ __forceinline__ void fill_expert_table(ExpertTable* t, const int32_t* offsets, int E, int64_t rows, int tokens) {
    static_assert(kBlocksMaxExperts == 512, "two experts per thread");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool works = tid < 256;
    const int32_t most = (int32_t)rows;
    if (works) {
        int32_t r[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) r[i] = tid + 256 * i <= E ? __ldg(offsets + tid + 256 * i) : 0;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (tid + 256 * i <= E) t->row[tid + 256 * i] = min(max(r[i], 0), most);
    }
    __syncthreads();
    bool descends = false;
    for (int e = 1 + tid; works && e <= E; e += 256) descends = descends || t->row[e] < t->row[e - 1];
    if (__syncthreads_or(descends)) {
        if (warp == 0) {
            int32_t before_all = 0;
            for (int e0 = 0; e0 <= E; e0 += 32) {
                int32_t r = e0 + lane <= E ? t->row[e0 + lane] : most;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int32_t before = __shfl_up_sync(0xFFFFFFFFu, r, o);
                    if (lane >= o) r = max(r, before);
                }
                r = max(r, before_all);
                before_all = __shfl_sync(0xFFFFFFFFu, r, 31);
                if (e0 + lane <= E) t->row[e0 + lane] = r;
            }
        }
        __syncthreads();
    }
    int32_t own[2] = {0, 0}, sum = 0;
    if (works) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (2 * tid + i < E) own[i] = (t->row[2 * tid + i + 1] - t->row[2 * tid + i] + tokens - 1) / tokens;
        sum = own[0] + own[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t before = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += before;
        }
        if (lane == 31) t->sums[warp] = sum;
    }
    __syncthreads();
    if (works) {
#pragma unroll
        for (int w = 0; w < 8; ++w) sum += w < warp ? t->sums[w] : 0;
        if (2 * tid < E) t->tile[2 * tid] = sum - own[0] - own[1];
        if (2 * tid + 1 < E) t->tile[2 * tid + 1] = sum - own[1];
        if (tid == 255) t->tile[E] = sum;
    }
    __syncthreads();
}

// A tile: expert, rows, and where its channels begin.
struct BlocksTile {
    int e, nb, count;   // expert; first channel block (many tokens) or first channel; tokens
    int64_t row;        // first row
};
// The rows of token tile j.
__device__ __forceinline__ BlocksTile blocks_rows(const BlocksParams& p, const ExpertTable* t, int j) {
    BlocksTile b;
    b.nb = 0;
    if (p.offsets == nullptr) {
        b.e = 0;
        b.row = (int64_t)j * p.tokens;
        b.count = (int)min((int64_t)p.tokens, p.rows - b.row);
        return b;
    }
    int lo = 0, hi = p.E;   // the last expert whose tiles begin at or before j
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t->tile[mid] <= j) lo = mid; else hi = mid;
    }
    b.e = lo;
    const int at = (j - t->tile[lo]) * p.tokens;
    b.row = t->row[lo] + at;
    b.count = min(p.tokens, t->row[lo + 1] - t->row[lo] - at);
    return b;
}
// The channel tiles of a token tile follow one another.
__device__ __forceinline__ BlocksTile blocks_tile(const BlocksParams& p, const ExpertTable* t, int i) {
    const int j = i / p.row_tiles;
    BlocksTile b = blocks_rows(p, t, j);
    b.nb = (i - j * p.row_tiles) * p.channels;
    return b;
}

// Arrival on a barrier of a CTA of the cluster that also announces what this thread has written to that CTA's shared memory, or
// read from its own.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// A value into the shared memory of a CTA of the cluster; its four bytes complete on a barrier of that CTA.
__device__ __forceinline__ void st_async_f32(uint32_t addr, float v, uint32_t cluster_bar) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::"r"(addr), "r"(__float_as_uint(v)), "r"(cluster_bar)
                 : "memory");
}
// Behind a wait: what other CTAs of the cluster have sent is visible too.
__device__ __forceinline__ void acquire_cluster(uint32_t bar, uint32_t parity) {
    asm volatile(
        "{\n\t"
        ".reg .pred p;\n\t"
        "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%0], %1;\n\t"
        "}\n" ::"r"(bar), "r"(parity)
        : "memory");
}

template <int TMAX_>
struct BlocksCfg {
    static constexpr int TMAX = TMAX_;
    static constexpr int kAccCols = TMAX_ < 32 ? 32 : TMAX_;
    static constexpr int kTmemCols = kBlocksBuffers * kAccCols;
    static constexpr int kCtas = TMAX_ <= 32 ? 2 : 1;   // per SM
    static constexpr int G = TMAX_ <= 32 ? 1 : 2;       // groups of warps that add
    static constexpr int TG = TMAX_ / G;                // tokens of each
    static constexpr int kThreads = 128 + 128 * G;
};

// Eight channels of a token.
__device__ __forceinline__ void store8(const BlocksParams& p, int64_t at, int have, bool wide, const float (&v)[8]) {
    if (p.out_fp32) {
        float* y = static_cast<float*>(p.y) + at;
        if (wide) {
            reinterpret_cast<float4*>(y)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(y)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) y[i] = v[i];
        }
    } else {
        __nv_bfloat16* y = static_cast<__nv_bfloat16*>(p.y) + at;
        __nv_bfloat162 h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        if (wide) {
            *reinterpret_cast<uint4*>(y) = make_uint4(*reinterpret_cast<uint32_t*>(&h[0]), *reinterpret_cast<uint32_t*>(&h[1]),
                                                      *reinterpret_cast<uint32_t*>(&h[2]), *reinterpret_cast<uint32_t*>(&h[3]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) y[i] = i & 1 ? h[i >> 1].y : h[i >> 1].x;
        }
    }
}

template <class Cfg>
__global__ void __launch_bounds__(Cfg::kThreads, Cfg::kCtas)
linear_blocks_kernel(const __grid_constant__ CUtensorMap tmap_w,   // w8 [E][N][K], box 128 x channels x 1, 128B swizzle
                     const __grid_constant__ CUtensorMap tmap_x,   // x8 [rows][K], box 128 x 32, 128B swizzle
                     const BlocksParams p) {
    constexpr int TMAX = Cfg::TMAX, NBUF = kBlocksBuffers, G = Cfg::G, TG = Cfg::TG;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - raw_addr);
    const BlocksSmem lay = blocks_smem(TMAX, p.channels, p.tokens, p.stages, p.cut, p.share, p.part_buffers, p.offsets != nullptr);
    const uint32_t wslot = (uint32_t)p.channels * 128u, stage_bytes = wslot + (uint32_t)p.xslot;
    const uint32_t bars = base + (uint32_t)lay.bars;
    const uint32_t bar_full = bars, bar_free = bar_full + 8u * kBlocksMaxStages;
    const uint32_t bar_acc = bar_free + 8u * kBlocksMaxStages, bar_acc_free = bar_acc + 8u * NBUF;
    const uint32_t bar_parts = bar_acc_free + 8u * NBUF, bar_parts_free = bar_parts + 16u, bar_drain = bar_parts_free + 16u;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + lay.bars + 8 * kBlocksBars);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    float* scales = reinterpret_cast<float*>(sm + lay.scales);   // [2 buffers][2 channel blocks][k-block][TMAX]
    ExpertTable* table = reinterpret_cast<ExpertTable*>(sm + lay.table);
    const uint32_t parts_addr = base + (uint32_t)lay.parts;      // [buffer][CTA][token][channel of the share]

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cut = p.cut, rank = cut > 1 ? (int)ptx::cluster_ctarank() : 0, share = p.share;
    const int kb0 = rank * p.KB / cut, KB = (rank + 1) * p.KB / cut - kb0;
    // A tile's channels are dealt out to the CTAs that write them in units of eight, at least one each: a CTA without any would have
    // nothing to wait for, and run ahead of those that send to it.
    const int units = p.channels >> 3, mine0 = rank * units / cut * 8, mine_n = (rank + 1) * units / cut * 8 - mine0;
    const int first = (int)blockIdx.x / cut, step = (int)gridDim.x / cut;
    const bool grouped = p.offsets != nullptr;

    if (warp == 0) {
        if (lane == 0) {
            for (int i = 0; i < p.stages; ++i) {
                ptx::mbar_init(bar_full + 8u * i, 1);
                ptx::mbar_init(bar_free + 8u * i, 1);
            }
            for (int i = 0; i < NBUF; ++i) {
                ptx::mbar_init(bar_acc + 8u * i, 1);
                ptx::mbar_init(bar_acc_free + 8u * i, 4 * G);
            }
            for (int i = 0; i < 2; ++i) {
                ptx::mbar_init(bar_parts + 8u * i, cut > 1 ? 1u : 4u * G);   // (bytes of all CTAs; or this one's warps)
                ptx::mbar_init(bar_parts_free + 8u * i, (uint32_t)cut);
            }
            ptx::mbar_init(bar_drain, 1);
            *abort_flag = 0u;
            ptx::fence_mbar_init();
        }
        __syncwarp();
    } else if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), Cfg::kTmemCols);
        ptx::tmem_relinquish();
        // The next kernel's CTAs may come only once this one's have their tensor memory: they hold theirs until they have run, and
        // they run only when this kernel is done.
        ptx::griddep_launch_dependents();
    } else if (warp == 2 && lane == 0) {
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_x);
    }
    if (cut > 1) ptx::cluster_arrive_relaxed();   // (behind the barriers' set-up; waited for ahead of the first access to another CTA)
    ptx::griddep_wait();
    ptx::tc_fence_before_sync();
    if (grouped) {
        fill_expert_table(table, p.offsets, p.E, p.rows, p.tokens);
    } else if (warp == 0) {   // (the loads need none of the others)
        asm volatile("bar.arrive 2, %0;" ::"n"(Cfg::kThreads) : "memory");
    } else {
        asm volatile("bar.sync 2, %0;" ::"n"(Cfg::kThreads) : "memory");
    }
    ptx::tc_fence_after_sync();
    const int token_tiles = grouped ? table->tile[p.E] : (int)((p.rows + p.tokens - 1) / p.tokens);
    const int tiles = token_tiles * p.row_tiles;

    if (warp == 0) {
        // ------------------------------------------------------------------ loads (whole warp, one lane issues)
        bool ok = true;
        ptx::Ring r;
        int issued = 0;
        for (int i = first; i < tiles && ok; i += step) {
            const BlocksTile t = blocks_tile(p, table, i);
            const int boxes = (t.count + 31) >> 5;
            const uint32_t bytes = wslot + (uint32_t)boxes * 4096u;
            for (int b = 0; b < KB; ++b) {
                if (issued >= p.stages) ok = ptx::mbar_wait_warp(bar_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                const uint32_t full = bar_full + 8u * r.idx, dst = base + (uint32_t)r.idx * stage_bytes;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(full, bytes);
                    ptx::tma_load_3d(dst, &tmap_w, (kb0 + b) * 128, t.nb, t.e, full);
                    for (int q = 0; q < boxes; ++q)
                        ptx::tma_load_2d(dst + wslot + (uint32_t)q * 4096u, &tmap_x, (kb0 + b) * 128, (int)t.row + 32 * q, full);
                }
                r.advance(p.stages);
                ++issued;
            }
        }
        if (!ok && lane == 0) {   // gave up: let the copies in flight land before the CTA goes away
            const uint64_t t0 = ptx::globaltimer_ns();
            for (int i = issued > p.stages ? issued - p.stages : 0; i < issued; ++i)
                while (!ptx::mbar_try_wait(bar_full + 8u * (i % p.stages), (uint32_t)((i / p.stages) & 1)) &&
                       ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs / 20) {
                }
        }
        __syncwarp();
        if (cut > 1) ptx::cluster_wait();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMAs (whole warp, one lane issues)
        const uint32_t tmem = *tmem_slot;
        bool ok = true;
        ptx::Ring r, a;
        int made = 0;
        for (int i = first; i < tiles && ok; i += step) {
            const BlocksTile t = blocks_tile(p, table, i);
            const uint32_t idesc = ptx::umma_idesc_e4m3_f32(128, 0) | (uint32_t)(((t.count + 15) & ~15) >> 3) << 17;
            for (int b = 0; b < KB; ++b) {
                if (made >= NBUF) ok = ptx::mbar_wait_warp(bar_acc_free + 8u * a.idx, a.phase ^ 1u, abort_flag, p.status);
                ok = ok && ptx::mbar_wait_warp(bar_full + 8u * r.idx, r.phase, abort_flag, p.status);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t w = base + (uint32_t)r.idx * stage_bytes;
                const uint32_t a_lo = ptx::umma_desc_lo(w), b_lo = ptx::umma_desc_lo(w + wslot);
                if (ptx::elect_one()) {
                    ptx::umma_f8_kblock(tmem + (uint32_t)(a.idx * Cfg::kAccCols), a_lo, b_lo, idesc, 0u);
                    ptx::umma_commit(bar_acc + 8u * a.idx);
                    ptx::umma_commit(bar_free + 8u * r.idx);
                }
                r.advance(p.stages);
                a.advance(NBUF);
                ++made;
            }
        }
        if (!ok && lane == 0) {   // gave up: wait for the MMAs already issued before tensor memory is freed
            ptx::umma_commit(bar_drain);
            const uint64_t t0 = ptx::globaltimer_ns();
            while (!ptx::mbar_try_wait(bar_drain, 0u) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {
            }
        }
        __syncwarp();
        if (cut > 1) ptx::cluster_wait();
    } else {
        // The CTAs' parts of this CTA's channels of a tile, added in ascending order of K and written: eight channels of a token at a
        // time, by `n` threads.  Returns whether the parts came.
        const bool wide = ((p.ldy * (p.out_fp32 ? 4 : 2)) & 15) == 0;   // rows of y 16-byte aligned (y itself is)
        const int part_floats = cut * p.tokens * share;
        auto write_tile = [&](const BlocksTile& t, int at, uint32_t phase, int me, int n) -> bool {
            if (!ptx::mbar_wait_warp(bar_parts + 8u * at, phase, abort_flag, p.status)) return false;
            if (cut > 1) acquire_cluster(bar_parts + 8u * at, phase);
            const int n0 = t.nb + mine0, have = min(mine_n, p.N - n0), groups = (have + 7) >> 3;
            const uint32_t from = parts_addr + (uint32_t)(at * part_floats * 4);
            for (int u = me; u < groups * t.count; u += n) {
                const int tok = u / groups, c = (u - tok * groups) * 8;
                float v[8] = {};
                for (int q = 0; q < cut; ++q) {
                    const uint32_t a = from + (uint32_t)(((q * p.tokens + tok) * share + c) * 4);
                    float w[8];
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]) : "r"(a) : "memory");
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(w[4]), "=f"(w[5]), "=f"(w[6]), "=f"(w[7]) : "r"(a + 16u) : "memory");
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = q == 0 ? w[k] : v[k] + w[k];
                }
                store8(p, (t.row + tok) * p.ldy + n0 + c, have - c, wide && have - c >= 8, v);
            }
            return true;
        };
        const int last_tile = first < tiles ? first + (tiles - 1 - first) / step * step : -1;
        if (warp < 4) {
            // -------------------------------------------------------------- outputs
            if (cut > 1) ptx::cluster_wait();
            int use = 0;
            bool ok = true;
            // (after a wait that gave up these two warps still walk all tiles, without waiting or writing: they meet at a barrier)
            for (int i = first; i < tiles; i += step, ++use) {
                const int at = p.part_buffers == 2 ? use & 1 : 0, times = p.part_buffers == 2 ? use >> 1 : use;
                const BlocksTile t = blocks_tile(p, table, i);
                if (cut > 1 && warp == 2 && lane == 0)
                    ptx::mbar_arrive_expect_tx(bar_parts + 8u * at, (uint32_t)(cut * t.count * mine_n * 4));
                // (the last tile's are written by the warps that add as well)
                ok = ok && write_tile(t, at, (uint32_t)times & 1u, (int)threadIdx.x - 64, i == last_tile ? 64 + 128 * G : 64);
                if (i + (int64_t)p.part_buffers * step < tiles) {   // the buffer's next tile may come
                    asm volatile("bar.sync 3, 64;" ::: "memory");
                    if (ok && warp == 2 && lane < cut) mbar_arrive_release_cluster(ptx::map_to_cta(bar_parts_free + 8u * at, (uint32_t)lane));
                }
            }
        } else {
            // -------------------------------------------------------------- sums: thread = channel of the tile, and a group's tokens
            const int all = (int)threadIdx.x - 128, tid = all & 127, g0 = all >> 7 ? TG : 0;   // (all: token in the scale fetches)
            const uint32_t lanes = *tmem_slot + ((uint32_t)((warp & 3) * 32) << 16);
            if (cut > 1) ptx::cluster_wait();
            bool ok = true;
            ptx::Ring a;
            int use = 0, c = 0;
            const bool channel = tid < p.channels, any = (warp & 3) * 32 < p.channels;
            const int owner = channel ? (((tid >> 3) + 1) * cut - 1) / units : 0, column = tid - owner * units / cut * 8;   // who writes this channel
            // (after a wait that gave up these warps still walk all tiles, without waiting or writing: they meet at a barrier)
            for (int i = first; i < tiles; i += step, ++use) {
                const BlocksTile t = blocks_tile(p, table, i);
                const int blk = t.nb >> 7, mine = (min(t.nb + tid, p.N - 1) >> 7) - blk;   // channel block: the tile's first, or the next
                const float* sw_row = p.s_w + ((int64_t)t.e * p.NB + blk) * p.KB + kb0;
                // (lanes 0..7 fetch the scales of eight k-blocks of the first block, 8..15 of the next)
                const float* sw_lane = sw_row + (lane >= 8 && blk + 1 < p.NB ? p.KB : 0) + (lane & 7);
                const float* sx_row = p.s_x + (t.row + all) * p.lds + kb0;
                const bool token = all < t.count;
                const int mine_count = t.count - g0;   // tokens of this group and later ones
                unsigned long long acc[TG / 2];
#pragma unroll
                for (int j = 0; j < TG / 2; ++j) acc[j] = 0ull;
                float next[kBlocksChunk];   // this thread's token's scales of the next chunk of k-blocks
#pragma unroll
                for (int j = 0; j < kBlocksChunk; ++j) next[j] = token && j < KB ? __ldg(sx_row + j) : 0.0f;
                float next_w = lane < 16 && (lane & 7) < KB ? __ldg(sw_lane) : 0.0f;
                for (int b0 = 0; b0 < KB; b0 += kBlocksChunk, c ^= 1) {
                    float* cur = scales + c * 2 * kBlocksChunk * TMAX;
#pragma unroll
                    for (int j = 0; j < kBlocksChunk; ++j) {
                        const float w0 = __shfl_sync(0xFFFFFFFFu, next_w, j), w1 = __shfl_sync(0xFFFFFFFFu, next_w, 8 + j);
                        if (all < TMAX) {
                            cur[j * TMAX + all] = next[j] * w0;
                            cur[(kBlocksChunk + j) * TMAX + all] = next[j] * w1;
                        }
                    }
                    // (two buffers: a warp writes a chunk's scales only when all have finished with the chunk before the last)
                    asm volatile("bar.sync 1, %0;" ::"n"(128 * G) : "memory");
#pragma unroll
                    for (int j = 0; j < kBlocksChunk; ++j) {
                        const int b = b0 + kBlocksChunk + j;
                        next[j] = token && b < KB ? __ldg(sx_row + b) : 0.0f;
                    }
                    next_w = lane < 16 && b0 + kBlocksChunk + (lane & 7) < KB ? __ldg(sw_lane + b0 + kBlocksChunk) : 0.0f;
                    const int end = min(kBlocksChunk, KB - b0);
                    for (int j = 0; j < end; ++j) {
                        ok = ok && ptx::mbar_wait_warp(bar_acc + 8u * a.idx, a.phase, abort_flag, p.status);
                        if (!ok) break;   // (warp-uniform)
                        ptx::tc_fence_after_sync();
                        const ulonglong2* f = reinterpret_cast<const ulonglong2*>(cur + (mine * kBlocksChunk + j) * TMAX + g0);
                        const uint32_t src = lanes + (uint32_t)(a.idx * Cfg::kAccCols + g0);
                        if (any && mine_count > 0) {
                            uint32_t v[2][16];   // sixteen tokens are on their way while those before are added
                            ptx::tmem_ld_32x32b_x16(src, v[0]);
#pragma unroll
                            for (int q = 0; q < TG / 16; ++q) {
                                if (q * 16 >= mine_count) break;
                                ptx::tmem_ld_wait_for(v[q & 1]);
                                if (q + 1 < TG / 16 && (q + 1) * 16 < mine_count) ptx::tmem_ld_32x32b_x16(src + (uint32_t)(q * 16 + 16), v[(q + 1) & 1]);
#pragma unroll
                                for (int h = 0; h < 4; ++h) {
                                    const ulonglong2 s = f[q * 4 + h];   // the scales of four tokens
                                    const uint32_t* x = &v[q & 1][4 * h];
                                    acc[q * 8 + 2 * h] = fma_f32x2(pack_f32x2(__uint_as_float(x[0]), __uint_as_float(x[1])), s.x, acc[q * 8 + 2 * h]);
                                    acc[q * 8 + 2 * h + 1] = fma_f32x2(pack_f32x2(__uint_as_float(x[2]), __uint_as_float(x[3])), s.y, acc[q * 8 + 2 * h + 1]);
                                }
                            }
                        }
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(bar_acc_free + 8u * a.idx);
                        a.advance(NBUF);
                    }
                }
                // The sums of this thread's channel go to the CTA that writes it, once that has read those of an earlier tile.
                const int at = p.part_buffers == 2 ? use & 1 : 0, times = p.part_buffers == 2 ? use >> 1 : use;
                if (times > 0) ok = ok && ptx::mbar_wait_warp(bar_parts_free + 8u * at, (uint32_t)(times - 1) & 1u, abort_flag, p.status);
                if (ok) {
                    const uint32_t off = (uint32_t)((at * part_floats + (rank * p.tokens + g0) * share + column) * 4);
                    if (cut > 1) {   // (their bytes complete on the owner's barrier)
                        if (channel) {
                            const uint32_t to = ptx::map_to_cta(parts_addr, (uint32_t)owner) + off, bar = ptx::map_to_cta(bar_parts + 8u * at, (uint32_t)owner);
#pragma unroll
                            for (int j = 0; j < TG / 2; ++j) {
                                float lo, hi;
                                unpack_f32x2(acc[j], lo, hi);
                                if (2 * j < mine_count) st_async_f32(to + (uint32_t)(2 * j * share * 4), lo, bar);
                                if (2 * j + 1 < mine_count) st_async_f32(to + (uint32_t)((2 * j + 1) * share * 4), hi, bar);
                            }
                        }
                    } else {
                        if (channel) {
                            const uint32_t to = parts_addr + off;
#pragma unroll
                            for (int j = 0; j < TG / 2; ++j) {
                                float lo, hi;
                                unpack_f32x2(acc[j], lo, hi);
                                if (2 * j < mine_count) asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + (uint32_t)(2 * j * share * 4)), "f"(lo) : "memory");
                                if (2 * j + 1 < mine_count) asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + (uint32_t)((2 * j + 1) * share * 4)), "f"(hi) : "memory");
                            }
                        }
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(bar_parts + 8u * at);
                    }
                    if (i == last_tile) ok = write_tile(t, at, (uint32_t)times & 1u, all + 64, 64 + 128 * G);
                }
            }
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(*tmem_slot, Cfg::kTmemCols);
    }
    // What is sent to another CTA is waited for there (parts by those that write them; a buffer's release is sent only where its
    // next use will wait), so a CTA leaves when it is done -- but for one whose wait gave up: it stays until all others are done
    // or have given up too, and 2 ms more for what may be on its way.
    if (cut > 1 && *abort_flag != 0u) {
        ptx::cluster_arrive();
        ptx::cluster_wait();
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs / 1000) {
        }
    }
}

// ---- many tokens ---------------------------------------------------------------------------------------------------------------
// A tile is 128 tokens x 256 channels: the tokens are the A operand, so that a thread of the warps that add has one token and needs
// one product s_x * s_w per k-block and 128 channels.  The sums of a tile are 128 registers in each of 256 threads; a k-block's MMAs
// (512 cycles) go into one of two buffers of tensor memory while the other is fetched (256 columns: 256 cycles) and added.
//
// Bound by that exchange of the buffers -- a k-block's 512 cycles, then the way from the MMAs' completion to the warps that add, their
// fetch and the way back, of which only a part hides behind the other buffer's MMAs; tensor memory holds no third one of 256 columns --
// and, where a launch lasts, by the power limit.  On different GPUs (2048, 8192, 8192) 136 to 146 us, 1.9 to 2.0 PFLOP/s; (8192, 8192,
// 4096) 254 to 264 us, 2.1 PFLOP/s; (8192, 28672, 8192) 1970 to 2180 us, 1.75 to 1.95 PFLOP/s, at 1.1 to 1.4 GHz, and 1650 to 1980 with
// weights of zeros, which draw little power: the exchange comes first.  Tiles of 256 x 256 on pairs of CTAs, each with half of the
// channels' weights, load two thirds of this, but their buffers' way back leads through the other CTA, and experts fill them worse, on
// one GPU: 158 us instead of 146, 282 instead of 264, 2190 instead of 1970; 64 experts of (4096, 2048) with 512 rows each 379 instead of
// 334, with 128 rows each 186 instead of 134.  Without gain on pairs, and not tried on single CTAs: sixteen warps that add, buffers of
// 128 columns, a second warp that issues, the first columns of the next k-block fetched ahead.
//
// Warps: 0..7 sums and outputs (warp % 4 = lane quarter, warp / 4 = 128 of the channels), 8 loads, 9 MMAs, 10 scales (11 idle): the
// products s_x * s_w of eight k-blocks at a time, through shared memory.  (Fetched by the warps that add, a k-block's scales cost
// each of them a load of 32 lines, and its latency.)
constexpr int kWideThreads = 384, kWideTokens = 128;
constexpr int kWideStages = 3;                                          // with two (1024, 4096, 4096) 30.1 us instead of 22.7; four gain nothing
constexpr int kWideStageBytes = 16384 + 32768;                          // 128 tokens, 256 channels
constexpr int kWideScaleBytes = 2 * 2 * kBlocksChunk * 128 * 4;         // [2 buffers][2 channel blocks][k-block][token]
constexpr int kWideOutBytes = 8 * 4096;                                 // outputs on their way, 32 rows of 128 bytes per warp
constexpr int kWideScales = kWideStages * kWideStageBytes, kWideOut = kWideScales + kWideScaleBytes, kWideBars = kWideOut + kWideOutBytes;
constexpr int kWideNumBars = 2 * kWideStages + 4 + 4 + 1;
constexpr int kWideTiles = kWideBars + (8 * kWideNumBars + 8 + 15) / 16 * 16;   // where tiles are described, 16 bytes each
constexpr int kWideTable = kWideTiles + 4 * 16;
constexpr int kWideBand = 64;                                           // token tiles (8192 tokens) that share the channels' weights while they are in L2 (8 to 64: within 4 %)
constexpr int wide_smem(bool grouped) { return 1024 + kWideTable + (grouped ? (int)sizeof(ExpertTable) : 0); }
static_assert(wide_smem(true) <= kBlocksSmemMax, "shared memory");

// Tile index -> expert, first of two channel blocks and rows.
__device__ __forceinline__ BlocksTile wide_blocks_tile(const BlocksParams& p, const ExpertTable* t, int i, int token_tiles) {
    const int NT = (p.NB + 1) >> 1;
    BlocksTile b;
    if (p.offsets != nullptr) {
        const int j = i / NT;
        b = blocks_rows(p, t, j);
        b.nb = 2 * (i - j * NT);
        return b;
    }
    const int per = kWideBand * NT, band = i / per, in = i - band * per;
    const int high = min(kWideBand, token_tiles - band * kWideBand), n = in / high;
    b = blocks_rows(p, t, band * kWideBand + in - n * high);
    b.nb = 2 * n;
    return b;
}

__global__ void __launch_bounds__(kWideThreads, 1)
linear_blocks_wide_kernel(const __grid_constant__ CUtensorMap tmap_w,   // w8 [E][N][K], box 128 x 128 x 1, 128B swizzle
                          const __grid_constant__ CUtensorMap tmap_x,   // x8 [rows][K], box 128 x 128, 128B swizzle
                          const __grid_constant__ CUtensorMap tmap_y,   // y [rows][N] where its rows are 16-byte aligned, box 128 bytes x 32, 128B swizzle
                          const BlocksParams p) {
    constexpr int S = kWideStages;
    constexpr uint32_t kStageBytes = (uint32_t)kWideStageBytes;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - raw_addr);
    const uint32_t bar_full = base + (uint32_t)kWideBars, bar_free = bar_full + 8u * S, bar_acc = bar_free + 8u * S, bar_acc_free = bar_acc + 16u,
                   bar_scales = bar_acc_free + 16u, bar_scales_free = bar_scales + 16u, bar_drain = bar_scales_free + 16u;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + kWideBars + 8 * kWideNumBars);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    const uint32_t tile_info = base + (uint32_t)kWideTiles;   // [4] first row, tokens, first channel block
    ExpertTable* table = reinterpret_cast<ExpertTable*>(sm + kWideTable);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            ptx::mbar_init(bar_full + 8u * i, 1);
            ptx::mbar_init(bar_free + 8u * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(bar_acc + 8u * i, 1);
            ptx::mbar_init(bar_acc_free + 8u * i, 8);
            ptx::mbar_init(bar_scales + 8u * i, 1);
            ptx::mbar_init(bar_scales_free + 8u * i, 8);
        }
        ptx::mbar_init(bar_drain, 1);
        *abort_flag = 0u;
        ptx::fence_mbar_init();
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_x);
    }
    if (warp == 9) {
        ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), 512);
        ptx::tmem_relinquish();
        ptx::griddep_launch_dependents();   // (not before: see linear_blocks_kernel)
    }
    ptx::griddep_wait();
    ptx::tc_fence_before_sync();
    if (p.offsets != nullptr) fill_expert_table(table, p.offsets, p.E, p.rows, p.tokens);
    else __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const int token_tiles = p.offsets != nullptr ? table->tile[p.E] : (int)((p.rows + p.tokens - 1) / p.tokens);
    const int tiles = token_tiles * ((p.NB + 1) >> 1);
    const int first = (int)blockIdx.x, step = (int)gridDim.x, KB = p.KB;
    const int n_it = first < tiles ? ((tiles - first + step - 1) / step) * KB : 0;   // k-blocks of all tiles of this CTA

    // Registers: 64 x 128 + 216 x 256 threads of the 168 x 384 that the block is launched with.  setmaxnreg is one instruction for all four
    // warps of a group, ahead of the roles in which they part.
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 8) {
            // ------------------------------------------------------------------ loads (whole warp, one lane issues)
            bool ok = true;
            ptx::Ring r;
            int issued = 0;
            for (int i = first; i < tiles && ok; i += step) {
                const BlocksTile t = wide_blocks_tile(p, table, i, token_tiles);
                for (int b = 0; b < KB; ++b) {
                    if (issued >= S) ok = ptx::mbar_wait_warp(bar_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                    if (!ok) break;
                    const uint32_t full = bar_full + 8u * r.idx, dst = base + (uint32_t)r.idx * kStageBytes;
                    if (ptx::elect_one()) {   // (channels and rows that are not there come as zeros)
                        ptx::mbar_arrive_expect_tx(full, kStageBytes);
                        ptx::tma_load_2d(dst, &tmap_x, b * 128, (int)t.row, full);
                        ptx::tma_load_3d(dst + 16384u, &tmap_w, b * 128, t.nb * 128, t.e, full);
                        ptx::tma_load_3d(dst + 32768u, &tmap_w, b * 128, t.nb * 128 + 128, t.e, full);
                    }
                    r.advance(S);
                    ++issued;
                }
            }
            if (!ok && lane == 0) {   // gave up: let the copies in flight land before the CTA goes away
                const uint64_t t0 = ptx::globaltimer_ns();
                for (int i = issued > S ? issued - S : 0; i < issued; ++i)
                    while (!ptx::mbar_try_wait(bar_full + 8u * (i % S), (uint32_t)((i / S) & 1)) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs / 20) {
                    }
            }
            __syncwarp();
        } else if (warp == 9) {
            // ------------------------------------------------------------------ MMAs (whole warp, one lane issues)
            constexpr uint32_t idesc = ptx::umma_idesc_e4m3_f32(kWideTokens, 256);
            bool ok = true;
            ptx::Ring r, a;
            for (int it = 0; it < n_it; ++it) {
                // (the buffer is waited for last: it is what comes last)
                ok = ptx::mbar_wait_warp(bar_full + 8u * r.idx, r.phase, abort_flag, p.status);
                if (it >= 2) ok = ok && ptx::mbar_wait_warp(bar_acc_free + 8u * a.idx, a.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t s = base + (uint32_t)r.idx * kStageBytes;
                const uint32_t a_lo = ptx::umma_desc_lo(s), b_lo = ptx::umma_desc_lo(s + 16384u);
                if (ptx::elect_one()) {
                    ptx::umma_f8_kblock(tmem + (uint32_t)(a.idx * 256), a_lo, b_lo, idesc, 0u);
                    ptx::umma_commit(bar_acc + 8u * a.idx);
                    ptx::umma_commit(bar_free + 8u * r.idx);
                }
                r.advance(S);
                a.advance(2);
            }
            if (!ok && lane == 0) {   // gave up: wait for the MMAs already issued before tensor memory is freed
                ptx::umma_commit(bar_drain);
                const uint64_t t0 = ptx::globaltimer_ns();
                while (!ptx::mbar_try_wait(bar_drain, 0u) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {
                }
            }
            __syncwarp();
        } else if (warp == 10) {
            // ------------------------------------------------------------------ scales (a lane has four tokens), and what the tiles are
            bool ok = true;
            ptx::Ring r;
            int filled = 0, n = 0;
            const bool wide = (p.lds & 3) == 0 && (reinterpret_cast<uintptr_t>(p.s_x) & 15u) == 0;
            for (int i = first; i < tiles && ok; i += step, ++n) {
                const BlocksTile t = wide_blocks_tile(p, table, i, token_tiles);
                const float* sw0 = p.s_w + ((int64_t)t.e * p.NB + t.nb) * KB;
                const float* sw1 = t.nb + 1 < p.NB ? sw0 + KB : sw0;
                for (int b0 = 0; b0 < KB; b0 += kBlocksChunk) {
                    float w0 = 0.0f, w1 = 0.0f;
                    const int len = min(kBlocksChunk, KB - b0);
                    if (lane < len) {
                        w0 = __ldg(sw0 + b0 + lane);
                        w1 = __ldg(sw1 + b0 + lane);
                    }
                    if (filled >= 2) ok = ptx::mbar_wait_warp(bar_scales_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                    if (!ok) break;
                    // (four places: the chunk of a tile that comes two tiles later waits for all warps to be done with this tile's)
                    if (b0 == 0 && lane == 0) ptx::st_shared_v4(tile_info + (uint32_t)((n & 3) * 16), make_uint4((uint32_t)t.row, (uint32_t)t.count, (uint32_t)t.nb, 0u));
                    float* f = reinterpret_cast<float*>(sm + kWideScales) + r.idx * 2 * kBlocksChunk * 128 + lane;
    #pragma unroll 2
                    for (int k = 0; k < 4; ++k) {
                        const int in = k * 32 + lane;
                        const float* sx = p.s_x + (t.row + min(in, t.count - 1)) * p.lds + b0;   // (a row that exists)
                        float x[kBlocksChunk];
                        if (wide && len == kBlocksChunk) {
                            const float4 u = __ldg(reinterpret_cast<const float4*>(sx)), v = __ldg(reinterpret_cast<const float4*>(sx) + 1);
                            x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
                        } else {
    #pragma unroll
                            for (int j = 0; j < kBlocksChunk; ++j) x[j] = j < len ? __ldg(sx + j) : 0.0f;
                        }
    #pragma unroll
                        for (int j = 0; j < kBlocksChunk; ++j) {
                            f[j * 128 + k * 32] = x[j] * __shfl_sync(0xFFFFFFFFu, w0, j);
                            f[(kBlocksChunk + j) * 128 + k * 32] = x[j] * __shfl_sync(0xFFFFFFFFu, w1, j);
                        }
                    }
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar_scales + 8u * r.idx);
                    r.advance(2);
                    ++filled;
                }
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ------------------------------------------------------------------ sums and outputs: thread = token
        // (128 registers of sums and 64 of columns leave few: the loop over k-blocks keeps next to nothing, and what is needed
        // around it is read again.  With spills in it, it took a third longer; with the tile worked out twice by each of these warps,
        // it took 8 % longer for 32768 rows of 64 experts of (4096, 2048).)
        const uint32_t src = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * 128);
        const uint32_t sc_mine = base + (uint32_t)kWideScales + (uint32_t)((warp >> 2) * kBlocksChunk * 512 + (warp & 3) * 128 + lane * 4);
        bool ok = true;
        int it = 0, chunk = 0;   // k-blocks and chunks of eight of them so far
        for (int n = 0; it < n_it && ok; ++n) {   // tiles
            auto this_tile = [&](int& row, int& count, int& nb) {
                asm volatile(
                    "{\n\t.reg .b32 none;\n\tld.shared.v4.b32 {%0, %1, %2, none}, [%3];\n\t}"
                    : "=r"(row), "=r"(count), "=r"(nb)
                    : "r"(tile_info + (uint32_t)((n & 3) * 16))
                    : "memory");
            };
            bool any = false;   // (warp-uniform) a token of this warp, and its channels, are there
            unsigned long long acc[64];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j] = 0ull;
            for (int left = p.KB; left > 0 && ok; ++chunk) {
                ok = ptx::mbar_wait_warp(bar_scales + 8u * (chunk & 1), (uint32_t)(chunk >> 1) & 1u, abort_flag, p.status);
                if (!ok) break;
                const uint32_t sc = sc_mine + (uint32_t)((chunk & 1) * 2 * kBlocksChunk * 512);
                {
                    int row, count, nb;
                    this_tile(row, count, nb);
                    any = (warp & 3) * 32 < count && nb + (warp >> 2) < p.NB;
                }
                const int end = min(kBlocksChunk, left);
                left -= end;
#pragma unroll 1
                for (int j = 0; j < end; ++j, ++it) {
                    float fs;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(fs) : "r"(sc + (uint32_t)(j * 512)) : "memory");
                    ok = ptx::mbar_wait_warp(bar_acc + 8u * (it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, p.status);
                    if (!ok) break;
                    ptx::tc_fence_after_sync();
                    const unsigned long long f = pack_f32x2(fs, fs);
                    auto release = [&]() {   // the buffer has been read
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0 && it + 2 < n_it) ptx::mbar_arrive(bar_acc_free + 8u * (it & 1));
                    };
                    if (any) {
                        // 32 columns are on their way while those before are added
                        const uint32_t from = src + (uint32_t)((it & 1) * 256);
                        uint32_t v[2][2][16];
                        ptx::tmem_ld_32x32b_x16(from, v[0][0]);
                        ptx::tmem_ld_32x32b_x16(from + 16u, v[0][1]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            ptx::tmem_ld_wait_for(v[c & 1][0], v[c & 1][1]);
                            if (c < 3) {
                                ptx::tmem_ld_32x32b_x16(from + (uint32_t)(32 * c + 32), v[(c + 1) & 1][0]);
                                ptx::tmem_ld_32x32b_x16(from + (uint32_t)(32 * c + 48), v[(c + 1) & 1][1]);
                            } else {
                                release();
                            }
#pragma unroll
                            for (int z = 0; z < 2; ++z)
#pragma unroll
                                for (int k = 0; k < 8; ++k)
                                    acc[16 * c + 8 * z + k] =
                                        fma_f32x2(pack_f32x2(__uint_as_float(v[c & 1][z][2 * k]), __uint_as_float(v[c & 1][z][2 * k + 1])), f, acc[16 * c + 8 * z + k]);
                        }
                    } else {
                        release();
                    }
                }
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_scales_free + 8u * (chunk & 1));
            }
            if (ok && any) {
                // Outputs, 128 bytes of 32 rows at a time, through shared memory (pieces of 16 bytes permuted by their row as in the 128-byte
                // swizzle, so that neither side meets a bank twice) and from there by bulk stores: read back and stored by the warps,
                // that took 3 % longer for 32768 rows of 64 experts of (4096, 2048).  Where a bulk store would write rows behind an
                // expert's last, or y's rows are not 16-byte aligned, the warps store; an instruction then touches four lines.
                int tile_row, count, nb;
                this_tile(tile_row, count, nb);
                nb += warp >> 2;
                const int q = warp & 3;
                const uint32_t out_s = base + (uint32_t)(kWideOut + warp * 4096);
                const int es = p.out_fp32 ? 4 : 2;
                const bool wide = ((p.ldy * es) & 15) == 0;   // rows 16-byte aligned (y itself is)
                const int row0 = q * 32, rows = min(32, count - row0);
                uint8_t* y0 = static_cast<uint8_t*>(p.y) + (((int64_t)tile_row + row0) * p.ldy + nb * 128) * es;
                const int have = min(128, p.N - nb * 128) * es;   // bytes of a row of this channel block
                const bool bulk = wide && (rows == 32 || p.offsets == nullptr);
                auto store = [&](int piece) {   // the piece's rows, four of them per round
                    if (bulk) {
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0 && piece * 128 < have) {
                            ptx::tma_store_2d(&tmap_y, nb * 128 + piece * (128 / es), tile_row + row0, out_s);
                            ptx::bulk_commit();
                        }
                        return;
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int row = 4 * k + (lane >> 3), byte = piece * 128 + (lane & 7) * 16;
                        uint4 o;
                        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(o.x), "=r"(o.y), "=r"(o.z), "=r"(o.w)
                                     : "r"(out_s + (uint32_t)(row * 128 + (((lane ^ row) & 7) << 4)))
                                     : "memory");
                        if (row >= rows || byte >= have) continue;
                        uint8_t* to = y0 + (int64_t)row * p.ldy * es + byte;
                        if (wide) {
                            *reinterpret_cast<uint4*>(to) = o;
                        } else if (es == 4) {
                            const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                            for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(to)[i] = w[i];
                        } else {
                            const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                            for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
                        }
                    }
                    __syncwarp();
                };
                const uint32_t mine = out_s + (uint32_t)(lane * 128);
                auto room = [&]() {   // bulk stores have read what is written over next
                    if (lane == 0) ptx::bulk_wait_read();
                    __syncwarp();
                };
                if (p.out_fp32) {
#pragma unroll
                    for (int piece = 0; piece < 4; ++piece) {
                        room();
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            float f[4];
                            unpack_f32x2(acc[16 * piece + 2 * c], f[0], f[1]);
                            unpack_f32x2(acc[16 * piece + 2 * c + 1], f[2], f[3]);
                            ptx::st_shared_v4(mine + (uint32_t)(((c ^ lane) & 7) << 4),
                                              make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
                        }
                        store(piece);
                    }
                } else {
#pragma unroll
                    for (int piece = 0; piece < 2; ++piece) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            uint32_t o[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                float lo, hi;
                                unpack_f32x2(acc[32 * piece + 4 * c + k], lo, hi);
                                const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
                                o[k] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            if (c == 0) room();
                            ptx::st_shared_v4(mine + (uint32_t)(((c ^ lane) & 7) << 4), make_uint4(o[0], o[1], o[2], o[3]));
                        }
                        store(piece);
                    }
                }
            }
        }
    }

    if (lane == 0) ptx::bulk_wait();   // (outputs)
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 9) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace w4a8
