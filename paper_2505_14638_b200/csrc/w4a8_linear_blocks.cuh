// FP8 linear layers with a scale per block of 128 (activations: one per token and 128 columns; weights: one per 128 x 128):
//   y[m][n] = sum_b s_x[m][b] * s_w[n / 128][b] * P_b[m][n],   P_b[m][n] = sum over the 128 columns of block b of x8 * w8,
// of one layer, or of several experts whose rows lie one behind the other.
//
// linear_blocks_kernel: a tile is 128 output channels x up to TMAX tokens.  P_b is one k-block's MMAs into a buffer of its own in
// tensor memory (FP32); four warps, a thread per channel, fetch it and add s_x * s_w times it to sums in registers -- the scales
// change with every k-block, so the tensor cores cannot go on adding.  The weights are the A operand (128 rows), the tokens the
// B operand (N = the tile's tokens rounded up to 16), so that few tokens cost few columns.
//
// Few tokens are bound by the weight stream: one stage of the ring is a k-block of weights (16 KB) with its activations, loaded by
// TMA in the 128-byte swizzle.  Where the tiles do not fill the SMs, the CTAs of a cluster take a part of K each and exchange
// their sums through distributed shared memory: each adds the parts of its share of the channels, in ascending order of K, so
// results repeat.  No workspace is needed, so nothing of one call can meet another's.
//
// Warps: 0 loads, 1 MMAs (and tensor memory's allocation), 2 and 3 idle after the start, 4..7 sums and outputs.
#pragma once

#include <cuda_bf16.h>

#include "w4a8_common.cuh"
#include "w4a8_ptx.cuh"

namespace w4a8 {

constexpr int kBlocksMaxExperts = 512;
constexpr int kBlocksThreads = 256;
constexpr int kBlocksMaxStages = 16, kBlocksBuffers = 4;
constexpr int kBlocksChunk = 8;    // k-blocks whose activation scales are fetched at a time

struct BlocksParams {
    const float *s_x, *s_w;
    const int32_t* offsets;   // [E + 1]; NULL: one layer, all rows
    void* y;
    int64_t lds, ldy, rows;
    int E, N, KB, NB;         // experts; channels; k-blocks; channel blocks
    int cut;                  // CTAs (a cluster) that share a tile's K
    int stages, xslot;        // ring: stages, bytes of a stage's activations (whole boxes of 32 tokens)
    int tokens;               // tokens of a tile at most
    int out_fp32;
    unsigned int* status;
};

// Where the experts' rows and token tiles begin, in shared memory.
struct ExpertTable {
    int32_t row[kBlocksMaxExperts + 1];    // first row; row[E] = end of the last
    int32_t tile[kBlocksMaxExperts + 1];   // token tiles of the experts before
};

// The first warp fills the table.  Offsets are taken into [0, rows] and in ascending order, whatever they hold.
__device__ __forceinline__ void fill_expert_table(ExpertTable* t, const int32_t* offsets, int E, int64_t rows, int tokens) {
    const int lane = threadIdx.x & 31;
    const int32_t most = (int32_t)rows;
    int32_t begin_all = 0, tiles = 0;
    for (int e0 = 0; e0 <= E; e0 += 32) {
        const int e = e0 + lane;
        int32_t r = e <= E ? min(max(__ldg(offsets + e), 0), most) : most;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t before = __shfl_up_sync(0xFFFFFFFFu, r, o);
            if (lane >= o) r = max(r, before);
        }
        r = max(r, begin_all);
        begin_all = __shfl_sync(0xFFFFFFFFu, r, 31);
        if (e <= E) t->row[e] = r;
    }
    __syncwarp();
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane;
        const int32_t own = e < E ? (t->row[e + 1] - t->row[e] + tokens - 1) / tokens : 0;
        int32_t sum = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int32_t before = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += before;
        }
        if (e < E) t->tile[e] = tiles + sum - own;
        tiles += __shfl_sync(0xFFFFFFFFu, sum, 31);
    }
    if (lane == 0) t->tile[E] = tiles;
}

// A tile: expert, first channel block, rows.
struct BlocksTile {
    int e, nb, count;   // expert, channel block, tokens
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
// The channel blocks of a token tile follow one another.
__device__ __forceinline__ BlocksTile blocks_tile(const BlocksParams& p, const ExpertTable* t, int i) {
    const int j = i / p.NB;
    BlocksTile b = blocks_rows(p, t, j);
    b.nb = i - j * p.NB;
    return b;
}

// Arrival on a barrier of a CTA of the cluster that also announces this thread's writes to that CTA's shared memory, and the wait
// that goes with it.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

template <int TMAX_>
struct BlocksCfg {
    static constexpr int TMAX = TMAX_;
    static constexpr int kAccCols = TMAX_ < 32 ? 32 : TMAX_;
    static constexpr int kTmemCols = kBlocksBuffers * kAccCols;
    static constexpr int kBarBytes = 8 * (2 * kBlocksMaxStages + 2 * kBlocksBuffers + 2 + 1) + 16;
    // (behind the ring) barriers, scales [2][chunk][TMAX], experts, parts of other CTAs [cut][TMAX][channels of a share]
    static constexpr int kScaleBytes = 2 * kBlocksChunk * TMAX_ * 4;
    __host__ __device__ static constexpr int table_bytes(bool grouped) { return grouped ? (int)sizeof(ExpertTable) : 0; }
    __host__ __device__ static constexpr int part_bytes(int cut) { return cut > 1 ? cut * ((128 + cut - 1) / cut) * TMAX_ * 4 : 0; }
    static constexpr int kSmemMax = 232448;
    __host__ __device__ static constexpr int fixed_bytes(bool grouped, int cut) {
        return 1024 + ((kBarBytes + 15) / 16 * 16) + kScaleBytes + (table_bytes(grouped) + 15) / 16 * 16 + part_bytes(cut);
    }
};

template <class Cfg>
__global__ void __launch_bounds__(kBlocksThreads, 1)
linear_blocks_kernel(const __grid_constant__ CUtensorMap tmap_w,   // w8 [E][N][K], box 128 x 128 x 1, 128B swizzle
                     const __grid_constant__ CUtensorMap tmap_x,   // x8 [rows][K], box 128 x 32, 128B swizzle
                     const BlocksParams p) {
    constexpr int TMAX = Cfg::TMAX, NBUF = kBlocksBuffers;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - raw_addr);
    const uint32_t stage_bytes = 16384u + (uint32_t)p.xslot;
    uint32_t off = (uint32_t)p.stages * stage_bytes;
    const uint32_t bars = base + off;
    const uint32_t bar_full = bars, bar_free = bar_full + 8u * kBlocksMaxStages;
    const uint32_t bar_acc = bar_free + 8u * kBlocksMaxStages, bar_acc_free = bar_acc + 8u * NBUF;
    const uint32_t bar_parts = bar_acc_free + 8u * NBUF, bar_parts_free = bar_parts + 8u, bar_drain = bar_parts + 16u;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + off + 8u * (2 * kBlocksMaxStages + 2 * NBUF + 3));
    volatile uint32_t* abort_flag = tmem_slot + 1;
    off += (uint32_t)(Cfg::kBarBytes + 15) / 16u * 16u;
    float* scales = reinterpret_cast<float*>(sm + off);   // [2][chunk][TMAX]
    off += (uint32_t)Cfg::kScaleBytes;
    ExpertTable* table = reinterpret_cast<ExpertTable*>(sm + off);
    off += (uint32_t)(Cfg::table_bytes(p.offsets != nullptr) + 15) / 16u * 16u;
    float* parts = reinterpret_cast<float*>(sm + off);    // [cut][TMAX][share]
    const uint32_t parts_addr = base + off;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cut = p.cut, rank = cut > 1 ? (int)ptx::cluster_ctarank() : 0;
    const int share = (128 + cut - 1) / cut;
    const int kb0 = rank * p.KB / cut, KB = (rank + 1) * p.KB / cut - kb0;

    if (warp == 1) {
        ptx::tmem_alloc(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), Cfg::kTmemCols);
        ptx::tmem_relinquish();
    } else if (warp == 2) {
        if (lane == 0) {
            for (int i = 0; i < p.stages; ++i) {
                ptx::mbar_init(bar_full + 8u * i, 1);
                ptx::mbar_init(bar_free + 8u * i, 1);
            }
            for (int i = 0; i < NBUF; ++i) {
                ptx::mbar_init(bar_acc + 8u * i, 1);
                ptx::mbar_init(bar_acc_free + 8u * i, 4);
            }
            ptx::mbar_init(bar_parts, (uint32_t)cut * 4u);
            ptx::mbar_init(bar_parts_free, (uint32_t)cut);
            ptx::mbar_init(bar_drain, 1);
            *abort_flag = 0u;
            ptx::fence_mbar_init();
        }
    } else if (warp == 3 && lane == 0) {
        ptx::prefetch_tensormap(&tmap_w);
        ptx::prefetch_tensormap(&tmap_x);
    }
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (warp == 0 && p.offsets != nullptr) fill_expert_table(table, p.offsets, p.E, p.rows, p.tokens);
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (cut > 1) ptx::cluster_sync_all();   // (barriers of the peers are there before anything arrives on them)
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const int token_tiles = p.offsets != nullptr ? table->tile[p.E] : (int)((p.rows + p.tokens - 1) / p.tokens);
    const int tiles = token_tiles * p.NB;
    const int first = (int)blockIdx.x / cut, step = (int)gridDim.x / cut;

    if (warp == 0) {
        // ------------------------------------------------------------------ loads (whole warp, one lane issues)
        bool ok = true;
        ptx::Ring r;
        int issued = 0;
        for (int i = first; i < tiles && ok; i += step) {
            const BlocksTile t = blocks_tile(p, table, i);
            const int boxes = (t.count + 31) >> 5;
            const uint32_t bytes = 16384u + (uint32_t)boxes * 4096u;
            for (int b = 0; b < KB; ++b) {
                if (issued >= p.stages) ok = ptx::mbar_wait_warp(bar_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                const uint32_t full = bar_full + 8u * r.idx, dst = base + (uint32_t)r.idx * stage_bytes;
                if (ptx::elect_one()) {
                    ptx::mbar_arrive_expect_tx(full, bytes);
                    ptx::tma_load_3d(dst, &tmap_w, (kb0 + b) * 128, t.nb * 128, t.e, full);
                    for (int q = 0; q < boxes; ++q)
                        ptx::tma_load_2d(dst + 16384u + (uint32_t)q * 4096u, &tmap_x, (kb0 + b) * 128, (int)t.row + 32 * q, full);
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
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMAs (whole warp, one lane issues)
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
                const uint32_t a_lo = ptx::umma_desc_lo(w), b_lo = ptx::umma_desc_lo(w + 16384u);
                if (ptx::elect_one()) {
                    ptx::umma_f8_kblock(tmem + (uint32_t)(a.idx * Cfg::kAccCols), a_lo, b_lo, idesc, 0u);
                    ptx::umma_commit(bar_free + 8u * r.idx);
                    ptx::umma_commit(bar_acc + 8u * a.idx);
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
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ sums and outputs: thread = channel of the tile
        const int tid = (int)threadIdx.x - 128;   // channel within the tile; token in the scale fetches
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        bool ok = true;
        ptx::Ring a;
        uint32_t exchanged = 0;
        int c = 0;
        // (after a wait that gave up these warps still walk all tiles, without waiting or writing: they meet at a barrier)
        for (int i = first; i < tiles; i += step) {
            const BlocksTile t = blocks_tile(p, table, i);
            const float* sw_row = p.s_w + ((int64_t)t.e * p.NB + t.nb) * p.KB + kb0;
            const float* sx_row = p.s_x + (t.row + tid) * p.lds + kb0;
            const bool token = tid < t.count;
            unsigned long long acc[TMAX / 2];
#pragma unroll
            for (int j = 0; j < TMAX / 2; ++j) acc[j] = 0ull;
            float next[kBlocksChunk];   // this thread's token's scales of the next chunk of k-blocks
#pragma unroll
            for (int j = 0; j < kBlocksChunk; ++j) next[j] = token && j < KB ? __ldg(sx_row + j) * __ldg(sw_row + j) : 0.0f;
            for (int b0 = 0; b0 < KB; b0 += kBlocksChunk, c ^= 1) {
                float* cur = scales + c * kBlocksChunk * TMAX;
                if (tid < TMAX) {
#pragma unroll
                    for (int j = 0; j < kBlocksChunk; ++j) cur[j * TMAX + tid] = next[j];
                }
                // (two buffers: a warp writes a chunk's scales only when all have finished with the chunk before the last)
                asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
                for (int j = 0; j < kBlocksChunk; ++j) {
                    const int b = b0 + kBlocksChunk + j;
                    next[j] = token && b < KB ? __ldg(sx_row + b) * __ldg(sw_row + b) : 0.0f;
                }
                const int end = min(kBlocksChunk, KB - b0);
                for (int j = 0; j < end; ++j) {
                    ok = ok && ptx::mbar_wait_warp(bar_acc + 8u * a.idx, a.phase, abort_flag, p.status);
                    if (!ok) break;   // (warp-uniform)
                    ptx::tc_fence_after_sync();
                    const ulonglong2* f = reinterpret_cast<const ulonglong2*>(cur + j * TMAX);
                    const uint32_t src = lanes + (uint32_t)(a.idx * Cfg::kAccCols);
#pragma unroll
                    for (int q = 0; q < TMAX / 16; ++q) {
                        if (q * 16 >= t.count) break;
                        uint32_t v[16];
                        ptx::tmem_ld_32x32b_x16(src + (uint32_t)(q * 16), v);
                        ptx::tmem_ld_wait_for(v);
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const ulonglong2 s = f[q * 4 + h];   // the scales of four tokens
                            acc[q * 8 + 2 * h] = fma_f32x2(pack_f32x2(__uint_as_float(v[4 * h]), __uint_as_float(v[4 * h + 1])), s.x, acc[q * 8 + 2 * h]);
                            acc[q * 8 + 2 * h + 1] = fma_f32x2(pack_f32x2(__uint_as_float(v[4 * h + 2]), __uint_as_float(v[4 * h + 3])), s.y, acc[q * 8 + 2 * h + 1]);
                        }
                    }
                    ptx::tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) ptx::mbar_arrive(bar_acc_free + 8u * a.idx);
                    a.advance(NBUF);
                }
            }
            if (cut == 1) {
                const int n = t.nb * 128 + tid;
                if (ok && n < p.N) {
#pragma unroll
                    for (int j = 0; j < TMAX / 2; ++j) {
                        float lo, hi;
                        unpack_f32x2(acc[j], lo, hi);
                        const int64_t at = (t.row + 2 * j) * p.ldy + n;
                        if (p.out_fp32) {
                            if (2 * j < t.count) static_cast<float*>(p.y)[at] = lo;
                            if (2 * j + 1 < t.count) static_cast<float*>(p.y)[at + p.ldy] = hi;
                        } else {
                            if (2 * j < t.count) static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(lo);
                            if (2 * j + 1 < t.count) static_cast<__nv_bfloat16*>(p.y)[at + p.ldy] = __float2bfloat16_rn(hi);
                        }
                    }
                }
                continue;
            }
            // The parts of this thread's channel go to the CTA that adds them, once that has read those of the tile before.
            if (exchanged > 0) ok = ok && ptx::mbar_wait_warp(bar_parts_free, (exchanged - 1u) & 1u, abort_flag, p.status);
            if (ok) {
                const int owner = tid / share;
                const uint32_t to = ptx::map_to_cta(parts_addr, (uint32_t)owner) + (uint32_t)((rank * TMAX * share + tid - owner * share) * 4);
#pragma unroll
                for (int j = 0; j < TMAX / 2; ++j) {
                    float lo, hi;
                    unpack_f32x2(acc[j], lo, hi);
                    if (2 * j < t.count) st_cluster_f32(to + (uint32_t)(2 * j * share * 4), lo);
                    if (2 * j + 1 < t.count) st_cluster_f32(to + (uint32_t)((2 * j + 1) * share * 4), hi);
                }
                asm volatile("fence.acq_rel.cluster;" ::: "memory");
                __syncwarp();
                if (lane < cut) mbar_arrive_release_cluster(ptx::map_to_cta(bar_parts, (uint32_t)lane));
                ok = ptx::mbar_wait_warp(bar_parts, exchanged & 1u, abort_flag, p.status);
                asm volatile("fence.acq_rel.cluster;" ::: "memory");
            }
            if (ok) {
                const int n0 = t.nb * 128 + rank * share, have = min(share, 128 - rank * share);
                for (int e = tid; e < t.count * share; e += 128) {
                    const int tok = e / share, c = e - tok * share;
                    if (c >= have || n0 + c >= p.N) continue;
                    float s = 0.0f;
                    for (int q = 0; q < cut; ++q) s += parts[(q * TMAX + tok) * share + c];
                    const int64_t at = (t.row + tok) * p.ldy + n0 + c;
                    if (p.out_fp32)
                        static_cast<float*>(p.y)[at] = s;
                    else
                        static_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(s);
                }
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (warp == 4 && lane < cut) mbar_arrive_release_cluster(ptx::map_to_cta(bar_parts_free, (uint32_t)lane));
            ++exchanged;
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc(tmem, Cfg::kTmemCols);
    }
    if (cut > 1) ptx::cluster_sync_all();   // (no CTA goes away while another writes to its shared memory or arrives on its barriers)
}

// ---- many tokens: CTA pairs ----------------------------------------------------------------------------------------------------
// Bound by the tensor cores.  A tile is 256 tokens x 256 channels of a CTA pair (cta_group::2): the tokens are the A operand, so that
// a thread of the warps that add has one token and needs one product s_x * s_w per k-block and 128 channels; each CTA holds 128
// tokens and the sums of all 256 channels: 128 registers in each of 256 threads.  Its k-block's MMAs (512 cycles) go into one of two
// buffers of tensor memory while the other is fetched (256 columns: 256 cycles) and added.
//
// Warps: 0..7 sums and outputs (warp % 4 = lane quarter, warp / 4 = 128 of the channels), 8 loads, 9 MMAs, 10 scales (11 idle): the
// products s_x * s_w of eight k-blocks at a time, through shared memory.  (Fetched by the warps that add, a k-block's scales cost
// each of them a load of 32 lines, and its latency.)
constexpr int kPairBlocksThreads = 384, kPairBlocksStages = 5;
constexpr int kPairBlocksOutBytes = 8 * 4096;  // outputs on their way, 32 rows of 128 bytes per warp
constexpr int kPairBlocksScaleBytes = 2 * 2 * kBlocksChunk * 128 * 4;   // [2 buffers][2 channel blocks][k-block][token]
constexpr int kPairBlocksStageBytes = 32768;   // 128 tokens, 128 channels
constexpr int kPairBlocksBand = 32;            // token tiles (8192 tokens) that share the channels' weights while they are in L2
constexpr int kPairBlocksBars = 2 * kPairBlocksStages + 4 + 4 + 1;
__host__ __device__ constexpr int pair_blocks_smem(bool grouped) {
    return 1024 + kPairBlocksStages * kPairBlocksStageBytes + kPairBlocksScaleBytes + kPairBlocksOutBytes + 8 * kPairBlocksBars + 16 + (grouped ? (int)sizeof(ExpertTable) : 0);
}

// Tile index -> expert, pair of channel blocks and rows.
__device__ __forceinline__ BlocksTile pair_blocks_tile(const BlocksParams& p, const ExpertTable* t, int i, int token_tiles) {
    const int NT = (p.NB + 1) >> 1;
    BlocksTile b;
    if (p.offsets != nullptr) {
        const int j = i / NT;
        b = blocks_rows(p, t, j);
        b.nb = 2 * (i - j * NT);
        return b;
    }
    const int per = kPairBlocksBand * NT, band = i / per, in = i - band * per;
    const int high = min(kPairBlocksBand, token_tiles - band * kPairBlocksBand), n = in / high;
    b = blocks_rows(p, t, band * kPairBlocksBand + in - n * high);
    b.nb = 2 * n;
    return b;
}

__global__ void __launch_bounds__(kPairBlocksThreads, 1)
linear_blocks_pair_kernel(const __grid_constant__ CUtensorMap tmap_w,   // w8 [E][N][K], box 128 x 128 x 1, 128B swizzle
                          const __grid_constant__ CUtensorMap tmap_x,   // x8 [rows][K], box 128 x 128, 128B swizzle
                          const BlocksParams p) {
    constexpr int S = kPairBlocksStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = ptx::smem_addr(smem_raw);
    const uint32_t base = (raw_addr + 1023u) & ~1023u;
    uint8_t* sm = smem_raw + (base - raw_addr);
    constexpr uint32_t kScales = (uint32_t)(S * kPairBlocksStageBytes), kOut = kScales + (uint32_t)kPairBlocksScaleBytes,
                       kBars = kOut + (uint32_t)kPairBlocksOutBytes;
    const uint32_t bar_full = base + kBars, bar_free = bar_full + 8u * S, bar_acc = bar_free + 8u * S, bar_acc_free = bar_acc + 16u,
                   bar_scales = bar_acc_free + 16u, bar_scales_free = bar_scales + 16u, bar_drain = bar_scales_free + 16u;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sm + kBars + 8 * kPairBlocksBars);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    ExpertTable* table = reinterpret_cast<ExpertTable*>(sm + kBars + 8 * kPairBlocksBars + 16);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = ptx::cluster_ctarank();
    const bool leader = rank == 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S; ++i) {
            ptx::mbar_init(bar_full + 8u * i, 1);
            ptx::mbar_init(bar_free + 8u * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            ptx::mbar_init(bar_acc + 8u * i, 1);
            ptx::mbar_init(bar_acc_free + 8u * i, 16);   // eight warps of each CTA
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
        ptx::tmem_alloc_pair(ptx::smem_addr(const_cast<uint32_t*>(tmem_slot)), 512);
        ptx::tmem_relinquish_pair();
    }
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (warp == 8 && p.offsets != nullptr) fill_expert_table(table, p.offsets, p.E, p.rows, p.tokens);
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::cluster_sync_all();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const int token_tiles = p.offsets != nullptr ? table->tile[p.E] : (int)((p.rows + p.tokens - 1) / p.tokens);
    const int tiles = token_tiles * ((p.NB + 1) >> 1);
    const int first = (int)blockIdx.x >> 1, step = (int)gridDim.x >> 1, KB = p.KB;
    const int n_it = first < tiles ? ((tiles - first + step - 1) / step) * KB : 0;   // k-blocks of all tiles of this pair

    if (warp == 8) {
        // ------------------------------------------------------------------ loads (whole warp, one lane issues)
        // (registers: 64 x 128 + 216 x 256 threads of the 168 x 384 that the block is launched with)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        bool ok = true;
        ptx::Ring r;
        int issued = 0;
        for (int i = first; i < tiles && ok; i += step) {
            const BlocksTile t = pair_blocks_tile(p, table, i, token_tiles);
            const int y = (int)t.row + (int)rank * 128, n = t.nb * 128 + (int)rank * 128;
            for (int b = 0; b < KB; ++b) {
                if (issued >= S) ok = ptx::mbar_wait_warp(bar_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                const uint32_t full = bar_full + 8u * r.idx, to = ptx::map_to_cta(full, 0u), dst = base + (uint32_t)(r.idx * kPairBlocksStageBytes);
                if (ptx::elect_one()) {
                    if (leader) ptx::mbar_arrive_expect_tx(full, 2u * kPairBlocksStageBytes);
                    ptx::tma_load_2d_pair(dst, &tmap_x, b * 128, y, to);
                    ptx::tma_load_3d_pair(dst + 16384u, &tmap_w, b * 128, n, t.e, to);
                }
                r.advance(S);
                ++issued;
            }
        }
        if (!ok && leader && lane == 0) {   // gave up: let both CTAs' copies in flight land before either goes away
            const uint64_t t0 = ptx::globaltimer_ns();
            for (int i = issued > S ? issued - S : 0; i < issued; ++i)
                while (!ptx::mbar_try_wait(bar_full + 8u * (i % S), (uint32_t)((i / S) & 1)) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs / 20) {
                }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ------------------------------------------------------------------ MMAs (one lane of the leader issues)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (leader) {
            constexpr uint32_t idesc = ptx::umma_idesc_e4m3_f32(256, 256);
            bool ok = true;
            ptx::Ring r, a;
            for (int it = 0; it < n_it; ++it) {
                // (the buffer is waited for last: it is what comes last)
                ok = ptx::mbar_wait_warp(bar_full + 8u * r.idx, r.phase, abort_flag, p.status);
                if (it >= 2) ok = ok && ptx::mbar_wait_warp(bar_acc_free + 8u * a.idx, a.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                ptx::tc_fence_after_sync();
                const uint32_t s = base + (uint32_t)(r.idx * kPairBlocksStageBytes);
                const uint32_t a_lo = ptx::umma_desc_lo(s), b_lo = ptx::umma_desc_lo(s + 16384u);
                if (ptx::elect_one()) {
                    ptx::umma_f8_kblock_pair(tmem + (uint32_t)(a.idx * 256), a_lo, b_lo, idesc, 0u);
                    ptx::umma_commit_pair(bar_acc + 8u * a.idx, 3);
                    if (it + S < n_it) ptx::umma_commit_pair(bar_free + 8u * r.idx, 3);   // (the slot is used again: see the closing barrier)
                }
                r.advance(S);
                a.advance(2);
            }
            if (!ok && lane == 0) {   // gave up: wait for the MMAs already issued before tensor memory is freed
                ptx::umma_commit_pair(bar_drain, 1);
                const uint64_t t0 = ptx::globaltimer_ns();
                while (!ptx::mbar_try_wait(bar_drain, 0u) && ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs) {
                }
            }
        }
        __syncwarp();
    } else if (warp == 10) {
        // ------------------------------------------------------------------ scales (a lane has four tokens)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        bool ok = true;
        ptx::Ring r;
        int filled = 0;
        const bool wide = (p.lds & 3) == 0 && (reinterpret_cast<uintptr_t>(p.s_x) & 15u) == 0;
        for (int i = first; i < tiles && ok; i += step) {
            const BlocksTile t = pair_blocks_tile(p, table, i, token_tiles);
            const float* sw0 = p.s_w + ((int64_t)t.e * p.NB + t.nb) * KB;
            const float* sw1 = t.nb + 1 < p.NB ? sw0 + KB : sw0;
            for (int b0 = 0; b0 < KB; b0 += kBlocksChunk) {
                float w0 = 0.0f, w1 = 0.0f;
                const int n = min(kBlocksChunk, KB - b0);
                if (lane < n) {
                    w0 = __ldg(sw0 + b0 + lane);
                    w1 = __ldg(sw1 + b0 + lane);
                }
                if (filled >= 2) ok = ptx::mbar_wait_warp(bar_scales_free + 8u * r.idx, r.phase ^ 1u, abort_flag, p.status);
                if (!ok) break;
                float* f = reinterpret_cast<float*>(sm + kScales) + r.idx * 2 * kBlocksChunk * 128 + lane;
#pragma unroll 2
                for (int k = 0; k < 4; ++k) {
                    const int in = (int)rank * 128 + k * 32 + lane;
                    const float* sx = p.s_x + (t.row + min(in, t.count - 1)) * p.lds + b0;   // (a row that exists)
                    float x[kBlocksChunk];
                    if (wide && n == kBlocksChunk) {
                        const float4 u = __ldg(reinterpret_cast<const float4*>(sx)), v = __ldg(reinterpret_cast<const float4*>(sx) + 1);
                        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w, x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
                    } else {
#pragma unroll
                        for (int j = 0; j < kBlocksChunk; ++j) x[j] = j < n ? __ldg(sx + j) : 0.0f;
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
    } else if (warp == 11) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    } else {
        // ------------------------------------------------------------------ sums and outputs: thread = token
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // (128 registers of sums and 64 of columns leave few: the loop over k-blocks keeps next to nothing, and what is needed
        // around it is worked out again.  With spills in it, it took a third longer.)
        const uint32_t src = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)((warp >> 2) * 128);
        const uint32_t sc_mine = base + kScales + (uint32_t)((warp >> 2) * kBlocksChunk * 512 + (warp & 3) * 128 + lane * 4);
        bool ok = true;
        int it = 0, chunk = 0;   // k-blocks and chunks of eight of them so far
        for (int i = first; i < tiles && ok; i += step) {
            bool any;   // (warp-uniform) a token of this warp, and its channels, are there
            {
                const BlocksTile t = pair_blocks_tile(p, table, i, token_tiles);
                any = (int)rank * 128 + (warp & 3) * 32 < t.count && t.nb + (warp >> 2) < p.NB;
            }
            unsigned long long acc[64];
#pragma unroll
            for (int j = 0; j < 64; ++j) acc[j] = 0ull;
            for (int left = p.KB; left > 0 && ok; ++chunk) {
                ok = ptx::mbar_wait_warp(bar_scales + 8u * (chunk & 1), (uint32_t)(chunk >> 1) & 1u, abort_flag, p.status);
                if (!ok) break;
                const uint32_t sc = sc_mine + (uint32_t)((chunk & 1) * 2 * kBlocksChunk * 512);
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
                        if (lane == 0 && it + 2 < n_it) ptx::mbar_arrive_cluster(ptx::map_to_cta(bar_acc_free + 8u * (it & 1), 0u));
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
                // Outputs, 128 bytes of 32 rows at a time, through shared memory (pieces of 16 bytes permuted by their row, so that
                // neither side meets a bank twice): a store then touches four lines, not one for each of 32 rows.
                const BlocksTile t = pair_blocks_tile(p, table, i, token_tiles);
                const int q = warp & 3, nb = t.nb + (warp >> 2);
                const uint32_t out_s = base + kOut + (uint32_t)(warp * 4096);
                const int es = p.out_fp32 ? 4 : 2;
                const bool wide = ((p.ldy * es) & 15) == 0;   // rows 16-byte aligned (y itself is)
                const int row0 = (int)rank * 128 + q * 32, rows = min(32, t.count - row0);
                uint8_t* y0 = static_cast<uint8_t*>(p.y) + ((t.row + row0) * p.ldy + nb * 128) * es;
                const int have = min(128, p.N - nb * 128) * es;   // bytes of a row of this channel block
                auto store = [&](int piece) {   // the piece's rows, four of them per round
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
                if (p.out_fp32) {
#pragma unroll
                    for (int piece = 0; piece < 4; ++piece) {
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
                            ptx::st_shared_v4(mine + (uint32_t)(((c ^ lane) & 7) << 4), make_uint4(o[0], o[1], o[2], o[3]));
                        }
                        store(piece);
                    }
                }
            }
        }
    }

    ptx::tc_fence_before_sync();
    __syncthreads();
    // Closing barrier: neither CTA leaves while the other may still reach into its shared memory or barriers.  What is sent to
    // the other CTA has been waited for there: stages and freed buffers by the MMA warp (freed buffers are not announced after
    // the last use), freed stages by the load warps (the same), complete buffers by the warps that add.
    ptx::cluster_sync_all();
    if (*abort_flag != 0u) {   // (not all of it, after a wait that gave up: late arrivals have 2 ms)
        const uint64_t t0 = ptx::globaltimer_ns();
        while (ptx::globaltimer_ns() - t0 < ptx::kWaitLimitNs / 1000) {
        }
    }
    __syncwarp();
    if (warp == 9) {
        ptx::tc_fence_after_sync();
        ptx::tmem_dealloc_pair(tmem, 512);
    }
}

}  // namespace w4a8
