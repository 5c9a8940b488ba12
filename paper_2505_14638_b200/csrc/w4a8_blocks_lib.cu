// C-ABI entry points for FP8 layers with block scales and for mixture-of-experts blocks (see include/w4a8.h): argument
// validation, plans and launches.  Nothing here allocates device memory.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

#include "../../include/w4a8.h"
#include "w4a8_block_kernels.cuh"
#include "w4a8_blocks_plan.h"
#include "w4a8_internal.h"
#include "w4a8_linear_blocks.cuh"
#include "w4a8_route.cuh"

namespace w4a8 {

// Launch with programmatic stream serialization (every kernel here waits for the one before it ahead of its first access) and,
// for cluster > 1, as thread-block clusters.
template <class... Params, class... Args>
static int launch(void (*kernel)(Params...), unsigned grid, unsigned block, size_t smem, int cluster, cudaStream_t st, Args... args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...);
    count_launch();
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return W4A8_ERR_CUDA;
    }
    return launch_status();
}

// The most dynamic shared memory a block may have, for `kernel` on the current device (set once per kernel and device).
template <class Kernel>
static bool allow_smem(Kernel kernel, std::atomic<uint64_t>& done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
    if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev & 1u)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBlocksSmemMax) != cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return true;
}

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

static unsigned grid_for(int64_t units, int64_t per_block, int sms, int per_sm) {
    const int64_t want = ceil_div(units, per_block), most = (int64_t)sms * per_sm;
    return (unsigned)(want < most ? want : most);
}

static int quantize_blocks_impl(const void* x, int64_t M, int64_t K, int64_t ldx, int kind, const int32_t* slots, int top_k,
                                uint8_t* x8, int64_t rows, int64_t ldx8, float* s_x, int64_t lds, cudaStream_t st) {
    if (!x || !x8 || !s_x) return W4A8_ERR_INVALID_ARG;
    if (M <= 0 || K <= 0 || rows <= 0 || top_k < 0) return W4A8_ERR_INVALID_ARG;
    if (kind != W4A8_CHAIN_INPUT_PLAIN && kind != W4A8_CHAIN_INPUT_SILU_MUL) return W4A8_ERR_INVALID_ARG;
    if ((slots == nullptr) != (top_k == 0)) return W4A8_ERR_INVALID_ARG;
    const int64_t width = kind == W4A8_CHAIN_INPUT_SILU_MUL ? 2 * K : K;
    if (M > INT32_MAX || rows > INT32_MAX || K > INT32_MAX / 2) return W4A8_ERR_BAD_SHAPE;
    if (K % 16 != 0 || ldx < width || ldx8 < K || lds < ceil_div(K, 128)) return W4A8_ERR_BAD_SHAPE;
    if (top_k == 0 && rows < M) return W4A8_ERR_BAD_SHAPE;
    if (!aligned16(x) || !aligned16(x8) || ldx % 8 != 0 || ldx8 % 16 != 0 || !aligned4(s_x) || !aligned4(slots))
        return W4A8_ERR_BAD_ALIGNMENT;
    const int rc = check_device();
    if (rc != W4A8_OK) return rc;
    const int sms = sm_count();
    if (sms <= 0) return W4A8_ERR_CUDA;
    const unsigned grid = grid_for(M * ceil_div(K, 512), 8, sms, 8);
    return kind == W4A8_CHAIN_INPUT_SILU_MUL
               ? launch(quantize_blocks_kernel<true>, grid, 256, 0, 1, st, static_cast<const uint16_t*>(x), (int)M, (int)K, ldx, slots, top_k, x8, rows, ldx8, s_x, lds)
               : launch(quantize_blocks_kernel<false>, grid, 256, 0, 1, st, static_cast<const uint16_t*>(x), (int)M, (int)K, ldx, slots, top_k, x8, rows, ldx8, s_x, lds);
}

// ------------------------------------------------------------------------------ linear layers
static bool make_map(CUtensorMap* m, const void* ptr, uint32_t rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box,
                     CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_UINT8) {
    EncodeTiledFn fn = encode_tiled_fn();
    const cuuint32_t step[3] = {1, 1, 1};
    return fn && fn(m, type, rank, const_cast<void*>(ptr), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static_assert(sizeof(ExpertTable) <= (size_t)kBlocksTableBytes, "the table's place in shared memory");

template <int TMAX>
static int launch_blocks(const CUtensorMap& tw, const CUtensorMap& tx, const BlocksParams& p, const BlocksPlan& pl, int sms, int64_t tiles, cudaStream_t st) {
    using Cfg = BlocksCfg<TMAX>;
    static std::atomic<uint64_t> allowed{0};
    if (!allow_smem(linear_blocks_kernel<Cfg>, allowed)) return W4A8_ERR_CUDA;
    const int64_t most = (int64_t)sms * pl.ctas / pl.cut, clusters = tiles < most ? tiles : most;
    return launch(linear_blocks_kernel<Cfg>, (unsigned)(clusters * pl.cut), Cfg::kThreads, (size_t)pl.smem, pl.cut, st, tw, tx, p);
}

static int linear_blocks_impl(const uint8_t* x8, int64_t ldx8, const float* s_x, int64_t lds, int64_t rows, const int32_t* offsets,
                              int64_t experts, const uint8_t* w8, int64_t ldw, int64_t w_stride, const float* s_w, int64_t N, int64_t K,
                              void* y, int64_t ldy, int out_dtype, cudaStream_t st) {
    if (!x8 || !s_x || !w8 || !s_w || !y) return W4A8_ERR_INVALID_ARG;
    if (rows <= 0 || N <= 0 || K <= 0 || experts <= 0) return W4A8_ERR_INVALID_ARG;
    if (out_dtype != W4A8_OUT_BF16 && out_dtype != W4A8_OUT_FP32) return W4A8_ERR_INVALID_ARG;
    if (rows > INT32_MAX - 256 || N > INT32_MAX / 2 || K > INT32_MAX / 2 || experts > kBlocksMaxExperts) return W4A8_ERR_BAD_SHAPE;
    const int64_t KB = ceil_div(K, 128), NB = ceil_div(N, 128);
    if (K % 16 != 0 || N % 16 != 0 || ldx8 < K || ldw < K || ldy < N || lds < KB) return W4A8_ERR_BAD_SHAPE;
    if (experts > 1 && w_stride < (N - 1) * ldw + K) return W4A8_ERR_BAD_SHAPE;
    if (!aligned16(x8) || !aligned16(w8) || !aligned16(y) || ldx8 % 16 != 0 || ldw % 16 != 0 || w_stride % 16 != 0 || !aligned4(s_x) ||
        !aligned4(s_w) || !aligned4(offsets))
        return W4A8_ERR_BAD_ALIGNMENT;
    int rc = check_device();
    if (rc != W4A8_OK) return rc;
    const int sms = sm_count();
    unsigned int* status = status_word_ptr();
    if (sms <= 0 || !status) return W4A8_ERR_CUDA;
    const BlocksPlan pl = blocks_plan(rows, experts, N, K, sms, offsets != nullptr);
    // (with experts: at most)
    const int64_t tiles = ceil_div(N, pl.wide ? 256 : pl.channels) * (ceil_div(rows, pl.tokens) + (offsets ? experts : 0));
    if (tiles > INT32_MAX / 2) return W4A8_ERR_BAD_SHAPE;
    CUtensorMap tw, tx;
    {
        const cuuint64_t dims[3] = {(cuuint64_t)K, (cuuint64_t)N, (cuuint64_t)experts};
        const cuuint64_t strides[2] = {(cuuint64_t)ldw, (cuuint64_t)(experts > 1 ? w_stride : N * ldw)};
        const cuuint32_t box[3] = {128, pl.wide ? 128u : (cuuint32_t)pl.channels, 1};
        if (!make_map(&tw, w8, 3, dims, strides, box)) return W4A8_ERR_CUDA;
    }
    {
        const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ldx8};
        const cuuint32_t box[2] = {128, pl.wide ? 128u : 32u};
        if (!make_map(&tx, x8, 2, dims, strides, box)) return W4A8_ERR_CUDA;
    }
    BlocksParams p = {};
    p.s_x = s_x;
    p.s_w = s_w;
    p.offsets = offsets;
    p.y = y;
    p.lds = lds;
    p.ldy = ldy;
    p.rows = rows;
    p.E = (int)experts;
    p.N = (int)N;
    p.KB = (int)KB;
    p.NB = (int)NB;
    p.tokens = pl.tokens;
    p.out_fp32 = out_dtype == W4A8_OUT_FP32 ? 1 : 0;
    p.status = status;
    if (pl.wide) {
        CUtensorMap ty = tx;   // (not used where rows of y are not 16-byte aligned)
        const int es = p.out_fp32 ? 4 : 2;
        if (ldy * es % 16 == 0) {
            const cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(ldy * es)};
            const cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32};
            if (!make_map(&ty, y, 2, dims, strides, box, p.out_fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16)) return W4A8_ERR_CUDA;
        }
        static std::atomic<uint64_t> allowed{0};
        if (!allow_smem(linear_blocks_wide_kernel, allowed)) return W4A8_ERR_CUDA;
        return launch(linear_blocks_wide_kernel, (unsigned)(tiles < sms ? tiles : sms), kWideThreads, (size_t)wide_smem(offsets != nullptr), 1, st, tw, tx, ty, p);
    }
    p.channels = pl.channels;
    p.row_tiles = (int)ceil_div(N, pl.channels);
    p.cut = pl.cut;
    p.share = pl.share;
    p.stages = pl.stages;
    p.xslot = (pl.tokens + 31) / 32 * 4096;
    p.part_buffers = pl.part_buffers;
    switch (pl.tmax) {
        case 16: return launch_blocks<16>(tw, tx, p, pl, sms, tiles, st);
        case 32: return launch_blocks<32>(tw, tx, p, pl, sms, tiles, st);
        case 64: return launch_blocks<64>(tw, tx, p, pl, sms, tiles, st);
        default: return launch_blocks<128>(tw, tx, p, pl, sms, tiles, st);
    }
}

// ------------------------------------------------------------------------------ routing
// Whole clusters of CTAs; up to a token per warp of a cluster: a single one.
static void route_chunks(int64_t M, int* chunk, int* chunks) {
    int64_t per = ceil_div(M, M <= kRouteCluster * kRouteWarps ? kRouteCluster : kRouteChunks);
    if (M > kRouteCluster * kRouteWarps && per < kRouteWarps) per = kRouteWarps;
    *chunk = (int)per;
    *chunks = (int)(ceil_div(ceil_div(M, per), kRouteCluster) * kRouteCluster);
}

template <int V>
static int launch_choose(const RouteParams& p, bool wide, cudaStream_t st) {
    return wide ? launch(route_choose_kernel<V, true>, (unsigned)p.chunks, kRouteWarps * 32, 0, kRouteCluster, st, p)
                : launch(route_choose_kernel<V, false>, (unsigned)p.chunks, kRouteWarps * 32, 0, kRouteCluster, st, p);
}

}  // namespace w4a8

using namespace w4a8;

extern "C" {

int w4a8_quantize_act_blocks(const void* x_bf16, int64_t M, int64_t K, int64_t ldx, int input_kind, const int32_t* slots, int top_k,
                             uint8_t* x8, int64_t rows, int64_t ldx8, float* s_x, int64_t lds, void* stream) {
    return quantize_blocks_impl(x_bf16, M, K, ldx, input_kind, slots, top_k, x8, rows, ldx8, s_x, lds, static_cast<cudaStream_t>(stream));
}

int w4a8_linear_fp8_blocks(const uint8_t* x8, int64_t ldx8, const float* s_x, int64_t lds, int64_t M, const uint8_t* w8, int64_t ldw,
                           const float* s_w, int64_t N, int64_t K, void* y, int64_t ldy, int out_dtype, void* stream) {
    return linear_blocks_impl(x8, ldx8, s_x, lds, M, nullptr, 1, w8, ldw, 0, s_w, N, K, y, ldy, out_dtype, static_cast<cudaStream_t>(stream));
}

int w4a8_linear_fp8_experts(const uint8_t* x8, int64_t ldx8, const float* s_x, int64_t lds, int64_t rows, const int32_t* offsets,
                            int64_t experts, const uint8_t* w8, int64_t ldw, int64_t w_stride, const float* s_w, int64_t N, int64_t K,
                            void* y, int64_t ldy, int out_dtype, void* stream) {
    if (!offsets) return W4A8_ERR_INVALID_ARG;
    return linear_blocks_impl(x8, ldx8, s_x, lds, rows, offsets, experts, w8, ldw, w_stride, s_w, N, K, y, ldy, out_dtype, static_cast<cudaStream_t>(stream));
}

size_t w4a8_route_experts_workspace_bytes(int64_t M, int64_t experts) {
    if (M <= 0 || experts <= 0 || experts > kRouteMaxExperts) return 0;
    int chunk, chunks;
    route_chunks(M, &chunk, &chunks);
    return chunks > kRouteCluster ? (size_t)(chunks / kRouteCluster) * (size_t)experts * sizeof(uint32_t) : 0;
}

int w4a8_route_experts(const void* logits, int logits_dtype, int64_t M, int64_t ldl, int64_t experts, int top_k, int score,
                       const float* bias, int groups, int top_groups, int group_best, int renormalize, float scale, int32_t* ids,
                       float* weights, int32_t* offsets, int32_t* slots, void* workspace, size_t workspace_bytes, void* stream) {
    if (!logits || !ids || !weights || !offsets || !slots) return W4A8_ERR_INVALID_ARG;
    if (M <= 0 || experts <= 0 || top_k <= 0 || groups <= 0 || top_groups <= 0) return W4A8_ERR_INVALID_ARG;
    if (logits_dtype != W4A8_OUT_BF16 && logits_dtype != W4A8_OUT_FP32) return W4A8_ERR_INVALID_ARG;
    if (score != W4A8_SCORE_SOFTMAX && score != W4A8_SCORE_SIGMOID) return W4A8_ERR_INVALID_ARG;
    if (group_best != 1 && group_best != 2) return W4A8_ERR_INVALID_ARG;
    if (renormalize != 0 && renormalize != 1) return W4A8_ERR_INVALID_ARG;
    if (experts > kRouteMaxExperts || top_k > kRouteMaxTopK || groups > kRouteMaxGroups) return W4A8_ERR_BAD_SHAPE;
    if (experts % groups != 0 || top_groups > groups || top_k > experts / groups * top_groups) return W4A8_ERR_BAD_SHAPE;
    if (ldl < experts || M > INT32_MAX / top_k) return W4A8_ERR_BAD_SHAPE;
    if ((reinterpret_cast<uintptr_t>(logits) & (logits_dtype == W4A8_OUT_FP32 ? 3u : 1u)) || !aligned4(bias) || !aligned4(ids) ||
        !aligned4(weights) || !aligned4(offsets) || !aligned4(slots) || !aligned4(workspace))
        return W4A8_ERR_BAD_ALIGNMENT;
    const size_t need = w4a8_route_experts_workspace_bytes(M, experts);
    if (need > 0 && (!workspace || workspace_bytes < need)) return W4A8_ERR_WORKSPACE_TOO_SMALL;
    int rc = check_device();
    if (rc != W4A8_OK) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    RouteParams p = {};
    p.logits = logits;
    p.ldl = ldl;
    p.bias = bias;
    p.ids = ids;
    p.offsets = offsets;
    p.slots = slots;
    p.weights = weights;
    p.counts = static_cast<uint32_t*>(workspace);
    p.M = M;
    p.E = (int)experts;
    p.top_k = top_k;
    p.groups = groups;
    p.top_groups = top_groups;
    p.group_best = group_best;
    p.logits_fp32 = logits_dtype == W4A8_OUT_FP32 ? 1 : 0;
    p.sigmoid = score == W4A8_SCORE_SIGMOID ? 1 : 0;
    p.renormalize = renormalize;
    p.scale = scale;
    route_chunks(M, &p.chunk, &p.chunks);
    const bool wide = bias != nullptr || (groups > 1 && group_best == 2);
    if (experts <= 32) rc = launch_choose<1>(p, wide, st);
    else if (experts <= 64) rc = launch_choose<2>(p, wide, st);
    else if (experts <= 128) rc = launch_choose<4>(p, wide, st);
    else if (experts <= 256) rc = launch_choose<8>(p, wide, st);
    else rc = launch_choose<16>(p, wide, st);
    if (rc != W4A8_OK || p.chunks == kRouteCluster) return rc;
    return launch(route_place_kernel, (unsigned)p.chunks, kRouteWarps * 32, 0, 1, st, p);
}

int w4a8_combine_experts(const void* y, int y_dtype, int64_t rows, int64_t ldy, const int32_t* slots, const float* weights, int64_t M,
                         int top_k, int64_t N, const void* add, int64_t ldadd, void* out, int64_t ldo, int out_dtype, void* stream) {
    if (!y || !slots || !weights || !out) return W4A8_ERR_INVALID_ARG;
    if (M <= 0 || rows <= 0 || N <= 0 || top_k <= 0) return W4A8_ERR_INVALID_ARG;
    if (y_dtype != W4A8_OUT_BF16 && y_dtype != W4A8_OUT_FP32) return W4A8_ERR_INVALID_ARG;
    if (out_dtype != W4A8_OUT_BF16 && out_dtype != W4A8_OUT_FP32) return W4A8_ERR_INVALID_ARG;
    if (rows > INT32_MAX || N > INT32_MAX / 2 || M > INT32_MAX / top_k) return W4A8_ERR_BAD_SHAPE;
    if (N % 16 != 0 || ldy < N || ldo < N || (add && ldadd < N)) return W4A8_ERR_BAD_SHAPE;
    const int64_t unit_y = y_dtype == W4A8_OUT_FP32 ? 4 : 8, unit_o = out_dtype == W4A8_OUT_FP32 ? 4 : 8;   // values in 16 bytes
    if (!aligned16(y) || !aligned16(out) || !aligned16(add) || ldy % unit_y != 0 || ldo % unit_o != 0 || (add && ldadd % unit_o != 0) ||
        !aligned4(slots) || !aligned4(weights))
        return W4A8_ERR_BAD_ALIGNMENT;
    const int rc = check_device();
    if (rc != W4A8_OK) return rc;
    const int sms = sm_count();
    if (sms <= 0) return W4A8_ERR_CUDA;
    const unsigned grid = grid_for(M * (N / 8), 256, sms, 8);
    auto kernel = y_dtype == W4A8_OUT_FP32 ? (out_dtype == W4A8_OUT_FP32 ? combine_experts_kernel<true, true> : combine_experts_kernel<true, false>)
                                           : (out_dtype == W4A8_OUT_FP32 ? combine_experts_kernel<false, true> : combine_experts_kernel<false, false>);
    return launch(kernel, grid, 256, 0, 1, static_cast<cudaStream_t>(stream), y, rows, ldy, slots, weights, M, top_k, (int)N, add, ldadd, out, ldo);
}

}  // extern "C"
