// blocks.cu -- copies of whole cache blocks (C5) by (source, destination) pairs, in the pools of every
// layer at once: the tails of forked branches, the moves of a compaction, a pool that is replaced by a
// larger or smaller one. Layers share their block tables, so one list of pairs serves all of them.
#include "common.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kPiece = 8;    // 16-byte pieces a lane
constexpr int kPools = 32;   // pools of one launch (their addresses travel as kernel arguments)

struct CopyArgs {
    const uint4 *src[2 * kPools];   // K and V of each pool
    uint4 *dst[2 * kPools];
    const float *src_scales[2 * kPools];
    float *dst_scales[2 * kPools];
    const int32_t *src_blocks, *dst_blocks;
    int32_t src_num, dst_num, vecs, scales;   // 16-byte pieces and fp32 scales of a block
    int32_t parts, count;                     // warps a block, pairs
    int *err;
};

// A warp takes kPiece 16-byte pieces a lane of one array (a pool's K or V, blockIdx.y) of one pair; the loads of a
// piece are all in flight together. Bound by HBM: a block is read once and written once. 6001 FP8 blocks (98.5 MB
// both ways) took 20.8 us with a CTA per (pair, array), one load a thread.
__global__ void __launch_bounds__(kThreads) copy_blocks_kernel(const __grid_constant__ CopyArgs p)
{
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int64_t pair = p.parts == 1 ? w : w / p.parts;
    if (pair >= p.count) return;
    const int part = (int)(w - pair * p.parts), lane = threadIdx.x & 31;
    const int32_t s = p.src_blocks[pair], d = p.dst_blocks[pair];
    const bool s_ok = s >= 0 && s < p.src_num;
    if (!s_ok || d < 0 || d >= p.dst_num) {
        if (lane == 0) padoc_record_error(p.err, PADOC_DEVERR_BLOCK_ID, s_ok ? d : s);
        return;
    }
    const int first = part * 32 * kPiece + lane;
    const uint4 *src = p.src[blockIdx.y] + (int64_t)s * p.vecs + first;
    uint4 *dst = p.dst[blockIdx.y] + (int64_t)d * p.vecs + first;
    uint4 x[kPiece];
#pragma unroll
    for (int j = 0; j < kPiece; ++j)
        if (first + 32 * j < p.vecs) x[j] = src[32 * j];
    if (part == 0)
        for (int i = lane; i < p.scales; i += 32)
            p.dst_scales[blockIdx.y][(int64_t)d * p.scales + i] = p.src_scales[blockIdx.y][(int64_t)s * p.scales + i];
#pragma unroll
    for (int j = 0; j < kPiece; ++j)
        if (first + 32 * j < p.vecs) dst[32 * j] = x[j];
}

// Launches the copies of all pools, kPools at a time; fill(j, a, i) puts pool j's addresses at entry i.
template <typename Fill>
padoc_status copy_pools(CopyArgs &p, int32_t num_pools, int32_t count, padoc_stream_t stream, Fill fill)
{
    p.count = count;
    p.parts = (p.vecs + 32 * kPiece - 1) / (32 * kPiece);
    const int64_t ctas = ((int64_t)count * p.parts + kThreads / 32 - 1) / (kThreads / 32);
    if (ctas > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    for (int32_t first = 0; first < num_pools; first += kPools) {
        const int32_t n = num_pools - first < kPools ? num_pools - first : kPools;
        for (int32_t i = 0; i < n; ++i) fill(first + i, p, i);
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3((unsigned)ctas, (unsigned)(2 * n));
        lc.blockDim = dim3(kThreads);
        lc.stream = (cudaStream_t)stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // see the kernel's wait
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        lc.attrs = attr;
        lc.numAttrs = 1;
        PADOC_CUDA_TRY(cudaLaunchKernelEx(&lc, copy_blocks_kernel, p));
        const padoc_status st = padoc_launch_status();
        if (st != PADOC_OK) return st;
    }
    return PADOC_OK;
}

bool aligned(const void *p, uintptr_t mask) { return p && !(((uintptr_t)p) & mask); }

}  // namespace

extern "C" padoc_status padoc_copy_kv_blocks(const padoc_kv_pool *dst, const padoc_kv_pool *src, int32_t num_pools,
                                             const int32_t *src_blocks, const int32_t *dst_blocks, int32_t count,
                                             padoc_stream_t stream)
{
    if (!dst || !src || num_pools < 0 || count < 0) return PADOC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < num_pools; ++i) {
        for (const padoc_kv_pool *q : {&dst[i], &src[i]})
            if (q->block_size != dst[0].block_size || q->num_kv_heads != dst[0].num_kv_heads ||
                q->head_dim != dst[0].head_dim || q->dtype != dst[0].dtype || !aligned(q->k_pool, 15) || !aligned(q->v_pool, 15))
                return PADOC_ERR_INVALID_ARGUMENT;
        if (dst[i].num_blocks != dst[0].num_blocks || src[i].num_blocks != src[0].num_blocks) return PADOC_ERR_INVALID_ARGUMENT;
    }
    if (num_pools == 0) return PADOC_OK;
    const padoc_kv_pool &d0 = dst[0];
    if (d0.num_blocks < 1 || src[0].num_blocks < 1 || d0.block_size < 1 || d0.num_kv_heads < 1 || d0.head_dim < 1)
        return PADOC_ERR_INVALID_ARGUMENT;
    if (d0.dtype != PADOC_DTYPE_BF16 && d0.dtype != PADOC_DTYPE_F32) return PADOC_ERR_INVALID_ARGUMENT;
    const int64_t elts = (int64_t)d0.block_size * d0.num_kv_heads;
    if (elts > (1 << 24) || d0.head_dim > (1 << 12)) return PADOC_ERR_UNSUPPORTED;
    const int64_t bytes = elts * d0.head_dim * (d0.dtype == PADOC_DTYPE_BF16 ? 2 : 4);
    if (bytes % 16 != 0 || bytes / 16 > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    if (count == 0) return PADOC_OK;
    if (!aligned(src_blocks, 3) || !aligned(dst_blocks, 3)) return PADOC_ERR_INVALID_ARGUMENT;
    CopyArgs p = {};
    p.src_blocks = src_blocks, p.dst_blocks = dst_blocks;
    p.src_num = src[0].num_blocks, p.dst_num = d0.num_blocks;
    p.vecs = (int32_t)(bytes / 16);
    p.err = padoc_device_error_word();
    if (!p.err) return PADOC_ERR_CUDA;
    return copy_pools(p, num_pools, count, stream, [&](int32_t j, CopyArgs &a, int32_t i) {
        a.src[2 * i] = (const uint4 *)src[j].k_pool, a.src[2 * i + 1] = (const uint4 *)src[j].v_pool;
        a.dst[2 * i] = (uint4 *)dst[j].k_pool, a.dst[2 * i + 1] = (uint4 *)dst[j].v_pool;
    });
}

extern "C" padoc_status padoc_copy_kv_blocks_e4m3(const padoc_kv_pool_e4m3 *dst, const padoc_kv_pool_e4m3 *src,
                                                  int32_t num_pools, const int32_t *src_blocks, const int32_t *dst_blocks,
                                                  int32_t count, padoc_stream_t stream)
{
    if (!dst || !src || num_pools < 0 || count < 0) return PADOC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < num_pools; ++i) {
        for (const padoc_kv_pool_e4m3 *q : {&dst[i], &src[i]})
            if (q->block_size != dst[0].block_size || q->num_kv_heads != dst[0].num_kv_heads ||
                q->head_dim != dst[0].head_dim || !aligned(q->k_codes, 15) || !aligned(q->v_codes, 15) ||
                !aligned(q->k_scales, 3) || !aligned(q->v_scales, 3))
                return PADOC_ERR_INVALID_ARGUMENT;
        if (dst[i].num_blocks != dst[0].num_blocks || src[i].num_blocks != src[0].num_blocks) return PADOC_ERR_INVALID_ARGUMENT;
    }
    if (num_pools == 0) return PADOC_OK;
    const padoc_kv_pool_e4m3 &d0 = dst[0];
    if (d0.num_blocks < 1 || src[0].num_blocks < 1 || d0.num_kv_heads < 1) return PADOC_ERR_INVALID_ARGUMENT;
    if (d0.block_size != 16 || d0.head_dim != 128 || d0.num_kv_heads > 65535) return PADOC_ERR_UNSUPPORTED;
    if (count == 0) return PADOC_OK;
    if (!aligned(src_blocks, 3) || !aligned(dst_blocks, 3)) return PADOC_ERR_INVALID_ARGUMENT;
    CopyArgs p = {};
    p.src_blocks = src_blocks, p.dst_blocks = dst_blocks;
    p.src_num = src[0].num_blocks, p.dst_num = d0.num_blocks;
    p.vecs = d0.num_kv_heads * (16 * 128 / 16);
    p.scales = d0.num_kv_heads;
    p.err = padoc_device_error_word();
    if (!p.err) return PADOC_ERR_CUDA;
    return copy_pools(p, num_pools, count, stream, [&](int32_t j, CopyArgs &a, int32_t i) {
        a.src[2 * i] = (const uint4 *)src[j].k_codes, a.src[2 * i + 1] = (const uint4 *)src[j].v_codes;
        a.dst[2 * i] = (uint4 *)dst[j].k_codes, a.dst[2 * i + 1] = (uint4 *)dst[j].v_codes;
        a.src_scales[2 * i] = src[j].k_scales, a.src_scales[2 * i + 1] = src[j].v_scales;
        a.dst_scales[2 * i] = (float *)dst[j].k_scales, a.dst_scales[2 * i + 1] = (float *)dst[j].v_scales;
    });
}
