// rotary.cu -- what stands between a model's projections and the attention kernels: the RMS norm of every
// query and key head (or none) and rotary positions with up to four axes (time, height, width of images
// and video), for packed rows (the training forward) with their gradients, and for a step's or a
// prefix's rows on their way into the paged pool (C5, Algorithm 1's append).
#include <cfloat>
#include <cmath>

#include "common.cuh"
#include "rotary.cuh"

namespace padoc_rotary_dev {

namespace {

constexpr int kWarps = 4;   // warps per CTA

// See row_part. kCtas: CTAs an SM that the registers have to allow. With the norm a row's steps take longer than its
// loads, so many rows want one more CTA on an SM than the compiler's own choice gives (96 registers, 5 CTAs), even at a
// few spilled values (8 bytes, 24 in the general form); few rows want the loads first. 16 + 2 heads of 128 dims in bf16,
// own choice / 6 / 7 CTAs: 10001 rows 18.7 / 19.0 / 20.8 us, 32768 49.4 / 48.0 / 53.3; 64 dims, 65536 rows 59.9 / 57.1 /
// 55.7; 256 dims, 16384 rows 51.8 / 50.1 / 53.7; 80 dims (the general form), 10001 rows 17.3 / 16.0 / 15.8, 52428 70.3 /
// 62.2 / 59.9. Adjacent pairs, which are turned one by one, lose by it: 26041 rows 43.3 / 46.9 / 49.1. Appends: see
// steps_of.
template <typename T, int V, bool kAdjacent, bool kNorm, int kMode, int kGroup, int kCtas>
__global__ void __launch_bounds__(32 * kWarps, kCtas) rotary_kernel(const __grid_constant__ Args p)
{
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int64_t i = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (i < p.count) row_part<T, V, kAdjacent, kNorm, kMode, kGroup>(p, i, blockIdx.y);
}

constexpr int kBwdWarps = 8;    // warps per CTA of the backward with the norm
constexpr int kBwdStages = 3;   // steps of a warp whose loads are in flight (2: 80.9, 3: 79.3, 4: 79.9, 6: 84.9 us for 32768 rows)

struct BwdArgs {
    Spec sp;                                // turns back
    const void *q, *k;                      // the forward's inputs
    int64_t q_stride, k_stride;
    const int32_t *pos;
    int64_t rows;
    int32_t hq, hkv, group;
    const void *dq_out, *dk_out;
    int64_t dq_out_stride, dk_out_stride;
    void *dq, *dk;
    int64_t dq_stride, dk_stride;
    float *part;                            // [CTAs][2][d]
};

// A vector of 16 or 8 bytes; bytes 0 writes zeros and reads nothing.
template <int kBytes>
__device__ __forceinline__ void cp_async_vec(uint32_t dst, const void *src, uint32_t bytes)
{
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// The backward with the norm. Persistent CTAs, a warp per row, as many heads a step as fit. Registers hold
// the weights' gradient sums and the angles, so the rows' values come through shared memory: every lane copies its
// own vectors kBwdStages steps ahead (cp.async) and reads them back itself, without a barrier. A CTA joins its
// warps' sums in a fixed order and writes one partial row, which rotary_weight_grad_kernel adds up (no atomics:
// the same call gives the same bits). Arithmetic is on packed pairs, weights come from shared memory in fp32.
// The packed batch of 32768 rows (453 MB): 276 us with plain loads, one step at a time, at 178 registers; 115 us
// through the ring with scalar arithmetic (2620 instructions a row); 76.3 us now (87% of the copy rate), bound by the
// latency of a step's chain (two sums over the head) at the 16 warps an SM that the sums' registers leave. Steps of
// query and of key heads apart take 74.4 us there, but 79.9 instead of 69.7 at 7 + 1 heads and 95 instead of 87 at
// 80 dims, where they leave lanes without a head. The general form (kGroup 0) in bf16 spills 4 to 8 bytes.
// kGroup: see Lane.
template <typename T, int V, bool kAdjacent, int kGroup>
__global__ void __launch_bounds__(32 * kBwdWarps, 2) rotary_norm_bwd_kernel(const __grid_constant__ BwdArgs p)
{
    using Vec = Raw<T, V>;
    constexpr int kPairs = V / 2;
    // [2][kPairs][group] weights in fp32, four to a piece, the pieces of a lane's two vectors; then
    // [kBwdWarps][kBwdStages][4][32] vectors; at the end [kBwdWarps][2][d] sums
    extern __shared__ uint4 smem_raw[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Lane l = warp_lane<kGroup>(p.group);
    const int group = l.group, heads = l.heads, sub = l.sub, chunk = l.chunk;
    const Place pl = lane_place<V>(chunk, l.used, p.sp.d, p.sp.rot);
    const int d = p.sp.d;
    Vec *ring = reinterpret_cast<Vec *>(smem_raw + 2 * kPairs * group) + (size_t)warp * kBwdStages * 4 * 32 + lane;
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    for (int e = threadIdx.x; e < 2 * kPairs * group; e += 32 * kBwdWarps) {
        const int kind = e >= kPairs * group, piece = e / group - kind * kPairs;
        const Place at = lane_place<V>(e % group, true, d, p.sp.rot);
        const T *w = static_cast<const T *>(kind ? p.sp.k_weight : p.sp.q_weight) +
                     (piece < kPairs / 2 ? at.a + 4 * piece : at.b + 4 * (piece - kPairs / 2));
        reinterpret_cast<float4 *>(smem_raw)[e] = make_float4((float)w[0], (float)w[1], (float)w[2], (float)w[3]);
    }
    __syncthreads();
    // a CTA's rows lie behind one another (a grid apart: 3% slower)
    const int64_t first = p.rows * blockIdx.x / gridDim.x + warp, row_end = p.rows * (blockIdx.x + 1) / gridDim.x;

    // the next step to be copied: its row and first head (the queries', then the keys'), the addresses of the lane's
    // first vectors there (of a query head), and its stage; lanes without a head there get zeros
    const int total = p.hq + p.hkv;
    int64_t ahead_row = first;
    int ahead_head = 0;
    uint32_t ahead_at = smem_u32(ring);
    const uint32_t ring_end = ahead_at + kBwdStages * 4 * 32 * (uint32_t)sizeof(Vec);
    const int lane_at = sub * d + pl.a, to_b = pl.b - pl.a, step_at = heads * d;
    const T *ax = static_cast<const T *>(p.q) + first * p.q_stride + lane_at;
    const T *ag = static_cast<const T *>(p.dq_out) + first * p.dq_out_stride + lane_at;
    auto copy_ahead = [&]() {
        if (ahead_row < row_end) {
            constexpr uint32_t kNext = 32 * sizeof(Vec);
            const uint32_t bytes = pl.active && ahead_head + sub < total ? (uint32_t)sizeof(Vec) : 0u;
            const T *x = ax, *g = ag;
            if (ahead_head + heads > p.hq && ahead_head + sub >= p.hq) {
                const int at = (ahead_head - p.hq) * d + lane_at;
                x = static_cast<const T *>(p.k) + ahead_row * p.k_stride + at;
                g = static_cast<const T *>(p.dk_out) + ahead_row * p.dk_out_stride + at;
            }
            cp_async_vec<sizeof(Vec)>(ahead_at, x, bytes);
            cp_async_vec<sizeof(Vec)>(ahead_at + kNext, x + to_b, bytes);
            cp_async_vec<sizeof(Vec)>(ahead_at + 2 * kNext, g, bytes);
            cp_async_vec<sizeof(Vec)>(ahead_at + 3 * kNext, g + to_b, bytes);
            ax += step_at;
            ag += step_at;
            ahead_head += heads;
            if (ahead_head >= total) {
                ahead_head = 0;
                ahead_row += kBwdWarps;
                ax = static_cast<const T *>(p.q) + ahead_row * p.q_stride + lane_at;
                ag = static_cast<const T *>(p.dq_out) + ahead_row * p.dq_out_stride + lane_at;
            }
        }
        cp_async_commit();
        ahead_at += 4 * 32 * (uint32_t)sizeof(Vec);
        if (ahead_at == ring_end) ahead_at -= kBwdStages * 4 * 32 * (uint32_t)sizeof(Vec);
    };
#pragma unroll
    for (int j = 0; j < kBwdStages; ++j) copy_ahead();

    const float inv_d = 1.f / (float)d;
    const bool whole = p.sp.rot == d;
    // sums of g h, the pairs of the lane's first, then of its second vector: the queries' in registers, the keys' (a
    // step in five at 16 + 2 heads) in shared memory
    uint64_t acc[V];
    ulonglong2 *acc_k = reinterpret_cast<ulonglong2 *>(smem_raw + 2 * kPairs * group + kBwdWarps * kBwdStages * 4 * 32 * sizeof(Vec) / 16) + warp * kPairs * 32 + lane;
#pragma unroll
    for (int j = 0; j < V; ++j) acc[j] = 0;
#pragma unroll
    for (int j = 0; j < V / 2; ++j) acc_k[j * 32] = make_ulonglong2(0, 0);
    int stage = 0;
    for (int64_t row = first; row < row_end; row += kBwdWarps) {
        uint64_t c[kPairs], s[kPairs];
        lane_angles<V, kAdjacent, sizeof(T) == 2, kGroup>(p.sp, p.pos, row, l, pl.turned, c, s);
        T *out_q = static_cast<T *>(p.dq) + row * p.dq_stride + lane_at;
#pragma unroll 1
        for (int h0 = 0; h0 < total; h0 += heads, out_q += step_at) {
            cp_async_wait<kBwdStages - 1>();
            const bool is_q = h0 + sub < p.hq;
            const ulonglong2 *w = reinterpret_cast<const ulonglong2 *>(smem_raw) + (is_q ? 0 : kPairs * group) + chunk;
            auto read_weights = [&](uint64_t(&wa)[kPairs], uint64_t(&wb)[kPairs]) {
#pragma unroll
                for (int j = 0; j < kPairs / 2; ++j) {
                    const ulonglong2 a = w[j * group], b = w[(kPairs / 2 + j) * group];
                    wa[2 * j] = a.x, wa[2 * j + 1] = a.y;
                    wb[2 * j] = b.x, wb[2 * j + 1] = b.y;
                }
            };
            const Vec *in = ring + stage * 4 * 32;
            uint64_t xa[kPairs], xb[kPairs], a[kPairs], b[kPairs], wa[kPairs], wb[kPairs];
            unpack2(in[0], xa);
            unpack2(in[32], xb);
            unpack2(in[64], a);
            unpack2(in[96], b);
            if (whole) turn_pairs<V, kAdjacent>(a, b, c, s);
            else if (pl.turned) turn_pairs<V, kAdjacent>(a, b, c, s);
            read_weights(wa, wb);
            uint64_t s2 = 0, d2 = 0;
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                s2 = f2_fma(xa[j], xa[j], f2_fma(xb[j], xb[j], s2));
                d2 = f2_fma(f2_mul(a[j], wa[j]), xa[j], f2_fma(f2_mul(b[j], wb[j]), xb[j], d2));
            }
            float r = rsqrtf(group_sum<kGroup>(f2_sum(s2), l) * inv_d + p.sp.eps);
            if (h0 + sub >= total) r = 0.f;   // no head: its zeros must not meet an infinite scale
            const float m = group_sum<kGroup>(f2_sum(d2), l) * r * inv_d;   // the mean of w g h
            // with t = r g: dw += t x, dx = r (w g - h m) = w t - (r r m) x
            const uint64_t r2 = f2_pack(r, r), c2 = f2_pack(-(r * r) * m, -(r * r) * m);
            read_weights(wa, wb);
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                a[j] = f2_mul(a[j], r2);
                b[j] = f2_mul(b[j], r2);
            }
            if (is_q) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    acc[j] = f2_fma(a[j], xa[j], acc[j]);
                    acc[kPairs + j] = f2_fma(b[j], xb[j], acc[kPairs + j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    ulonglong2 v = acc_k[j * 32];
                    v.x = f2_fma(a[j], xa[j], v.x);
                    v.y = f2_fma(b[j], xb[j], v.y);
                    acc_k[j * 32] = v;
                }
            }
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                a[j] = f2_fma(a[j], wa[j], f2_mul(xa[j], c2));
                b[j] = f2_fma(b[j], wb[j], f2_mul(xb[j], c2));
            }
            if (pl.active && h0 + sub < total) {
                T *out = is_q ? out_q : static_cast<T *>(p.dk) + row * p.dk_stride + (h0 - p.hq) * d + lane_at;
                store_vec2<V>(out, a);
                store_vec2<V>(out + to_b, b);
            }
            copy_ahead();   // into the stage just read
            stage = stage + 1 == kBwdStages ? 0 : stage + 1;
        }
    }
    cp_async_wait<0>();
    uint64_t acc_all[2][V];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const ulonglong2 v = acc_k[j * 32];
        acc_all[0][j] = acc[j], acc_all[0][kPairs + j] = acc[kPairs + j];
        acc_all[1][j] = v.x, acc_all[1][kPairs + j] = v.y;
    }
    __syncthreads();   // every warp is done with its stages
    float *sums = reinterpret_cast<float *>(smem_raw);
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float lo, hi;
            f2_unpack(acc_all[kind][j], lo, hi);
            if constexpr (kGroup != 0) {
#pragma unroll
                for (int m = kGroup; m < 32; m <<= 1) {
                    lo += __shfl_xor_sync(0xffffffffu, lo, m);
                    hi += __shfl_xor_sync(0xffffffffu, hi, m);
                }
            } else {   // the first head's lanes collect the others'
                const float own_lo = lo, own_hi = hi;
                for (int g = 1; g < heads; ++g) {
                    lo += __shfl_sync(0xffffffffu, own_lo, chunk + g * group);
                    hi += __shfl_sync(0xffffffffu, own_hi, chunk + g * group);
                }
            }
            if (sub == 0 && pl.active)
                *reinterpret_cast<float2 *>(sums + (warp * 2 + kind) * d + (j < kPairs ? pl.a + 2 * j : pl.b + 2 * (j - kPairs))) = make_float2(lo, hi);
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * d; e += 32 * kBwdWarps) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kBwdWarps; ++w) v += sums[w * 2 * d + e];
        p.part[(int64_t)blockIdx.x * 2 * d + e] = v;
    }
}

// Column sums of the CTAs' partial rows: 32 columns a CTA, a warp takes every 32nd row and has eight of them in
// flight (with 8 warps and a load at a time the 304 rows of the largest grid took 6 us).
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(32 * kSumWarps) rotary_weight_grad_kernel(const float *__restrict__ part, int n, int d, float *dqw, float *dkw)
{
    __shared__ float sums[kSumWarps][32];
    pdl_wait_prerequisite();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float v = 0.f;
    for (int r0 = warp; r0 < n; r0 += 8 * kSumWarps) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int r = r0 + j * kSumWarps;
            x[j] = r < n && col < 2 * d ? part[(int64_t)r * 2 * d + col] : 0.f;
        }
        v += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    sums[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && col < 2 * d) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kSumWarps; ++w) t += sums[w][lane];
        (col < d ? dqw[col] : dkw[col - d]) = t;
    }
}

size_t elt_size(padoc_dtype t) { return t == PADOC_DTYPE_BF16 ? 2 : 4; }

padoc_status check_ptr(const void *p, int64_t stride, int64_t rows, int64_t least, size_t esz)
{
    if (!p) return PADOC_ERR_INVALID_ARGUMENT;
    if (((uintptr_t)p) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if (stride < least || (stride * (int64_t)esz) % 16 != 0) return PADOC_ERR_INVALID_ARGUMENT;
    if (rows > 0 && stride > INT64_MAX / 8 / rows) return PADOC_ERR_INVALID_ARGUMENT;
    return PADOC_OK;
}

template <typename K>
padoc_status launch(K kernel, dim3 grid, int block, size_t smem, padoc_stream_t stream, void **argv)
{
    cudaLaunchConfig_t lc = {};
    lc.gridDim = grid;
    lc.blockDim = dim3(block);
    lc.dynamicSmemBytes = smem;
    lc.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // every kernel here waits for its predecessor
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = attr;
    lc.numAttrs = 1;
    PADOC_CUDA_TRY(cudaLaunchKernelExC(&lc, (const void *)kernel, argv));
    return padoc_launch_status();
}

template <typename T, int V, int kMode, int kGroup>
padoc_status launch_group(const Args &p, bool adjacent, bool norm, dim3 grid, padoc_stream_t stream)
{
    auto *k = adjacent ? (norm ? rotary_kernel<T, V, true, true, kMode, kGroup, kMode == kAppend ? 7 : 1> : rotary_kernel<T, V, true, false, kMode, kGroup, kMode == kAppend ? 7 : 1>)
                       : (norm ? rotary_kernel<T, V, false, true, kMode, kGroup, kMode == kAppend ? 7 : 1> : rotary_kernel<T, V, false, false, kMode, kGroup, kMode == kAppend ? 7 : 1>);
    if constexpr (kMode == kPacked && V == 8)
        if (norm && !adjacent && (int64_t)grid.x * grid.y * kWarps >= 64 * (int64_t)padoc_default_ctas())   // 64 warps an SM
            k = rotary_kernel<T, V, false, true, kMode, kGroup, 6>;
    void *argv[1] = {const_cast<Args *>(&p)};
    return launch(k, grid, 32 * kWarps, 0, stream, argv);
}
template <typename T, int V, int kMode>
padoc_status launch_rows(const Args &p, bool adjacent, bool norm, dim3 grid, padoc_stream_t stream)
{
    // (64, 128 and 256 dims in bf16, 64 and 128 in fp32; other heads, and bf16 ones in 8-byte vectors, take the general form)
    if constexpr (V == 8)
        if (p.group == 4) return launch_group<T, V, kMode, 4>(p, adjacent, norm, grid, stream);
    if constexpr (V == 8 || sizeof(T) == 4) {
        if (p.group == 8) return launch_group<T, V, kMode, 8>(p, adjacent, norm, grid, stream);
        if (p.group == 16) return launch_group<T, V, kMode, 16>(p, adjacent, norm, grid, stream);
    }
    return launch_group<T, V, kMode, 0>(p, adjacent, norm, grid, stream);
}

template <int kMode>
padoc_status launch_any(Args &p, const padoc_rotary *rot, padoc_dtype dtype, padoc_stream_t stream)
{
    const int vec = vec_of(rot, dtype);
    const int parts = split_rows(p, vec, (p.q ? p.hq : 0) + (kMode == kAppend ? 2 : 1) * p.hkv, steps_of(kMode));
    const dim3 grid((unsigned)((p.count + kWarps - 1) / kWarps), (unsigned)parts);
    const bool adj = rot->adjacent != 0, norm = rot->q_weight != nullptr;
    if (dtype == PADOC_DTYPE_F32) return launch_rows<float, 4, kMode>(p, adj, norm, grid, stream);
    return vec == 8 ? launch_rows<__nv_bfloat16, 8, kMode>(p, adj, norm, grid, stream)
                    : launch_rows<__nv_bfloat16, 4, kMode>(p, adj, norm, grid, stream);
}

// CTAs of the backward with the norm, two an SM; each leaves a partial row of weight gradients.
int bwd_ctas(int64_t rows)
{
    const int64_t need = (rows + kBwdWarps - 1) / kBwdWarps, most = 2 * (int64_t)padoc_default_ctas();
    return (int)(need < most ? need : most);
}

template <typename T, int V, int kGroup>
padoc_status launch_bwd_group(const BwdArgs &p, bool adjacent, int ctas, padoc_stream_t stream)
{
    auto *k = adjacent ? rotary_norm_bwd_kernel<T, V, true, kGroup> : rotary_norm_bwd_kernel<T, V, false, kGroup>;
    constexpr size_t kRing = (size_t)kBwdWarps * kBwdStages * 4 * 32 * sizeof(Raw<T, V>), kSums = (size_t)kBwdWarps * (V / 2) * 32 * 16;
    static_assert(kRing >= (size_t)kBwdWarps * 2 * 256 * sizeof(float), "the joined sums fit where the ring was");
    const int smem = (int)((size_t)V * p.group * 16 + kRing + kSums);
    // the limit for the longest heads, whatever this call's: it stays with the kernel, and a later call may need more
    const padoc_status st = padoc_set_max_smem((const void *)k, (int)((size_t)V * 32 * 16 + kRing + kSums));
    void *argv[1] = {const_cast<BwdArgs *>(&p)};
    return st != PADOC_OK ? st : launch(k, dim3((unsigned)ctas), 32 * kBwdWarps, smem, stream, argv);
}
template <typename T, int V>
padoc_status launch_bwd(const BwdArgs &p, bool adjacent, int ctas, padoc_stream_t stream)
{
    if constexpr (V == 8)
        if (p.group == 4) return launch_bwd_group<T, V, 4>(p, adjacent, ctas, stream);
    if constexpr (V == 8 || sizeof(T) == 4) {
        if (p.group == 8) return launch_bwd_group<T, V, 8>(p, adjacent, ctas, stream);
        if (p.group == 16) return launch_bwd_group<T, V, 16>(p, adjacent, ctas, stream);
    }
    return launch_bwd_group<T, V, 0>(p, adjacent, ctas, stream);
}

}  // namespace

int vec_of(const padoc_rotary *r, padoc_dtype t)
{
    return t == PADOC_DTYPE_BF16 && r->head_dim % 16 == 0 && r->rotary_dim % 16 == 0 ? 8 : 4;
}

int split_rows(Args &p, int vec, int heads_total, int most_steps)
{
    p.group = group_of(p.sp.d, vec);
    const int heads = 32 / p.group;
    const int steps = (heads_total + heads - 1) / heads, least = (steps + most_steps - 1) / most_steps;
    const int64_t want = ((int64_t)padoc_default_ctas() * 8 + p.count - 1) / p.count;
    const int parts = want < least ? least : want > steps ? steps : (int)want;
    p.steps = (steps + parts - 1) / parts;
    return (steps + p.steps - 1) / p.steps;
}

padoc_status check_spec(const padoc_rotary *r)
{
    if (!r || !r->freq || (((uintptr_t)r->freq) & 7)) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->head_dim < 1 || r->rotary_dim < 1 || r->rotary_dim > r->head_dim) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->num_axes < 1 || r->num_axes > 4 || (r->adjacent != 0 && r->adjacent != 1)) return PADOC_ERR_INVALID_ARGUMENT;
    if (!std::isfinite(r->amplitude)) return PADOC_ERR_INVALID_ARGUMENT;
    if ((r->q_weight == nullptr) != (r->k_weight == nullptr)) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->q_weight && (!(r->eps >= 0.f) || !std::isfinite(r->eps))) return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)r->q_weight) | ((uintptr_t)r->k_weight)) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if (r->head_dim > 256 || r->head_dim % 8 != 0 || r->rotary_dim % 8 != 0) return PADOC_ERR_UNSUPPORTED;
    return PADOC_OK;
}

padoc_status check_rows(const padoc_qkv_rows *in, const padoc_rotary *rot, bool with_v)
{
    if (!in || in->rows < 0 || in->num_kv_heads < 1 || in->num_q_heads < 0 || (in->q && in->num_q_heads < 1))
        return PADOC_ERR_INVALID_ARGUMENT;
    if (in->dtype != PADOC_DTYPE_BF16 && in->dtype != PADOC_DTYPE_F32) return PADOC_ERR_INVALID_ARGUMENT;
    if (in->rows > INT32_MAX || in->num_q_heads > 4096 || in->num_kv_heads > 4096) return PADOC_ERR_UNSUPPORTED;
    if (in->rows == 0) return PADOC_OK;
    const size_t e = elt_size(in->dtype);
    if (!in->pos || (((uintptr_t)in->pos) & 3)) return PADOC_ERR_INVALID_ARGUMENT;
    padoc_status st = check_ptr(in->k, in->k_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    if (st == PADOC_OK && in->q) st = check_ptr(in->q, in->q_stride, in->rows, (int64_t)in->num_q_heads * rot->head_dim, e);
    if (st == PADOC_OK && with_v) st = check_ptr(in->v, in->v_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    return st;
}

}  // namespace padoc_rotary_dev

using namespace padoc_rotary_dev;

extern "C" padoc_status padoc_build_rotary_table(const double *inv_freq, const int32_t *axis_of, int32_t num_freqs,
                                                 int32_t num_axes, uint64_t *table)
{
    if (!inv_freq || !table || num_freqs < 1 || num_axes < 1 || num_axes > 4 || (num_axes > 1 && !axis_of))
        return PADOC_ERR_INVALID_ARGUMENT;
    for (int32_t i = 0; i < num_freqs; ++i) {
        if (!std::isfinite(inv_freq[i])) return PADOC_ERR_INVALID_ARGUMENT;
        if (axis_of && (axis_of[i] < 0 || axis_of[i] >= num_axes)) return PADOC_ERR_INVALID_ARGUMENT;
    }
    for (int32_t i = 0; i < num_freqs; ++i) {
        const double turns = inv_freq[i] / 6.283185307179586476925;
        const double frac = turns - std::floor(turns);                     // [0, 1]
        const double units = std::nearbyint(std::ldexp(frac, 62));         // the axis takes the two lowest bits
        const uint64_t u = units >= 0x1p62 ? 0 : (uint64_t)units;          // (a whole turn is none)
        table[i] = u << 2 | (uint64_t)(axis_of ? axis_of[i] : 0);
    }
    return PADOC_OK;
}

extern "C" padoc_status padoc_qk_rotary(const padoc_rotary *rot, const padoc_qkv_rows *in, void *q_out, int64_t q_out_stride,
                                        void *k_out, int64_t k_out_stride, padoc_stream_t stream)
{
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    st = check_rows(in, rot, false);
    if (st != PADOC_OK) return st;
    if (in->num_q_heads < 1) return PADOC_ERR_INVALID_ARGUMENT;
    if (in->rows == 0) return PADOC_OK;
    if (!in->q) return PADOC_ERR_INVALID_ARGUMENT;
    const size_t e = elt_size(in->dtype);
    st = check_ptr(q_out, q_out_stride, in->rows, (int64_t)in->num_q_heads * rot->head_dim, e);
    if (st == PADOC_OK) st = check_ptr(k_out, k_out_stride, in->rows, (int64_t)in->num_kv_heads * rot->head_dim, e);
    if (st != PADOC_OK) return st;
    Args p = {};
    p.sp = make_spec(rot);
    p.q = in->q, p.k = in->k;
    p.q_stride = in->q_stride, p.k_stride = in->k_stride;
    p.pos = in->pos;
    p.rows = p.count = in->rows;
    p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
    p.q_out = q_out, p.k_out = k_out;
    p.q_out_stride = q_out_stride, p.k_out_stride = k_out_stride;
    return launch_any<kPacked>(p, rot, in->dtype, stream);
}

extern "C" padoc_status padoc_append_rotary_inputs(const padoc_kv_pool *pool, const padoc_rotary *rot, const padoc_qkv_rows *in,
                                                   void *q_dst, const int32_t *src_rows, const int32_t *slots, int32_t count,
                                                   padoc_stream_t stream)
{
    if (!pool || count < 0) return PADOC_ERR_INVALID_ARGUMENT;
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    st = check_rows(in, rot, true);
    if (st != PADOC_OK) return st;
    if (pool->dtype != in->dtype || pool->head_dim != rot->head_dim || pool->num_kv_heads != in->num_kv_heads ||
        pool->num_blocks < 1 || pool->block_size < 1)
        return PADOC_ERR_INVALID_ARGUMENT;
    if (count == 0) return PADOC_OK;
    if (in->rows == 0 || !slots || !pool->k_pool || !pool->v_pool || (in->q && !q_dst)) return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)pool->k_pool) | ((uintptr_t)pool->v_pool) | ((uintptr_t)q_dst)) & 15) return PADOC_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)src_rows) | ((uintptr_t)slots)) & 3) return PADOC_ERR_INVALID_ARGUMENT;
    int *err = padoc_device_error_word();
    if (!err) return PADOC_ERR_CUDA;
    Args p = {};
    p.sp = make_spec(rot);
    p.q = in->q, p.k = in->k, p.v = in->v;
    p.q_stride = in->q_stride, p.k_stride = in->k_stride, p.v_stride = in->v_stride;
    p.pos = in->pos;
    p.rows = in->rows;
    p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
    p.q_out = q_dst, p.q_out_stride = (int64_t)in->num_q_heads * rot->head_dim;
    p.k_out = const_cast<void *>(pool->k_pool), p.v_out = const_cast<void *>(pool->v_pool);
    p.src_rows = src_rows, p.slots = slots;
    p.count = count;
    p.pool_slots = (int64_t)pool->num_blocks * pool->block_size;
    p.block_size = pool->block_size;
    p.err = err;
    return launch_any<kAppend>(p, rot, in->dtype, stream);
}

extern "C" padoc_status padoc_qk_rotary_bwd_workspace_size(const padoc_rotary *rot, int64_t rows, size_t *bytes)
{
    const padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    if (rows < 0 || !bytes) return PADOC_ERR_INVALID_ARGUMENT;
    if (rows > INT32_MAX) return PADOC_ERR_UNSUPPORTED;
    *bytes = rot->q_weight ? (size_t)bwd_ctas(rows) * 2 * rot->head_dim * sizeof(float) : 0;
    return PADOC_OK;
}

extern "C" padoc_status padoc_qk_rotary_bwd(const padoc_rotary *rot, const padoc_qkv_rows *in, const void *dq_out,
                                            int64_t dq_out_stride, const void *dk_out, int64_t dk_out_stride, void *dq,
                                            int64_t dq_stride, void *dk, int64_t dk_stride, float *dq_weight, float *dk_weight,
                                            void *workspace, size_t workspace_bytes, padoc_stream_t stream)
{
    padoc_status st = check_spec(rot);
    if (st != PADOC_OK) return st;
    if (!in || in->num_q_heads < 1) return PADOC_ERR_INVALID_ARGUMENT;
    const bool norm = rot->q_weight != nullptr;
    padoc_qkv_rows rows = *in;
    if (!norm) {   // the rotation's gradient does not depend on the rows: dk_out stands in for their checks
        rows.q = nullptr;
        rows.k = dk_out;
        rows.k_stride = dk_out_stride;
    }
    st = check_rows(&rows, rot, false);
    if (st != PADOC_OK) return st;
    if (norm) {
        if (!dq_weight || !dk_weight || ((((uintptr_t)dq_weight) | ((uintptr_t)dk_weight)) & 3)) return PADOC_ERR_INVALID_ARGUMENT;
        if (in->rows > 0 && !in->q) return PADOC_ERR_INVALID_ARGUMENT;
    }
    if (in->rows > 0) {
        const size_t e = elt_size(in->dtype);
        const int64_t nq = (int64_t)in->num_q_heads * rot->head_dim, nk = (int64_t)in->num_kv_heads * rot->head_dim;
        st = check_ptr(dq_out, dq_out_stride, in->rows, nq, e);
        if (st == PADOC_OK) st = check_ptr(dk_out, dk_out_stride, in->rows, nk, e);
        if (st == PADOC_OK) st = check_ptr(dq, dq_stride, in->rows, nq, e);
        if (st == PADOC_OK) st = check_ptr(dk, dk_stride, in->rows, nk, e);
        if (st != PADOC_OK) return st;
    }
    Spec back = make_spec(rot);
    back.sin_amplitude = -back.sin_amplitude;
    if (!norm) {   // the rotation back is the forward's kernel
        if (in->rows == 0) return PADOC_OK;
        Args p = {};
        p.sp = back;
        p.q = dq_out, p.k = dk_out;
        p.q_stride = dq_out_stride, p.k_stride = dk_out_stride;
        p.pos = in->pos;
        p.rows = p.count = in->rows;
        p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
        p.q_out = dq, p.k_out = dk;
        p.q_out_stride = dq_stride, p.k_out_stride = dk_stride;
        return launch_any<kPacked>(p, rot, in->dtype, stream);
    }
    const int ctas = bwd_ctas(in->rows), d = rot->head_dim;
    if (ctas > 0) {
        if (!workspace || (((uintptr_t)workspace) & 255)) return PADOC_ERR_INVALID_ARGUMENT;
        if (workspace_bytes < (size_t)ctas * 2 * d * sizeof(float)) return PADOC_ERR_WORKSPACE_TOO_SMALL;
    }
    // both are written, by threads without an order between them
    if ((uintptr_t)dq_weight < (uintptr_t)(dk_weight + d) && (uintptr_t)dk_weight < (uintptr_t)(dq_weight + d))
        return PADOC_ERR_INVALID_ARGUMENT;
    if (ctas > 0) {
        BwdArgs p = {};
        p.sp = back;
        p.q = in->q, p.k = in->k;
        p.q_stride = in->q_stride, p.k_stride = in->k_stride;
        p.pos = in->pos;
        p.rows = in->rows;
        p.hq = in->num_q_heads, p.hkv = in->num_kv_heads;
        p.dq_out = dq_out, p.dk_out = dk_out;
        p.dq_out_stride = dq_out_stride, p.dk_out_stride = dk_out_stride;
        p.dq = dq, p.dk = dk;
        p.dq_stride = dq_stride, p.dk_stride = dk_stride;
        p.part = (float *)workspace;
        const int vec = vec_of(rot, in->dtype);
        p.group = group_of(d, vec);
        const bool adj = rot->adjacent != 0;
        st = in->dtype == PADOC_DTYPE_F32 ? launch_bwd<float, 4>(p, adj, ctas, stream)
             : vec == 8                   ? launch_bwd<__nv_bfloat16, 8>(p, adj, ctas, stream)
                                          : launch_bwd<__nv_bfloat16, 4>(p, adj, ctas, stream);
        if (st != PADOC_OK) return st;
    }
    // (with no rows there are no partial sums: zeros)
    const float *part = (const float *)workspace;
    int n = ctas, dim = d;
    void *argv[5] = {&part, &n, &dim, &dq_weight, &dk_weight};
    return launch(rotary_weight_grad_kernel, dim3((unsigned)((2 * d + 31) / 32)), 32 * kSumWarps, 0, stream, argv);
}
